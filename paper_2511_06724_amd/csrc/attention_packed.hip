// Attention of packed sequences: o = softmax(q k^T scale) v for each sequence and head, causal or
// not, with groups of query heads that share a key head (gfx950).
//
// A work unit is BM query rows of one (sequence, key head). The rows are the sequence's tokens times
// the `group` query heads of that key head (row r: token r / group, head r % group), so one pass over
// the keys serves the whole group, a single new token fills as many rows as the group has heads, and the
// causal border of a tile is BM / group tokens wide. Causal masks are aligned to the end: the last
// token sees all keys of its sequence, token i of n the first kv_len - n + i + 1 (none if that is not
// positive: its output is zero).
//
// Units are found on the device, so lengths may change between calls and replays: sequence s owns the
// slots from floor(q_start[s] group / BM) + s on, which leaves room for its last, partial tile.
//
// Per 64 keys a wave takes S^T = K Q^T with 32 x 32 matrix instructions: a lane holds one query
// column, whose statistics are its own registers and one exchange with lane ^ 32, and the
// probabilities already lie in the operand layout of O^T = V^T P^T. V stays as rows of keys: the
// transposed operand comes from LDS transposed as it is read (bf16) or by rows (fp32).
//
// Softmax in base 2: P = 2^(s scale log2 e - m), where m moves only when a tile's maximum exceeds it
// by more than 2^8 in the exponent (any m gives the same quotient). It starts at the lowest finite
// number, so that a masked score (-inf) gives 0 also while nothing has been seen. Scores, m, the row
// sum and O are fp32; P is rounded to bf16 for the matrix instruction (half a step, 2^-8 of a
// probability, independent from key to key), the row sum adds the rounded values.
//
// Masked keys carry no value, also if theirs is an infinity or a NaN: 0 * inf in the matrix product
// would be NaN. Key rows past the range are not read (the last one is, instead), and if a workgroup's
// result has a non-finite value, it computes its rows again and takes such values out of the
// product, adding them where they are seen. That costs nothing where all results are finite.
#include <algorithm>
#include <cmath>

#include "lane_swap.h"
#include "packed.h"

namespace dn {
namespace {

constexpr int kKT = 64;        // keys per tile
constexpr float kLazy = 8.0f;  // log2 headroom before the reference maximum moves
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// One (sequence, tile of BM rows): rows [row0, row0 + BM) of `rows`.
struct Unit {
  int rows, row0, len_q, len_k;
  long long q0, k0;  // first packed row, first key row
};

__device__ __forceinline__ int from_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ long long from_lane(long long x, int lane) {
  return (long long)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// The unit of a slot, by a whole wave. False: the slot is not used. Up to 64 sequences lie in the lanes at once, which
// saves a load that waits for another.
template <int BM> __device__ __forceinline__ bool find_unit(const PackedAttnParams& p, int group, long long slot, Unit& u) {
  const int* qs = p.seqs.q_start;
  auto place = [&](int q, int i) { return (long long)q * group / BM + i; };
  int s, a, b;
  if (p.seqs.n <= 64) {
    const int i = min((int)(threadIdx.x & 63), p.seqs.n - 1);
    const int qa = qs[i], qb = qs[i + 1], len = p.seqs.kv_len[i];
    const long long k0 = p.seqs.kv_start[i];
    s = __popcll(__ballot((int)(threadIdx.x & 63) < p.seqs.n && place(qa, i) <= slot)) - 1;
    if (s < 0) return false;
    a = from_lane(qa, s);
    b = from_lane(qb, s);
    u.len_k = from_lane(len, s);
    u.k0 = from_lane(k0, s);
  } else {
    s = __builtin_amdgcn_readfirstlane(search_group<64>(p.seqs.n, slot, [&](int i) { return place(qs[i], i); }));
    if (s < 0) return false;
    a = __builtin_amdgcn_readfirstlane(qs[s]);
    b = __builtin_amdgcn_readfirstlane(qs[s + 1]);
    u.len_k = __builtin_amdgcn_readfirstlane(p.seqs.kv_len[s]);
    u.k0 = from_lane(p.seqs.kv_start[s], 0);
  }
  if (!sequence_attends(a, b, p.T, u.len_k, u.k0, p.kv_rows)) return false;
  u.q0 = a;
  u.len_q = b - a;
  const long long rows = (long long)u.len_q * group, row0 = (slot - place(a, s)) * BM;
  if (row0 < 0 || row0 >= rows) return false;  // (below: starts that are not in order)
  u.rows = (int)rows;
  u.row0 = (int)row0;
  return true;
}

// Keys a token of the unit's sequence sees.
__device__ __forceinline__ int limit(const PackedAttnParams& p, const Unit& u, int token) {
  return p.causal ? max(0, token - u.len_q + u.len_k + 1) : u.len_k;
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
// x f; an infinity or a NaN of a value that is seen stays what it is also when its weight f has become zero beside a larger one.
__device__ __forceinline__ float weigh(float x, float f) { return not_finite(x) ? x : x * f; }
__device__ __forceinline__ bool is_nan(float x) { return (__float_as_uint(x) & 0x7fffffffu) > 0x7f800000u; }

// Maximum of scores. (fmaxf would quiet every matrix-core result first, one operation each; this one
// hands a NaN on, whose row is NaN with any reference.)
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Whether a result of the workgroup is an infinity or a NaN; `flags`: LDS that nothing is read from any more, one int a wave.
template <int DB, int NW> __device__ __forceinline__ bool any_not_finite(const f32x16* o, int* flags) {
  bool bad = false;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) bad |= not_finite(o[d][r]);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) flags[threadIdx.x >> 6] = 0;
  __syncthreads();
  if (bad) flags[threadIdx.x >> 6] = 1;
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) any |= flags[w];
  return any != 0;
}

template <typename T> __device__ __forceinline__ T* row_out(const PackedAttnParams& p, const Unit& u, int token, int head, int D) {
  return static_cast<T*>(p.o) + (u.q0 + token) * p.ldo + (long long)head * D;
}

// A lane's half of 32 values of an output row: 8 g + 4 (lane / 32) .. + 3 in registers 4 g .. 4 g + 3.
template <typename T> __device__ __forceinline__ void store_block(T* op, const f32x16& o, float l) {
  const float inv = l != 0.f ? 1.f / l : 0.f;
  op += 4 * ((threadIdx.x & 63) >> 5);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    T v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = from_f32<T>(o[4 * g + e] * inv);
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(op + 8 * g) = __builtin_bit_cast(uint2, bf16x4{v[0], v[1], v[2], v[3]});
    else
      *reinterpret_cast<f32x4*>(op + 8 * g) = f32x4{v[0], v[1], v[2], v[3]};
  }
}

template <typename T> struct Pv;
template <> struct Pv<bf16> {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  static constexpr int STEPS = 2;  // matrix instructions per 32 keys
  // Step c of a 32-key block takes keys 16 c + 4 h + {0..3} and 16 c + 8 + 4 h + {0..3} in lane half h:
  // score registers 8 c .. 8 c + 7.
  __device__ static __forceinline__ bf16x8 p(const f32x16& s, int c) {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = static_cast<bf16>(s[8 * c + e]);
    return r;
  }
  // V[those keys][d0 + lane % 32]: a transposing read gives lane i of 16 the column i of 4 rows of 16
  // values, whose 16 pieces of 4 the lanes point at (lane i: row i / 4, columns 4 (i % 4) ..).
  __device__ static __forceinline__ bf16x8 v(const bf16* vs, int ld, int kb, int c, int d0, int lane) {
    const bf16* a = vs + (kb * 32 + 16 * c + 4 * (lane >> 5) + ((lane & 15) >> 2)) * ld + d0 + (lane & 16) + 4 * (lane & 3);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 8 * ld));
    bf16x8 r;
    const bf16x4 l = __builtin_bit_cast(bf16x4, lo), h = __builtin_bit_cast(bf16x4, hi);
    r[0] = l[0]; r[1] = l[1]; r[2] = l[2]; r[3] = l[3];
    r[4] = h[0]; r[5] = h[1]; r[6] = h[2]; r[7] = h[3];
    return r;
  }
  // Value e of a fragment: finite part; +1 / -1 counts of infinities (a NaN counts as both).
  static constexpr int N = 8;
  __device__ static __forceinline__ float get(const bf16x8& f, int e) { return static_cast<float>(f[e]); }
  __device__ static __forceinline__ void set(bf16x8& f, int e, float x) { f[e] = static_cast<bf16>(x); }
};
template <> struct Pv<float> {
  static constexpr int STEPS = 16;
  // Register c of a 32-key block belongs to key 8 (c / 4) + 4 h + c % 4.
  __device__ static __forceinline__ float p(const f32x16& s, int c) { return s[c]; }
  __device__ static __forceinline__ float v(const float* vs, int ld, int kb, int c, int d0, int lane) {
    return vs[(kb * 32 + 8 * (c >> 2) + 4 * (lane >> 5) + (c & 3)) * ld + d0 + (lane & 31)];
  }
  static constexpr int N = 1;
  __device__ static __forceinline__ float get(const float& f, int) { return f; }
  __device__ static __forceinline__ void set(float& f, int, float x) { f = x; }
};

// The rows of a unit again (32 per wave) over keys [begin, end), when a result was not finite: infinities and NaN of V are
// taken out of the product and counted where their keys are seen.
template <typename T, int D, int NW, typename F>
__device__ __forceinline__ void careful_rows(const PackedAttnParams& p, const Unit& u, int group, int kvh, T* lds, int begin, int end, F emit) {
  using MM = Mma<T>;
  using V = Pv<T>;
  constexpr int NT = 64 * NW, VEC = 16 / sizeof(T), LD = D + VEC, NS = D / MM::KS, DB = D / 32, CH = D / VEC;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int first = u.row0 + (tid >> 6) * 32, row = min(first + (lane & 31), u.rows - 1);
  const int token = row / group, head = kvh * group + row - token * group;
  const int lim = limit(p, u, token);
  const T* qp = static_cast<const T*>(p.q) + (u.q0 + token) * p.ldq + (long long)head * D + half * MM::KPL;
  const T* kp = static_cast<const T*>(p.k) + u.k0 * p.ldk + (long long)kvh * D;
  const T* vp = static_cast<const T*>(p.v) + u.k0 * p.ldv + (long long)kvh * D;
  T* ks = lds;
  T* vs = lds + kKT * LD;
#pragma unroll 1
  for (int d = 0; d < DB; ++d) {  // 32 output values at a time: few registers, for a path that is hardly ever taken
    f32x16 o;
    float m = kLowest, l = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) o[r] = 0.f;
#pragma unroll 1
    for (int k0 = begin; k0 < end; k0 += kKT) {
      __syncthreads();
#pragma unroll 1
      for (int w = tid; w < kKT * CH; w += NT) {
        const int r = w / CH, c = w - r * CH;
        const long long key = min(k0 + r, end - 1);
        st16(ks + r * LD + c * VEC, ld16(kp + key * p.ldk + c * VEC));
        st16(vs + r * LD + c * VEC, ld16(vp + key * p.ldv + c * VEC));
      }
      __syncthreads();
#pragma unroll 1
      for (int kb = 0; kb < 2; ++kb) {
        f32x16 s, n;
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll 1
        for (int i = 0; i < NS; ++i)
          s = MM::mma(MM::load(&ks[(kb * 32 + (lane & 31)) * LD + i * MM::KS + half * MM::KPL]), MM::load(qp + i * MM::KS), s);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = k0 + kb * 32 + acc_row(r, lane) < min(lim, end) ? s[r] * p.scale_log2 : -INFINITY;
          mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          o[r] = weigh(o[r], alpha);
          s[r] = to_f32(from_f32<T>(fast_exp2(s[r] - m)));
          l += s[r];
        }
#pragma unroll 1
        for (int sign = 0; sign < 3; ++sign) {  // the finite values; +inf (and NaN); -inf (and NaN)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (sign > 0) s[r] = k0 + kb * 32 + acc_row(r, lane) < min(lim, end) ? 1.f : 0.f;  // count where a key is seen
            n[r] = sign == 0 ? o[r] : 0.f;
          }
#pragma unroll
          for (int c = 0; c < V::STEPS; ++c) {
            typename MM::frag f = V::v(vs, LD, kb, c, d * 32, lane);
#pragma unroll
            for (int e = 0; e < V::N; ++e) {
              const float x = V::get(f, e);
              const bool finite = !not_finite(x), other = sign == 1 ? x < 0 : x > 0;
              V::set(f, e, sign == 0 ? (finite ? x : 0.f) : (finite || (other && !is_nan(x)) ? 0.f : 1.f));
            }
            n = MM::mma(f, V::p(s, c), n);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int r = 0; r < 16; ++r)
            o[r] = sign == 0 ? n[r] : n[r] == 0.f ? o[r] : o[r] + (sign == 1 ? INFINITY : -INFINITY);
        }
      }
    }
    l += __shfl_xor(l, 32, 64);
    if (first + (lane & 31) < u.rows) emit(token, head, d, o, m, l);
  }
}

// fp32 tiles: four waves of 32 rows, key tiles through registers into LDS, double-buffered. Bound by the fp32 matrix
// instructions (256 operations a cycle and CU, 154 TFLOP/s) where there are tiles for the CUs, by one tile's keys where there
// are not. A lane reads four head dims of K (and held four of Q) at a time, in the same order on both sides. 10/10 x 64, 2 x 1024
// tokens 79 us; 16/4 x 128, 4 x 300 tokens 52.7.
template <int D> __global__ __launch_bounds__(256) void packed_f32_kernel(PackedAttnParams p, int group) {
  using MM = Mma<float>;
  using V = Pv<float>;
  constexpr int NW = 4, BM = 32 * NW, NT = 64 * NW;
  constexpr int LD = D + 4;         // LDS row of a key (elements)
  constexpr int NV = D / 8;         // 16-byte operands of a row per lane
  constexpr int DB = D / 32;
  constexpr int CH = D / 4;         // 16-byte pieces per row
  constexpr int PER = kKT * CH / NT;
  constexpr int STAGE = 2 * kKT * LD;
  __shared__ __align__(16) float lds[2 * STAGE];

  Unit u;
  if (!find_unit<BM>(p, group, blockIdx.x, u)) return;
  const int kvh = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = u.row0 + wave * 32;  // first row of the wave
  const int row = min(first + (lane & 31), u.rows - 1);
  const int token = row / group, head = kvh * group + row - token * group;
  const int lim = limit(p, u, token);
  const int lo = limit(p, u, min(first, u.rows - 1) / group);                // the wave's shortest range
  const int end = limit(p, u, min(u.row0 + BM - 1, u.rows - 1) / group);     // the workgroup's longest
  const int ntiles = (end + kKT - 1) / kKT;

  const float* qp = static_cast<const float*>(p.q) + (u.q0 + token) * p.ldq + (long long)head * D + half * 4;
  f32x4 qv[NV];
#pragma unroll
  for (int n = 0; n < NV; ++n) qv[n] = __builtin_bit_cast(f32x4, ld16(qp + n * 8));
  const float* kp = static_cast<const float*>(p.k) + u.k0 * p.ldk + (long long)kvh * D;
  const float* vp = static_cast<const float*>(p.v) + u.k0 * p.ldv + (long long)kvh * D;
  uint4 rk[PER], rv[PER];
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int w = tid + i * NT, r = w / CH, c = w - r * CH;
      const long long key = min(t * kKT + r, end - 1);
      rk[i] = ld16(kp + key * p.ldk + c * 4);
      rv[i] = ld16(vp + key * p.ldv + c * 4);
    }
  };
  auto store = [&](int buf) {
    float* ks = lds + buf * STAGE;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int w = tid + i * NT, r = w / CH, c = w - r * CH;
      st16(ks + r * LD + c * 4, rk[i]);
      st16(ks + kKT * LD + r * LD + c * 4, rv[i]);
    }
  };

  f32x16 o[DB];
  float m = kLowest, l = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  if (ntiles > 0) {
    load(0);
    store(0);
    if (ntiles > 1) load(1);
  }
  __syncthreads();
  for (int t = 0; t < ntiles; ++t) {
    const int k0 = t * kKT;
    const float* ks = lds + (t & 1) * STAGE;
    const float* vs = ks + kKT * LD;
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      f32x4 ka[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        ka[kb] = __builtin_bit_cast(f32x4, ld16(&ks[(kb * 32 + (lane & 31)) * LD + n * 8 + half * 4]));
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[kb] = MM::mma(ka[kb][e], qv[n][e], s[kb]);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] *= p.scale_log2;
    if (k0 + kKT > lo) {  // keys past a range
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + kb * 32 + acc_row(r, lane) >= lim) s[kb][r] = -INFINITY;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = max2(mx, s[kb][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    if (__any(mx > m + kLazy)) {
      const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = m_new;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = fast_exp2(s[kb][r] - m);
        l += s[kb][r];
      }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int c = 0; c < V::STEPS; ++c)
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = MM::mma(V::v(vs, LD, kb, c, d * 32, lane), s[kb][c], o[d]);
    if (t + 1 < ntiles) {
      store((t + 1) & 1);
      if (t + 2 < ntiles) load(t + 2);
    }
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);  // each half has summed its own keys
  if (any_not_finite<DB, NW>(o, reinterpret_cast<int*>(lds)))
    return careful_rows<float, D, NW>(p, u, group, kvh, lds, 0, end, [&](int tok, int h, int d, const f32x16& x, float, float sum) {
      store_block<float>(row_out<float>(p, u, tok, h, D) + 32 * d, x, sum);
    });
  if (first + (lane & 31) < u.rows) {
    float* op = row_out<float>(p, u, token, head, D);
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<float>(op + 32 * d, o[d], l);
  }
}

// ---------------------------------------------------------------------------
// bf16: the matrix cores and the vector unit kept busy at once.
//
// Tiles of KT keys (rows of K, rows of V) go global -> LDS without registers into a ring of R slots. Work
// is pipelined over blocks of 32 keys: while the exponentials of block j run on the vector unit,
// the matrix cores take the scores of block j + 1 and add the values of block j - 1 with the
// probabilities of the step before. None of the three waits for another, so they are laid out by hand
// in chunks of one matrix instruction, the load of a fragment two chunks ahead and a share of the
// exponentials, held apart by scheduling barriers. Then comes the one decision of a step: whether the
// maximum of the new scores moves the reference; if so, the pending values are added first and O and l scaled.
//
// At the top of tile t a wave waits for its loads of tile t + 1 and meets the others: theirs have
// landed then, and all are done with tile t - 2, whose slot takes tile t + R - 2. Of the waves on a SIMD the
// older one is served first and would run ahead into that barrier, leaving the other alone: priorities
// fall over the steps of a tile, so that the wave that is behind is served first.
//
// LDS rows are D * 2 bytes in 16-byte pieces, stored xor a function of the row so that reads are free
// of bank conflicts: a lane reads one piece of K row lane % 32; a transposing read of V takes 32 bytes (a pair
// of pieces) of each of 4 rows.
//
// Bound by the matrix cores at the clock that power leaves them (a large product of the BLAS library on random data reaches
// 1.14 to 1.22 PFLOP/s). Measured: 32/8 x 128, 4 prompts of 7,000 to 16,000 tokens, causal,
// 2.55 ms (1.11 PFLOP/s, the matrix cores busy 63 % of the CUs' time, no bank conflicts); 20/20 x 128, two images of 4173
// tokens, 356 us (1.0 PFLOP/s; 2.66 tiles a CU); 10/10 x 64, 2 x 4096 tokens, 117 us (734 TFLOP/s, whose exponentials weigh twice).
template <int D, int KT> struct Tile {
  static constexpr int CH = D / 8;                            // 16-byte pieces per row
  static constexpr int BYTES = KT * D * 2;                    // of K, and of V
  // low bits of a step of K (two pieces) and of a block of V (two pairs) that the xor reaches
  static constexpr int XS = D == 128 ? 7 : D == 64 ? 3 : 1, XD = D == 128 ? 3 : D == 64 ? 1 : 0;
  // 8 rows' pieces lie in different 16-byte columns of 128 bytes and 16 rows' of 256
  __device__ static __forceinline__ int k_piece(int row, int c) {
    return c ^ (D == 128  ? row & 15
                : D == 64 ? (row & 7) ^ ((row >> 3) & 1)
                : D == 32 ? (((row >> 1) ^ (row >> 3)) & 1) | ((row >> 1) & 2)
                          : row & 3);
  }
  // 4 rows' pairs in different 32-byte columns of 128 bytes, 4 rows' two neighbouring pairs of 256
  __device__ static __forceinline__ int v_piece(int row, int c) {
    return c ^ (D == 128  ? ((row & 1) << 2) | ((row & 2) ? 10 : 0)
                : D == 64 ? (row & 3) << 1
                : D == 32 ? row & 2
                          : (row & 1) << 1);
  }
};

template <int D, int KT, int NW, int R, int WPE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(WPE, WPE))) void packed_pipe_kernel(PackedAttnParams p, int group,
                                                                                                         int slots) {
  using TL = Tile<D, KT>;
  using V = Pv<bf16>;
  constexpr int BM = 32 * NW, H = KT / 32;
  constexpr int NS = D / 16, DB = D / 32;    // steps of the scores, blocks of the values
  constexpr int C = NS + 2 * DB, PF = 2;     // chunks; how many ahead a fragment is loaded
  constexpr int PW = KT * TL::CH / 64 / NW;  // 1 KB loads of K (and of V) per wave and tile
  static_assert(KT * TL::CH % (64 * NW) == 0, "whole loads per wave");
  static_assert(C % PF == 0, "a fragment's place is the same in every step");
  static_assert(R >= 4 && (H == 1 || H == 2) && 2 * PW * (H == 1 ? 2 : 1) <= C, "ring and loads");
  constexpr int LDS = R * 2 * TL::BYTES;
  static_assert(2 * kKT * (D + 8) * 2 <= LDS, "careful_rows fits");
  __shared__ __align__(16) unsigned char lds[LDS];

  // ids are dealt to the eight XCDs in turn: each gets a contiguous range of key heads, whose keys stay in its L2
  const int total = gridDim.x, xcd = blockIdx.x % 8;
  const int logical = xcd * (total / 8) + min(xcd, total % 8) + blockIdx.x / 8;
  const int kvh = logical / slots;
  int slot = logical - kvh * slots;
  if (p.causal) slot = slots - 1 - slot;  // the longest key ranges first
  Unit u;
  if (!find_unit<BM>(p, group, slot, u)) return;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = u.row0 + wave * 32;
  const int row = min(first + (lane & 31), u.rows - 1), token = row / group, head = kvh * group + row - token * group;
  const int lim = limit(p, u, token);
  const int lo = __builtin_amdgcn_readfirstlane(limit(p, u, min(first, u.rows - 1) / group));      // the wave's shortest range
  const int hi = __builtin_amdgcn_readfirstlane(limit(p, u, min(first + 31, u.rows - 1) / group)); // and longest
  const int end = __builtin_amdgcn_readfirstlane(limit(p, u, min(u.row0 + BM - 1, u.rows - 1) / group));
  const int ntiles = (end + KT - 1) / KT, mine = first < u.rows ? (hi + KT - 1) / KT : 0;

  // a negative scale is one of -q (exactly), scale 0 one of 0 q: a masked score then is -inf
  float c = p.scale_log2;
  bf16x8 qf[NS];
  {
    const bf16* qp = static_cast<const bf16*>(p.q) + (u.q0 + token) * p.ldq + (long long)head * D + half * 8;
    const unsigned flip = c < 0.f ? 0x80008000u : 0u, keep = c == 0.f ? 0u : ~0u;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const uint4 w = ld16(qp + s * 16);
      qf[s] = __builtin_bit_cast(bf16x8, make_uint4((w.x ^ flip) & keep, (w.y ^ flip) & keep, (w.z ^ flip) & keep, (w.w ^ flip) & keep));
    }
  }
  c = c == 0.f ? 1.f : fabsf(c);

  // loads of a tile: piece i * 64 + lane of K and of V, wave-uniform bases and 32-bit lane offsets
  const char* kbase = reinterpret_cast<const char*>(static_cast<const bf16*>(p.k) + u.k0 * p.ldk + (long long)kvh * D);
  const char* vbase = reinterpret_cast<const char*>(static_cast<const bf16*>(p.v) + u.k0 * p.ldv + (long long)kvh * D);
  unsigned koff[PW], voff[PW];
  auto set_offsets = [&](int t) {
#pragma unroll
    for (int j = 0; j < PW; ++j) {
      const int w = (wave * PW + j) * 64 + lane, r = w / TL::CH, ch = w - r * TL::CH;
      const unsigned key = (unsigned)(min(t * KT + r, end - 1) - t * KT);
      koff[j] = 2u * (key * (unsigned)p.ldk + 8u * TL::k_piece(r, ch));
      voff[j] = 2u * (key * (unsigned)p.ldv + 8u * TL::v_piece(r, ch));
    }
  };
  auto load_k = [&](int at, int j) { dma16_base(kbase, koff[j], (lds_void*)(lds + at * 2 * TL::BYTES + (wave * PW + j) * 1024)); };
  auto load_v = [&](int at, int j) { dma16_base(vbase, voff[j], (lds_void*)(lds + at * 2 * TL::BYTES + TL::BYTES + (wave * PW + j) * 1024)); };
  int issued = 0;
  // past the last tile it is loaded again: the same count of loads per tile, which nothing reads
  auto advance = [&] {
    if (issued < ntiles - 1) {
      ++issued;
      kbase += 2 * KT * p.ldk;
      vbase += 2 * KT * p.ldv;
      if (issued == ntiles - 1) set_offsets(issued);
    }
  };
  auto issue = [&](int at) {
#pragma unroll
    for (int j = 0; j < PW; ++j) load_k(at, j);
#pragma unroll
    for (int j = 0; j < PW; ++j) load_v(at, j);
    advance();
  };

  // lane offsets of the fragments within a slot. Step s of K is piece 2 s + half, block d of V the pieces from 4 d:
  // their low bits go into the xor with the row, the rest is added
  constexpr int XS = TL::XS, XD = TL::XD;
  const int kfo = (lane & 31) * D * 2 + TL::k_piece(lane & 31, half) * 16;
  const int vrow = 4 * half + ((lane & 15) >> 2), vcol = (lane & 16) + 4 * (lane & 3);
  const int vfo = TL::BYTES + vrow * D * 2 + TL::v_piece(vrow, vcol >> 3) * 16 + (vcol & 7) * 2;
  auto k_frag = [&](const unsigned char* T, int kb, int s) {
    return *reinterpret_cast<const bf16x8*>(T + (kfo ^ ((s & XS) << 5)) + ((s & ~XS) << 5) + kb * 32 * D * 2);
  };
  // fragment n of a block's values: keys 16 (n / DB) .., values 32 (n % DB) ..
  auto v_frag = [&](const unsigned char* T, int kb, int n) {
    const int cc = n / DB, d = n % DB;
    const unsigned char* a = T + (vfo ^ ((d & XD) << 6)) + ((d & ~XD) << 6) + (kb * 32 + 16 * cc) * D * 2;
    const bf16x4 l = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((V::lds_s16x4*)a));
    const bf16x4 h = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((V::lds_s16x4*)(a + 8 * D * 2)));
    return __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  f32x16 o[DB];
  float sa[16], m = kLowest, l = 0.f, top = 0.f;  // scores at hand, reference maximum, row sum, the scores' maximum
  bool move = false;                              // that maximum exceeds the reference somewhere in the wave
  bf16x8 pf[2][2], fr[PF];
  const bf16x8 none = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0));
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  pf[1][0] = pf[1][1] = none;

  // eight scores leave the accumulators; their maximum
  auto take = [&](const f32x16& x, float* y) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = x[e];
      asm("" : "+v"(y[e]));
    }
    return max2(max2(max2(max2(max2(y[0], y[1]), y[2]), max2(max2(y[3], y[4]), y[5])), y[6]), y[7]);
  };
  auto compare = [&](float x) {
    top = x * c;
    move = __any(top > m + kLazy);
  };
  auto zero16 = [] {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
  };
  // O^T += V^T P^T of one block
  auto values = [&](const unsigned char* T, int kb, const bf16x8 (&pp)[2]) {
#pragma unroll
    for (int n = 0; n < 2 * DB; ++n) {
      o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(T, kb, n), pp[n / DB], o[n % DB], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Block j: its exponentials into pn; scores of block j + 1 (block kn of tile Tn); values of block j - 1 (kp of Tp) with
  // pp; first fragments of the values of block j (kc of Tc) for the next step; loads into slot `in`.
  auto step = [&](int j, const unsigned char* Tp, int kp, const unsigned char* Tn, int kn, const unsigned char* Tc, int kc, int in,
                  bf16x8 (&pp)[2], bf16x8 (&pn)[2]) {
    if ((j + 1) * 32 > lo) {  // keys past a range
      float x = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (j * 32 + acc_row(r, lane) >= lim) sa[r] = -INFINITY;
        x = fmaxf(x, sa[r]);
      }
      compare(x);
    }
    if (move) {
      values(Tp, kp, pp);
      const float m_new = fmaxf(m, fmaxf(top, __shfl_xor(top, 32, 64)));
      const float alpha = fast_exp2(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      m = m_new;
      pp[0] = pp[1] = none;
    }
    f32x16 sn;
    float w[2], ev[4], sv[16];
    // probabilities 2 k, 2 k + 1 to bf16, and into the row sum
    auto round_pair = [&](int k) {
      const bf16x2 ones = {static_cast<bf16>(1.f), static_cast<bf16>(1.f)};
      unsigned pair = pack_bf16(ev[(2 * k) & 3], ev[(2 * k + 1) & 3]);
      asm volatile("" : "+v"(pair));
      const bf16x2 pr = __builtin_bit_cast(bf16x2, pair);
      pn[k >> 2][(2 * k) & 7] = pr[0];
      pn[k >> 2][(2 * k + 1) & 7] = pr[1];
      l = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l, false);
    };
    // chunks: the first PF values, the scores, the other values (beside which the scores are taken)
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const bf16x8 f = fr[i % PF];
      if (H == 2 && i % (C / 2) == 0) {
        if (kc == 0 && i == 0) __builtin_amdgcn_s_setprio(3);
        if (kc == 0 && i != 0) __builtin_amdgcn_s_setprio(2);
        if (kc == 1 && i == 0) __builtin_amdgcn_s_setprio(1);
        if (kc == 1 && i != 0) __builtin_amdgcn_s_setprio(0);
      }
      if (i % 2 == 1) {  // tiles of two blocks: K beside the first, V beside the second
        const int n = i / 2;
        if (H == 1 ? n < PW : kc == 0 && n < PW) load_k(in, n);
        if (H == 1 ? n >= PW && n < 2 * PW : kc == 1 && n < PW) load_v(in, H == 1 ? n - PW : n);
      }
      {
        const int n = i + PF;
        fr[i % PF] = n < PF + NS ? k_frag(Tn, kn, n - PF) : n < C ? v_frag(Tp, kp, n - NS) : v_frag(Tc, kc, n - C);
      }
      if (i >= PF && i < PF + NS) {
        sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i - PF], i == PF ? zero16() : sn, 0, 0, 0);
      } else {
        const int n = i < PF ? i : i - NS;
        o[n % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, pp[n / DB], o[n % DB], 0, 0, 0);
      }
#pragma unroll
      for (int e = i * 16 / C; e < (i + 1) * 16 / C; ++e) {
        if (e >= 2 && e % 2 == 0) round_pair(e / 2 - 1);
        ev[e & 3] = fast_exp2(fmaf(sa[e], c, -m));
        asm volatile("" : "+v"(ev[e & 3]));
      }
      constexpr int S1 = PF + NS + 1;
      if (i == (S1 < C - 1 ? S1 : C - 1)) w[0] = take(__builtin_shufflevector(sn, sn, 0, 1, 2, 3, 4, 5, 6, 7, 0, 1, 2, 3, 4, 5, 6, 7), sv);
      if (i == (S1 + 1 < C - 1 ? S1 + 1 : C - 1))
        w[1] = take(__builtin_shufflevector(sn, sn, 8, 9, 10, 11, 12, 13, 14, 15, 8, 9, 10, 11, 12, 13, 14, 15), sv + 8);
      if (i == (S1 + 2 < C - 1 ? S1 + 2 : C - 1)) compare(max2(w[0], w[1]));
      __builtin_amdgcn_sched_barrier(0);
    }
    round_pair(7);
#pragma unroll
    for (int r = 0; r < 16; ++r) sa[r] = sv[r];
  };

  if (ntiles > 0) {
    set_offsets(0);
#pragma unroll
    for (int t = 0; t < R - 2; ++t) issue(t);
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((R - 3) * 2 * PW));
    __builtin_amdgcn_s_barrier();
    f32x16 s0 = zero16();
#pragma unroll
    for (int s = 0; s < NS; ++s) s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(lds, 0, s), qf[s], s0, 0, 0, 0);
    const float x0 = take(__builtin_shufflevector(s0, s0, 0, 1, 2, 3, 4, 5, 6, 7, 0, 1, 2, 3, 4, 5, 6, 7), sa);
    const float x1 = take(__builtin_shufflevector(s0, s0, 8, 9, 10, 11, 12, 13, 14, 15, 8, 9, 10, 11, 12, 13, 14, 15), sa + 8);
    compare(max2(x0, x1));
#pragma unroll
    for (int i = 0; i < PF; ++i) fr[i] = v_frag(lds, H - 1, i);
    int at = 0;  // slot of tile t
    const unsigned char* Tp = lds;
    auto turn = [&] {
      __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((R - 4) * 2 * PW));
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    // the loop's place within 32 bytes of instructions, whatever comes before: 64 wide, 8192 tokens 255.7 us here, 260.1 at the
    // worst of eight; 128 wide 0.7 % between them
    asm volatile(".p2align 5\n\ts_nop 0\n\ts_nop 0");
    for (int t = 0; t < mine; ++t) {
      turn();
      const unsigned char* T = lds + at * 2 * TL::BYTES;
      const int in = at < 2 ? at + R - 2 : at - 2;
      at = at == R - 1 ? 0 : at + 1;
      const unsigned char* Tn = lds + at * 2 * TL::BYTES;
      if constexpr (H == 2) {
        step(2 * t, Tp, 1, T, 1, T, 0, in, pf[1], pf[0]);
        step(2 * t + 1, T, 0, Tn, 0, T, 1, in, pf[0], pf[1]);
      } else {
        step(t, Tp, 0, Tn, 0, T, 0, in, pf[1], pf[0]);
        pf[1][0] = pf[0][0];
        pf[1][1] = pf[0][1];
      }
      advance();
      Tp = T;
    }
    values(Tp, H - 1, pf[1]);
    for (int t = mine; t < ntiles; ++t) {  // the other waves' tiles: this one's share of the loads
      turn();
      issue(at < 2 ? at + R - 2 : at - 2);
      at = at == R - 1 ? 0 : at + 1;
    }
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(0));
  }
  l += __shfl_xor(l, 32, 64);  // each half has summed its own keys
  if (any_not_finite<DB, NW>(o, reinterpret_cast<int*>(lds))) 
    return careful_rows<bf16, D, NW>(p, u, group, kvh, reinterpret_cast<bf16*>(lds), 0, end, [&](int tok, int h, int d, const f32x16& x, float, float sum) {
      store_block<bf16>(row_out<bf16>(p, u, tok, h, D) + 32 * d, x, sum);
    });
  if (first + (lane & 31) < u.rows) {
    bf16* op = row_out<bf16>(p, u, token, head, D);
#pragma unroll
    for (int d = 0; d < DB; ++d) store_block<bf16>(op + 32 * d, o[d], l);
  }
}

template <int D, int KT, int NW, int R, int WPE> void launch_pipe(const PackedAttnParams& p, hipStream_t s) {
  constexpr int BM = 32 * NW;
  const int group = p.heads / p.kv_heads;
  const long long slots = p.T * group / BM + p.seqs.n;
  DN_CHECK(slots * p.kv_heads * (64 * NW) < (1ll << 32), "dn_op_attention_packed: too many rows for one launch");
  hipLaunchKernelGGL((packed_pipe_kernel<D, KT, NW, R, WPE>), dim3((unsigned)(slots * p.kv_heads)), dim3(64 * NW), 0, s, p, group, (int)slots);
  DN_HIP(hipGetLastError());
}

// ---------------------------------------------------------------------------
// 16 bytes per lane global -> LDS as dma16_base, for data that is read once: past the caches the same reads reach 6.5 TB/s,
// through them 5.6 (1.07 GB, rows of 256 bytes 2 KB apart).
__device__ __forceinline__ void dma16_stream(const char* base, unsigned off, lds_void* lds) {
  const unsigned a = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(reinterpret_cast<__UINTPTR_TYPE__>(lds)));
  const unsigned long long b = reinterpret_cast<__UINTPTR_TYPE__>(base);
  const unsigned long long u = static_cast<unsigned long long>(__builtin_amdgcn_readfirstlane(static_cast<unsigned>(b >> 32))) << 32 |
                               static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<unsigned>(b)));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(off), "s"(u), "s"(a) : "memory", "m0");
}

// Few rows per sequence (single tokens, short drafts) over many keys: bound by reading K and V once.
//
// Work units are 32 rows of one (sequence, key head), each as many blocks of 32 keys long as its sequence. `shares`
// workgroups divide all blocks of the call evenly, whatever the lengths: workgroup w takes blocks [w B / shares,
// (w + 1) B / shares) of their concatenation, found from the lengths on the device. Within a unit each of its NW
// waves takes every NW-th block, loaded global -> LDS into a ring of its own, so nothing waits for another wave until
// the unit's end, where the waves' (m, l, O) meet in LDS in wave order. A unit that one workgroup has to itself is stored;
// one that is divided goes to the workspace in parts, which a second kernel joins in order: results do not depend on timing.
// 32/8 x 128, 32 contexts of 1 to 54 k keys (1.07 GB): 176 us and 6.7 of the join, 6.1 TB/s while a large copy moves 5.1.
template <typename T, int D> struct Block {
  static constexpr int RB = D * (int)sizeof(T), CH = RB / 16;  // bytes and 16-byte pieces per row
  static constexpr int BYTES = 32 * RB;                        // of K, and of V
  static constexpr int KX = CH % 16 == 0 ? 15 : CH % 8 == 0 ? 7 : 3, VX = sizeof(T) == 4 ? 0 : CH % 8 == 0 ? 3 : 1;
  __device__ static __forceinline__ int k_piece(int row, int c) { return c ^ (row & KX); }
  __device__ static __forceinline__ int v_piece(int row, int c) { return c ^ ((row & VX) << 1); }
};

// The workspace of divided units. A workgroup has at most two: one it comes into (part 0), one it leaves (part 1).
// A divided unit belongs to the workgroup that begins it: `rows` (0: the workgroup leaves none) from row0 of the
// sequence at packed row q0, workgroups up to `last`.
struct DividedUnit {
  int rows, row0, kvh, last;
  long long q0;
};
struct Partials {
  DividedUnit* unit = nullptr;  // [shares]
  float2* ml = nullptr;         // [shares][2][32] (m, l)
  float* o = nullptr;           // [shares][2][32][D]
};

__device__ __forceinline__ int key_blocks(int len) { return max(1, (len + 31) / 32); }  // (one that stores zeros, without keys)

// Sequences in order, 64 at a time in the lanes of a wave: blocks of the units (for one key head) before and in each.
struct Walk {
  int first = 0;             // sequence of lane 0
  long long base = 0;        // blocks before it
  long long incl = 0, cost = 0, k0 = 0;
  int qa = 0, qb = 0, len = 0;
  __device__ __forceinline__ void load(const PackedAttnParams& p, int group) {
    const int i = first + (threadIdx.x & 63);
    cost = 0;
    if (i < p.seqs.n) {
      qa = p.seqs.q_start[i], qb = p.seqs.q_start[i + 1], len = p.seqs.kv_len[i];
      k0 = p.seqs.kv_start[i];
      if (sequence_attends(qa, qb, p.T, len, k0, p.kv_rows))
        cost = ((long long)(qb - qa) * group + 31) / 32 * key_blocks(len);
    }
    incl = cost;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const long long x = __shfl_up(incl, d, 64);
      if ((int)(threadIdx.x & 63) >= d) incl += x;
    }
  }
  __device__ __forceinline__ long long last() const { return base + from_lane(incl, 63); }
  __device__ __forceinline__ void next(const PackedAttnParams& p, int group) {
    base = last();
    first += 64;
    load(p, group);
  }
  __device__ __forceinline__ void restart(const PackedAttnParams& p, int group) {
    if (first == 0) return;
    first = 0;
    base = 0;
    load(p, group);
  }
  // lane of the sequence that block y belongs to; y < all blocks, not before `base`
  __device__ __forceinline__ int find(const PackedAttnParams& p, int group, long long y) {
    while (y >= last()) next(p, group);
    return __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(base + incl > y)) - 1);
  }
};

template <typename T, int D, int NW, int R, bool DIVIDED>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(D * sizeof(T) <= 64 ? 2 : 1))) void packed_narrow_kernel(
    PackedAttnParams p, int group, int shares, Partials part) {
  using MM = Mma<T>;
  using BL = Block<T, D>;
  constexpr int NV = BL::CH / 2;             // 16-byte operands of a K or Q row per lane
  constexpr int DB = D / 32;
  constexpr int LW = 32 * BL::CH / 64;       // 1 KB loads of K (and of V) per block
  constexpr int RING = NW * R * 2 * BL::BYTES, CARE = 2 * kKT * (D + 16 / (int)sizeof(T)) * (int)sizeof(T), JOIN = NW * (DB * 16 * 64 + 64) * 4;
  constexpr int LDS = RING > CARE ? (RING > JOIN ? RING : JOIN) : (CARE > JOIN ? CARE : JOIN);
  __shared__ __align__(16) unsigned char lds[LDS];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, r32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  Walk walk;
  long long per_head = 1, x0 = 0, x1 = 1;  // blocks of one key head; the workgroup's
  if constexpr (DIVIDED) {
    walk.load(p, group);
    per_head = walk.last();
    while (walk.first + 64 < p.seqs.n) {
      walk.next(p, group);
      per_head = walk.last();
    }
    walk.restart(p, group);
    const long long blocks = per_head * p.kv_heads;
    const long long g = min((long long)shares, blocks);  // (with fewer blocks than workgroups the last have none)
    if (tid == 0) part.unit[blockIdx.x].rows = 0;
    if (blockIdx.x >= g) return;
    x0 = blocks * blockIdx.x / g;
    x1 = blocks * (blockIdx.x + 1) / g;
  }
  while (x0 < x1) {
    Unit u;
    int kvh = blockIdx.y, b0 = 0, b1;
    bool whole = true;
    long long unit_part = 0;
    if constexpr (DIVIDED) {
      kvh = (int)(x0 / per_head);
      const long long y = x0 - kvh * per_head;
      if (y < walk.base) walk.restart(p, group);
      const int i = walk.find(p, group, y);
      const int qa = from_lane(walk.qa, i);
      u.q0 = qa;
      u.len_q = from_lane(walk.qb, i) - qa;
      u.len_k = from_lane(walk.len, i);
      u.k0 = from_lane(walk.k0, i);
      const int nb = key_blocks(u.len_k);
      const long long in = y - (walk.base + from_lane(walk.incl - walk.cost, i));
      const int tile = (int)(in / nb);
      b0 = (int)(in - (long long)tile * nb);
      b1 = b0 + (int)min((long long)(nb - b0), x1 - x0);
      u.row0 = tile * 32;
      u.rows = (int)min((long long)u.len_q * group, u.row0 + 32ll);
      whole = b0 == 0 && b1 == nb;
      unit_part = 2ll * blockIdx.x + (b0 == 0 ? 1 : 0);
      if (b0 == 0 && !whole && tid == 0) {
        // the last workgroup w with w blocks / g <= the unit's last block
        const long long blocks = per_head * p.kv_heads, g = min((long long)shares, blocks);
        part.unit[blockIdx.x] = DividedUnit{u.rows - u.row0, u.row0, kvh, (int)(((x0 + nb) * g - 1) / blocks), u.q0};
      }
      x0 += b1 - b0;
    } else {
      if (!find_unit<32>(p, group, blockIdx.x, u)) return;
      u.rows = min(u.rows, u.row0 + 32);
      b1 = key_blocks(u.len_k);
      ++x0;
    }

    const int row = min(u.row0 + r32, u.rows - 1), token = row / group, head = kvh * group + row - token * group;
    const int lim = limit(p, u, token);
    const int range = __builtin_amdgcn_readfirstlane(limit(p, u, (u.rows - 1) / group));
    const int lo = __builtin_amdgcn_readfirstlane(limit(p, u, u.row0 / group));
    const int end = min(range, b1 * 32);
    auto emit = [&](int tok, int h, int d, const f32x16& x, float m, float sum) {
      if (whole) return store_block<T>(row_out<T>(p, u, tok, h, D) + 32 * d, x, sum);
      float* o = part.o + (unit_part * 32 + r32) * D + 32 * d + 4 * half;
#pragma unroll
      for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(o + 8 * g) = f32x4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
      if (d == 0 && half == 0) part.ml[unit_part * 32 + r32] = make_float2(m, sum);
    };

    const T* qp = static_cast<const T*>(p.q) + (u.q0 + token) * p.ldq + (long long)head * D + half * (16 / sizeof(T));
    uint4 qv[NV];
#pragma unroll
    for (int s = 0; s < NV; ++s) qv[s] = ld16(qp + s * (32 / sizeof(T)));
    const char* kbase = reinterpret_cast<const char*>(static_cast<const T*>(p.k) + u.k0 * p.ldk + (long long)kvh * D);
    const char* vbase = reinterpret_cast<const char*>(static_cast<const T*>(p.v) + u.k0 * p.ldv + (long long)kvh * D);
    unsigned char* ring = lds + wave * R * 2 * BL::BYTES;
    unsigned koff[LW], voff[LW];
    auto set_offsets = [&](int keys) {  // of a block that has `keys` keys: the rows past them read the last one
#pragma unroll
      for (int j = 0; j < LW; ++j) {
        const int w = j * 64 + lane, r = w / BL::CH, ch = w - r * BL::CH;
        const unsigned key = (unsigned)min(r, keys - 1) * (unsigned)sizeof(T);
        koff[j] = key * (unsigned)p.ldk + 16u * BL::k_piece(r, ch);
        voff[j] = key * (unsigned)p.ldv + 16u * BL::v_piece(r, ch);
      }
    };
    set_offsets(32);
    auto issue = [&](int b, int slot) {
      const char* kb = kbase + (long long)b * 32 * p.ldk * (int)sizeof(T);
      const char* vb = vbase + (long long)b * 32 * p.ldv * (int)sizeof(T);
      unsigned char* to = ring + slot * 2 * BL::BYTES;
      const bool partial = (b + 1) * 32 > end;
      if (partial) set_offsets(end - b * 32);
#pragma unroll
      for (int j = 0; j < LW; ++j) dma16_stream(kb, koff[j], (lds_void*)(to + j * 1024));
#pragma unroll
      for (int j = 0; j < LW; ++j) dma16_stream(vb, voff[j], (lds_void*)(to + BL::BYTES + j * 1024));
      if (partial) set_offsets(32);
    };

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    float m = kLowest, l = 0.f;
    const int nk = (end + 31) / 32 - b0;                                   // blocks with keys (some rows see)
    const int mine = nk > wave ? (nk - wave + NW - 1) / NW : 0;            // of the wave
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < R - 1; ++i) issue(b0 + wave + min(i, mine - 1) * NW, i);
    }
    int slot = 0;
    for (int i = 0; i < mine; ++i) {
      // reads of the slot that is loaded now are done; past the last block it is loaded again, so that the count of
      // loads behind a block is the same
      __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(63));
      issue(b0 + wave + min(i + R - 1, mine - 1) * NW, slot == 0 ? R - 1 : slot - 1);
      __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((R - 1) * 2 * LW));
      __builtin_amdgcn_sched_barrier(0);
      const unsigned char* K = ring + slot * 2 * BL::BYTES;
      const T* vs = reinterpret_cast<const T*>(K + BL::BYTES);
      const int k0 = (b0 + wave + i * NW) * 32;
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const uint4 kv = *reinterpret_cast<const uint4*>(K + r32 * BL::RB + BL::k_piece(r32, 2 * n + half) * 16);
        if constexpr (sizeof(T) == 4) {
          const f32x4 ka = __builtin_bit_cast(f32x4, kv), qa = __builtin_bit_cast(f32x4, qv[n]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s = MM::mma(ka[e], qa[e], s);
        } else {
          s = MM::mma(__builtin_bit_cast(bf16x8, kv), __builtin_bit_cast(bf16x8, qv[n]), s);
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= p.scale_log2;
      if (k0 + 32 > min(lo, end)) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (k0 + acc_row(r, lane) >= min(lim, end)) s[r] = -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      if (__any(mx > m + kLazy)) {
        const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - m_new);
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
        m = m_new;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = to_f32(from_f32<T>(fast_exp2(s[r] - m)));
        l += s[r];
      }
      if constexpr (sizeof(T) == 4) {
        // register 4 g + e: key 8 g + 4 half + e (V is stored as it is)
#pragma unroll
        for (int c = 0; c < 16; ++c)
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d] = MM::mma(vs[(8 * (c >> 2) + 4 * half + (c & 3)) * D + d * 32 + r32], s[c], o[d]);
      } else {
        const int vrow = 4 * half + ((lane & 15) >> 2), vcol = (lane & 16) + 4 * (lane & 3);
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          const bf16x8 pf = Pv<bf16>::p(s, cc);
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const int col = d * 32 + vcol, r0 = 16 * cc + vrow;  // rows r0 and r0 + 8 have one xor
            const unsigned char* a = K + BL::BYTES + r0 * BL::RB + BL::v_piece(r0, col >> 3) * 16 + (col & 7) * 2;
            const bf16x4 x = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Pv<bf16>::lds_s16x4*)a));
            const bf16x4 y = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Pv<bf16>::lds_s16x4*)(a + 8 * BL::RB)));
            o[d] = MM::mma(__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7), pf, o[d]);
          }
        }
      }
      slot = slot == R - 1 ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(0));
    l += __shfl_xor(l, 32, 64);
    if (any_not_finite<DB, NW>(o, reinterpret_cast<int*>(lds))) {
      __syncthreads();
      careful_rows<T, D, NW>(p, u, group, kvh, reinterpret_cast<T*>(lds), b0 * 32, end, emit);
      __syncthreads();
      continue;
    }
    __syncthreads();

    // the waves' results in order: thread (unit w of 32 values d, lane) sums over the waves
    float* so = reinterpret_cast<float*>(lds);         // [wave][DB][16][64]
    float* sm = so + NW * DB * 16 * 64;                // [wave][32] m, then [wave][32] l
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) so[((wave * DB + d) * 16 + r) * 64 + lane] = o[d][r];
    if (half == 0) {
      sm[wave * 32 + r32] = m;
      sm[NW * 32 + wave * 32 + r32] = l;
    }
    __syncthreads();
    if (u.row0 + r32 < u.rows) {
      float top = sm[r32], sum = 0.f, f[NW];
#pragma unroll
      for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w * 32 + r32]);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        f[w] = fast_exp2(sm[w * 32 + r32] - top);
        sum += f[w] * sm[NW * 32 + w * 32 + r32];
      }
      for (int d = wave; d < DB; d += NW) {
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          x[r] = 0.f;
#pragma unroll
          for (int w = 0; w < NW; ++w) x[r] += f[w] * so[((w * DB + d) * 16 + r) * 64 + lane];
        }
        emit(token, head, d, x, top, sum);
      }
    }
    __syncthreads();
  }
}

// A row of a divided unit from its parts first, first + step, ..: reference maximum, row sum and this lane's D / 64 values
// against it. A lane holds the statistics of one part.
template <int D> struct JoinedRow {
  static constexpr int E = (D + 63) / 64;
  float top = kLowest, sum = 0.f, v[E] = {};
  // Parts first, first + step, .. of n. Again with weigh() if a value is a NaN, so that the usual sum costs no more.
  template <int W> __device__ __forceinline__ void add(const Partials& part, int w0, int n, int r, int first, int step) {
    add_parts<W, false>(part, w0, n, r, first, step);
    bool nan = false;
#pragma unroll
    for (int e = 0; e < E; ++e) nan |= is_nan(v[e]);
    if (__builtin_expect(__any(nan), 0)) {
      *this = JoinedRow();
      add_parts<1, true>(part, w0, n, r, first, step);
    }
  }
  // (with loads of W parts side by side)
  template <int W, bool WEIGH> __device__ __forceinline__ void add_parts(const Partials& part, int w0, int n, int r, int first, int step) {
    const int lane = threadIdx.x & 63;
    auto at = [&](int k) { return (2ll * (w0 + k) + (k == 0 ? 1 : 0)) * 32 + r; };
    for (int c = first; c < n; c += 64 * step) {
      const int mine = c + lane * step, cnt = min(64, (n - c + step - 1) / step);
      const float2 ml = mine < n ? part.ml[at(mine)] : make_float2(kLowest, 0.f);
      // values and statistics come from another XCD's writes: one wait for both
      float x[W][E];
      auto load = [&](int k0) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float* o = part.o + at(c + min(k0 + j, cnt - 1) * step) * D;
#pragma unroll
          for (int e = 0; e < E; ++e) x[j][e] = o[min(e * 64 + lane, D - 1)];
        }
      };
      load(0);
      const float up = fmaxf(top, wave_max(ml.x)), alpha = fast_exp2(top - up);
      top = up;
      sum *= alpha;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = WEIGH ? weigh(v[e], alpha) : v[e] * alpha;
      const float f = ml.y == 0.f ? 0.f : fast_exp2(ml.x - top), fl = f * ml.y;
      for (int k0 = 0; k0 < cnt; k0 += W) {
        if (k0) load(k0);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (k0 + j < cnt) {
            const float fk = __shfl(f, k0 + j, 64);
            sum += __shfl(fl, k0 + j, 64);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += WEIGH ? weigh(x[j][e], fk) : fk * x[j][e];
          }
        }
      }
    }
  }
  template <typename T> __device__ __forceinline__ void store(const PackedAttnParams& p, int group, const DividedUnit& u, int r) const {
    const int lane = threadIdx.x & 63, row = u.row0 + r, token = row / group;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    T* o = static_cast<T*>(p.o) + (u.q0 + token) * p.ldo + (long long)(u.kvh * group + row - token * group) * D;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * 64 + lane < D) o[e * 64 + lane] = from_f32<T>(v[e] * inv);
  }
};

// Joins units of few parts: four waves (of each of gridDim.y workgroups) take the rows of the units that four shares begin in turn.
template <typename T, int D> __global__ __launch_bounds__(256) void join_rows_kernel(PackedAttnParams p, int group, int shares, Partials part) {
  const int waves = 4 * gridDim.y, wave = __builtin_amdgcn_readfirstlane(4 * blockIdx.y + (threadIdx.x >> 6));
  DividedUnit units[4];  // (loads side by side)
#pragma unroll
  for (int i = 0; i < 4; ++i) units[i] = part.unit[min((int)blockIdx.x * 4 + i, shares - 1)];
  int before = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const DividedUnit u = units[i];
    const int w0 = blockIdx.x * 4 + i;
    if (w0 >= shares) return;
    for (int r = (wave + waves - before) % waves; r < u.rows; r += waves) {
      JoinedRow<D> row;
      row.template add<16>(part, w0, u.last - w0 + 1, r, 0, 1);
      row.template store<T>(p, group, u, r);
    }
    before = (before + u.rows) % waves;
  }
}

// Joins units of many parts: a workgroup per row, whose wave w takes parts w, w + kJoin, ..; then the waves' sums in order.
constexpr int kJoin = 8;
template <typename T, int D> __global__ __launch_bounds__(64 * kJoin) void join_kernel(PackedAttnParams p, int group, Partials part) {
  constexpr int E = JoinedRow<D>::E;
  __shared__ float s_v[kJoin][E * 64], s_top[kJoin], s_sum[kJoin];
  const int w0 = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const DividedUnit u = part.unit[w0];
  for (int r = blockIdx.y; r < u.rows; r += gridDim.y) {
    JoinedRow<D> row;
    row.template add<4>(part, w0, u.last - w0 + 1, r, wave, kJoin);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) s_v[wave][e * 64 + lane] = row.v[e];
    if (lane == 0) {
      s_top[wave] = row.top;
      s_sum[wave] = row.sum;
    }
    __syncthreads();
    if (wave == 0) {
      JoinedRow<D> all;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) all.top = fmaxf(all.top, s_top[k]);
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const float f = fast_exp2(s_top[k] - all.top);
        all.sum += f * s_sum[k];
#pragma unroll
        for (int e = 0; e < E; ++e) all.v[e] += weigh(s_v[k][e * 64 + lane], f);
      }
      all.template store<T>(p, group, u, r);
    }
  }
}

// Workspace layout and size (0 where every unit has a workgroup to itself).
size_t partials(void* ws, int D, int shares, Partials& r) {
  unsigned char* b = static_cast<unsigned char*>(ws);
  size_t n = 0;
  auto take = [&](size_t bytes) {
    unsigned char* x = b ? b + n : nullptr;
    n += (bytes + 255) / 256 * 256;
    return x;
  };
  r.unit = reinterpret_cast<DividedUnit*>(take(sizeof(DividedUnit) * shares));
  r.ml = reinterpret_cast<float2*>(take(sizeof(float2) * 64 * shares));
  r.o = reinterpret_cast<float*>(take(sizeof(float) * 64 * shares * D));
  return n;
}

// Divided calls: one wave a workgroup, up to 1024 of them: 32 contexts up to 54 k, 32/8 heads of 128: 181 us, with two waves and
// 512 200, with four and 256 212. Their LDS lets four run on a CU at once, but of wide fp32 heads fewer (96: three, 128: two, by
// careful_rows' tiles): the last of those shares start as others end. Undivided units have four
// waves, of wide fp32 heads two.
constexpr int most_shares(int row_bytes) { return row_bytes <= 64 ? 2048 : 1024; }

// Of few blocks the shares are fewer: with a block's time t and a part's time in the join c, s shares of B blocks, of which the
// largest unit has `most`, take t B / s + c s most / B, least at s = sqrt(t / c) B / sqrt(most). The root is 5 for bf16 and 12
// for fp32, by measurement (fp32, one context of 3483 keys: 18.5 us with 8, 15.7 with 12 or 16; bf16, six contexts up to
// 48 k, 4/1 x 32: 22.0 with 5, 23.1 with 7.5, 26.2 with 10).
int shares_of(long long blocks, long long most, long long units, int elem, int D) {
  const double s = (elem == 2 ? 5.0 : 12.0) * blocks / std::sqrt((double)most);
  return (int)std::min<long long>({std::max((long long)std::min(s, 1e9), units), blocks, most_shares(D * elem)});
}

// Rows of a unit, in the mean.
int rows_of_unit(long long rows, int n) { return (int)std::min<long long>(32, (rows + n - 1) / n); }

template <typename T, int D> void launch_narrow(const PackedAttnParams& p, const PackedPlan& plan, hipStream_t s) {
  constexpr int R = D * sizeof(T) <= 128 ? 4 : 2;
  const long long group = p.heads / p.kv_heads, rows = p.T * group;
  Partials part;
  if (plan.most) {
    const int shares = plan.shares;
    partials(p.ws, D, plan.most, part);
    hipLaunchKernelGGL((packed_narrow_kernel<T, D, 1, R, true>), dim3(shares), dim3(64), 0, s, p, (int)group, shares, part);
    DN_HIP(hipGetLastError());
    if (plan.join == kJoinRows) {
      hipLaunchKernelGGL((join_rows_kernel<T, D>), dim3((shares + 3) / 4, plan.split), dim3(256), 0, s, p, (int)group, shares, part);
    } else {
      hipLaunchKernelGGL((join_kernel<T, D>), dim3(shares, rows_of_unit(rows, p.seqs.n)), dim3(64 * kJoin), 0, s, p, (int)group, part);
    }
  } else {
    constexpr int NW = D * sizeof(T) > 256 ? 2 : 4;
    const long long slots = rows / 32 + p.seqs.n;
    DN_CHECK(slots * (64 * NW) < (1ll << 32), "dn_op_attention_packed: too many rows for one launch");
    hipLaunchKernelGGL((packed_narrow_kernel<T, D, NW, R, false>), dim3((unsigned)slots, p.kv_heads), dim3(64 * NW), 0, s, p, (int)group, 0, part);
  }
  DN_HIP(hipGetLastError());
}

template <int D> void launch_f32(const PackedAttnParams& p, hipStream_t s) {
  const int group = p.heads / p.kv_heads;
  const long long slots = p.T * group / 128 + p.seqs.n;
  DN_CHECK(slots * 256 < (1ll << 32), "dn_op_attention_packed: too many rows for one launch");
  hipLaunchKernelGGL((packed_f32_kernel<D>), dim3((unsigned)slots, p.kv_heads), dim3(256), 0, s, p, group);
  DN_HIP(hipGetLastError());
}

}  // namespace

bool attention_packed_dim(int D) { return D == 32 || D == 64 || D == 96 || D == 128; }

// A call is run in one way, by the mean of its sequences. Where they are unlike, the fewer ones pay: a prompt of 2048 and four tokens
// behind 64 k keys, 32/8 x 128, take 1085 us as tiles, whose keys' bytes take 218.
// Measured, us (heads/kv_heads x head dim):
//  - few rows a sequence: narrow. Up to 256 keys a unit is one workgroup's (77 keys, 20/20 x 64: 6.1); longer ones are divided.
//  - too few tiles to fill the CUs and long keys: narrow, divided. A tile's time goes with the keys (0.017 us each of 128
//    wide heads), a divided call's with keys and tiles behind about 20 us, so the most tiles that are divided fall from 112
//    as the keys get fewer (16/2 x 128, 128 tokens behind 16 k keys: 71, tiles 273; 32/8 x 128, 4 x 64 behind 8 k: 125, 143;
//    16/4 x 128, 8 x 32 behind 2 k: 33.6, 41.4; but 8/8 x 64, 4 x 50 behind 700: 47, tiles 12.8; 2 x 300 behind 700: 27, 14.4).
//    Many units that read the same keys gain less: 64 (12/3 x 128, 662 of 2253: 57.6, tiles 44.6; 1/1, 3000: 36.2, 56.4).
//  - fp32, bound by the matrix cores either way: narrow while its smaller units fill more CUs (10/2 x 64, 7 chunks behind up
//    to 825 keys: 24.7, tiles 64.8; 12/12 x 64, 16 x 77 tokens: 21.0, 26.0; 10/10 x 64, 2 x 1024 tokens: 87, tiles 79).
//    Divided past 256 keys of wide heads, whose units have two waves by their LDS (8/2 x 128, 4 x 20 behind 500: 19.5, else
//    44.7), and past 1024 of others, with four (16/4 x 64, 8 x 10 behind 900: 25.8, else 29.0; 8/8 x 64, 500 of 1000: 22.4, 17.8).
//  - tiles: 8 waves of 32 rows where there are tiles for every CU and the border is small beside them (20/20 x 128, two
//    images of 4173 tokens: 357, 4 waves 402; 8 x 512 tokens: 40.0, 36.3); 2 waves for short prompts (20/20 x 64,
//    64 of 49 tokens in the mean: 18.1, 4 waves 20.6, 8 waves 39.2); else 4 (64 wide: 2 x 10/10, 4096 tokens: 120, 8 waves 141).
PackedPlan attention_packed_plan(int elem, int D, long long T, int heads, int kv_heads, int n, int max_kv, long long kv_rows) {
  const long long group = heads / kv_heads, rows = T * group, units = (rows / 32 + n) * kv_heads;
  auto tiles = [&](int bm) { return (rows / bm + n) * kv_heads; };
  const bool few = rows <= 32ll * n, some = rows < 96ll * n;
  PackedPlan r;
  if (!(few || (elem == 4 ? some || tiles(128) < 128 : tiles(128) <= (rows < 1024ll * n ? 112 : 64) - 100000 / max_kv))) {
    r.waves = elem == 4 ? 4 : some ? 2 : D == 128 && rows >= 1024ll * n && tiles(256) >= 256 ? 8 : D == 96 ? 6 : 4;
    return r;
  }
  if (max_kv <= (few || elem == 2 || D > 64 ? 256 : 1024)) return r;
  r.most = (int)std::min<long long>(most_shares(D * elem), units * ((max_kv + 31ll) / 32));
  // the tensors' rows bound the blocks, too
  const long long blocks = (kv_rows / 32 + n) * kv_heads * ((rows + 32ll * n - 1) / (32ll * n));
  const long long longest = std::min(blocks, (max_kv + 31ll) / 32);
  r.shares = std::min(r.most, shares_of(blocks, longest, units, elem, D));
  // rows' joining: up to about 32 parts of the largest unit, and not so few rows that every one can have a workgroup (16/2 x
  // 128, 128 tokens behind 16 k keys: 71 us, with a workgroup per row 128; 13 single tokens, 1/1 x 96: 14.8 and 10.4). The rows
  // of few units go over several workgroups, a row or so a wave (the former: 98 with one)
  const long long per = rows_of_unit(rows, n);
  r.join = r.shares * per > 1024 && r.shares * longest <= 32 * blocks ? kJoinRows : kJoinUnits;
  if (r.join == kJoinRows) r.split = (int)std::max<long long>(1, std::min(per / 4, 1024 / units));
  return r;
}

namespace {

template <typename T, int D> void run(const PackedAttnParams& p, hipStream_t s) {
  const PackedPlan r = attention_packed_plan(sizeof(T), D, p.T, p.heads, p.kv_heads, p.seqs.n, p.max_kv, p.kv_rows);
  if (!r.waves) return launch_narrow<T, D>(p, r, s);
  if constexpr (sizeof(T) == 4) {
    launch_f32<D>(p, s);
  } else if constexpr (D == 128) {
    r.waves == 8 ? launch_pipe<D, 64, 8, 4, 2>(p, s) : r.waves == 4 ? launch_pipe<D, 32, 4, 5, 2>(p, s) : launch_pipe<D, 32, 2, 5, 2>(p, s);
  } else if constexpr (D == 96) {  // (six waves: whole loads)
    r.waves == 6 ? launch_pipe<D, 32, 6, 5, 3>(p, s) : launch_pipe<D, 32, 2, 5, 2>(p, s);
  } else if constexpr (D == 64) {
    r.waves == 4 ? launch_pipe<D, 32, 4, 5, 3>(p, s) : launch_pipe<D, 32, 2, 5, 2>(p, s);
  } else {
    r.waves == 4 ? launch_pipe<D, 64, 4, 4, 3>(p, s) : launch_pipe<D, 64, 2, 4, 3>(p, s);
  }
}

}  // namespace

size_t attention_packed_bytes(int elem, long long T, int heads, int kv_heads, int D, int n, int max_kv) {
  const PackedPlan r = attention_packed_plan(elem, D, T, heads, kv_heads, n, max_kv, 0);  // (of the most shares)
  Partials part;
  return r.most ? partials(nullptr, D, r.most, part) : 0;
}

template <typename T> void attention_packed(const PackedAttnParams& p, int D, hipStream_t s) {
  switch (D) {
    case 32: return run<T, 32>(p, s);
    case 64: return run<T, 64>(p, s);
    case 96: return run<T, 96>(p, s);
    default: return run<T, 128>(p, s);
  }
}

template void attention_packed<float>(const PackedAttnParams&, int, hipStream_t);
template void attention_packed<bf16>(const PackedAttnParams&, int, hipStream_t);

}  // namespace dn
