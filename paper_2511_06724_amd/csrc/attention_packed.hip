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
// would be NaN. Key rows past the range are not read (the last one is, instead), and if the result of
// a workgroup with a masked tile has a non-finite value, it runs again and takes non-finite values
// out of masked tiles, adding them back where they are seen (one tile a work unit at most, plus the
// border of the range).
#include <algorithm>

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

// The unit of a slot, by a whole wave. False: the slot is not used.
template <int BM> __device__ __forceinline__ bool find_unit(const PackedAttnParams& p, int group, long long slot, Unit& u) {
  const int* qs = p.seqs.q_start;
  const int s = __builtin_amdgcn_readfirstlane(
      search_group<64>(p.seqs.n, slot, [&](int i) { return (long long)qs[i] * group / BM + i; }));
  if (s < 0) return false;
  const int a = qs[s], b = qs[s + 1];
  u.len_k = p.seqs.kv_len[s];
  u.k0 = p.seqs.kv_start[s];
  if (a < 0 || b <= a || b > p.T || u.len_k < 0 || u.k0 < 0 || u.k0 > p.kv_rows - u.len_k) return false;
  u.q0 = a;
  u.len_q = b - a;
  const long long rows = (long long)u.len_q * group, row0 = (slot - ((long long)a * group / BM + s)) * BM;
  if (row0 >= rows) return false;
  u.rows = (int)rows;
  u.row0 = (int)row0;
  return true;
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

// O^T += V^T P^T of one 64-key tile of which some keys are masked, when the values may hold infinities
// or NaN: the finite values by the product; the others are counted where they are seen.
template <typename T, int DB>
__device__ __forceinline__ void pv_careful(const T* vs, int ld, const f32x16* pr, const f32x16* seen, f32x16* o, int lane) {
  using MM = Mma<T>;
  using V = Pv<T>;
#pragma unroll 1
  for (int sign = 0; sign < 3; ++sign) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      f32x16 n;
#pragma unroll
      for (int r = 0; r < 16; ++r) n[r] = sign == 0 ? o[d][r] : 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int c = 0; c < V::STEPS; ++c) {
          typename MM::frag f = V::v(vs, ld, kb, c, d * 32, lane);
#pragma unroll
          for (int e = 0; e < V::N; ++e) {
            const float x = V::get(f, e);
            const bool finite = fabsf(x) <= -kLowest, other = sign == 1 ? x < 0 : x > 0;
            V::set(f, e, sign == 0 ? (finite ? x : 0.f) : (finite || other ? 0.f : 1.f));
          }
          n = MM::mma(f, V::p(sign == 0 ? pr[kb] : seen[kb], c), n);
        }
#pragma unroll
      for (int r = 0; r < 16; ++r)
        o[d][r] = sign == 0 ? n[r] : n[r] == 0.f ? o[d][r] : o[d][r] + (sign == 1 ? INFINITY : -INFINITY);
    }
  }
}

// Any head dim and type: key tiles go through registers into LDS, double-buffered; NW waves of 32 rows.
template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW) void packed_kernel(PackedAttnParams p, int group) {
  using MM = Mma<T>;
  using V = Pv<T>;
  constexpr int BM = 32 * NW;
  constexpr int NT = 64 * NW;
  constexpr int VEC = 16 / sizeof(T);
  constexpr int LD = D + VEC;       // LDS row of a key (elements)
  constexpr int NS = D / MM::KS;    // matrix steps over the head dim
  constexpr int DB = D / 32;
  constexpr int CH = D / VEC;       // 16-byte pieces per row
  constexpr int PER = (kKT * CH + NT - 1) / NT;
  constexpr int STAGE = 2 * kKT * LD;
  __shared__ __align__(16) T lds[2 * STAGE];

  Unit u;
  if (!find_unit<BM>(p, group, blockIdx.x, u)) return;
  const int kvh = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = u.row0 + wave * 32;  // first row of the wave
  const int row = min(first + (lane & 31), u.rows - 1);
  const int token = row / group, head = kvh * group + row - token * group;
  const int shift = u.len_k - u.len_q;
  auto limit = [&](int tok) { return p.causal ? max(0, tok + shift + 1) : u.len_k; };
  const int lim = limit(token);
  const int lim_min = limit(min(first, u.rows - 1) / group);                 // of the wave
  const int end = limit(min(u.row0 + BM - 1, u.rows - 1) / group);            // of the workgroup
  T* op = static_cast<T*>(p.o) + (u.q0 + token) * p.ldo + (long long)head * D;
  const bool store_row = first + (lane & 31) < u.rows;

  const T* qp = static_cast<const T*>(p.q) + (u.q0 + token) * p.ldq + (long long)head * D;
  typename MM::frag qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) qf[s] = MM::load(qp + s * MM::KS + half * MM::KPL);
  const T* kp = static_cast<const T*>(p.k) + u.k0 * p.ldk + (long long)kvh * D;
  const T* vp = static_cast<const T*>(p.v) + u.k0 * p.ldv + (long long)kvh * D;

  const int ntiles = (end + kKT - 1) / kKT;
  const bool any_masked = limit(u.row0 / group) < ntiles * kKT;  // a masked key in a tile (workgroup-uniform)
  f32x16 o[DB];
  float m_ref, l_run;
  uint4 rk[PER], rv[PER];
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int w = tid + i * NT;
      if (PER * NT != kKT * CH && w >= kKT * CH) break;
      const int r = w / CH, c = w - r * CH;
      const long long key = min(t * kKT + r, end - 1);
      rk[i] = ld16(kp + key * p.ldk + c * VEC);
      rv[i] = ld16(vp + key * p.ldv + c * VEC);
    }
  };
  auto store = [&](int buf) {
    T* ks = lds + buf * STAGE;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int w = tid + i * NT;
      if (PER * NT != kKT * CH && w >= kKT * CH) break;
      const int r = w / CH, c = w - r * CH;
      st16(ks + r * LD + c * VEC, rk[i]);
      st16(ks + kKT * LD + r * LD + c * VEC, rv[i]);
    }
  };

  for (bool careful = false;; careful = true) {
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    m_ref = kLowest;
    l_run = 0.f;
    if (ntiles > 0) {
      load(0);
      store(0);
      if (ntiles > 1) load(1);
    }
    __syncthreads();
    for (int t = 0; t < ntiles; ++t) {
      const int k0 = t * kKT;
      const T* ks = lds + (t & 1) * STAGE;
      const T* vs = ks + kKT * LD;
      f32x16 s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          s[kb] = MM::mma(MM::load(&ks[(kb * 32 + (lane & 31)) * LD + i * MM::KS + half * MM::KPL]), qf[i], s[kb]);
      const bool masked = k0 + kKT > lim_min;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] *= p.scale_log2;
      if (masked) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (k0 + kb * 32 + acc_row(r, lane) >= lim) s[kb][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      if (__any(mx > m_ref + kLazy)) {
        const float m_new = fmaxf(m_ref, mx);
        const float alpha = fast_exp2(m_ref - m_new);
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
        m_ref = m_new;
      }
      float rs = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = to_f32(from_f32<T>(fast_exp2(s[kb][r] - m_ref)));
          s[kb][r] = e;
          rs += e;
        }
      l_run += rs + __shfl_xor(rs, 32, 64);
      if (masked && careful) {
        f32x16 seen[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) seen[kb][r] = k0 + kb * 32 + acc_row(r, lane) < lim ? 1.f : 0.f;
        pv_careful<T, DB>(vs, LD, s, seen, o, lane);
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int c = 0; c < V::STEPS; ++c) {
            const typename MM::frag pf = V::p(s[kb], c);
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] = MM::mma(V::v(vs, LD, kb, c, d * 32, lane), pf, o[d]);
          }
      }
      if (t + 1 < ntiles) {
        store((t + 1) & 1);
        if (t + 2 < ntiles) load(t + 2);
      }
      __syncthreads();
    }
    if (careful || !any_masked) break;
    float bad = 0.f;  // NaN if a result is not finite
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) bad += o[d][r] * 0.f;
    if (!__syncthreads_or(bad != bad)) break;
  }

  if (store_row) {
    const float inv = l_run != 0.f ? 1.f / l_run : 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        T v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = from_f32<T>(o[d][4 * g + e] * inv);
        T* dst = op + d * 32 + 8 * g + 4 * half;
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, bf16x4{v[0], v[1], v[2], v[3]});
        else
          *reinterpret_cast<f32x4*>(dst) = f32x4{v[0], v[1], v[2], v[3]};
      }
  }
}

template <typename T, int D, int NW> void launch(const PackedAttnParams& p, hipStream_t s) {
  constexpr int BM = 32 * NW;
  const int group = p.heads / p.kv_heads;
  const long long slots = p.T * group / BM + p.seqs.n;
  DN_CHECK(slots * (64 * NW) < (1ll << 32), "dn_op_attention_packed: too many rows for one launch");
  hipLaunchKernelGGL((packed_kernel<T, D, NW>), dim3((unsigned)slots, p.kv_heads), dim3(64 * NW), 0, s, p, group);
  DN_HIP(hipGetLastError());
}

}  // namespace

bool attention_packed_dim(int D) { return D == 32 || D == 64 || D == 96 || D == 128; }

size_t attention_packed_bytes(int, long long, int, int, int, int, int) { return 0; }

template <typename T> void attention_packed(const PackedAttnParams& p, int D, hipStream_t s) {
  switch (D) {
    case 32: return launch<T, 32, 4>(p, s);
    case 64: return launch<T, 64, 4>(p, s);
    case 96: return launch<T, 96, 4>(p, s);
    default: return launch<T, 128, 4>(p, s);
  }
}

template void attention_packed<float>(const PackedAttnParams&, int, hipStream_t);
template void attention_packed<bf16>(const PackedAttnParams&, int, hipStream_t);

}  // namespace dn
