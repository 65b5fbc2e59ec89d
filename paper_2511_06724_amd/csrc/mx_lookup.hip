// Top-1 cosine search over a prompt-embedding table in microscaled rows (mx.h; gfx950).
//
// score(q, row) = q . c / |c| with c the values the row's codes stand for; the cosine divides by |q| at
// the end. A positive factor of a row cancels, so block scales are taken relative to the row's largest:
// no sum over- or underflows for any scales. A zero row, or one with a NaN block, never wins; ties go to
// the lowest row at every stage.
//
// Rows of 8 .. 1024 values (mx_scan_mfma_kernel): codes converted to fp16 (exact) against up to 64 queries (32 past
// 768 values) held in registers, on the matrix cores; the table is read once per pass, 17/32 (33/32) bytes a value.
// Bound by that for few queries: 100000 x 768 E2M1 rows (41 MB) 10.8 us for one query (one pass at 5.1 TB/s: 8.0),
// 11.1 for 16, a million rows 66.0 (79.7; from the cache between memory and L2 in part), E4M3 rows (79 MB) 16.9
// (15.5), and 4 to 5 for the reduction. For 64 queries 19.0 (E4M3 24.1): a third of it the queries' way into the
// registers of every CU (98 KB each), the rest products and conversions (16 cycles per product, 8 per conversion of
// two values).
// Other rows (mx_scan_kernel): two queries per pass (one past 8192 values), packed dot products in fp32; 100000 x
// 1280 E2M1 rows (68 MB) 24 to 26 us a pass.
#include <algorithm>
#include <type_traits>

#include "mx.h"

namespace dn {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Cand {
  float s;
  int pad;
  long long i;
};

constexpr int kScanBlocks = 1024;   // workgroups of a scan at most
constexpr int kScanQ = 2;           // queries per pass of the vector scan at most
constexpr int kMfmaQ = 64;          // and of the matrix-core scan
constexpr int kMfmaMinDim = 8, kMfmaMaxDim = 1024;  // the queries are held in registers
constexpr int kCus = 256;
template <int FMT, int H, int G> constexpr int kWaves = G == 1 && (FMT == kMx4 || H < 8) ? 2 : 1;  // per SIMD, as many as registers allow

__device__ __forceinline__ bool better(float s, long long i, float bs, long long bi) {
  return s > bs || (s == bs && i < bi);
}

// Eight codes of a block -> fp16 values times the scale `sc` (as the conversions take it).
template <int FMT> struct Codes;
template <> struct Codes<kMx4> {
  static constexpr int kWords = 4;  // 32-bit words of a block
  // values 8 U + 2 P, + 1
  template <int U, int P> __device__ static __forceinline__ h2 pair(const unsigned* w, float sc) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[U], sc, P);
  }
};
template <> struct Codes<kMx8> {
  static constexpr int kWords = 8;
  template <int U, int P> __device__ static __forceinline__ h2 pair(const unsigned* w, float sc) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * U + P / 2], sc, P % 2 == 1);
  }
};
template <int FMT, int U> __device__ __forceinline__ f16x8 eight(const unsigned* w, float sc) {
  const h2 a = Codes<FMT>::template pair<U, 0>(w, sc), b = Codes<FMT>::template pair<U, 1>(w, sc);
  const h2 c = Codes<FMT>::template pair<U, 2>(w, sc), d = Codes<FMT>::template pair<U, 3>(w, sc);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// f(integral constant) for I .. E - 1
template <int I, int E, typename F> __device__ __forceinline__ void each(F&& f) {
  if constexpr (I < E) {
    f(std::integral_constant<int, I>());
    each<I + 1, E>(f);
  }
}

__device__ __forceinline__ float dot8(const f16x8& a, const f16x8& b, float acc) {
#pragma unroll
  for (int e = 0; e < 8; e += 2)
    acc = __builtin_amdgcn_fdot2(h2{a[e], a[e + 1]}, h2{b[e], b[e + 1]}, acc, false);
  return acc;
}

template <int FMT> __device__ __forceinline__ void load_block(const unsigned char* codes, long long block, unsigned* w) {
  constexpr int W = Codes<FMT>::kWords;
#pragma unroll
  for (int e = 0; e < W; e += 4) {
    const uint4 v = ld16(codes + block * (4 * W) + 4 * e);
    w[e] = v.x, w[e + 1] = v.y, w[e + 2] = v.z, w[e + 3] = v.w;
  }
}

// Values [c, c + 8) of a query, zero past dim >= 8. Without a branch, so that many such loads can be in flight:
// the last eight values that there are, which are then moved down.
struct Query8 {
  uint4 v;
  int shift;
};
__device__ __forceinline__ Query8 query_load(const _Float16* q, int c, int dim) {
  struct __attribute__((packed, aligned(2))) Bytes {
    unsigned w[4];
  };
  const int o = min(c, dim - 8);
  const Bytes b = *reinterpret_cast<const Bytes*>(q + o);
  return Query8{make_uint4(b.w[0], b.w[1], b.w[2], b.w[3]), c - o};
}
__device__ __forceinline__ f16x8 query_value(const Query8& r) {
  unsigned w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
  const bool s4 = r.shift & 4, s2 = r.shift & 2, s1 = r.shift & 1, none = r.shift >= 8;
  w[0] = s4 ? w[2] : w[0], w[1] = s4 ? w[3] : w[1], w[2] = s4 ? 0u : w[2], w[3] = s4 ? 0u : w[3];
  w[0] = s2 ? w[1] : w[0], w[1] = s2 ? w[2] : w[1], w[2] = s2 ? w[3] : w[2], w[3] = s2 ? 0u : w[3];
  w[0] = s1 ? __builtin_amdgcn_alignbit(w[1], w[0], 16) : w[0];
  w[1] = s1 ? __builtin_amdgcn_alignbit(w[2], w[1], 16) : w[1];
  w[2] = s1 ? __builtin_amdgcn_alignbit(w[3], w[2], 16) : w[2];
  w[3] = s1 ? w[3] >> 16 : w[3];
  const uint4 v = none ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(w[0], w[1], w[2], w[3]);
  return __builtin_bit_cast(f16x8, v);
}

// 2^(s - smax) as a number, 0 where that underflows.
__device__ __forceinline__ float rel_scale(unsigned s, unsigned smax) {
  return __uint_as_float((unsigned)max((int)s - (int)smax + 127, 0) << 23);
}

__device__ __forceinline__ float row_score(float dot, float cc, bool ok) { return ok && cc > 0.f ? dot * rsqrtf(cc) : -INFINITY; }

template <int CTRL> __device__ __forceinline__ float dpp_fadd(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// c + the product of 16 rows' E2M1 blocks, scale bytes s, with themselves (16x16x128; a lane's block is its row's
// l / 16-th).
__device__ __forceinline__ f32x4 norm4(const unsigned* w, unsigned s, const f32x4& c) {
  typedef int v8i __attribute__((ext_vector_type(8)));
  const v8i a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, a, c, 4, 4, 0, (int)s, 0, (int)s);
}

// Over the four lanes l % 16 of a wave, in each of them.
__device__ __forceinline__ unsigned quad_umax(unsigned v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max(b[0], b[1]);
}
__device__ __forceinline__ float quad_sum(float x) {
  unsigned v = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// The best pair, the lowest r (unsigned) of equal scores.
__device__ __forceinline__ void quad_best(float& s, int& r) {
  const unsigned v = __float_as_uint(s), u = r;
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false), i = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const float a0 = __uint_as_float(a[0]), a1 = __uint_as_float(a[1]);
  const bool p = a1 > a0 || (a1 == a0 && i[1] < i[0]);
  const unsigned v2 = p ? a[1] : a[0], u2 = p ? i[1] : i[0];
  const auto b = __builtin_amdgcn_permlane16_swap(v2, v2, false, false), j = __builtin_amdgcn_permlane16_swap(u2, u2, false, false);
  const float b0 = __uint_as_float(b[0]), b1 = __uint_as_float(b[1]);
  const bool o = b1 > b0 || (b1 == b0 && j[1] < j[0]);
  s = o ? b1 : b0;
  r = o ? j[1] : j[0];
}
// Sum over eight lanes, in each of them.
__device__ __forceinline__ float oct_sum(float v) { return dpp_fadd<0x141>(dpp_fadd<0x4e>(dpp_fadd<0xb1>(v))); }

// Eight lanes a row, R rows at once; the queries lie in LDS as [Q][blocks 32] fp16.
template <int FMT, int Q>
__global__ __launch_bounds__(256) void mx_scan_kernel(const _Float16* q, const unsigned char* codes, const unsigned char* scales,
                                                      long long n, int dim, int blocks, Cand* part) {
  constexpr int R = 2;
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ Cand red[4][Q];
  const int t = threadIdx.x, lane = t & 63, li = lane & 7;
  for (int e = t; e < Q * blocks * 32; e += 256) {
    const int k = e / (blocks * 32), c = e - k * blocks * 32;
    reinterpret_cast<_Float16*>(lds)[e] = c < dim ? q[(long long)k * dim + c] : static_cast<_Float16>(0.f);
  }
  __syncthreads();
  const f16x8* ql = reinterpret_cast<const f16x8*>(lds);
  float bs[Q];
  long long bi[Q];
#pragma unroll
  for (int k = 0; k < Q; ++k) bs[k] = -INFINITY, bi[k] = n;
  const long long step = (long long)gridDim.x * 32 * R;
  for (long long r0 = (long long)blockIdx.x * 32 * R + (t >> 3) * R; r0 < n; r0 += step) {
    for (int r = 0; r < R; ++r) {
      const long long row = min(r0 + r, n - 1);
      unsigned smax = 0;
      for (int b = li; b < blocks; b += 8) smax = max(smax, (unsigned)scales[row * blocks + b]);
      smax = oct_umax(smax);
      float d[Q], cc = 0.f;
#pragma unroll
      for (int k = 0; k < Q; ++k) d[k] = 0.f;
      for (int b = li; b < blocks; b += 8) {
        unsigned w[Codes<FMT>::kWords];
        load_block<FMT>(codes, row * blocks + b, w);
        const float sc = rel_scale(scales[row * blocks + b], smax);
        float c1 = 0.f, d1[Q];
#pragma unroll
        for (int k = 0; k < Q; ++k) d1[k] = 0.f;
        each<0, 4>([&](auto u) {
          const f16x8 v = eight<FMT, u>(w, 1.f);
          c1 = dot8(v, v, c1);
#pragma unroll
          for (int k = 0; k < Q; ++k) d1[k] = dot8(ql[(k * blocks + b) * 4 + u], v, d1[k]);
        });
        cc += c1 * sc * sc;
#pragma unroll
        for (int k = 0; k < Q; ++k) d[k] += d1[k] * sc;
      }
      cc = oct_sum(cc);
#pragma unroll
      for (int k = 0; k < Q; ++k) {
        const float sc = row_score(oct_sum(d[k]), cc, smax < 255u && r0 + r < n);
        if (better(sc, r0 + r, bs[k], bi[k])) {
          bs[k] = sc;
          bi[k] = r0 + r;
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < Q; ++k) {
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) {
      const float s2 = __shfl_xor(bs[k], o, 64);
      const long long i2 = __shfl_xor(bi[k], o, 64);
      if (better(s2, i2, bs[k], bi[k])) {
        bs[k] = s2;
        bi[k] = i2;
      }
    }
    if (lane == 0) red[t >> 6][k] = Cand{bs[k], 0, bi[k]};
  }
  __syncthreads();
  if (t < Q) {
    Cand b = red[0][t];
    for (int w = 1; w < 4; ++w)
      if (better(red[w][t].s, red[w][t].i, b.s, b.i)) b = red[w][t];
    part[(long long)blockIdx.x * Q + t] = b;
  }
}

// Sixteen scale bytes from any address (the buffer has 16 bytes to spare).
struct __attribute__((packed, aligned(1))) Bytes16 {
  unsigned w[4];
};

// 16-row tiles against 16 G queries on the matrix cores (16x16x32 f16). Lane: row (query) l % 16 and, of block
// quad j, block 4 j + l / 16: the k order of a product is free, so a lane takes whole blocks and both operands
// agree on it; four lanes then load adjacent blocks of a row, 64 (128) contiguous bytes. A wave holds its
// queries' H quads in registers (they reach them through LDS, once a workgroup) and walks over tiles; the
// codes of the next tile replace a block's as soon as it is converted.
template <int FMT, int H, int G>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(kWaves<FMT, H, G>, kWaves<FMT, H, G>))) void mx_scan_mfma_kernel(
    const _Float16* q, int nq, const unsigned char* codes, const unsigned char* scales, long long n, int dim, int blocks, Cand* part) {
  // scale of the row's largest block: its values stay below 2^16 (fp16) and those of blocks 2^-22 times as
  // large are still exact
  constexpr int kTop = FMT == kMx4 ? 10 : 7;
  constexpr int W = Codes<FMT>::kWords;
  __shared__ __align__(16) f16x8 ql[G * H * 4 * 64];
  __shared__ __align__(16) float inv[4][32];
  __shared__ Cand red[4][16 * G];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int r16 = lane & 15, g = lane >> 4;

  const long long tiles = (n + 15) / 16, stride = (long long)gridDim.x * 4;
  long long tile = (long long)blockIdx.x * 4 + wave;
  auto row_of = [&](long long tl) { return min(min(tl, tiles - 1) * 16 + r16, n - 1); };
  unsigned w[H][W];
  Bytes16 sb[(H + 3) / 4];
  auto load = [&](long long row, int j) { load_block<FMT>(codes, row * blocks + min(4 * j + g, blocks - 1), w[j]); };
  auto load_scales = [&](long long row) {
#pragma unroll
    for (int e = 0; e < (H + 3) / 4; ++e) sb[e] = *reinterpret_cast<const Bytes16*>(scales + row * blocks + 16 * e);
  };

  // Fragment f = (c H + j) 4 + u, lane l: values 8 u .. of block 4 j + l / 16 of query 16 c + l % 16, in LDS at
  // position l ^ 4 u, so that writes of four fragments side by side touch all banks. Load c H + j of a wave
  // takes 64 bytes, block 4 j + wave, of 16 queries, four adjacent lanes a query.
  {
    const int u = lane & 3, k0 = lane >> 2;
    Query8 x[G * H];
#pragma unroll
    for (int i = 0; i < G * H; ++i) {
      const int b = 4 * (i % H) + wave, k = 16 * (i / H) + k0;
      x[i] = query_load(q + (long long)min(k, nq - 1) * dim, b * 32 + 8 * u, dim);
      if (k >= nq) x[i].shift = 8;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < H; ++j) load(row_of(tile), j);
    load_scales(row_of(tile));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < G * H; ++i) {
      const uint4 z = make_uint4(0u, 0u, 0u, 0u);
      ql[(i * 4 + u) * 64 + ((wave * 16 + k0) ^ (4 * u))] =
          dim % 8 == 0 ? __builtin_bit_cast(f16x8, x[i].shift >= 8 ? z : x[i].v) : query_value(x[i]);
    }
  }
  __syncthreads();
  f16x8 qf[G][H][4];
#pragma unroll
  for (int c = 0; c < G; ++c)
#pragma unroll
    for (int j = 0; j < H; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        // as whole operands, accumulation registers first: left to itself the compiler gathers them from
        // single registers before each use
        qf[c][j][u] = ql[((c * H + j) * 4 + u) * 64 + (lane ^ (4 * u))];
        if ((c * H + j) * 4 + u < 52)
          asm volatile("" : "+a"(qf[c][j][u]));
        else
          asm volatile("" : "+v"(qf[c][j][u]));
      }

  float best[G];
  int best_r[G];  // row of the tile, with the wave's tile count above; -1: none
#pragma unroll
  for (int c = 0; c < G; ++c) best[c] = -INFINITY, best_r[c] = -1;
  const long long tile0 = tile;
  for (int count = 0; tile < tiles; tile += stride, count += 16) {
    const long long next = row_of(tile + stride);
    // scales of this tile's blocks, relative to the row's largest
    unsigned s[H], smax = 0;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      s[j] = (sb[j / 4].w[j % 4] >> (8 * g)) & 255u;
      if (4 * j + g < blocks) smax = max(smax, s[j]);
    }
    smax = quad_umax(smax);
    load_scales(next);
    f32x4 acc[G], nrm = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < G; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float cc = 0.f;
    float sc[H];
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int e = (int)s[j] - (int)smax + 127;  // 2^-127 and what no fp16 value is: 0
      s[j] = 4 * j + g < blocks && e > 0 ? (unsigned)e : 0u;
      sc[j] = s[j] > (unsigned)kTop ? __uint_as_float((s[j] + kTop) << 23) : 0.f;
    }
    // each conversion (eight cycles) between two products, for the values after these
    f16x8 v = eight<FMT, 0>(w[0], sc[0]);
    each<0, 4 * H>([&](auto f) {
      constexpr int j = f / 4, u = f % 4, jn = (f + 1) / 4, un = (f + 1) % 4;
      h2 x[4];
      each<0, G>([&](auto c) {
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, qf[c][j][u], acc[c], 0, 0, 0);
        if constexpr (f + 1 < 4 * H)
          each<c * 4 / G, (c + 1) * 4 / G>([&](auto e) { x[e] = Codes<FMT>::template pair<un, e>(w[jn], sc[jn]); });
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (FMT == kMx8) cc = dot8(v, v, cc);
      if constexpr (FMT == kMx4 && u == 0) nrm = norm4(w[j], s[j], nrm);
      if constexpr (u == 3) {
        load(next, j);  // not later: it has this tile's time to arrive
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (f + 1 < 4 * H) v = f16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
    });
    // |row|^2 (E2M1: the diagonal of the product of the rows with themselves, lane row r16 and column r16 / 4 == g)
    float c2;
    if constexpr (FMT == kMx4)
      c2 = r16 & 2 ? (r16 & 1 ? nrm[3] : nrm[2]) : (r16 & 1 ? nrm[1] : nrm[0]);
    else
      c2 = quad_sum(cc);
    const bool ok = c2 > 0.f && smax < 255u && tile * 16 + r16 < n;
    // NaN scores never win; without a branch, into which the compiler would move the products for c2
    inv[wave][FMT == kMx8 || (r16 >> 2) == g ? r16 : 16 + r16] = ok ? rsqrtf(c2) : NAN;
    const f32x4 iv = *reinterpret_cast<const f32x4*>(&inv[wave][4 * g]);
    // lane: query r16 of each group, rows 4 g ..
#pragma unroll
    for (int c = 0; c < G; ++c) {
      acc[c] *= iv;
      const float ts = fmaxf(fmaxf(acc[c][0], acc[c][1]), fmaxf(acc[c][2], acc[c][3]));
      const int r = acc[c][0] == ts ? 0 : acc[c][1] == ts ? 1 : acc[c][2] == ts ? 2 : 3;
      const bool up = ts > best[c];  // a wave's tiles ascend
      best[c] = up ? ts : best[c];
      best_r[c] = up ? count + 4 * g + r : best_r[c];
    }
  }
  if constexpr (FMT == kMx4) {
#pragma unroll
    for (int c = 0; c < G; ++c) best[c] *= 1.f / (1 << kTop);
  }
#pragma unroll
  for (int c = 0; c < G; ++c) {
    // a wave's rows ascend with best_r, -1 comes last
    quad_best(best[c], best_r[c]);
    const long long best_i = best_r[c] < 0 ? n : (tile0 + (best_r[c] >> 4) * stride) * 16 + (best_r[c] & 15);
    if (g == 0) red[wave][16 * c + r16] = Cand{best[c], 0, best_i};
  }
  __syncthreads();
  if (t < 16 * G) {
    Cand b = red[0][t];
    for (int k = 1; k < 4; ++k)
      if (better(red[k][t].s, red[k][t].i, b.s, b.i)) b = red[k][t];
    part[(long long)blockIdx.x * (16 * G) + t] = b;
  }
}

// One workgroup per query: the winners of its column (pitch entries apart), and |q|^2.
__global__ __launch_bounds__(256) void mx_reduce_kernel(const Cand* part, int nb, int pitch, const _Float16* q, int dim,
                                                        long long n, long long* idx, float* score, KTable kt, int* kout) {
  __shared__ float ws_s[4], ws_q[4];
  __shared__ long long ws_i[4];
  const int j = blockIdx.x, t = threadIdx.x, lane = t & 63, w = t >> 6;
  float bs = -INFINITY, qq = 0.f;
  long long bi = n;
  // few iterations of many loads: in a chain of dependent ones the latency of each would be most of the kernel
  const _Float16* const qj = q + (long long)j * dim;
  for (int k = t; k < nb; k += 512) {
    const Cand c = part[(long long)k * pitch + j], d = part[(long long)min(k + 256, nb - 1) * pitch + j];
    if (better(c.s, c.i, bs, bi)) {
      bs = c.s;
      bi = c.i;
    }
    if (better(d.s, d.i, bs, bi)) {
      bs = d.s;
      bi = d.i;
    }
  }
  if (dim >= 8) {
    for (int e = 8 * t; e < dim; e += 2048) {
      const f16x8 x = query_value(query_load(qj, e, dim));
#pragma unroll
      for (int i = 0; i < 8; ++i) qq = fmaf(static_cast<float>(x[i]), static_cast<float>(x[i]), qq);
    }
  } else if (t < dim) {
    qq = static_cast<float>(qj[t]) * static_cast<float>(qj[t]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float s2 = __shfl_xor(bs, o, 64);
    const long long i2 = __shfl_xor(bi, o, 64);
    if (better(s2, i2, bs, bi)) {
      bs = s2;
      bi = i2;
    }
    qq += __shfl_xor(qq, o, 64);
  }
  if (lane == 0) {
    ws_s[w] = bs;
    ws_i[w] = bi;
    ws_q[w] = qq;
  }
  __syncthreads();
  if (t == 0) {
    float qn = ws_q[0];
    for (int k = 1; k < 4; ++k) {
      if (better(ws_s[k], ws_i[k], bs, bi)) {
        bs = ws_s[k];
        bi = ws_i[k];
      }
      qn += ws_q[k];
    }
    // a zero query, or one that is not finite, has no cosine; nor has a table of such rows
    const bool ok = qn > 0.f && qn < INFINITY && bs > -INFINITY;
    const float sc = ok ? bs * rsqrtf(qn) : 0.f;
    idx[j] = ok ? bi : -1;
    if (score) score[j] = sc;
    if (kout) {
      int l = 0;
      for (int i = 0; i < kt.n; ++i)
        if (sc >= kt.thr[i]) l = i + 1;
      kout[j] = ok ? kt.level[l] : 0;
    }
  }
}

struct Scan {
  const unsigned char* codes;
  const unsigned char* scales;
  long long n;
  int dim, blocks;
  Cand* part;
  hipStream_t s;
};

template <int FMT, int Q> int launch_scan(const Scan& a, const _Float16* q) {
  const int nb = static_cast<int>(std::min<long long>((a.n + 63) / 64, kScanBlocks));
  hipLaunchKernelGGL((mx_scan_kernel<FMT, Q>), dim3(nb), dim3(256), (size_t)Q * a.blocks * 64, a.s, q, a.codes, a.scales, a.n, a.dim,
                     a.blocks, a.part);
  return nb;
}
template <int FMT, int H, int G> int launch_mfma(const Scan& a, const _Float16* q, int nq) {
  const int nb = static_cast<int>(std::min<long long>((a.n + 63) / 64, kCus * kWaves<FMT, H, G>));
  hipLaunchKernelGGL((mx_scan_mfma_kernel<FMT, H, G>), dim3(nb), dim3(256), 0, a.s, q, nq, a.codes, a.scales, a.n, a.dim, a.blocks, a.part);
  return nb;
}
template <int FMT, int G> int mfma_blocks(const Scan& a, const _Float16* q, int nq) {
  if (a.blocks <= 8) return launch_mfma<FMT, 2, G>(a, q, nq);
  if (a.blocks <= 16) return launch_mfma<FMT, 4, G>(a, q, nq);
  if (G == 4 || a.blocks <= 24) return launch_mfma<FMT, 6, G>(a, q, nq);
  if constexpr (G < 4)
    return launch_mfma<FMT, 8, G>(a, q, nq);
  else
    throw Error(-1, "mx_lookup: 64 queries of 768 values at most");
}

template <int FMT>
void lookup_fmt(const Scan& a, const _Float16* q, int nq, long long* idx, float* score, const KTable& kt, int* kout) {
  while (nq > 0) {
    int m, nb, pitch;
    if (a.dim >= kMfmaMinDim && a.dim <= kMfmaMaxDim) {
      // 64 queries of up to 768 values fit the registers, 32 of 1024
      m = std::min(nq, a.blocks <= 24 ? kMfmaQ : kMfmaQ / 2);
      pitch = m <= 16 ? 16 : m <= 32 ? 32 : 64;
      nb = m <= 16 ? mfma_blocks<FMT, 1>(a, q, m) : m <= 32 ? mfma_blocks<FMT, 2>(a, q, m) : mfma_blocks<FMT, 4>(a, q, m);
    } else {
      // the queries lie in LDS, at most 32 KB of them
      m = pitch = nq >= 2 && a.blocks <= 256 ? 2 : 1;
      nb = m == 2 ? launch_scan<FMT, 2>(a, q) : launch_scan<FMT, 1>(a, q);
    }
    hipLaunchKernelGGL(mx_reduce_kernel, dim3(m), dim3(256), 0, a.s, a.part, nb, pitch, q, a.dim, a.n, idx, score, kt, kout);
    DN_HIP(hipGetLastError());
    q += (long long)m * a.dim;
    idx += m;
    if (score) score += m;
    if (kout) kout += m;
    nq -= m;
  }
}

}  // namespace

size_t mx_lookup_workspace() {
  return sizeof(Cand) * std::max((size_t)kScanBlocks * kScanQ, (size_t)kCus * kMfmaQ);
}

void mx_lookup(int fmt, const uint16_t* q, int nq, const void* table, long long n, int dim, void* ws, long long* idx_out,
               float* score_out, const KTable* kt, int* k_out, hipStream_t s) {
  DN_CHECK(dim >= 1 && dim <= kMxLookupMaxDim, "ac_mx_lookup: dim must be in [1, 16384]");
  Scan a;
  a.codes = static_cast<const unsigned char*>(table);
  a.scales = a.codes + mx_scale_offset(fmt, n, dim);
  a.n = n;
  a.dim = dim;
  a.blocks = static_cast<int>(mx_blocks(dim));
  a.part = static_cast<Cand*>(ws);
  a.s = s;
  const KTable tab = kt ? *kt : KTable();
  const _Float16* qh = reinterpret_cast<const _Float16*>(q);
  if (fmt == kMx4)
    lookup_fmt<kMx4>(a, qh, nq, idx_out, score_out, tab, kt ? k_out : nullptr);
  else
    lookup_fmt<kMx8>(a, qh, nq, idx_out, score_out, tab, kt ? k_out : nullptr);
}

}  // namespace dn
