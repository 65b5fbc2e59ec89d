// Top-1 cosine search over a prompt-embedding table in microscaled rows (mx.h; gfx950).
//
// score(q, row) = q . c / |c| with c the values the row's codes stand for; the cosine divides by |q| at
// the end. A positive factor of a row cancels, so block scales are taken relative to the row's largest:
// no sum over- or underflows for any scales. A zero row, or one with a NaN block, never wins; ties go to
// the lowest row at every stage.
//
// Few queries (mx_scan_kernel): eight lanes a row, a lane's blocks 8 apart (128 contiguous bytes a row and
// load), codes converted to fp16 (exact) and multiplied with packed dot products in fp32.
// More (mx_scan_mfma_kernel): 32-row tiles against 32 queries held in registers on the matrix cores
// (32x32x16 f16). Both read the table once per pass, 17/32 (33/32) bytes a value.
#include <algorithm>

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
constexpr int kScanQ = 4;           // queries per pass of the vector scan
constexpr int kMfmaQ = 64;          // and of the matrix-core scan
constexpr int kMfmaBlocks = 256;    // one workgroup per CU
constexpr int kMfmaMaxDim = 1024;   // the queries are held in registers

__device__ __forceinline__ bool better(float s, long long i, float bs, long long bi) {
  return s > bs || (s == bs && i < bi);
}

// Eight codes of a block -> fp16 values times the scale `sc` (as the conversions take it).
template <int FMT> struct Codes;
template <> struct Codes<kMx4> {
  static constexpr int kWords = 4;  // 32-bit words of a block
  // word u / 2 holds values 8 u' ..: eight values from word u
  __device__ static __forceinline__ f16x8 eight(const unsigned* w, int u, float sc) {
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[u], sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[u], sc, 1);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[u], sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[u], sc, 3);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
};
template <> struct Codes<kMx8> {
  static constexpr int kWords = 8;
  __device__ static __forceinline__ f16x8 eight(const unsigned* w, int u, float sc) {
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * u], sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * u], sc, true);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * u + 1], sc, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * u + 1], sc, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
};

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

// Values [c, c + 8) of a query, zero past dim.
__device__ __forceinline__ f16x8 query8(const _Float16* q, int c, int dim, bool vec) {
  if (vec && c + 8 <= dim) return *reinterpret_cast<const f16x8*>(q + c);
  f16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < dim ? q[c + e] : static_cast<_Float16>(0.f);
  return v;
}

// 2^(s - smax) as a number, 0 where that underflows.
__device__ __forceinline__ float rel_scale(unsigned s, unsigned smax) {
  return __uint_as_float((unsigned)max((int)s - (int)smax + 127, 0) << 23);
}

__device__ __forceinline__ float row_score(float dot, float cc, bool ok) { return ok && cc > 0.f ? dot * rsqrtf(cc) : -INFINITY; }

template <int CTRL> __device__ __forceinline__ float dpp_fadd(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Sum over eight lanes, in each of them.
__device__ __forceinline__ float oct_sum(float v) { return dpp_fadd<0x141>(dpp_fadd<0x4e>(dpp_fadd<0xb1>(v))); }

// NB blocks a lane (a row has at most 8 NB), the Q queries in registers; NB = 0: any number of blocks,
// the queries in LDS as [Q][blocks 32] fp16.
template <int FMT, int NB, int Q>
__global__ __launch_bounds__(256) void mx_scan_kernel(const _Float16* q, const unsigned char* codes, const unsigned char* scales,
                                                      long long n, int dim, int blocks, bool qvec, Cand* part) {
  constexpr int R = 2;  // rows per lane group and step
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ Cand red[4][Q];
  const int t = threadIdx.x, lane = t & 63, li = lane & 7;
  f16x8 qv[NB > 0 ? Q : 1][NB > 0 ? NB : 1][4];
  if constexpr (NB > 0) {
#pragma unroll
    for (int k = 0; k < Q; ++k)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) qv[k][j][u] = query8(q + (long long)k * dim, (li + 8 * j) * 32 + 8 * u, dim, qvec);
  } else {
    f16x8* ql = reinterpret_cast<f16x8*>(lds);
    for (int e = t; e < Q * blocks * 4; e += 256) {
      const int k = e / (blocks * 4);
      ql[e] = query8(q + (long long)k * dim, (e - k * blocks * 4) * 8, dim, qvec);
    }
    __syncthreads();
  }
  float bs[Q];
  long long bi[Q];
#pragma unroll
  for (int k = 0; k < Q; ++k) bs[k] = -INFINITY, bi[k] = n;
  const long long step = (long long)gridDim.x * 32 * R;
  for (long long r0 = (long long)blockIdx.x * 32 * R + (t >> 3) * R; r0 < n; r0 += step) {
    float d[R][Q], cc[R];
    bool ok[R];
    if constexpr (NB > 0) {
      unsigned w[R][NB][Codes<FMT>::kWords], s[R][NB];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const long long row = min(r0 + r, n - 1);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const long long b = row * blocks + min(li + 8 * j, blocks - 1);
          load_block<FMT>(codes, b, w[r][j]);
          s[r][j] = scales[b];
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        unsigned smax = 0;
#pragma unroll
        for (int j = 0; j < NB; ++j) smax = max(smax, s[r][j]);  // a repeated last block changes nothing
        smax = oct_umax(smax);
        ok[r] = smax < 255u;
        cc[r] = 0.f;
#pragma unroll
        for (int k = 0; k < Q; ++k) d[r][k] = 0.f;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const float sc = li + 8 * j < blocks ? rel_scale(s[r][j], smax) : 0.f;
          float c1 = 0.f, d1[Q];
#pragma unroll
          for (int k = 0; k < Q; ++k) d1[k] = 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const f16x8 v = Codes<FMT>::eight(w[r][j], u, 1.f);
            c1 = dot8(v, v, c1);
#pragma unroll
            for (int k = 0; k < Q; ++k) d1[k] = dot8(qv[k][j][u], v, d1[k]);
          }
          cc[r] += c1 * sc * sc;
#pragma unroll
          for (int k = 0; k < Q; ++k) d[r][k] += d1[k] * sc;
        }
      }
    } else {
      const f16x8* ql = reinterpret_cast<const f16x8*>(lds);
      for (int r = 0; r < R; ++r) {
        const long long row = min(r0 + r, n - 1);
        unsigned smax = 0;
        for (int b = li; b < blocks; b += 8) smax = max(smax, (unsigned)scales[row * blocks + b]);
        smax = oct_umax(smax);
        ok[r] = smax < 255u;
        cc[r] = 0.f;
        for (int k = 0; k < Q; ++k) d[r][k] = 0.f;
        for (int b = li; b < blocks; b += 8) {
          unsigned w[Codes<FMT>::kWords];
          load_block<FMT>(codes, row * blocks + b, w);
          const float sc = rel_scale(scales[row * blocks + b], smax);
          float c1 = 0.f, d1[Q];
#pragma unroll
          for (int k = 0; k < Q; ++k) d1[k] = 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const f16x8 v = Codes<FMT>::eight(w, u, 1.f);
            c1 = dot8(v, v, c1);
#pragma unroll
            for (int k = 0; k < Q; ++k) d1[k] = dot8(ql[(k * blocks + b) * 4 + u], v, d1[k]);
          }
          cc[r] += c1 * sc * sc;
#pragma unroll
          for (int k = 0; k < Q; ++k) d[r][k] += d1[k] * sc;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float c = oct_sum(cc[r]);
#pragma unroll
      for (int k = 0; k < Q; ++k) {
        const float sc = row_score(oct_sum(d[r][k]), c, ok[r] && r0 + r < n);
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

// H: blocks a lane half may have. Lane: row (queries: query) l % 32 of a tile and blocks
// [half hb, + hb) of it, half = l / 32: the k order of a product is free, so a lane takes whole blocks and
// both operands agree on it. A wave holds 32 queries for all blocks; waves of a workgroup take query halves
// (nq > 32) and row tiles. The codes of the next tile replace a block's as soon as it is converted.
template <int FMT, int H>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void mx_scan_mfma_kernel(
    const _Float16* q, int nq, const unsigned char* codes, const unsigned char* scales, long long n, int dim, int blocks, bool qvec,
    Cand* part) {
  // scale of the row's largest block: its values stay below 2^16 (fp16) and those of blocks 2^-22 times as
  // large are still exact
  constexpr int kTop = FMT == kMx4 ? 10 : 7;
  constexpr int W = Codes<FMT>::kWords;
  __shared__ __align__(16) float inv[4][32];
  __shared__ Cand red[4][32];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int halves = nq > 32 ? 2 : 1, streams = 4 / halves;
  const int qh = halves == 2 ? wave & 1 : 0, stream = halves == 2 ? wave >> 1 : wave;
  const int hb = (blocks + 1) / 2, b0 = h * hb;
  const int last = min(hb, blocks - b0) - 1;  // this half's last block (-1: none)

  f16x8 qf[H][4];
  {
    const int qi = 32 * qh + r32;
    const _Float16* qp = q + (long long)min(qi, nq - 1) * dim;
#pragma unroll
    for (int j = 0; j < H; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) qf[j][u] = query8(qp, j <= last ? (b0 + j) * 32 + 8 * u : dim, dim, qvec);
  }
  const long long tiles = (n + 31) / 32, stride = (long long)gridDim.x * streams;
  long long tile = (long long)blockIdx.x * streams + stream;
  auto row_of = [&](long long tl) { return min(tl * 32 + r32, n - 1); };
  unsigned w[H][W];
  Bytes16 sb;
  const int bl = max(min(b0, blocks - 1), 0);
  {
    const long long row = row_of(min(tile, tiles - 1));
#pragma unroll
    for (int j = 0; j < H; ++j) load_block<FMT>(codes, row * blocks + min(bl + j, blocks - 1), w[j]);
    sb = *reinterpret_cast<const Bytes16*>(scales + row * blocks + bl);
  }
  float best = -INFINITY;
  long long best_i = n;
  for (; tile < tiles; tile += stride) {
    const long long next = row_of(min(tile + stride, tiles - 1));
    // scales of this tile's blocks, relative to the row's largest
    unsigned s[H], smax = 0;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      s[j] = (sb.w[j / 4] >> (8 * (j % 4))) & 255u;
      if (j <= last) smax = max(smax, s[j]);
    }
    const auto both = __builtin_amdgcn_permlane32_swap(smax, smax, false, false);
    smax = max(both[0], both[1]);
    sb = *reinterpret_cast<const Bytes16*>(scales + next * blocks + bl);
    f32x16 acc[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][r] = acc[1][r] = 0.f;
    float cc = 0.f;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int e = (int)s[j] - (int)smax + 127 + kTop;
      const float sc = j <= last && e > 0 ? __uint_as_float((unsigned)e << 23) : 0.f;  // 0: 2^-127, no fp16 value
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f16x8 v = Codes<FMT>::eight(w[j], u, sc);
        acc[u & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, qf[j][u], acc[u & 1], 0, 0, 0);
        cc = dot8(v, v, cc);
      }
      load_block<FMT>(codes, next * blocks + min(bl + j, blocks - 1), w[j]);
    }
    const unsigned cu = __float_as_uint(cc);
    const auto cs = __builtin_amdgcn_permlane32_swap(cu, cu, false, false);
    const float c2 = __uint_as_float(cs[0]) + __uint_as_float(cs[1]);
    const bool ok = c2 > 0.f && smax < 255u && tile * 32 + r32 < n;
    inv[wave][r32] = ok ? rsqrtf(c2) : NAN;  // NaN scores never win
    // lane: query r32, rows 8 (r / 4) + 4 h + r % 4, ascending with r
    float iv[16];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(&inv[wave][8 * g + 4 * h]);
#pragma unroll
      for (int e = 0; e < 4; ++e) iv[4 * g + e] = x[e];
    }
    float ts = -INFINITY;
    int ti = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float sc = (acc[0][r] + acc[1][r]) * iv[r];
      if (sc > ts) {
        ts = sc;
        ti = 8 * (r >> 2) + (r & 3);
      }
    }
    if (ts > best) {  // a wave's tiles ascend
      best = ts;
      best_i = tile * 32 + ti + 4 * h;
    }
  }
  const float s2 = __shfl_xor(best, 32, 64);
  const long long i2 = __shfl_xor(best_i, 32, 64);
  if (better(s2, i2, best, best_i)) {
    best = s2;
    best_i = i2;
  }
  if (h == 0) red[wave][r32] = Cand{best, 0, best_i};
  __syncthreads();
  if (t < 32 * halves) {
    const int hq = t >> 5;
    Cand b = red[hq][t & 31];
    for (int k = 1; k < streams; ++k) {
      const Cand c = red[hq + k * halves][t & 31];
      if (better(c.s, c.i, b.s, b.i)) b = c;
    }
    part[(long long)blockIdx.x * kMfmaQ + t] = b;
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
  for (int k = t; k < nb; k += 256) {
    const Cand c = part[(long long)k * pitch + j];
    if (better(c.s, c.i, bs, bi)) {
      bs = c.s;
      bi = c.i;
    }
  }
  for (int e = t; e < dim; e += 256) {
    const float x = static_cast<float>(q[(long long)j * dim + e]);
    qq += x * x;
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

template <int FMT, int NB, int Q> int launch_scan(const Scan& a, const _Float16* q) {
  const bool vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && a.dim % 8 == 0;
  const int nb = static_cast<int>(std::min<long long>((a.n + 63) / 64, kScanBlocks));
  const size_t lds = NB > 0 ? 0 : (size_t)Q * a.blocks * 64;
  hipLaunchKernelGGL((mx_scan_kernel<FMT, NB, Q>), dim3(nb), dim3(256), lds, a.s, q, a.codes, a.scales, a.n, a.dim, a.blocks, vec,
                     a.part);
  return nb;
}
template <int FMT, int Q> int scan_blocks(const Scan& a, const _Float16* q) {
  if (a.blocks <= 8) return launch_scan<FMT, 1, Q>(a, q);
  if (a.blocks <= 16) return launch_scan<FMT, 2, Q>(a, q);
  if (a.blocks <= 24) return launch_scan<FMT, 3, Q>(a, q);
  if (a.blocks <= 32) return launch_scan<FMT, 4, Q>(a, q);
  if constexpr (Q <= 2)
    return launch_scan<FMT, 0, Q>(a, q);
  else
    throw Error(-1, "mx_lookup: long rows take two queries at most");
}
template <int FMT, int H> int launch_mfma(const Scan& a, const _Float16* q, int nq) {
  const bool vec = reinterpret_cast<uintptr_t>(q) % 16 == 0 && a.dim % 8 == 0;
  const long long tiles = (a.n + 31) / 32, streams = nq > 32 ? 2 : 4;
  const int nb = static_cast<int>(std::min<long long>((tiles + streams - 1) / streams, kMfmaBlocks));
  hipLaunchKernelGGL((mx_scan_mfma_kernel<FMT, H>), dim3(nb), dim3(256), 0, a.s, q, nq, a.codes, a.scales, a.n, a.dim, a.blocks, vec,
                     a.part);
  return nb;
}

template <int FMT>
void lookup_fmt(const Scan& a, const _Float16* q, int nq, long long* idx, float* score, const KTable& kt, int* kout) {
  while (nq > 0) {
    int m, nb, pitch;
    if (nq > kScanQ && a.dim <= kMfmaMaxDim) {
      m = std::min(nq, kMfmaQ);
      pitch = kMfmaQ;
      const int hb = (a.blocks + 1) / 2;
      nb = hb <= 4 ? launch_mfma<FMT, 4>(a, q, m)
           : hb <= 8 ? launch_mfma<FMT, 8>(a, q, m)
           : hb <= 12 ? launch_mfma<FMT, 12>(a, q, m)
                      : launch_mfma<FMT, 16>(a, q, m);
    } else {
      // long rows: the queries lie in LDS, at most 32 KB of them
      m = pitch = nq >= 4 && a.blocks <= 32 ? 4 : nq >= 2 && a.blocks <= 256 ? 2 : 1;
      nb = m == 4 ? scan_blocks<FMT, 4>(a, q) : m == 2 ? scan_blocks<FMT, 2>(a, q) : scan_blocks<FMT, 1>(a, q);
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
  return sizeof(Cand) * std::max((size_t)kScanBlocks * kScanQ, (size_t)kMfmaBlocks * kMfmaQ);
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
