// 4-bit GEMM on microscaled operands (mx.h; gfx950).
//
// The 32x32x64 matrix-core step takes 32 E2M1 codes (16 bytes) per lane and one E8M0 scale: a lane
// supplies row (l % 32) and block (l / 32) of a 64-deep step, which is exactly a block of an MX row,
// so operands go from memory to the matrix core without a conversion, and the sums are fp32.
//  - B, the packed weights (pack_mx4): per 32 columns and step the lanes' 16 bytes in 1 KB of
//    contiguous memory, loaded straight into registers D stages ahead;
//  - A, MX rows: stages of 128 values (64 bytes of codes and 4 of scales a row) go global -> LDS
//    without passing registers, shared by the four waves; 16-byte chunk c of row r lies at
//    position c ^ ((r / 2) % 4), so that eight consecutive rows' reads of a chunk touch all banks;
//  - C^T = B A^T, a lane then holds four consecutive columns of a row per register group;
//  - tiles go to XCDs in contiguous ranges, row tiles fastest, so that a band of B stays in one L2.
#include <type_traits>

#include "mx.h"

namespace dn {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kXcds = 8;
constexpr int kStageK = 128;

__device__ __forceinline__ v8i operand(const uint4& a) {
  v8i r = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  return r;
}

// One 64-deep step of a 32 x 32 block: step S of a stage, whose scales are bytes S of `bs` and 2 S of `as`.
template <int S>
__device__ __forceinline__ f32x16 mma4(const uint4& b, int bs, const uint4& a, int as, const f32x16& c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(b), operand(a), c, 4, 4, S, bs, 2 * S, as);
}

// 4 bytes per lane of the first N lanes, global -> LDS (lane i writes lds + 4 i); see dma16 (common.h).
// The execution mask is narrowed inside the block: a branch around the load would end the basic
// block, and the compiler then sinks the matrix instructions before it past it.
template <int N> __device__ __forceinline__ void dma4(const void* g, lds_void* lds) {
  const unsigned a = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(reinterpret_cast<__UINTPTR_TYPE__>(lds)));
  unsigned long long all;
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %0, exec\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dword %1, off\n\ts_mov_b64 exec, %0"
               : "=&s"(all)
               : "v"(g), "s"(a), "s"((1ull << N) - 1)
               : "memory", "m0");
}

// x * Phi(x), erf from Abramowitz & Stegun 7.1.26, as max(x, 0) - |x| q, q = (1 - erf(|x| / sqrt 2)) / 2.
__device__ __forceinline__ float gelu_q(float x) {
  const float ax = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(fmaf(ax, 0.3275911f * 0.70710678118654752f, 1.0f));
  const float poly = t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
  const float e = __builtin_amdgcn_exp2f(x * (x * -0.72134752044448170f));
  return fmaf(-fminf(ax, 3.4e38f), poly * e, fmaxf(x, 0.0f));  // finite |x| times zero at x = +-inf
}

__device__ __forceinline__ bool aligned(const void* q, unsigned n) {
  return (reinterpret_cast<__UINTPTR_TYPE__>(q) & (n - 1)) == 0;
}

// Four consecutive columns [n, n + 4) of row m (n % 4 == 0): bias, residual, store.
__device__ __forceinline__ void finish4(const GemmMx4Params& p, int m, int n, int ld, f32x4 v, bool vec) {
  const long long o = (long long)m * ld + n;
  if (p.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += p.bias[n + e];
  }
  if (vec) {
    if (p.resid && p.resid_f32) v += *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.resid) + o);
    if (p.resid && !p.resid_f32) {
      const bf16x4 r = *reinterpret_cast<const bf16x4*>(static_cast<const bf16*>(p.resid) + o);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += static_cast<float>(r[e]);
    }
    if (p.out_f32) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + o) = v;
    } else {
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = static_cast<bf16>(v[e]);
      *reinterpret_cast<bf16x4*>(static_cast<bf16*>(p.out) + o) = w;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x = v[e];
    if (p.resid) x += p.resid_f32 ? static_cast<const float*>(p.resid)[o + e] : static_cast<float>(static_cast<const bf16*>(p.resid)[o + e]);
    if (p.out_f32)
      static_cast<float*>(p.out)[o + e] = x;
    else
      static_cast<bf16*>(p.out)[o + e] = static_cast<bf16>(x);
  }
}

// Whether rows of the output (and the residual) can be accessed four columns at a time.
__device__ __forceinline__ bool out_vec(const GemmMx4Params& p) {
  return aligned(p.out, p.out_f32 ? 16 : 8) && aligned(p.resid, p.resid_f32 ? 16 : 8);
}

// ---------------------------------------------------------------- tiles of 32 FM x 128 FN

// Scheduling groups: NM matrix instructions, each of the first NR followed by an LDS read.
template <int I, int NM, int NR> struct KSched {
  __device__ static __forceinline__ void apply() {
    if constexpr (I < NM) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (I < NR) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      KSched<I + 1, NM, NR>::apply();
    }
  }
};

template <int FM, int FN> constexpr int stage_bytes() { return 32 * FM * 68; }
template <int FM, int FN, int S, bool GE> constexpr size_t tile_lds() {
  constexpr size_t ring = size_t(S) * stage_bytes<FM, FN>();
  constexpr size_t ep = 4 * 32 * (32 * FN + 4) * 4;
  return ring > ep ? ring : ep;
}

// S LDS stages; A and B are loaded S - 1 stages ahead.
template <int FM, int FN, int S, bool GE>
__device__ __forceinline__ void mx4_tile(const GemmMx4Params& p, const int m0, const int n0) {
  constexpr int BM = 32 * FM, D = S - 1, PW = BM / 64, SR = BM / 4;  // code DMA per wave, scale rows per wave
  constexpr int STAGE = stage_bytes<FM, FN>(), SCALES = BM * 64;
  static_assert(BM % 64 == 0 && (!GE || FN % 2 == 0), "whole DMA instructions, whole GEGLU pairs");
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nk = p.K / kStageK;
  const int r32 = lane & 31, h = lane >> 5;

  // A: DMA instruction j of this wave fills rows [16 q, 16 q + 16), q = wave PW + j
  const unsigned char* const codes = static_cast<const unsigned char*>(p.a);
  const unsigned char* const ascales = codes + (long long)p.M * (p.K / 2);
  const unsigned char* pa[PW];
#pragma unroll
  for (int j = 0; j < PW; ++j) {
    const int row = 16 * (wave * PW + j) + (lane >> 2);
    pa[j] = codes + (long long)min(m0 + row, p.M - 1) * (p.K / 2) + (((lane & 3) ^ ((row >> 1) & 3)) * 16);
  }
  const unsigned char* const ps = ascales + (long long)min(m0 + wave * SR + (lane & (SR - 1)), p.M - 1) * (p.K / 32);
  auto issue_a = [&](int kt_in, int slot) {
    const int kt = min(kt_in, nk - 1);  // stages past the end repeat the last one
    unsigned char* stage = smem + slot * STAGE;
#pragma unroll
    for (int j = 0; j < PW; ++j) dma16(pa[j] + kt * 64, (lds_void*)(stage + (wave * PW + j) * 1024));
    dma4<SR>(ps + kt * 4, (lds_void*)(stage + SCALES + wave * SR * 4));
  };

  // B: column blocks (n0 + 32 FN wave) / 32 + j, past the matrix the last one
  // scales: one word per lane and pair of column blocks, two bytes (steps) of each
  struct BStage {
    uint4 c[2][FN];
    unsigned s[(FN + 1) / 2];
  };
  const unsigned char* bc[FN];
  const unsigned char* bs[(FN + 1) / 2];
  const int nb0 = (n0 + wave * 32 * FN) / 32;
  static_assert(FN <= 2, "the column blocks of a wave share their scale words");
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const long long nb = min(nb0 + j, p.N / 32 - 1);
    bc[j] = static_cast<const unsigned char*>(p.b) + nb * nk * 2048 + lane * 16;
    if (j % 2 == 0)
      bs[j / 2] = static_cast<const unsigned char*>(p.b) + (long long)p.N * (p.K / 2) + nb / 2 * nk * 256 + lane * 4;
  }
  const int bshift = FN == 1 ? 16 * (min(nb0, p.N / 32 - 1) & 1) : 0;
  auto load_b = [&](int kt_in, BStage& d) {
    const long long kt = min(kt_in, nk - 1);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      d.c[0][j] = ld16(bc[j] + kt * 2048);
      d.c[1][j] = ld16(bc[j] + kt * 2048 + 1024);
      if (j % 2 == 0) d.s[j / 2] = *reinterpret_cast<const unsigned*>(bs[j / 2] + kt * 256);
    }
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // Loads of a stage: 2 FN and a scale word of B, then PW + 1 of A. Before stage kt is read, its DMA has landed when at
  // most those of the D - 1 stages issued after it are out. The last D - 1 stages (TAIL > 0, counted
  // from 1) load nothing more: the compiler would drop B loads that nothing uses, and the count with
  // them.
  constexpr int kLoads = 2 * FN + 1 + PW + 1;
  static_assert((D - 1) * kLoads < 64, "vmcnt range");
  const int sw = (r32 >> 1) & 3;
  auto stage = [&](int kt, BStage& b, auto tail) {
    constexpr int TAIL = decltype(tail)::value;
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((TAIL > 0 ? D - TAIL : D - 1) * kLoads));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    const unsigned char* st = smem + (kt % S) * STAGE;
    uint4 a0[FM], a1[FM];
    int as[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const unsigned char* row = st + (32 * i + r32) * 64;
      a0[i] = ld16(row + (h ^ sw) * 16);
      as[i] = *reinterpret_cast<const int*>(st + SCALES + (32 * i + r32) * 4);
    }
    __builtin_amdgcn_sched_barrier(0);
    int bw[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) bw[j] = (int)(b.s[j / 2] >> (FN == 1 ? bshift : 16 * (j % 2)));
#pragma unroll
    for (int i = 0; i < FM; ++i) as[i] = (int)((unsigned)as[i] >> (8 * h));
#pragma unroll
    for (int i = 0; i < FM; ++i) a1[i] = ld16(st + (32 * i + r32) * 64 + ((2 + h) ^ sw) * 16);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mma4<0>(b.c[0][j], bw[j], a0[i], as[i], acc[i][j]);
    KSched<0, FM * FN, FM>::apply();
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mma4<1>(b.c[1][j], bw[j], a1[i], as[i], acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (TAIL == 0) {
      load_b(kt + D, b);
      __builtin_amdgcn_sched_barrier(0);
      issue_a(kt + D, (kt + D) % S);
    }
  };

  BStage b[D];
#pragma unroll
  for (int v = 0; v < D; ++v) {
    load_b(v, b[v]);
    __builtin_amdgcn_sched_barrier(0);
    issue_a(v, v);
  }
  int kt = 0;
  for (; kt + D <= nk; kt += D) {
#pragma unroll
    for (int v = 0; v < D; ++v) stage(kt + v, b[v], std::integral_constant<int, 0>());
  }
  static_assert(D == 3, "two stages at most are left");
  if (kt < nk) stage(kt, b[0], std::integral_constant<int, 1>());
  if (kt + 1 < nk) stage(kt + 1, b[1], std::integral_constant<int, 2>());
  __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(0));
  __syncthreads();

  // Epilogue. Lane: row r32 of block i, columns 8 g + 4 h .. + 3 in registers 4 g ...
  const int nw0 = n0 + wave * 32 * FN;
  if constexpr (GE) {
    const int n_out = p.N / 2;
#pragma unroll
    for (int j = 0; j < FN; j += 2) {
      const int n = nw0 + 32 * j, o = n / 2;  // value columns n .., gates n + 32 ..
      if (n >= p.N) break;
      f32x4 ba[4], bg[4];
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ba[g][e] = p.bias ? p.bias[n + 8 * g + 4 * h + e] : 0.f;
          bg[g][e] = p.bias ? p.bias[n + 32 + 8 * g + 4 * h + e] : 0.f;
        }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int m = m0 + 32 * i + r32;
        float v[16];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[4 * g + e] = (acc[i][j][4 * g + e] + ba[g][e]) * gelu_q(acc[i][j + 1][4 * g + e] + bg[g][e]);
        if (p.out_f32) {
          if (m < p.M) {
            float* y = static_cast<float*>(p.out) + (long long)m * n_out + o + 4 * h;
            const bool vec = aligned(p.out, 16);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              if (vec)
                *reinterpret_cast<f32x4*>(y + 8 * g) = f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
              else
                for (int e = 0; e < 4; ++e) y[8 * g + e] = v[4 * g + e];
            }
          }
          continue;
        }
        // the 32 columns are one block of the output row, in this lane and lane ^ 32
        unsigned am = mx_abs_bits(v[0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) am = max(am, mx_abs_bits(v[e]));
        const auto sw2 = __builtin_amdgcn_permlane32_swap(am, am, false, false);
        const unsigned s = mx_scale<kMx4>(max(sw2[0], sw2[1]));
        // codes of g = 0, 1 and of g = 2, 3: four (16 bits) each
        const unsigned p01 = mx4_codes8(v, s), p23 = mx4_codes8(v + 8, s);
        const auto x = __builtin_amdgcn_permlane32_swap(p01, p23, false, false);
        const uint2 w = make_uint2(__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[1], x[0], 0x07060302u));
        if (m < p.M) {
          unsigned char* oc = static_cast<unsigned char*>(p.out) + (long long)m * (n_out / 2) + o / 2;
          *reinterpret_cast<uint2*>(oc + 8 * h) = w;
          if (h == 0) static_cast<unsigned char*>(p.out)[(long long)p.M * (n_out / 2) + (long long)m * (n_out / 32) + o / 32] = (unsigned char)s;
        }
      }
    }
  } else {
    // whole rows of the wave's columns through LDS, 32 rows at a time
    constexpr int WN = 32 * FN, EPL = WN + 4, LPR = WN / 4, RPI = 64 / LPR;
    float* ep = reinterpret_cast<float*>(smem) + wave * 32 * EPL;
    const int c4 = (lane % LPR) * 4, n = nw0 + c4;
    const bool vec = out_vec(p), in = n < p.N;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(ep + r32 * EPL + j * 32 + 8 * g + 4 * h) =
              f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
#pragma unroll
      for (int t = 0; t < 32 / RPI; ++t) {
        const int rr = t * RPI + lane / LPR, m = m0 + 32 * i + rr;
        const f32x4 v = *reinterpret_cast<const f32x4*>(ep + rr * EPL + c4);
        if (m < p.M && in) finish4(p, m, n, p.N, v, vec);
      }
    }
  }
}

template <int FM, int FN, int S, bool GE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_mx4_kernel(GemmMx4Params p, int mt, int nt) {
  const int wg = blockIdx.x, units = mt * nt;
  const int xcd = wg % kXcds, idx = wg / kXcds;
  const int base = units / kXcds, rem = units % kXcds;
  const int u = xcd * base + min(xcd, rem) + idx;
  mx4_tile<FM, FN, S, GE>(p, (u % mt) * 32 * FM, (u / mt) * 128 * FN);
}

// ---------------------------------------------------------------- few rows
//
// 32 rows x 32 columns (GEGLU: a 64-column value / gate pair), the K stages dealt to the NW waves; the
// waves' partial sums meet in LDS in wave order. A is read straight from memory: with few rows the
// time is the weights' and the latency of a wave's few stages, and more waves shorten both.
template <int NW, bool GE>
__global__ __launch_bounds__(64 * NW) void gemm_mx4_rows_kernel(GemmMx4Params p, int nt) {
  constexpr int FN = GE ? 2 : 1, WN = 32 * FN, EPL = WN + 4;
  __shared__ __align__(16) float part[NW][32][EPL];
  const int t = threadIdx.x, lane = t & 63, r32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int nk = p.K / kStageK;
  const int n0 = (int)(blockIdx.x % nt) * WN, m0 = (int)(blockIdx.x / nt) * 32;
  const long long row = min(m0 + r32, p.M - 1);
  const unsigned char* a = static_cast<const unsigned char*>(p.a) + row * (p.K / 2) + h * 16;
  const unsigned char* as = static_cast<const unsigned char*>(p.a) + (long long)p.M * (p.K / 2) + row * (p.K / 32);
  const unsigned char* b = static_cast<const unsigned char*>(p.b) + (long long)(n0 / 32) * nk * 2048 + lane * 16;
  const unsigned char* bs = static_cast<const unsigned char*>(p.b) + (long long)p.N * (p.K / 2) + (long long)(n0 / 64) * nk * 256 + lane * 4;
  const int bshift = n0 & 32 ? 16 : 0;
  f32x16 acc[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
  for (int kt = wave; kt < nk; kt += NW) {
    const uint4 a0 = ld16(a + kt * 64), a1 = ld16(a + kt * 64 + 32);
    const int sa = (int)(*reinterpret_cast<const unsigned*>(as + kt * 4) >> (8 * h));
    const unsigned sw = *reinterpret_cast<const unsigned*>(bs + kt * 256);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const long long o = (long long)j * nk + kt;
      const uint4 b0 = ld16(b + o * 2048), b1 = ld16(b + o * 2048 + 1024);
      const int sb = (int)(sw >> (bshift + 16 * j));
      acc[j] = mma4<0>(b0, sb, a0, sa, acc[j]);
      acc[j] = mma4<1>(b1, sb, a1, sa, acc[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(&part[wave][r32][32 * j + 8 * g + 4 * h]) =
          f32x4{acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
  __syncthreads();
  // thread: row t / 8, columns 4 (t % 8) .. of the block (of the value and the gate block)
  if (t >= 256) return;
  const int rr = t >> 3, c = (t & 7) * 4, m = m0 + rr;
  f32x4 v[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    v[j] = *reinterpret_cast<const f32x4*>(&part[0][rr][32 * j + c]);
    for (int w = 1; w < NW; ++w) v[j] += *reinterpret_cast<const f32x4*>(&part[w][rr][32 * j + c]);
  }
  if constexpr (GE) {
    const int n_out = p.N / 2, o = n0 / 2 + c;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float ba = p.bias ? p.bias[n0 + c + e] : 0.f, bg = p.bias ? p.bias[n0 + 32 + c + e] : 0.f;
      y[e] = (v[0][e] + ba) * gelu_q(v[1][e] + bg);
    }
    if (p.out_f32) {
      if (m < p.M)
        for (int e = 0; e < 4; ++e) static_cast<float*>(p.out)[(long long)m * n_out + o + e] = y[e];
      return;
    }
    // the row's block lies in eight lanes
    const unsigned s = mx_scale<kMx4>(oct_umax(max(max(mx_abs_bits(y[0]), mx_abs_bits(y[1])), max(mx_abs_bits(y[2]), mx_abs_bits(y[3])))));
    const float z[8] = {y[0], y[1], y[2], y[3], 0.f, 0.f, 0.f, 0.f};
    const unsigned w = mx4_codes8(z, s);
    if (m < p.M) {
      unsigned char* oc = static_cast<unsigned char*>(p.out);
      *reinterpret_cast<unsigned short*>(oc + (long long)m * (n_out / 2) + o / 2) = (unsigned short)w;
      if ((t & 7) == 0) oc[(long long)p.M * (n_out / 2) + (long long)m * (n_out / 32) + o / 32] = (unsigned char)s;
    }
  } else {
    if (m < p.M) finish4(p, m, n0 + c, p.N, v[0], out_vec(p));
  }
}

template <int FM, int FN, bool GE> void launch_tile(const GemmMx4Params& p, hipStream_t s) {
  constexpr int S = 4;
  constexpr size_t lds = tile_lds<FM, FN, S, GE>();
  static_assert(lds <= 64 * 1024, "no attribute needed up to 64 KB");
  const int mt = ceil_div(p.M, 32 * FM), nt = ceil_div(p.N, 128 * FN);
  DN_CHECK((long long)mt * nt <= 0x7fffffffll, "gemm_mx4: too many tiles");
  hipLaunchKernelGGL((gemm_mx4_kernel<FM, FN, S, GE>), dim3(mt * nt), dim3(256), lds, s, p, mt, nt);
}

template <bool GE> void launch_rows(const GemmMx4Params& p, hipStream_t s) {
  constexpr int NW = 8;
  const int nt = p.N / (GE ? 64 : 32), mt = ceil_div(p.M, 32);
  DN_CHECK((long long)mt * nt <= 0x7fffffffll, "gemm_mx4: too many tiles");
  hipLaunchKernelGGL((gemm_mx4_rows_kernel<NW, GE>), dim3(mt * nt), dim3(64 * NW), 0, s, p, nt);
}

}  // namespace

bool gemm_mx4_layout(int N, int K) { return N >= 32 && N % 32 == 0 && K >= kStageK && K % kStageK == 0; }
size_t gemm_mx4_code_bytes(int N, int K) { return (size_t)N * (K / 2); }
size_t gemm_mx4_bytes(int N, int K) { return (size_t)N * (K / 2) + (size_t)((N + 63) / 64 * 64) * (K / 32); }

void gemm_mx4_check(const GemmMx4Params& p) {
  DN_CHECK(gemm_mx4_layout(p.N, p.K) && p.M >= 1, "gemm_mx4: N % 32 == 0 and K % 128 == 0 needed");
  DN_CHECK(p.a && p.b && p.out, "gemm_mx4: null operand");
  DN_CHECK(!p.geglu || (p.N % 64 == 0 && !p.resid), "gemm_mx4: GEGLU takes value / gate pairs of 64 columns, no residual");
  DN_CHECK(((uintptr_t)p.a | (uintptr_t)p.b) % 16 == 0 && (uintptr_t)p.bias % 4 == 0, "gemm_mx4: operands must be 16-byte aligned");
  DN_CHECK((uintptr_t)p.out % (p.out_f32 ? 4 : p.geglu ? 16 : 2) == 0 && (uintptr_t)p.resid % (p.resid_f32 ? 4 : 2) == 0,
           "gemm_mx4: misaligned output or residual");
}

void gemm_mx4(const GemmMx4Params& p, int cus, hipStream_t s) {
  gemm_mx4_check(p);
  if (p.M <= 64) {
    p.geglu ? launch_rows<true>(p, s) : launch_rows<false>(p, s);
  } else if (p.geglu) {
    launch_tile<4, 2, true>(p, s);
  } else {
    const long long wide = (long long)ceil_div(p.M, 128) * ceil_div(p.N, 256);
    if (wide >= 2 * cus)
      launch_tile<4, 2, false>(p, s);
    else if ((long long)ceil_div(p.M, 128) * ceil_div(p.N, 128) >= 2 * cus)
      launch_tile<4, 1, false>(p, s);
    else
      launch_tile<2, 1, false>(p, s);
  }
  DN_HIP(hipGetLastError());
}

}  // namespace dn
