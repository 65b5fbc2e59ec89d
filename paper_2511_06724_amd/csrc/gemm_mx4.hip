// 4-bit GEMM on microscaled operands (mx.h; gfx950).
//
// The 32x32x64 matrix-core step takes 32 E2M1 codes (16 bytes) per lane and one E8M0 scale: a lane
// supplies row (l % 32) and block (l / 32) of a 64-deep step, which is exactly a block of an MX row,
// so operands go from memory to the matrix core without a conversion, and the sums are fp32.
//  - B, the packed weights (pack_mx4): per 32 columns and step the lanes' 16 bytes in 1 KB of
//    contiguous memory, loaded straight into registers three or four stages ahead;
//  - A, MX rows: stages of 128 values (64 bytes of codes a row) go global -> LDS without passing
//    registers, shared by the waves; 16-byte chunk c of row r lies at position c ^ ((r / 4) % 4), so
//    that sixteen consecutive rows' reads of a chunk touch all banks. The scales are copied once;
//  - C^T = B A^T, a lane then holds four consecutive columns of a row per register group;
//  - tiles go to XCDs in contiguous ranges, row tiles fastest, so that a band of B stays in one L2.
// A step (65536 multiply-adds) takes the matrix core 32 cycles, 1.0e16 operations per second at 2.4 GHz, eight
// times what a large bf16 product through the library reaches; a loop of steps on random data sustains 6.5 to
// 7.1e15. Measured: 4096^3 40.9 us (3.4e15); 2048 x 1280, K = 5120, fp32 residual 15.5 us with a bf16 output, 19.4
// with an fp32 one; GEGLU 2048 x 5120, K = 1280 23.1 us; 32768 x 5120, K = 640 116 us (336 MB of output, 2.9 TB/s).
// The matrix cores are busy 51 % of the time that CUs are in the first, 20 to 30 % in the others: what bounds those
// is a tile's start, which waits for residual, bias and first stages one after the other, and its stores and GELUs.
#include <algorithm>
#include <limits>
#include <type_traits>

#include "lane_swap.h"
#include "mx.h"

namespace dn {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kXcds = 8;
constexpr int kStageK = 128;
constexpr int kMaxDim = 1 << 22;  // of N and K: offsets within a tile's rows have 32 bits
constexpr size_t kBSpare = 8192;  // of a packed matrix, for the loads past its last stage: four stages of 2 KB

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename V> __device__ __forceinline__ v8i operand(const V& a) {
  v8i r = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  return r;
}

// One 64-deep step of a 32 x 32 block: step S of a stage, whose scales are bytes S of `bs` and 2 S of `as`.
template <int S, typename V>
__device__ __forceinline__ f32x16 mma4(const V& b, int bs, const uint4& a, int as, const f32x16& c) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(b), operand(a), c, 4, 4, S, bs, 2 * S, as);
}

// A global pointer every lane of the wave has, in scalar registers.
typedef const unsigned char __attribute__((address_space(1))) * GlobalBytes;
typedef const unsigned __attribute__((address_space(1))) * Global4;
typedef const u32x4 __attribute__((address_space(1))) * Global16;
__device__ __forceinline__ GlobalBytes uniform(const void* q) {
  const unsigned long long b = reinterpret_cast<__UINTPTR_TYPE__>(q);
  return reinterpret_cast<GlobalBytes>(
      static_cast<unsigned long long>(__builtin_amdgcn_readfirstlane(static_cast<unsigned>(b >> 32))) << 32 |
      static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<unsigned>(b))));
}

// 16 bytes per lane global -> LDS (lane i writes lds + 16 i) from a wave-uniform base and a byte offset per
// lane; see dma16 (common.h) for why this is assembly, with a wait state after the write of M0. dma16_if: where
// `on` (wave-uniform), else nothing: with an empty execution mask rather than a branch, which would end the basic
// block (the compiler then sinks the matrix instructions before it past it).
__device__ __forceinline__ void dma16_to(GlobalBytes base, unsigned off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}
__device__ __forceinline__ void dma16_if(bool on, GlobalBytes base, unsigned off, unsigned lds) {
  const unsigned mask = __builtin_amdgcn_readfirstlane(on ? ~0u : 0u);
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dwordx4 %0, %1\n\t"
               "s_mov_b64 exec, -1" ::"v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)), "s"(mask)
               : "memory", "m0");
}

// x * Phi(x), erf from Abramowitz & Stegun 7.1.26, as max(x, 0) - |x| q, q = (1 - erf(|x| / sqrt 2)) / 2.
__device__ __forceinline__ float gelu_q(float x) {
  const float ax = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(fmaf(ax, 0.3275911f * 0.70710678118654752f, 1.0f));
  const float poly = t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
  const float e = __builtin_amdgcn_exp2f(x * (x * -0.72134752044448170f));
  // finite |x| times zero at x = +-inf; minimum and maximum pass a NaN on as it is
  return fmaf(-__builtin_elementwise_minimum(ax, 3.4e38f), poly * e, __builtin_elementwise_maximum(x, 0.0f));
}

__device__ __forceinline__ bool aligned(const void* q, unsigned n) {
  return (reinterpret_cast<__UINTPTR_TYPE__>(q) & (n - 1)) == 0;
}

// Registers 4 g .. 4 g + 3 of a block.
__device__ __forceinline__ f32x4 group_of(const f32x16& a, int g) { return f32x4{a[4 * g], a[4 * g + 1], a[4 * g + 2], a[4 * g + 3]}; }

__device__ __forceinline__ void set_group(f32x16& a, int g, const f32x4& v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a[4 * g + e] = v[e];
}
// Four bf16 values in two words.
__device__ __forceinline__ f32x4 bf16x4_values(unsigned lo, unsigned hi) {
  return f32x4{__uint_as_float(lo << 16), __uint_as_float(lo & 0xffff0000u), __uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)};
}

// Past the caches: a bf16 output would push the operands out of them (32768 x 5120, K = 640: 116.5 us, cached 122;
// 4096^3 38.8 and 40.3). The fp32 output, the residual stream that the next LayerNorm reads, gains as much by itself
// and loses it there (the feed-forward at 8192 x 640: 58.4, cached 57.3), so it is cached.
__device__ __forceinline__ void store_nt(bf16* d, const uint4& v) {
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(d));
}

// Whether output and residual can be accessed 16 bytes at a time.
__device__ __forceinline__ bool out_vec(const GemmMx4Params& p) { return aligned(p.out, 16) && aligned(p.resid, 16); }

// Four values of the residual, one by one.
__device__ __forceinline__ f32x4 resid4(const GemmMx4Params& p, long long o) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = p.resid_f32 ? static_cast<const float*>(p.resid)[o + e] : static_cast<float>(static_cast<const bf16*>(p.resid)[o + e]);
  return v;
}

// Four values to out + o one by one.
__device__ __forceinline__ void store_each(const GemmMx4Params& p, long long o, const f32x4& v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (p.out_f32)
      static_cast<float*>(p.out)[o + e] = v[e];
    else
      static_cast<bf16*>(p.out)[o + e] = static_cast<bf16>(v[e]);
  }
}

// ---------------------------------------------------------------- tiles of 32 FM x 32 FN NW

template <int I, int E, typename G> __device__ __forceinline__ void work_range(G& work) {
  if constexpr (I < E) {
    work(std::integral_constant<int, I>());
    work_range<I + 1, E>(work);
  }
}

// NM matrix instructions with NA other pieces of work (LDS reads, loads) dealt out between them, in this order
// in the program: memory instructions in a row stall a wave in their issue, with its matrix core idle.
template <int I, int NM, int NA, typename F, typename G> __device__ __forceinline__ void interleave(F& mfma, G& work) {
  if constexpr (I < NM) {
    mfma(std::integral_constant<int, I>());
    __builtin_amdgcn_sched_barrier(0);
    work_range<NA * I / NM, NA * (I + 1) / NM>(work);
    __builtin_amdgcn_sched_barrier(0);
    interleave<I + 1, NM, NA>(mfma, work);
  }
}

// LDS of a tile: S stages of codes, then the scales of its rows for up to kScaleK values, copied once instead
// of four bytes a row and stage (a line each time: that took as long as the codes).
constexpr int kScaleK = 8192;
template <int FM> constexpr int stage_bytes() { return 32 * FM * 64; }
constexpr size_t scale_lds(int bm, int K) { return (size_t)bm * 16 * (((K < kScaleK ? K : kScaleK) / 32 + 15) / 16); }
template <int FM, int S> size_t tile_lds(int K) { return size_t(S) * stage_bytes<FM>() + scale_lds(32 * FM, K); }

// S LDS stages and register sets of B, loaded up to S stages ahead. A stage is two 64-deep steps:
//   step 0's MFMAs and the LDS reads of step 1; hand-over: the DMA of the next stage has landed (wait),
//   and every wave is done with this stage's LDS (barrier); step 1's MFMAs and the LDS reads of the next
//   stage's step 0; then the loads of stage kt + S, into the LDS slot and the registers of this one.
// So LDS latency and the loads' issue lie under MFMAs of the same wave.
template <int FM, int FN, int S, int NW, bool GE>
__device__ __forceinline__ void mx4_tile(const GemmMx4Params& p, const int m0, const int n0) {
  constexpr int BM = 32 * FM, PW = BM / 64;  // code DMA of each of the first four waves
  constexpr int STAGE = stage_bytes<FM>();
  static_assert(NW == 4 || NW == 5, "four waves issue the DMA");
  static_assert(BM % 64 == 0 && FN <= 2 && (!GE || FN == 2), "whole DMA instructions, shared scale words, whole GEGLU pairs");
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* const scales = smem + S * STAGE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int nb0 = (n0 + wave * 32 * FN) / 32, nb_last = p.N / 32 - 1;
  const int bshift = FN == 1 ? 16 * (min(nb0, nb_last) & 1) : 0;

  // The accumulators begin with residual and bias, and the epilogue only stores. Both are waited for before the
  // first stages' loads are issued: a latency each at a tile's start. Lane: row r32 of block i, columns
  // 8 g + 4 h .. + 3 in registers 4 g ...
  // Rows are accessed in the store layout of a block, 64 bytes of each of 16 rows: row r16 and, for fp32 (a
  // pair of groups) and for bf16, the lane's first column.
  f32x16 acc[FM][FN];
  const bool vec = out_vec(p);
  const int r16 = lane & 15, c8 = 8 * ((lane >> 4) & 1) + 4 * h, c16 = 16 * ((lane >> 4) & 1) + 8 * h;
  auto row_at = [&](int i, int r) { return (long long)min(m0 + 32 * i + r, p.M - 1) * p.N; };
  if (GE || !p.resid) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  } else if (!vec) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) set_group(acc[i][j], g, resid4(p, row_at(i, r32) + min(nb0 + j, nb_last) * 32 + 4 * h + 8 * g));
  } else if (p.resid_f32) {
    const float* const r = static_cast<const float*>(p.resid) + c8;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = min(nb0 + j, nb_last) * 32;
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
          set_group(acc[i][j], g, *reinterpret_cast<const f32x4*>(r + row_at(i, r16) + n + 8 * g));
          set_group(acc[i][j], g + 1, *reinterpret_cast<const f32x4*>(r + row_at(i, r16 + 16) + n + 8 * g));
        }
      }
    __builtin_amdgcn_sched_barrier(0);  // every load before the first use
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
          f32x4 v = group_of(acc[i][j], g), w = group_of(acc[i][j], g + 1);
          rows16(v, w);
          set_group(acc[i][j], g, v);
          set_group(acc[i][j], g + 1, w);
        }
  } else {
    const bf16* const r = static_cast<const bf16*>(p.resid) + c16;
    uint4 x[FM][FN][2];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = min(nb0 + j, nb_last) * 32;
        x[i][j][0] = ld16(r + row_at(i, r16) + n);
        x[i][j][1] = ld16(r + row_at(i, r16 + 16) + n);
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        rows16(x[i][j][0], x[i][j][1]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint4 u = x[i][j][t];
          const Pair lo = swap32(u.x, u.z), hi = swap32(u.y, u.w);
          set_group(acc[i][j], 2 * t, bf16x4_values(lo.a, hi.a));
          set_group(acc[i][j], 2 * t + 1, bf16x4_values(lo.b, hi.b));
        }
      }
  }
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const float* const q = p.bias + min(nb0 + j, nb_last) * 32 + 4 * h;
      float bias[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) bias[r] = q[8 * (r >> 2) + (r & 3)];
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] += bias[r];
    }
  }

  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<__UINTPTR_TYPE__>((lds_void*)smem));
  const int rows = p.M - m0;  // rows past the matrix read its last one

  for (int k0 = 0; k0 < p.K; k0 += kScaleK) {
    const int kc = min(p.K - k0, kScaleK), nk = kc / kStageK, pitch = kc / 32;
    // scales of the tile's rows, as [16-byte chunk][row] (a lane's reads of consecutive rows then lie 16
    // bytes apart whatever the row length); a chunk past the row's end is other rows', or the buffer's spare
    // bytes, and not used
    const GlobalBytes gs =
        uniform(static_cast<const unsigned char*>(p.a) + (long long)p.M * (p.K / 2) + (long long)m0 * (p.K / 32) + k0 / 32);
    for (int e0 = wave * 64; e0 < BM * ((pitch + 15) / 16); e0 += 64 * NW) {
      const int e = e0 + lane, row = e % BM, c = e / BM;
      dma16_to(gs, (unsigned)min(row, rows - 1) * (unsigned)(p.K / 32) + c * 16, lds0 + S * STAGE + e0 * 16);
    }

    // A: DMA instruction j of this wave fills rows [16 q, 16 q + 16), q = wave PW + j
    const GlobalBytes ga = uniform(static_cast<const unsigned char*>(p.a) + (long long)m0 * (p.K / 2) + k0 / 2);
    unsigned oa[PW];
#pragma unroll
    for (int j = 0; j < PW; ++j) {
      const int row = 16 * (wave * PW + j) + (lane >> 2);
      oa[j] = (unsigned)min(row, rows - 1) * (unsigned)(p.K / 2) + (unsigned)(((lane & 3) ^ ((row >> 2) & 3)) * 16);
    }
    auto dma_a = [&](int kt, int slot, int j) {
      const GlobalBytes g = ga + (long long)min(kt, nk - 1) * 64;  // stages past the end repeat the last one
      const unsigned dst = lds0 + slot * STAGE + (wave * PW + j) * 1024;
      if constexpr (NW == 4)
        dma16_to(g, oa[j], dst);
      else
        dma16_if(wave < 4, g, oa[j], dst);
    };

    // B: column blocks nb0 + j, past the matrix the last one; scales: one word per lane and pair of column
    // blocks, two bytes (steps) of each. Loads run on past the last stage (a packed matrix has room for that).
    struct BStage {
      u32x4 c[2][FN];
      unsigned s;
    };
    const int nk_all = p.K / kStageK, kt0 = k0 / kStageK;
    GlobalBytes gb[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j)
      gb[j] = uniform(static_cast<const unsigned char*>(p.b) + ((long long)min(nb0 + j, nb_last) * nk_all + kt0) * 2048);
    GlobalBytes gbs = uniform(static_cast<const unsigned char*>(p.b) + (long long)p.N * (p.K / 2) +
                                       ((long long)(min(nb0, nb_last) / 2) * nk_all + kt0) * 256);
    const unsigned l16 = lane * 16, l4 = lane * 4;
    // from the pointers of stage kt: of a stage `ahead` further
    auto load_c0 = [&](int ahead, BStage& d, int j) { d.c[0][j] = *reinterpret_cast<Global16>(gb[j] + ahead * 2048 + l16); };
    auto load_c1 = [&](int ahead, BStage& d, int j) { d.c[1][j] = *reinterpret_cast<Global16>(gb[j] + ahead * 2048 + 1024 + l16); };
    auto load_s = [&](int ahead, BStage& d) { d.s = *reinterpret_cast<Global4>(gbs + ahead * 256 + l4); };

    // Loads of a stage, in order: FN codes of step 0 of B, PW of A (both for stage kt + S, during step 1 of
    // stage kt); FN codes of step 1 and the scale word of B (during step 0 of the stage after). At the
    // hand-over to stage kt + 1, its DMA has landed when at most the loads of the S - 2 stages issued after it and
    // the FN + 1 of the present stage are out. The last stages (TAIL > 0, counted from 1) load nothing more:
    // the compiler would drop B loads that nothing uses, and the count with them.
    constexpr int kLoads = 2 * FN + 1 + PW;
    static_assert((S - 1) * kLoads < 64, "vmcnt range");
    const unsigned char* const arow = smem + r32 * 64;
    const int sw = (r32 >> 2) & 3;
    const unsigned char* const row0 = arow + (h ^ sw) * 16;
    const unsigned char* const row1 = arow + ((2 + h) ^ sw) * 16;
    const unsigned char* const srow = scales + r32 * 16;
    uint4 a0[FM], a1[FM];
    unsigned aw[FM];
    // stage kt in LDS slot and register set V (a constant: every LDS address is a base and an offset in the
    // instruction; with one wave on a SIMD, address arithmetic is not hidden)
    auto stage = [&](int kt, auto v, BStage* b, auto tail) {
      constexpr int V = decltype(v)::value, TAIL = decltype(tail)::value;
      BStage& cur = b[V];
      BStage& prev = b[(V + S - 1) % S];
      int as[FM], bw[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) as[i] = (int)(aw[i] >> (8 * h));
#pragma unroll
      for (int j = 0; j < FN; ++j) bw[j] = (int)(cur.s >> (FN == 1 ? bshift : 16 * j));
      auto mfma0 = [&](auto e) {
        constexpr int i = decltype(e)::value / FN, j = decltype(e)::value % FN;
        acc[i][j] = mma4<0>(cur.c[0][j], bw[j], a0[i], as[i], acc[i][j]);
      };
      auto work0 = [&](auto e) {
        constexpr int w = decltype(e)::value;
        if constexpr (w < FM)
          a1[w] = ld16(row1 + V * STAGE + w * 2048);
        else if constexpr (w < FM + FN)
          load_c1(S - 1, prev, w - FM);
        else
          load_s(S - 1, prev);
      };
      __builtin_amdgcn_sched_barrier(0);
      interleave<0, FM * FN, FM + (TAIL == 0 ? FN + 1 : 0)>(mfma0, work0);
      __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(TAIL > 0 ? (S - 1 - TAIL) * kLoads : (S - 2) * kLoads + FN + 1));
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const int kn = min(kt + 1, nk - 1);
      const unsigned char* const sc = srow + ((kn >> 2) * (16 * BM) + (kn & 3) * 4);
      auto mfma1 = [&](auto e) {
        constexpr int i = decltype(e)::value / FN, j = decltype(e)::value % FN;
        acc[i][j] = mma4<1>(cur.c[1][j], bw[j], a1[i], as[i], acc[i][j]);
      };
      auto work1 = [&](auto e) {
        constexpr int w = decltype(e)::value;
        if constexpr (w < FM) {
          a0[w] = ld16(row0 + (V + 1) % S * STAGE + w * 2048);
          aw[w] = *reinterpret_cast<const unsigned*>(sc + w * 512);
        } else if constexpr (w < FM + FN) {
          load_c0(S, cur, w - FM);
        } else {
          dma_a(kt + S, V, w - FM - FN);
        }
      };
      interleave<0, FM * FN, FM + (TAIL == 0 ? FN + PW : 0)>(mfma1, work1);
#pragma unroll
      for (int j = 0; j < FN; ++j) gb[j] += 2048;
      gbs += 256;
    };

    BStage b[S];
#pragma unroll
    for (int v = 0; v < S; ++v) {
      if (v > 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j) load_c1(v - 1, b[v - 1], j);
        load_s(v - 1, b[v - 1]);
      }
#pragma unroll
      for (int j = 0; j < FN; ++j) load_c0(v, b[v], j);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < PW; ++j) dma_a(v, v, j);
    }
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((S - 1) * kLoads));  // the scales and stage 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      a0[i] = ld16(row0 + i * 2048);
      aw[i] = *reinterpret_cast<const unsigned*>(srow + i * 512);
    }
    int kt = 0;
    for (; kt + S <= nk; kt += S) {
      stage(kt, std::integral_constant<int, 0>(), b, std::integral_constant<int, 0>());
      stage(kt + 1, std::integral_constant<int, 1>(), b, std::integral_constant<int, 0>());
      stage(kt + 2, std::integral_constant<int, 2>(), b, std::integral_constant<int, 0>());
      if constexpr (S == 4) stage(kt + 3, std::integral_constant<int, 3 % S>(), b, std::integral_constant<int, 0>());
    }
    static_assert(S == 3 || S == 4, "the loop above and the stages below");
    if (kt < nk) {
      stage(kt, std::integral_constant<int, 0>(), b, std::integral_constant<int, 1>());
      if (kt + 1 < nk) {
        stage(kt + 1, std::integral_constant<int, 1>(), b, std::integral_constant<int, 2>());
        if constexpr (S == 4) {
          if (kt + 2 < nk) stage(kt + 2, std::integral_constant<int, 2>(), b, std::integral_constant<int, 3 % S>());
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(0));
    __syncthreads();
  }

  // Epilogue.
  const int nw0 = n0 + wave * 32 * FN;
  if constexpr (GE) {
    const int n_out = p.N / 2;
#pragma unroll
    for (int j = 0; j < FN; j += 2) {
      const int n = nw0 + 32 * j, o = n / 2;  // value columns n .., gates n + 32 ..
      if (n >= p.N) break;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int m = m0 + 32 * i + r32;
        float v[16];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            v[4 * g + e] = acc[i][j][4 * g + e] * gelu_q(acc[i][j + 1][4 * g + e]);
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
        float mx = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = __builtin_elementwise_maximum(mx, fabsf(v[e]));  // a NaN stays
        const unsigned am = mx_abs_bits(mx);
        const auto sw2 = __builtin_amdgcn_permlane32_swap(am, am, false, false);
        const unsigned s = mx_scale<kMx4>(max(sw2[0], sw2[1]));
        // codes of g = 0, 1 and of g = 2, 3: four (16 bits) each
        const unsigned p01 = mx4_codes8(v, s), p23 = mx4_codes8(v + 8, s);
        const auto x = __builtin_amdgcn_permlane32_swap(p01, p23, false, false);
        const uint2 w = make_uint2(__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[1], x[0], 0x07060302u));
        // codes [row][64 bytes], scales [row][4] of the tile
        *reinterpret_cast<uint2*>(smem + (32 * i + r32) * 64 + wave * 16 + 8 * h) = w;
        if (h == 0) smem[BM * 64 + (32 * i + r32) * 4 + wave] = (unsigned char)s;
      }
    }
    if (p.out_f32) return;
    // whole rows of the tile: 64 bytes of codes by four lanes, four scale bytes
    __syncthreads();
    const int o0 = n0 / 2, cols = min(n_out - o0, 128);  // output columns of the tile, a multiple of 32
    unsigned char* const oc = static_cast<unsigned char*>(p.out) + o0 / 2;
    unsigned char* const os = static_cast<unsigned char*>(p.out) + (long long)p.M * (n_out / 2) + o0 / 32;
    const int t = threadIdx.x, q = t & 3;
#pragma unroll
    for (int e = 0; e < BM / 64; ++e) {
      const int row = 64 * e + (t >> 2), m = m0 + row;
      if (m < p.M && 32 * q < cols) *reinterpret_cast<uint4*>(oc + (long long)m * (n_out / 2) + 16 * q) = ld16(smem + row * 64 + 16 * q);
    }
    if (t < BM && m0 + t < p.M) {
      const unsigned w = *reinterpret_cast<const unsigned*>(smem + BM * 64 + t * 4);
      unsigned char* d = os + (long long)(m0 + t) * (n_out / 32);
      if (cols == 128 && n_out % 128 == 0)
        *reinterpret_cast<unsigned*>(d) = w;
      else
        for (int e = 0; e < cols / 32; ++e) d[e] = (unsigned char)(w >> (8 * e));
    }
  } else {
    // straight from registers: lanes trade pieces so that a store covers 64 bytes of each of 16 rows
    auto blocks = [&](auto store) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          if (nw0 + 32 * j < p.N) store(acc[i][j], m0 + 32 * i, nw0 + 32 * j);
    };
    if (!vec) {
      blocks([&](const f32x16& a, int mb, int n) {
        if (mb + r32 < p.M)
#pragma unroll
          for (int g = 0; g < 4; ++g) store_each(p, (long long)(mb + r32) * p.N + n + 8 * g + 4 * h, group_of(a, g));
      });
    } else if (p.out_f32) {
      blocks([&](const f32x16& a, int mb, int n) {
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
          f32x4 v = group_of(a, g), w = group_of(a, g + 1);
          rows16(v, w);
          float* d = static_cast<float*>(p.out) + (long long)(mb + r16) * p.N + n + 8 * g + c8;
          if (mb + r16 < p.M) *reinterpret_cast<f32x4*>(d) = v;
          if (mb + r16 + 16 < p.M) *reinterpret_cast<f32x4*>(d + 16ll * p.N) = w;
        }
      });
    } else {
      blocks([&](const f32x16& a, int mb, int n) {
        const f32x4 v0 = group_of(a, 0), v1 = group_of(a, 1), v2 = group_of(a, 2), v3 = group_of(a, 3);
        uint4 v = bf16_row8(reinterpret_cast<const float*>(&v0), reinterpret_cast<const float*>(&v1));
        uint4 w = bf16_row8(reinterpret_cast<const float*>(&v2), reinterpret_cast<const float*>(&v3));
        rows16(v, w);
        bf16* d = static_cast<bf16*>(p.out) + (long long)(mb + r16) * p.N + n + c16;
        if (mb + r16 < p.M) store_nt(d, v);
        if (mb + r16 + 16 < p.M) store_nt(d + 16ll * p.N, w);
      });
    }
  }
}

// Workgroup wg of `units` tiles, in contiguous ranges per XCD.
__device__ __forceinline__ int xcd_unit(int wg, int units) {
  const int xcd = wg % kXcds, idx = wg / kXcds;
  return xcd * (units / kXcds) + min(xcd, units % kXcds) + idx;
}

template <int FM, int FN, int S, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_mx4_kernel(GemmMx4Params p, int mt, int nt) {
  const int u = xcd_unit(blockIdx.x, mt * nt);
  mx4_tile<FM, FN, S, NW, false>(p, (u % mt) * 32 * FM, (u / mt) * 32 * FN * NW);
}

// GEGLU: the first nt column bands in mt tiles of 128 rows, then bands in mt2 tiles of 64 rows.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_mx4_geglu_kernel(GemmMx4Params p, int mt, int nt, int mt2) {
  const int big = mt * nt, wg = blockIdx.x;
  if (wg < big) {
    const int u = xcd_unit(wg, big);
    mx4_tile<4, 2, 3, 4, true>(p, (u % mt) * 128, (u / mt) * 256);
  } else {
    const int u = xcd_unit(wg - big, gridDim.x - big);
    mx4_tile<2, 2, 4, 4, true>(p, (u % mt2) * 64, (nt + u / mt2) * 256);
  }
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
    if (m >= p.M) return;
    const int n = n0 + c;
    if (p.bias)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[0][e] += p.bias[n + e];
    if (p.resid) v[0] += resid4(p, (long long)m * p.N + n);
    store_each(p, (long long)m * p.N + n, v[0]);
  }
}

// A launch has less than 2^32 threads.
bool fits(long long groups, int threads) { return groups * threads <= 0xffffffffll; }
unsigned grid_of(long long groups, int threads) {
  DN_CHECK(fits(groups, threads), "gemm_mx4: too many tiles for one launch");
  return static_cast<unsigned>(groups);
}

template <int FM, int FN, int S, int NW> void launch_tile(const GemmMx4Params& p, hipStream_t s) {
  static_assert(S * stage_bytes<FM>() + scale_lds(32 * FM, kScaleK) <= 64 * 1024, "no attribute needed, two workgroups per CU");
  const size_t lds = tile_lds<FM, S>(p.K);
  const int mt = ceil_div(p.M, 32 * FM), nt = ceil_div(p.N, 32 * FN * NW);
  const unsigned grid = grid_of((long long)mt * nt, 64 * NW);
  hipLaunchKernelGGL((gemm_mx4_kernel<FM, FN, S, NW>), dim3(grid), dim3(64 * NW), lds, s, p, mt, nt);
}

// GEGLU with the last `small` column bands in tiles of 64 rows.
void launch_geglu(const GemmMx4Params& p, int small, hipStream_t s) {
  static_assert(3 * stage_bytes<4>() + scale_lds(128, kScaleK) <= 64 * 1024 && 4 * stage_bytes<2>() + scale_lds(64, kScaleK) <= 64 * 1024,
                "no attribute needed, two workgroups per CU");
  const size_t lds = std::max(tile_lds<4, 3>(p.K), tile_lds<2, 4>(p.K));
  const int mt = ceil_div(p.M, 128), mt2 = ceil_div(p.M, 64), nt = ceil_div(p.N, 256) - small;
  const unsigned grid = grid_of((long long)mt * nt + (long long)mt2 * small, 256);
  hipLaunchKernelGGL(gemm_mx4_geglu_kernel, dim3(grid), dim3(256), lds, s, p, mt, nt, mt2);
}

template <bool GE> void launch_rows(const GemmMx4Params& p, hipStream_t s) {
  constexpr int NW = 8;
  const int nt = p.N / (GE ? 64 : 32), mt = ceil_div(p.M, 32);
  const unsigned grid = grid_of((long long)mt * nt, 64 * NW);
  hipLaunchKernelGGL((gemm_mx4_rows_kernel<NW, GE>), dim3(grid), dim3(64 * NW), 0, s, p, nt);
}

}  // namespace

bool gemm_mx4_layout(int N, int K) {
  return N >= 32 && N % 32 == 0 && N <= kMaxDim && K >= kStageK && K % kStageK == 0 && K <= kMaxDim;
}
size_t gemm_mx4_code_bytes(int N, int K) { return (size_t)N * (K / 2); }
size_t gemm_mx4_bytes(int N, int K) {
  return (size_t)N * (K / 2) + (size_t)((N + 63) / 64 * 64) * (K / 32) + kBSpare;
}

void gemm_mx4_check(const GemmMx4Params& p) {
  DN_CHECK(gemm_mx4_layout(p.N, p.K) && p.M >= 1, "gemm_mx4: N % 32 == 0 and K % 128 == 0, both at most 2^22, needed");
  DN_CHECK(p.a && p.b && p.out, "gemm_mx4: null operand");
  // the largest tiles have to fit a launch; M is then at most 2^31 - 128, and no row number of a tile overflows
  DN_CHECK(fits((long long)ceil_div(p.M, 128) * ceil_div(p.N, 256), 256), "gemm_mx4: too many tiles for one launch");
  DN_CHECK(!p.geglu || (p.N % 64 == 0 && !p.resid), "gemm_mx4: GEGLU takes value / gate pairs of 64 columns, no residual");
  DN_CHECK(((uintptr_t)p.a | (uintptr_t)p.b) % 16 == 0 && (uintptr_t)p.bias % 4 == 0, "gemm_mx4: operands must be 16-byte aligned");
  DN_CHECK((uintptr_t)p.out % (p.out_f32 ? 4 : p.geglu ? 16 : 2) == 0 && (uintptr_t)p.resid % (p.resid_f32 ? 4 : 2) == 0,
           "gemm_mx4: misaligned output or residual");
}

namespace {

// Estimated time in microseconds of tiles of bm x bn on `cus` CUs: the busiest CU works off its tiles in pairs,
// two workgroups side by side, and a last one alone. Per stage a pair (`two`) costs about what its matrix
// instructions do, a workgroup alone (`one`) somewhat more than half of it, as waits are not covered; `fixed`
// is a tile's start and end. The constants are fitted to measured times of 20 shapes, M 100 .. 32768, N 160 ..
// 5120, K 640 .. 5120.
// A shape whose tiles do not fit a launch costs more than any other.
float tile_cost(int M, int N, int K, int cus, int bm, int bn, int threads, float one, float two, float fixed) {
  const long long tiles = (long long)ceil_div(M, bm) * ceil_div(N, bn), per_cu = (tiles + cus - 1) / cus;
  if (!fits(tiles, threads)) return std::numeric_limits<float>::max();
  return K / kStageK * (one * (per_cu % 2) + two * (per_cu / 2)) + fixed * per_cu;
}

}  // namespace

Mx4Plan gemm_mx4_plan(int M, int N, int K, bool geglu, int cus) {
  // Two rows kernel workgroups of 8 waves per CU: as long as all of its 32 x 32 blocks are resident at once, it
  // wins, since no tile fills the chip then (200 x 1280, K = 5120: 9.4 us, the 64 x 128 tiles 11.0; 77 x 5120
  // GEGLU, K = 1280: 5.8 and 8.6); with more it loses to re-reading B per 32 rows (128 x 5120, K = 2560: 8.4
  // and 6.2).
  const int pair = geglu ? 64 : 32;
  if ((long long)ceil_div(M, 32) * (N / pair) <= 2ll * cus) return Mx4Plan{32, pair, 0};
  if (geglu) {
    // 64-row tiles while all of them run at once, each on a CU of its own (300 x 2560, K = 640: 5.6 us, 128 rows
    // 7.2); with more, 128 rows are faster (8192 x 2560, K = 640: 33.7 and 29.0). After whole rounds of two tiles
    // per CU, a last one of half the CUs or fewer runs as 64-row tiles (2048 x 5120, K = 1280: 24.8 and 22.4 us; with
    // all CUs in it there is nothing to gain: 8192 x 2560, K = 640: 28.8 and 29.5), as whole column bands: also where
    // a band is longer than that round (33024 x 256, K = 640: 15.6 and 15.0 us), unless that takes in every band
    // (65664 x 128, K = 640: 15.8 and 17.0) or more tiles than a launch holds.
    const int mt = ceil_div(M, 128), mt2 = ceil_div(M, 64), nt = ceil_div(N, 256);
    const long long tail = (long long)mt * nt % (2 * cus), bands = (tail + mt - 1) / mt;
    int small = 0;
    if ((long long)mt2 * nt <= cus)
      small = nt;
    else if (2 * tail <= cus && bands < nt && fits(mt * (nt - bands) + mt2 * bands, 256))
      small = (int)bands;
    return Mx4Plan{128, 256, small};
  }
  // 128 x 256 does most work per byte from LDS and L2 (4096^3 39.8 us, 64 x 128 58, 64 x 160 68); the smaller
  // ones win where they even out the tiles per CU (2048 x 1280, K = 5120: 24.5, 19.8, 15.0; 700 x 1280,
  // K = 2560: 16.0, 8.4, 9.2)
  const float big = tile_cost(M, N, K, cus, 128, 256, 256, 0.43f, 0.86f, 4.2f);
  const float small = tile_cost(M, N, K, cus, 64, 128, 256, 0.18f, 0.39f, 1.2f);
  const float five = tile_cost(M, N, K, cus, 64, 160, 320, 0.21f, 0.48f, 2.5f);
  if (big <= small && big <= five) return Mx4Plan{128, 256, 0};
  return small <= five ? Mx4Plan{64, 128, 0} : Mx4Plan{64, 160, 0};
}

void gemm_mx4(const GemmMx4Params& p, int cus, hipStream_t s) {
  gemm_mx4_check(p);
  const Mx4Plan g = gemm_mx4_plan(p.M, p.N, p.K, p.geglu != 0, cus);
  if (g.bm == 32)
    p.geglu ? launch_rows<true>(p, s) : launch_rows<false>(p, s);
  else if (p.geglu)
    launch_geglu(p, g.small, s);
  else if (g.bm == 128)
    launch_tile<4, 2, 3, 4>(p, s);
  else if (g.bn == 128)
    launch_tile<2, 1, 4, 4>(p, s);
  else
    launch_tile<2, 1, 4, 5>(p, s);
  DN_HIP(hipGetLastError());
}

}  // namespace dn
