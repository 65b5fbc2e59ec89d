// Rotary positions and the RMS norm of query and key heads (gfx950).
//
// A head x of D values is rotated in pairs: (a, b) -> (a cos t - b sin t, a sin t + b cos t), pair i by
// the angle t = pos[axis_i] f_i. Before that a head may be normalised: x rsqrt(mean x^2 + eps) gain.
//
// Angles: positions of long contexts times a frequency lose their fraction of a turn in 32 bits (at
// position 10^6 an fp32 product is off by 0.06 radians). The table holds f_i / 2 pi as a 64-bit
// binary fraction of a turn; its product with the position modulo 2^64 is the angle modulo one turn
// exactly (to 2^-64 turns per position, at any frequency), of which the top 32 bits are kept. Sine and cosine of an
// eighth of a turn either way are Taylor polynomials (truncated below 2^-29), so all of an fp32
// result's error is rounding.
//
// Bound by memory: every value is read and written once. A group of G lanes holds one head, eight
// values a lane: four pairs, neighbours (DN_ROPE_PAIRS) or half the rotated width apart
// (DN_ROPE_HALVES), so no pair and no norm leaves the group. The group takes several heads of one row
// after another, which share the row's angles. 32,760 rows of 20 heads of 128 in fp32 122 us, 20 + 20 in bf16 with their norms
// 120 us: 5.5 TB/s of reads and writes, where a large copy moves 5.1. Of 80 values a group of 16 lanes uses 10: 3.8 TB/s.
#include <algorithm>
#include <cmath>

#include "packed.h"

namespace dn {
namespace {

constexpr int kThreads = 256;

__global__ void rope_table_kernel(RopeTableParams p, RopeEntry* t) {
  const int i = threadIdx.x;
  t[i] = RopeEntry{(unsigned)p.turn[i], (unsigned)(p.turn[i] >> 32), p.axis[i], 0};
}

// cos and sin of u / 2^32 turns.
__device__ __forceinline__ void turn_sincos(unsigned u, float& c, float& s) {
  const unsigned quarter = (u + 0x20000000u) >> 30;
  const float x = (float)(int)(u - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float z = x * x;
  const float ps = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float pc = 1.f + z * (-1.f / 2 + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 - z * (1.f / 3628800)))));
  c = quarter & 1 ? ps : pc;
  s = quarter & 1 ? pc : ps;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter >= 2) s = -s;
}

template <typename T> struct Quad;  // four values of a row as they are loaded
template <> struct Quad<float> {
  typedef uint4 raw;
  __device__ static __forceinline__ void get(raw r, float* v) {
    v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
  }
  __device__ static __forceinline__ raw put(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Quad<bf16> {
  typedef uint2 raw;
  __device__ static __forceinline__ void get(raw r, float* v) {
    v[0] = __uint_as_float(r.x << 16), v[1] = __uint_as_float(r.x & 0xffff0000u);
    v[2] = __uint_as_float(r.y << 16), v[3] = __uint_as_float(r.y & 0xffff0000u);
  }
  __device__ static __forceinline__ raw put(const float* v) {
    const bf16x4 r = {static_cast<bf16>(v[0]), static_cast<bf16>(v[1]), static_cast<bf16>(v[2]), static_cast<bf16>(v[3])};
    return __builtin_bit_cast(uint2, r);
  }
};

// Sum over the lanes of a group, in every lane.
template <int G> __device__ __forceinline__ float group_sum(float v) {
  v = dpp_add<0xb1, 0xf>(v);               // quad_perm [1, 0, 3, 2]
  v = dpp_add<0x4e, 0xf>(v);               // quad_perm [2, 3, 0, 1]
  if (G >= 8) v = dpp_add<0x141, 0xf>(v);  // row_half_mirror
  if (G >= 16) v = dpp_add<0x140, 0xf>(v); // row_mirror
  if (G >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

// Maximum over the lanes of a group, in every lane.
template <int G> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = 1; o < G; o *= 2) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

template <typename T, int G, bool HALVES, bool NORM, int HC>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p, int chunks, int width) {
  typedef typename Quad<T>::raw raw;
  const int c = threadIdx.x & (G - 1);
  const bool lane_in = 8 * c < p.D;
  // first values of the lane's two quads
  const bool turned = HALVES && 4 * c < p.half;
  const int a0 = lane_in ? (turned ? 4 * c : 8 * c) : 0;
  const int b0 = turned ? p.half + 4 * c : a0 + 4;
  const int all = p.heads + p.kv_heads + p.v_heads;
  const long long units = p.T * chunks, step = (long long)gridDim.x * (kThreads / G);
  unsigned tl[4], th[4];
  int ax[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const RopeEntry e = p.table[min(4 * c + j, kRopePairs - 1)];
    tl[j] = e.lo, th[j] = e.hi, ax[j] = min(e.axis, p.n_axes - 1);
  }
  float gq[8], gk[8];
  if (NORM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = e < 4 ? a0 + e : b0 + e - 4;
      gq[e] = p.gq[d];
      gk[e] = p.gk[d];
    }
  }
  for (long long u = (long long)blockIdx.x * (kThreads / G) + threadIdx.x / G; u < units; u += step) {
    const long long t = u / chunks;
    const int h0 = (int)(u - t * chunks) * width, h1 = min(h0 + width, all);  // width <= HC
    // the rows of keys and values this one goes to
    long long row = t;
    if (p.seqs.n) {
      const int s = search_group<G>(p.seqs.n, t, [&](int i) { return (long long)p.seqs.q_start[i]; });
      if (s < 0) continue;
      const int q0 = p.seqs.q_start[s], q1 = p.seqs.q_start[s + 1], len = p.seqs.kv_len[s];
      const long long k0 = p.seqs.kv_start[s];
      if (q0 < 0 || t < q0 || t >= q1 || q1 > p.T || len < q1 - q0 || k0 < 0 || k0 > p.kv_rows - len) continue;
      row = k0 + len - (q1 - t);
    }
    raw xa[HC], xb[HC];
    if (lane_in) {
#pragma unroll
      for (int j = 0; j < HC; ++j) {
        const int h = h0 + j;
        if (h < h1) {
          const int hk = h - p.heads, hv = hk - p.kv_heads;
          const T* src = hk < 0   ? static_cast<const T*>(p.q) + t * p.ldq + h * p.D
                         : hv < 0 ? static_cast<const T*>(p.k) + t * p.ldk + hk * p.D
                                  : static_cast<const T*>(p.v) + t * p.ldv + hv * p.D;
          xa[j] = *reinterpret_cast<const raw*>(src + a0);
          xb[j] = *reinterpret_cast<const raw*>(src + b0);
        }
      }
    }
    float cs[4], sn[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned at = (unsigned)p.pos[t * p.n_axes + ax[j]];
      // bits 32 .. 63 of the table's 64 times the position: the position's bits as an unsigned number
      // are 2^32 more than a negative position, whose surplus is taken off again
      unsigned turn = th[j] * at + __umulhi(tl[j], at);
      if ((int)at < 0) turn -= tl[j];
      turn_sincos(turn, cs[j], sn[j]);
    }
#pragma unroll
    for (int j = 0; j < HC; ++j) {
      const int h = h0 + j;
      if (h >= h1) break;
      const int hk = h - p.heads, hv = hk - p.kv_heads;
      T* dst = hk < 0   ? static_cast<T*>(p.qo) + t * p.ldqo + h * p.D
               : hv < 0 ? static_cast<T*>(p.ko) + row * p.ldko + hk * p.D
                        : static_cast<T*>(p.vo) + row * p.ldvo + hv * p.D;
      if (hv < 0) {
        float v[8];
        Quad<T>::get(xa[j], v);
        Quad<T>::get(xb[j], v + 4);
        if (NORM) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
          ss = group_sum<G>(lane_in ? ss : 0.f);
          float mean = ss / p.D + p.eps;
          // Squares of large or tiny values leave 32 bits (past 1.8e19; below 1e-23 where eps is no larger): the head, and the
          // root of eps with it, is brought to one by a power of two first. A group takes one side; the usual one does not pay
          // (48 tokens 3.63 us, without 3.60; 32,760 tokens no difference), but it would for a root here or a second look at
          // the heads behind the loop, which keep more registers (3.69, and 137 us for 124).
          const bool odd = !(mean >= 0x1p-80f && mean <= 0x1p120f);
          if (__builtin_expect(__any(odd), 0)) if (odd) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
            // (the exponent of an infinity or of zero is 0)
            float eps = p.eps;
            asm volatile("" : "+v"(eps));  // (or its root is taken ahead of the loop, in every call)
            const int root = eps > 0.f ? (__builtin_amdgcn_frexp_expf(eps) + 1) >> 1 : -1000;
            const int down = max(__builtin_amdgcn_frexp_expf(group_max<G>(lane_in ? top : 0.f)), root);
            ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = ldexpf(v[e], -down);
              ss = fmaf(v[e], v[e], ss);
            }
            mean = group_sum<G>(lane_in ? ss : 0.f) / p.D + ldexpf(eps, -2 * down);
          }
          const float r = 1.f / sqrtf(mean);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = v[e] * r * (hk < 0 ? gq[e] : gk[e]);
        }
        float y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = HALVES ? e : 2 * e, k = HALVES ? e + 4 : 2 * e + 1;
          // pairs past the rotated width pass as they are, an infinity among them too
          const bool on = 4 * c + e < p.half;
          y[i] = on ? fmaf(v[i], cs[e], -(v[k] * sn[e])) : v[i];
          y[k] = on ? fmaf(v[i], sn[e], v[k] * cs[e]) : v[k];
        }
        xa[j] = Quad<T>::put(y);
        xb[j] = Quad<T>::put(y + 4);
      }
      if (lane_in) {
        *reinterpret_cast<raw*>(dst + a0) = xa[j];
        *reinterpret_cast<raw*>(dst + b0) = xb[j];
      }
    }
  }
}

template <typename T, int G, bool HALVES, bool NORM, int HC> void launch(const RotaryParams& p, hipStream_t s) {
  const int all = p.heads + p.kv_heads + p.v_heads;
  const int chunks = (all + HC - 1) / HC, width = (all + chunks - 1) / chunks;
  const long long blocks = (p.T * chunks + kThreads / G - 1) / (kThreads / G);
  hipLaunchKernelGGL((rotary_kernel<T, G, HALVES, NORM, HC>), dim3((unsigned)std::min(blocks, 1ll << 20)), dim3(kThreads), 0, s,
                     p, chunks, width);
  DN_HIP(hipGetLastError());
}

// Heads a group takes in turn, by the waves that one head each would make: few rows want every lane at once, many share
// angles and the search for the sequence and keep more loads in flight. Measured, us, of 1, 2, 4 and 8 heads:
// 576 waves (48 tokens, 32 + 8 + 8 heads of 128) 3.6, 3.9, 4.6, 6.1; 2,250 (750 tokens, 4 + 1 + 1 of 256, fp32) 5.2, 4.8, 5.1,
// 6.1; 10,240 (8192 tokens, 10 of 64) 7.9, 6.0, 5.5, 5.9; 327,600 (32,760 tokens, 20 + 20 of 128) 212, 141, 123, 126; up to
// eight heads in all in one piece (4 + 1 + 1 of 80, 19 k tokens) 33.0, 22.9, 21.1, 16.5.
template <typename T, int G, bool HALVES, bool NORM> void launch_heads(const RotaryParams& p, hipStream_t s) {
  const int all = p.heads + p.kv_heads + p.v_heads;
  const long long waves = p.T * all * G / 64;
  if (waves >= 8192 && all > 4 && all <= 8)
    launch<T, G, HALVES, NORM, 8>(p, s);
  else if (waves >= 4096)
    launch<T, G, HALVES, NORM, 4>(p, s);
  else if (waves >= 1024)
    launch<T, G, HALVES, NORM, 2>(p, s);
  else
    launch<T, G, HALVES, NORM, 1>(p, s);
}

template <typename T, int G> void launch_kind(const RotaryParams& p, hipStream_t s) {
  if (p.halves)
    p.gq ? launch_heads<T, G, true, true>(p, s) : launch_heads<T, G, true, false>(p, s);
  else
    p.gq ? launch_heads<T, G, false, true>(p, s) : launch_heads<T, G, false, false>(p, s);
}

}  // namespace

// freq = m 2^e with 53 bits of m, times 128 bits of 1 / (2 pi), in integers: the whole turns drop off as bits past the
// 64th. In 64 bits of a long double they would take the place of the fraction's last bits, and 2 pi's own error grows with the
// frequency: 2^-21 of a turn at 3 10^4 radians a position and position 2^31, where this is within 2^-32.
unsigned long long rope_turn(double freq) {
  typedef unsigned __int128 u128;
  int e;
  const unsigned long long m = static_cast<unsigned long long>(std::ldexp(std::frexp(std::fabs(freq), &e), 53));
  e -= 53;
  const unsigned long long hi = 0x28be60db9391054aull, lo = 0x7f09d5f47d4d3770ull;  // 2^128 / (2 pi)
  const u128 top = static_cast<u128>(m) * hi + (static_cast<u128>(m) * lo >> 64);   // m 2^64 / (2 pi)
  const int drop = -e;  // at least 36 by the bound of freq
  if (drop >= 128) return 0;
  const unsigned long long turn = static_cast<unsigned long long>(top >> drop) + static_cast<unsigned long long>(top >> (drop - 1) & 1);
  return freq < 0 ? 0 - turn : turn;
}

void rope_table(const RopeTableParams& p, void* table, hipStream_t s) {
  hipLaunchKernelGGL(rope_table_kernel, dim3(1), dim3(kRopePairs), 0, s, p, static_cast<RopeEntry*>(table));
  DN_HIP(hipGetLastError());
}

template <typename T> void rotary(const RotaryParams& p, hipStream_t s) {
  if (p.D <= 32)
    launch_kind<T, 4>(p, s);
  else if (p.D <= 64)
    launch_kind<T, 8>(p, s);
  else if (p.D <= 128)
    launch_kind<T, 16>(p, s);
  else
    launch_kind<T, 32>(p, s);
}

template void rotary<float>(const RotaryParams&, hipStream_t);
template void rotary<bf16>(const RotaryParams&, hipStream_t);

}  // namespace dn
