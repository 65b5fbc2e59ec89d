// Packed sequences: rows of several requests of different lengths back to back, and the rows of a
// cache that belong to each of them; the parameter blocks of the kernels that work on them.
//
// Sequence s of n has the rows [q_start[s], q_start[s + 1]) of the packed tensors and the rows
// [kv_start[s], kv_start[s] + kv_len[s]) of the key and value tensors; its last packed row belongs to
// its last key. The arrays are device memory, so kernels check what they read there: a sequence
// whose rows lie outside the tensors is skipped, its outputs are left as they were.
#pragma once

#include "kernels.h"

namespace dn {

struct Sequences {
  int n = 0;                            // 0: one row after another, row t of the keys is row t
  const int* q_start = nullptr;         // [n + 1], non-decreasing
  const long long* kv_start = nullptr;  // [n]
  const int* kv_len = nullptr;          // [n]
};

// Whether attention takes a sequence: packed rows [a, b) of T, `len` keys from k0 of kv_rows. Key positions, a tile past the last
// one among them, are counted in 32 bits.
constexpr unsigned kMaxKeys = 0x7fffffff - 65536;
__host__ __device__ __forceinline__ bool sequence_attends(int a, int b, long long T, int len, long long k0, long long kv_rows) {
  return a >= 0 && b > a && b <= T && static_cast<unsigned>(len) <= kMaxKeys && k0 >= 0 && k0 <= kv_rows - len;
}

// Largest s in [0, n) with first(s) <= x for a non-decreasing first, or -1, by the G lanes of a lane
// group (G a power of two, the group's lanes converged): every step probes G places, so up to 64
// sequences take one or two dependent loads. It ends, in bounds, for any values of `first`.
template <int G, typename F> __device__ __forceinline__ int search_group(int n, long long x, const F& first) {
  const int lane = threadIdx.x & 63, c = lane & (G - 1);
  int lo = 0, cnt = n;  // the answer lies in [lo - 1, lo + cnt)
  while (cnt > 0) {
    const int step = (cnt + G - 1) / G;
    const int i = (c + 1) * step - 1;  // the last of block c
    const bool in = i < cnt && first(lo + i) <= x;
    const unsigned long long m = __ballot(in) >> (lane & ~(G - 1));
    const int k = G == 64 ? __popcll(m) : __popcll(m & ((1ull << (G & 63)) - 1));
    const int gone = k * step;
    lo += gone;
    cnt = min(step - 1, cnt - gone);
  }
  return lo - 1;
}

// ---------------------------------------------------------------- rotation
constexpr int kRopeMaxAxes = 4;
constexpr int kRopeMaxDim = 256;
constexpr int kRopePairs = kRopeMaxDim / 2;

// Entry i of a rotation table: turns per position of pair i as a 64-bit fraction, and its axis. Pairs
// past the rotated width turn by nothing.
struct RopeEntry {
  unsigned lo, hi;
  int axis, zero;
};
struct RopeTableParams {
  unsigned long long turn[kRopePairs];
  unsigned char axis[kRopePairs];
};
// freq radians in turns: the fraction, in units of 2^-64, within one of them (|freq| <= 2^16).
unsigned long long rope_turn(double freq);
void rope_table(const RopeTableParams& p, void* table, hipStream_t s);

// Rotates (and, with gains, RMS-normalises first) the heads of packed rows; copies the heads of v.
struct RotaryParams {
  const void* q = nullptr;
  const void* k = nullptr;
  const void* v = nullptr;
  void* qo = nullptr;
  void* ko = nullptr;
  void* vo = nullptr;
  long long ldq = 0, ldk = 0, ldv = 0, ldqo = 0, ldko = 0, ldvo = 0;
  long long T = 0, kv_rows = 0;
  int heads = 0, kv_heads = 0, v_heads = 0, D = 0;
  const float* gq = nullptr;
  const float* gk = nullptr;
  float eps = 0.f;
  const RopeEntry* table = nullptr;
  const int* pos = nullptr;
  int n_axes = 0, half = 0;  // half: rotated pairs
  bool halves = false;
  Sequences seqs;
};
template <typename T> void rotary(const RotaryParams& p, hipStream_t s);

// ---------------------------------------------------------------- attention
struct PackedAttnParams {
  const void* q = nullptr;
  const void* k = nullptr;
  const void* v = nullptr;
  void* o = nullptr;
  long long ldq = 0, ldk = 0, ldv = 0, ldo = 0;
  long long T = 0, kv_rows = 0;
  int heads = 0, kv_heads = 0, max_kv = 0;
  bool causal = false;
  float scale_log2 = 0.f;  // scale * log2(e)
  void* ws = nullptr;
  Sequences seqs;
};
bool attention_packed_dim(int D);
// How a call is run: a function of sizes alone (of the 256 CUs of the one GPU this is built for), so that the workspace does
// not depend on the device at hand.
enum PackedJoin { kJoinNone, kJoinRows, kJoinUnits };
struct PackedPlan {
  int waves = 0;   // of 32 rows, of a tile (fp32: four); 0: units of 32 rows (narrow)
  int most = 0;    // narrow: most workgroups over all key blocks, whatever kv_rows (0: one per unit)
  int shares = 0;  // and those that are launched
  int join = kJoinNone, split = 1;  // who joins a divided call's parts, workgroups of join_rows_kernel for four shares
};
PackedPlan attention_packed_plan(int elem, int D, long long T, int heads, int kv_heads, int n, int max_kv, long long kv_rows);
// Workspace bytes (0: none).
size_t attention_packed_bytes(int elem, long long T, int heads, int kv_heads, int D, int n, int max_kv);
template <typename T> void attention_packed(const PackedAttnParams& p, int D, hipStream_t s);

}  // namespace dn
