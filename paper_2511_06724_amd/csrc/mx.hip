// Microscaled rows (mx.h): quantisation of rows as they are written (in order, or scattered into
// the slots of a cache), reading back, and the packing of 4-bit weights (gfx950).
//
// Both directions move bytes and do little else: a thread handles eight values (16 or 32 bytes of
// the source, 4 or 8 of codes), four neighbouring lanes a block, whose largest magnitude meets in
// two DPP steps. Every thread issues the loads of its kUnroll groups before it uses the first.
#include <algorithm>

#include "mx.h"

namespace dn {
namespace {

constexpr int kUnroll = 4;
constexpr int kGroups = 256 * kUnroll;  // groups of eight values per workgroup
// Rows per call up to which a row looks for a later row of the same slot by itself; more are
// claimed by kernels of their own.
constexpr int kScanRows = 32;
constexpr int kClaimOneGroup = 16384;   // rows one workgroup claims in a single launch

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

// Elements [c, c + 8) of a row, zero past `cols`.
__device__ __forceinline__ void load8(const float* x, long long c, long long cols, bool vec, float* v) {
  if (vec && c + 8 <= cols) {
    const float4 a = *reinterpret_cast<const float4*>(x + c), b = *reinterpret_cast<const float4*>(x + c + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? x[c + e] : 0.f;
  }
}
template <typename H, typename H8>
__device__ __forceinline__ void load8_16(const H* x, long long c, long long cols, bool vec, float* v) {
  if (vec && c + 8 <= cols) {
    const H8 a = *reinterpret_cast<const H8*>(x + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(a[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? static_cast<float>(x[c + e]) : 0.f;
  }
}
__device__ __forceinline__ void load8(const bf16* x, long long c, long long cols, bool vec, float* v) {
  load8_16<bf16, bf16x8>(x, c, cols, vec, v);
}
__device__ __forceinline__ void load8(const _Float16* x, long long c, long long cols, bool vec, float* v) {
  load8_16<_Float16, half8>(x, c, cols, vec, v);
}

__device__ __forceinline__ unsigned amax8(const float* v) {
  unsigned a = mx_abs_bits(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) a = max(a, mx_abs_bits(v[e]));
  return a;
}

// Row and first value of each of a thread's groups; the row index is 64-bit, the offset in a
// workgroup's rows 32-bit (one 64-bit division per workgroup).
struct GroupPos {
  long long row;
  unsigned g;  // group of the row
};
struct GroupMap {
  long long row0;
  unsigned off, per_row;
  __device__ GroupMap(long long base, unsigned groups_per_row) : per_row(groups_per_row) {
    row0 = base / groups_per_row;
    off = (unsigned)(base - row0 * groups_per_row);
  }
  __device__ GroupPos at(unsigned local) const {
    const unsigned t = off + local;
    const unsigned q = per_row >= kGroups ? (t >= per_row ? 1u : 0u) : t / per_row;
    return GroupPos{row0 + q, t - q * per_row};
  }
};

struct StoreParams {
  const void* x;
  long long ldx, rows, cols;
  unsigned blocks;          // of a row
  int vec;                  // rows can be read 16 bytes at a time
  const long long* slots;   // nullptr: row j goes to slot j
  long long n_slots;
  const int* owner;         // nullptr: rows look for later rows of their slot themselves
  unsigned char* codes;
  unsigned char* scales;
};

// Destination of row j, -1 for none (a slot outside the table, or a later row of the same slot).
__device__ __forceinline__ long long store_slot(const StoreParams& p, long long j) {
  if (!p.slots) return j;
  const long long s = p.slots[j];
  if (s < 0 || s >= p.n_slots) return -1;
  if (p.owner) return p.owner[s] == (int)j ? s : -1;
  for (long long k = j + 1; k < p.rows; ++k)
    if (p.slots[k] == s) return -1;
  return s;
}

template <int FMT, typename T> __global__ __launch_bounds__(256) void mx_store_kernel(StoreParams p) {
  const unsigned G = p.blocks * 4;
  const long long base = (long long)blockIdx.x * kGroups, total = p.rows * G;
  const GroupMap map(base, G);
  float v[kUnroll][8];
  GroupPos pos[kUnroll];
  long long slot[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const unsigned local = u * 256 + threadIdx.x;
    slot[u] = -1;
    if (base + local >= total) continue;
    pos[u] = map.at(local);
    load8(static_cast<const T*>(p.x) + pos[u].row * p.ldx, 8ll * pos[u].g, p.cols, p.vec, v[u]);
    slot[u] = store_slot(p, pos[u].row);
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (slot[u] < 0) continue;  // the four lanes of a block together
    const unsigned s = mx_scale<FMT>(quad_umax(amax8(v[u])));
    const long long block = slot[u] * p.blocks + pos[u].g / 4;
    if constexpr (FMT == kMx4) {
      *reinterpret_cast<unsigned*>(p.codes + block * 16 + (pos[u].g & 3) * 4) = mx4_codes8(v[u], s);
    } else {
      *reinterpret_cast<uint2*>(p.codes + block * 32 + (pos[u].g & 3) * 8) =
          make_uint2(mx8_codes4(v[u], s), mx8_codes4(v[u] + 4, s));
    }
    if ((pos[u].g & 3) == 0) p.scales[block] = (unsigned char)s;
  }
}

// The last row of a slot owns it: the owner word of every slot in use is cleared, then takes the
// largest row index. PHASE 0: both, in one workgroup; 1, 2: one of them over a grid.
template <int PHASE>
__global__ __launch_bounds__(1024) void mx_claim_kernel(const long long* slots, long long rows, long long n_slots, int* owner) {
  const long long i0 = blockIdx.x * (long long)blockDim.x + threadIdx.x, step = (long long)gridDim.x * blockDim.x;
  if constexpr (PHASE != 2) {
    for (long long j = i0; j < rows; j += step) {
      const long long s = slots[j];
      if (s >= 0 && s < n_slots) owner[s] = -1;
    }
  }
  if constexpr (PHASE == 0) {
    __threadfence();
    __syncthreads();
  }
  if constexpr (PHASE != 1) {
    for (long long j = i0; j < rows; j += step) {
      const long long s = slots[j];
      if (s >= 0 && s < n_slots) atomicMax(owner + s, (int)j);
    }
  }
}

struct FetchParams {
  const unsigned char* codes;
  const unsigned char* scales;
  long long n_slots, rows, cols;
  unsigned blocks;
  const long long* idx;  // nullptr: row j is slot j
  float* y;
  long long ldy;
  int vec;
};

template <int FMT> __global__ __launch_bounds__(256) void mx_fetch_kernel(FetchParams p) {
  const unsigned G = p.blocks * 4;
  const long long base = (long long)blockIdx.x * kGroups, total = p.rows * G;
  const GroupMap map(base, G);
  GroupPos pos[kUnroll];
  bool on[kUnroll];
  uint2 code[kUnroll];
  unsigned s[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const unsigned local = u * 256 + threadIdx.x;
    on[u] = base + local < total;
    if (!on[u]) continue;
    pos[u] = map.at(local);
    const long long slot = p.idx ? p.idx[pos[u].row] : pos[u].row;
    on[u] = slot >= 0 && slot < p.n_slots;
    if (!on[u]) continue;
    const long long block = slot * p.blocks + pos[u].g / 4;
    if constexpr (FMT == kMx4)
      code[u].x = *reinterpret_cast<const unsigned*>(p.codes + block * 16 + (pos[u].g & 3) * 4);
    else
      code[u] = *reinterpret_cast<const uint2*>(p.codes + block * 32 + (pos[u].g & 3) * 8);
    s[u] = p.scales[block];
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (!on[u]) continue;
    float v[8];
    if constexpr (FMT == kMx4) {
      mx4_values8(code[u].x, s[u], v);
    } else {
      mx8_values4(code[u].x, s[u], v);
      mx8_values4(code[u].y, s[u], v + 4);
    }
    const long long c = 8ll * pos[u].g;
    float* y = p.y + pos[u].row * p.ldy + c;
    if (p.vec && c + 8 <= p.cols) {
      *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(y + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      for (int e = 0; e < 8; ++e)
        if (c + e < p.cols) y[e] = v[e];
    }
  }
}

// A weight matrix in the operand order of the 32x32x64 matrix-core step (gemm_mx4.hip): per 32 rows
// and 64-deep step the 64 lanes' 16 bytes (lane: row % 32, plus 32 for the second block of the step),
// and per 64 rows and 128 deep the lanes' four scale bytes (step 0, 1 of the first 32 rows, then of the others).
__global__ __launch_bounds__(256) void pack_mx4_kernel(PackParams p, unsigned char* scales) {
  const int per_row = p.cols / 8;
  const long long t = blockIdx.x * 256ll + threadIdx.x;
  if (t >= (long long)p.rows * per_row) return;
  const int r = (int)(t / per_row), c = (int)(t - (long long)r * per_row) * 8;
  const long long sr = pack_src_row(p, r);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = sr >= 0 ? p.src[sr * p.src_cols + c + e] : 0.f;
  const unsigned s = mx_scale<kMx4>(quad_umax(amax8(v)));
  const int lane = (r & 31) + 32 * ((c & 63) >> 5);
  unsigned char* codes = static_cast<unsigned char*>(p.dst);
  const long long step = (long long)(r >> 5) * (p.cols / 64) + c / 64, quad = (long long)(r >> 6) * (p.cols / 128) + c / 128;
  *reinterpret_cast<unsigned*>(codes + (step * 64 + lane) * 16 + (c & 31) / 2) = mx4_codes8(v, s);
  if ((c & 31) == 0) scales[(quad * 64 + lane) * 4 + ((r >> 5) & 1) * 2 + ((c >> 6) & 1)] = (unsigned char)s;
}

unsigned grid_for(long long groups) {
  const long long n = (groups + kGroups - 1) / kGroups;
  DN_CHECK(n <= 0x7fffffffll, "mx: too many values for one call");
  return static_cast<unsigned>(n);
}

}  // namespace

long long mx_bytes(int fmt, long long rows, long long cols) {
  DN_CHECK(rows >= 1 && cols >= 1 && cols <= kMxMaxCols, "mx: rows and columns must be >= 1, columns <= 2^31 - 32");
  const long long b = mx_blocks(cols);
  DN_CHECK(rows <= (1ll << 46) / b, "mx: buffer too large");
  return rows * b * mx_block_bytes(fmt) + (rows * b + 15) / 16 * 16 + 16;
}

size_t mx_scale_offset(int fmt, long long rows, long long cols) { return (size_t)(rows * mx_blocks(cols) * mx_block_bytes(fmt)); }

size_t mx_store_workspace(long long rows, long long n_slots) { return rows <= kScanRows ? 0 : (size_t)n_slots * sizeof(int); }

template <typename T>
void mx_store(int fmt, const T* x, long long ldx, long long rows, long long cols, const long long* slots, long long n_slots,
              void* table, int* owner, hipStream_t s) {
  StoreParams p;
  p.x = x;
  p.ldx = ldx;
  p.rows = rows;
  p.cols = cols;
  p.blocks = static_cast<unsigned>(mx_blocks(cols));
  p.vec = (reinterpret_cast<uintptr_t>(x) | (uintptr_t)ldx * sizeof(T)) % 16 == 0;
  p.slots = slots;
  p.n_slots = n_slots;
  p.owner = rows > kScanRows ? owner : nullptr;
  p.codes = static_cast<unsigned char*>(table);
  p.scales = p.codes + mx_scale_offset(fmt, n_slots, cols);
  const unsigned grid = grid_for(rows * p.blocks * 4);
  if (slots && rows > kScanRows) {
    if (rows <= kClaimOneGroup) {
      hipLaunchKernelGGL(mx_claim_kernel<0>, dim3(1), dim3(1024), 0, s, slots, rows, n_slots, owner);
    } else {
      const unsigned g = static_cast<unsigned>(std::min<long long>((rows + 1023) / 1024, 1024));
      hipLaunchKernelGGL(mx_claim_kernel<1>, dim3(g), dim3(1024), 0, s, slots, rows, n_slots, owner);
      hipLaunchKernelGGL(mx_claim_kernel<2>, dim3(g), dim3(1024), 0, s, slots, rows, n_slots, owner);
    }
  }
  if (fmt == kMx4)
    hipLaunchKernelGGL((mx_store_kernel<kMx4, T>), dim3(grid), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((mx_store_kernel<kMx8, T>), dim3(grid), dim3(256), 0, s, p);
  DN_HIP(hipGetLastError());
}

void mx_fetch(int fmt, const void* table, long long n_slots, long long cols, const long long* idx, long long rows, float* y,
              long long ldy, hipStream_t s) {
  FetchParams p;
  p.codes = static_cast<const unsigned char*>(table);
  p.scales = p.codes + mx_scale_offset(fmt, n_slots, cols);
  p.n_slots = n_slots;
  p.rows = rows;
  p.cols = cols;
  p.blocks = static_cast<unsigned>(mx_blocks(cols));
  p.idx = idx;
  p.y = y;
  p.ldy = ldy;
  p.vec = (reinterpret_cast<uintptr_t>(y) | (uintptr_t)ldy * 4) % 16 == 0;
  const unsigned grid = grid_for(rows * p.blocks * 4);
  if (fmt == kMx4)
    hipLaunchKernelGGL(mx_fetch_kernel<kMx4>, dim3(grid), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL(mx_fetch_kernel<kMx8>, dim3(grid), dim3(256), 0, s, p);
  DN_HIP(hipGetLastError());
}

void pack_mx4(const PackParams& p, unsigned char* scales, hipStream_t s) {
  DN_CHECK(p.col_mode == 0 && p.rows % 32 == 0 && p.cols % 128 == 0 && p.src_cols == p.cols,
           "pack_mx4: rows must be a multiple of 32, columns of 128");
  const long long n = (long long)p.rows * (p.cols / 8);
  hipLaunchKernelGGL(pack_mx4_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, s, p, scales);
  DN_HIP(hipGetLastError());
}

template void mx_store<float>(int, const float*, long long, long long, long long, const long long*, long long, void*, int*,
                              hipStream_t);
template void mx_store<bf16>(int, const bf16*, long long, long long, long long, const long long*, long long, void*, int*,
                             hipStream_t);
template void mx_store<_Float16>(int, const _Float16*, long long, long long, long long, const long long*, long long, void*,
                                 int*, hipStream_t);

}  // namespace dn
