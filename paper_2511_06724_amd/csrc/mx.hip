// Microscaled rows (mx.h): quantisation of rows as they are written (in order, or scattered into
// the slots of a cache), reading back, and the packing of 4-bit weights (gfx950).
//
// Both directions move bytes and do little else. A thread handles eight values (16 or 32 bytes of
// the source, 4 or 8 of codes), four neighbouring lanes a block, whose largest magnitude meets in
// two DPP steps. Slots are looked up once per row and workgroup. Bound by memory where rows are many: 100000 rows of
// 768 fp16 values into scattered slots of a table of E2M1 rows 59 us and 10 for the claims (195 MB: 38 us at
// 5.1 TB/s; in order 39), back as fp32 75 us (348 MB, 68); two groups of eight per thread take the store 15 % and the
// read 4 % less than one.
#include <algorithm>

#include "mx.h"

namespace dn {
namespace {

constexpr int kStoreUnroll = 2, kFetchUnroll = 2;
constexpr int kStoreGroups = 256 * kStoreUnroll;  // groups of eight values per workgroup
constexpr int kFetchGroups = 256 * kFetchUnroll;
// Rows per call up to which every workgroup looks for later rows of its rows' slots by itself; more are
// claimed by kernels of their own (64 states of 65536 values: 9.5 us with those).
constexpr int kScanRows = 256;
// Rows one workgroup claims in a single launch, in dependent rounds: 17.5 us for 4096 rows, 51 for 16384. (The two
// launches over a grid take 10 us for 100000.)
constexpr int kClaimOneGroup = 16384;

// Elements [c, c + 8) of a row, zero past `cols`; a row may begin at any element.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Eight {
  T v[8];
};
template <typename T> __device__ __forceinline__ void load8(const T* x, long long c, long long cols, float* v) {
  if (c + 8 <= cols) {
    const Eight<T> a = *reinterpret_cast<const Eight<T>*>(x + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(a.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? static_cast<float>(x[c + e]) : 0.f;
  }
}

__device__ __forceinline__ unsigned amax8(const float* v) {
  unsigned a = mx_abs_bits(v[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) a = max(a, mx_abs_bits(v[e]));
  return a;
}

// The value N lanes up in a row of sixteen (the last N lanes': 0).
template <int N> __device__ __forceinline__ unsigned dpp_row_shl(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x100 + N, 0xf, 0xf, true);
}

// The groups of eight values of a workgroup that covers N of them from group `base` on, rows of per_row groups
// one after the other: its first row, and a thread's groups, 256 apart, as row (counted from the first) and
// group of the row. One 64-bit division per workgroup, one of 32 bits per thread.
template <unsigned N> struct Groups {
  long long row0;
  unsigned off, per_row, rows;  // rows that it may touch
  unsigned row, g, dq, dr;
  __device__ Groups(long long base, unsigned groups_per_row, long long rows_all) : per_row(groups_per_row) {
    row0 = base / per_row;
    off = (unsigned)(base - row0 * per_row);
    rows = (unsigned)min((long long)((off + N - 1) / per_row + 1), rows_all - row0);
    const unsigned t = off + threadIdx.x;
    row = t / per_row;
    g = t - row * per_row;
    dq = 256 / per_row;
    dr = 256 - dq * per_row;
  }
  __device__ void next() {
    g += dr;
    const bool wrap = g >= per_row;
    row += dq + wrap;
    g -= wrap ? per_row : 0;
  }
};

struct StoreParams {
  const void* x;
  long long ldx, rows, cols;
  unsigned blocks;          // of a row
  const long long* slots;   // nullptr: row j goes to slot j
  long long n_slots;
  const int* owner;         // nullptr: rows look for later rows of their slot themselves
  unsigned char* codes;
  unsigned char* scales;
};

// First block of the destination of rows row0 .. row0 + n - 1, -1 for none (a slot outside the table, or a later
// row of the same slot), into LDS.
__device__ __forceinline__ void store_blocks(const StoreParams& p, long long row0, unsigned n, long long* first, long long* all) {
  const int t = threadIdx.x;
  if (p.owner) {
    for (unsigned i = t; i < n; i += 256) {
      const long long s = p.slots[row0 + i];
      first[i] = s >= 0 && s < p.n_slots && p.owner[s] == (int)(row0 + i) ? s * p.blocks : -1;
    }
  } else {
    if (t < p.rows) all[t] = p.slots[t];
    __syncthreads();
    for (unsigned i = t; i < n; i += 256) {
      const int j = (int)row0 + (int)i;
      const long long s = all[j];
      bool on = s >= 0 && s < p.n_slots;
#pragma unroll 8
      for (int k = j + 1; k < (int)p.rows; ++k) on &= all[k] != s;
      first[i] = on ? s * p.blocks : -1;
    }
  }
  __syncthreads();
}

template <int FMT, typename T> __global__ __launch_bounds__(256) void mx_store_kernel(StoreParams p) {
  __shared__ long long first[kStoreGroups / 4 + 1], all[kScanRows];
  const long long base = (long long)blockIdx.x * kStoreGroups, total = p.rows * (p.blocks * 4ll);
  Groups<kStoreGroups> at(base, p.blocks * 4, p.rows);
  const T* const x = static_cast<const T*>(p.x) + at.row0 * p.ldx;
  float v[kStoreUnroll][8];
  unsigned row[kStoreUnroll], g[kStoreUnroll];
#pragma unroll
  for (int u = 0; u < kStoreUnroll; ++u) {
    row[u] = at.row, g[u] = at.g;
    at.next();
    if (base + u * 256 + threadIdx.x < total) load8(x + row[u] * p.ldx, 8ll * g[u], p.cols, v[u]);
  }
  if (p.slots) store_blocks(p, at.row0, at.rows, first, all);
  // every load arrives before the first store is out: a wait for a load after it would wait for the store too
#pragma unroll
  for (int u = 0; u < kStoreUnroll; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(v[u][e]));
#pragma unroll
  for (int u = 0; u < kStoreUnroll; ++u) {
    if (base + u * 256 + threadIdx.x >= total) break;  // the four lanes of a block together, here and below
    const long long b0 = p.slots ? first[row[u]] : (at.row0 + row[u]) * p.blocks;
    if (b0 < 0) continue;
    const unsigned s = mx_scale<FMT>(quad_umax(amax8(v[u])));
    if constexpr (FMT == kMx4)
      *reinterpret_cast<unsigned*>(p.codes + b0 * 16 + g[u] * 4ull) = mx4_codes8(v[u], s);
    else
      *reinterpret_cast<uint2*>(p.codes + b0 * 32 + g[u] * 8ull) = make_uint2(mx8_codes4(v[u], s), mx8_codes4(v[u] + 4, s));
    if (p.blocks % 4 == 0) {
      // sixteen lanes hold four blocks of a row, whose scales are a word
      const unsigned w = s | dpp_row_shl<4>(s) << 8 | dpp_row_shl<8>(s) << 16 | dpp_row_shl<12>(s) << 24;
      if ((g[u] & 15) == 0) *reinterpret_cast<unsigned*>(p.scales + b0 + g[u] / 4) = w;
    } else if ((g[u] & 3) == 0) {
      p.scales[b0 + g[u] / 4] = (unsigned char)s;
    }
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
};

// Four values at any address, as one store (of a structure, the compiler splits one off for the short path).
typedef float Four __attribute__((ext_vector_type(4), aligned(4)));

template <int FMT> __global__ __launch_bounds__(256) void mx_fetch_kernel(FetchParams p) {
  __shared__ long long first[kFetchGroups / 4 + 1];
  const long long base = (long long)blockIdx.x * kFetchGroups, left = p.rows * (p.blocks * 4ll) - base;
  Groups<kFetchGroups> at(base, p.blocks * 4, p.rows);
  if (p.idx) {
    for (unsigned i = threadIdx.x; i < at.rows; i += 256) {
      const long long s = p.idx[at.row0 + i];
      first[i] = s >= 0 && s < p.n_slots ? s * p.blocks : -1;
    }
    __syncthreads();
  }
  unsigned row[kFetchUnroll], g[kFetchUnroll], s[kFetchUnroll];
  bool on[kFetchUnroll];
  uint2 code[kFetchUnroll];
#pragma unroll
  for (int u = 0; u < kFetchUnroll; ++u) {
    row[u] = min(at.row, at.rows - 1), g[u] = at.g;
    at.next();
    const long long b = p.idx ? first[row[u]] : (at.row0 + row[u]) * p.blocks, b0 = max(b, 0ll);  // none: read block 0
    on[u] = u * 256 + threadIdx.x < left && b >= 0;
    if constexpr (FMT == kMx4)
      code[u] = make_uint2(*reinterpret_cast<const unsigned*>(p.codes + b0 * 16 + g[u] * 4ull), 0u);
    else
      code[u] = *reinterpret_cast<const uint2*>(p.codes + b0 * 32 + g[u] * 8ull);
    s[u] = p.scales[b0 + g[u] / 4];
  }
  // every load arrives before the first store is out: a wait for a load after it would wait for the store too
#pragma unroll
  for (int u = 0; u < kFetchUnroll; ++u) asm volatile("" : "+v"(code[u].x), "+v"(code[u].y), "+v"(s[u]));
#pragma unroll
  for (int u = 0; u < kFetchUnroll; ++u) {
    if (!on[u]) continue;
    float v[8];
    if constexpr (FMT == kMx4) {
      mx4_values8(code[u].x, s[u], v);
    } else {
      mx8_values4(code[u].x, s[u], v);
      mx8_values4(code[u].y, s[u], v + 4);
    }
    const unsigned c = 8 * g[u], cols = (unsigned)p.cols;
    float* const y = p.y + (at.row0 + row[u]) * p.ldy + c;
    if (c + 8 <= cols) {
      reinterpret_cast<Four*>(y)[0] = Four{v[0], v[1], v[2], v[3]};
      reinterpret_cast<Four*>(y)[1] = Four{v[4], v[5], v[6], v[7]};
    } else {
      for (unsigned e = 0; e < 8; ++e)
        if (c + e < cols) y[e] = v[e];
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

unsigned grid_for(long long groups, int per_workgroup) {
  const long long n = (groups + per_workgroup - 1) / per_workgroup;
  DN_CHECK(n <= 0xffffffll, "mx: too many values for one call");  // a launch has less than 2^32 threads
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
  p.slots = slots;
  p.n_slots = n_slots;
  p.owner = rows > kScanRows ? owner : nullptr;
  p.codes = static_cast<unsigned char*>(table);
  p.scales = p.codes + mx_scale_offset(fmt, n_slots, cols);
  const unsigned grid = grid_for(rows * p.blocks * 4, kStoreGroups);
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
  const unsigned grid = grid_for(rows * p.blocks * 4, kFetchGroups);
  if (fmt == kMx4)
    hipLaunchKernelGGL(mx_fetch_kernel<kMx4>, dim3(grid), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL(mx_fetch_kernel<kMx8>, dim3(grid), dim3(256), 0, s, p);
  DN_HIP(hipGetLastError());
}

void pack_mx4(const PackParams& p, unsigned char* scales, hipStream_t s) {
  DN_CHECK(p.col_mode == 0 && p.rows % 32 == 0 && p.cols % 128 == 0 && p.src_cols == p.cols,
           "pack_mx4: rows must be a multiple of 32, columns of 128");
  const unsigned grid = grid_for((long long)p.rows * (p.cols / 8), 256);
  hipLaunchKernelGGL(pack_mx4_kernel, dim3(grid), dim3(256), 0, s, p, scales);
  DN_HIP(hipGetLastError());
}

template void mx_store<float>(int, const float*, long long, long long, long long, const long long*, long long, void*, int*,
                              hipStream_t);
template void mx_store<bf16>(int, const bf16*, long long, long long, long long, const long long*, long long, void*, int*,
                             hipStream_t);
template void mx_store<_Float16>(int, const _Float16*, long long, long long, long long, const long long*, long long, void*,
                                 int*, hipStream_t);

}  // namespace dn
