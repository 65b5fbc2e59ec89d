// C ABI of the denoise-loop library: argument checks, error mapping and the
// single-kernel entry points. Every entry point catches all C++ exceptions.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <mutex>
#include <string>
#include <vector>

#include "model.h"
#include "packed.h"

// Scratch of the no-allocation batched lookup: the per-workgroup winners of one pass
// (at most lookup_batch_workspace_bytes(), 256 KiB, which also covers the per-query
// scan's lookup_workspace_bytes()), then 64 floats that receive the cosines when the
// caller asks for none. Every GPU the library runs on holds its own copy until the
// process ends; its device address comes from hipGetSymbolAddress, once per device.
constexpr size_t kScratchWinnerBytes = 256 * 1024;
constexpr size_t kScratchBytes = kScratchWinnerBytes + 64 * sizeof(float);
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

namespace dn {
// probe.hip: the bf16 matrix-core rate (TFLOP/s) every CU sustains on back-to-back
// 32x32x16 MFMAs and the shader clock (GHz) meanwhile. Synchronous.
void mfma_rate(int iters, double* tflops, double* clock_ghz);
}  // namespace dn

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// Device address of `scratch` on the current device (looked up on the first call on
// that device, with the device current; later calls reuse it).
void* scratch_ptr() {
  int dev = 0;
  DN_HIP(hipGetDevice(&dev));
  DN_CHECK(dev >= 0 && dev < kMaxDevices, "scratch: device ordinal beyond 64");
  std::lock_guard<std::mutex> lk(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    DN_HIP(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
    DN_CHECK(p != nullptr, "scratch: no device address");
    g_scratch_ptr[dev] = p;
  }
  return g_scratch_ptr[dev];
}

thread_local std::string g_last_error;

dn_status fail(int code, const std::string& msg) {
  g_last_error = msg;
  return static_cast<dn_status>(code);
}

template <typename F> dn_status guarded(F&& f) {
  try {
    g_last_error.clear();
    f();
    return DN_OK;
  } catch (const dn::Error& e) {
    return fail(e.code, e.what());
  } catch (const std::bad_alloc&) {
    return fail(DN_ENOMEM, "host allocation failed");
  } catch (const std::exception& e) {
    return fail(DN_EHIP, e.what());
  } catch (...) {
    return fail(DN_EHIP, "unknown error");
  }
}

hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

// Per-device state of the cache lookup, allocated once: the device workspace of the
// per-workgroup winners, and a pinned host buffer the reduction writes the result to
// (index at byte 0, score at byte 8), so no copy follows the kernels.
struct LookupRes {
  long long idx;
  float score;
  int k;
};
struct LookupWs {
  std::mutex mu;
  std::vector<void*> ws;
  std::vector<LookupRes*> res;
  std::vector<void*> batch_ws;        // per-workgroup winners of the batched scan
  std::vector<long long*> batch_res;  // pinned: 64 indices, then 64 scores, then 64 levels
};
LookupWs g_lookup;

void lookup_state(int dev, void** ws, LookupRes** res) {
  std::lock_guard<std::mutex> lk(g_lookup.mu);
  if ((int)g_lookup.ws.size() <= dev) {
    g_lookup.ws.resize(dev + 1, nullptr);
    g_lookup.res.resize(dev + 1, nullptr);
  }
  if (!g_lookup.ws[dev]) DN_HIP(hipMalloc(&g_lookup.ws[dev], dn::lookup_workspace_bytes()));
  if (!g_lookup.res[dev]) DN_HIP(hipHostMalloc(reinterpret_cast<void**>(&g_lookup.res[dev]), 256));
  *ws = g_lookup.ws[dev];
  *res = g_lookup.res[dev];
}

void lookup_batch_state(int dev, void** ws, long long** idx, float** score, int** lev) {
  std::lock_guard<std::mutex> lk(g_lookup.mu);
  if ((int)g_lookup.batch_ws.size() <= dev) {
    g_lookup.batch_ws.resize(dev + 1, nullptr);
    g_lookup.batch_res.resize(dev + 1, nullptr);
  }
  const int mq = dn::lookup_batch_max_queries();
  if (!g_lookup.batch_ws[dev]) DN_HIP(hipMalloc(&g_lookup.batch_ws[dev], dn::lookup_batch_workspace_bytes()));
  if (!g_lookup.batch_res[dev])
    DN_HIP(hipHostMalloc(reinterpret_cast<void**>(&g_lookup.batch_res[dev]),
                         mq * (sizeof(long long) + sizeof(float) + sizeof(int))));
  *ws = g_lookup.batch_ws[dev];
  *idx = g_lookup.batch_res[dev];
  *score = reinterpret_cast<float*>(g_lookup.batch_res[dev] + mq);
  *lev = reinterpret_cast<int*>(*score + mq);
}

// Checks a similarity-to-level table and converts it for the kernels.
dn::KTable k_table(const ac_k_table* t) {
  DN_CHECK(t, "ac_k_table: null table");
  DN_CHECK(t->n_thresholds >= 0 && t->n_thresholds < AC_MAX_K_LEVELS,
           "ac_k_table: n_thresholds must be in [0, " + std::to_string(AC_MAX_K_LEVELS - 1) + "]");
  dn::KTable k;
  k.n = t->n_thresholds;
  for (int i = 0; i < k.n; ++i) {
    DN_CHECK(std::isfinite(t->threshold[i]), "ac_k_table: thresholds must be finite");
    DN_CHECK(i == 0 || t->threshold[i] > t->threshold[i - 1], "ac_k_table: thresholds must increase strictly");
    k.thr[i] = t->threshold[i];
  }
  for (int j = 0; j <= k.n; ++j) {
    DN_CHECK(t->level[j] >= 0, "ac_k_table: levels must be >= 0");
    DN_CHECK(j == 0 || t->level[j] >= t->level[j - 1], "ac_k_table: levels must not decrease");
    k.level[j] = t->level[j];
  }
  return k;
}

// The batched search of ac_lookup_batch / ac_lookup_batch_k (host results; level per
// query when kt is given).
void lookup_batch_host(const uint16_t* query_embs, int32_t nq, const uint16_t* cache_embs, int64_t n, int32_t dim,
                       int64_t* out_idx, float* out_score, const dn::KTable* kt, int32_t* out_k, const char* who) {
  const std::string w(who);
  DN_CHECK(query_embs && cache_embs && out_idx, w + ": null pointer");
  DN_CHECK(nq >= 1, w + ": nq must be >= 1");
  DN_CHECK(n >= 1, w + ": n must be >= 1");
  DN_CHECK(dim >= 1, w + ": dim must be >= 1");
  DN_CHECK(!kt || out_k, w + ": null level output");
  int dev = 0;
  DN_HIP(hipGetDevice(&dev));
  if (!dn::lookup_batch_supported(query_embs, cache_embs, n, dim)) {
    // other widths or alignments: one scan per query
    void* ws = nullptr;
    LookupRes* res = nullptr;
    lookup_state(dev, &ws, &res);
    for (int j = 0; j < nq; ++j) {
      res->idx = -1;
      res->score = 0.f;
      res->k = -1;
      dn::lookup(query_embs + (size_t)j * dim, cache_embs, n, dim, ws, &res->idx, &res->score, nullptr, kt,
                 &res->k);
      DN_HIP(hipStreamSynchronize(nullptr));
      out_idx[j] = *static_cast<volatile long long*>(&res->idx);
      if (out_score) out_score[j] = *static_cast<volatile float*>(&res->score);
      if (kt) out_k[j] = *static_cast<volatile int*>(&res->k);
    }
    return;
  }
  void* ws = nullptr;
  long long* ridx = nullptr;
  float* rscore = nullptr;
  int* rk = nullptr;
  lookup_batch_state(dev, &ws, &ridx, &rscore, &rk);
  const int mq = dn::lookup_batch_max_queries();
  for (int j0 = 0; j0 < nq; j0 += mq) {
    const int m = nq - j0 < mq ? nq - j0 : mq;
    for (int j = 0; j < m; ++j) ridx[j] = -2;
    dn::lookup_batch(query_embs + (size_t)j0 * dim, m, cache_embs, n, dim, ws, ridx, rscore, nullptr, kt, rk);
    DN_HIP(hipStreamSynchronize(nullptr));
    for (int j = 0; j < m; ++j) {
      const long long idx = static_cast<volatile long long*>(ridx)[j];
      DN_CHECK(idx >= -1 && idx < n, w + ": result not written");
      out_idx[j0 + j] = idx;
      if (out_score) out_score[j0 + j] = static_cast<volatile float*>(rscore)[j];
      if (kt) out_k[j0 + j] = static_cast<volatile int*>(rk)[j];
    }
  }
}

bool is_dtype(int32_t d) { return d == DN_FP32 || d == DN_BF16; }
bool is_dtype8(int32_t d) { return is_dtype(d) || d == DN_FP8; }
bool is_mx(int32_t d) { return d == DN_MXFP4 || d == DN_MXFP8; }
bool is_dtype_op(int32_t d) { return is_dtype8(d) || d == DN_MXFP4; }  // operand types of the dense layers and LayerNorm
static_assert(DN_MXFP4 == dn::kMx4 && DN_MXFP8 == dn::kMx8, "the kernels' format numbers");

// Whether `p` (which may be null) is aligned to its elements of n bytes.
bool on(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Arguments the MX row calls share: a table of n_slots rows of `cols` values, `rows` rows in fp32 / bf16 /
// fp16 (dense rows ld apart) on the other side.
void check_mx(const char* who, int32_t dtype, const void* table, int64_t n_slots, int64_t cols, const void* x, int64_t ld,
              int64_t rows) {
  const std::string w(who);
  DN_CHECK(is_mx(dtype), w + ": dtype must be DN_MXFP4 or DN_MXFP8");
  DN_CHECK(table && x, w + ": null pointer");
  DN_CHECK(n_slots >= 1 && cols >= 1 && rows >= 1 && rows <= 0x7fffffffll, w + ": bad sizes");
  (void)dn::mx_bytes(dtype, n_slots, cols);
  DN_CHECK(ld >= cols && ld <= (1ll << 40), w + ": row stride smaller than the row");
  DN_CHECK(reinterpret_cast<uintptr_t>(table) % 16 == 0, w + ": the MX buffer must be 16-byte aligned");
}

void store_rows(const char* who, int32_t dtype, int32_t src, const void* x, int64_t ldx, int64_t rows, int64_t cols,
                const int64_t* slots, int64_t n_slots, void* table, void* ws, void* stream) {
  const std::string w(who);
  DN_CHECK(src == DN_FP32 || src == DN_BF16 || src == DN_FP16, w + ": source dtype must be DN_FP32, DN_BF16 or DN_FP16");
  DN_CHECK(reinterpret_cast<uintptr_t>(x) % (src == DN_FP32 ? 4 : 2) == 0, w + ": misaligned source");
  const long long* sl = reinterpret_cast<const long long*>(slots);
  int* owner = static_cast<int*>(ws);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (src == DN_FP32)
    dn::mx_store<float>(dtype, static_cast<const float*>(x), ldx, rows, cols, sl, n_slots, table, owner, s);
  else if (src == DN_BF16)
    dn::mx_store<dn::bf16>(dtype, static_cast<const dn::bf16*>(x), ldx, rows, cols, sl, n_slots, table, owner, s);
  else
    dn::mx_store<_Float16>(dtype, static_cast<const _Float16*>(x), ldx, rows, cols, sl, n_slots, table, owner, s);
}

// Per-device state of the single-kernel GEMM entry points: CU count (tile
// planning) and a zero block for implicit-conv padding reads.
struct OpDev {
  int cus = 0;
  void* zero = nullptr;
  float* part = nullptr;  // split-K partial slabs, grown on demand
  size_t part_floats = 0;
  float* gn = nullptr;    // GroupNorm partial sums and per-channel scale / shift, grown on demand
  size_t gn_floats = 0;
};
std::mutex g_op_mu;
std::vector<OpDev> g_op_dev;

// Grows a per-device buffer of the single-kernel entry points. Work already enqueued
// may still read the old buffer, so the device is synchronised before it is freed.
void grow(float** buf, size_t* have, size_t need) {
  if (need <= *have) return;
  if (*buf) {
    DN_HIP(hipDeviceSynchronize());
    DN_HIP(hipFree(*buf));
    *buf = nullptr;
    *have = 0;
  }
  DN_HIP(hipMalloc(reinterpret_cast<void**>(buf), need * 4));
  *have = need;
}

// Compute units of the current device (no allocation: callers may be capturing).
int current_cus() {
  static std::atomic<int> known[64];  // by device; asking takes most of a microsecond
  int dev = 0, cus = 0;
  DN_HIP(hipGetDevice(&dev));
  if (dev < 64 && (cus = known[dev].load(std::memory_order_relaxed))) return cus;
  DN_HIP(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev));
  if (dev < 64) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

OpDev& op_dev_locked(int dev) {
  if ((int)g_op_dev.size() <= dev) g_op_dev.resize(dev + 1);
  OpDev& d = g_op_dev[dev];
  if (!d.cus) {
    hipDeviceProp_t prop;
    DN_HIP(hipGetDeviceProperties(&prop, dev));
    DN_HIP(hipMalloc(&d.zero, 256));
    DN_HIP(hipMemset(d.zero, 0, 256));
    d.cus = prop.multiProcessorCount;
  }
  return d;
}

template <typename T> dn::GemmPlan op_plan(const dn::GemmParams& p, int cus) {
  return p.wscale ? dn::gemm_plan_fp8(p.M, p.N, p.K, p.geglu, cus, false, p.out_f32)
                  : dn::gemm_plan<T>(p.M, p.N, p.K, p.geglu, cus, p.vt != nullptr, false, p.taps == 9, p.out_f32);
}

template <typename T> void op_gemm(dn::GemmParams& p, hipStream_t s) {
  int dev = 0;
  DN_HIP(hipGetDevice(&dev));
  OpDev w;
  {
    std::lock_guard<std::mutex> lk(g_op_mu);
    OpDev& d = op_dev_locked(dev);
    const dn::GemmPlan g0 = op_plan<T>(p, d.cus);
    grow(&d.part, &d.part_floats, dn::gemm_workspace_floats(g0, p.M, p.N));
    w = d;
  }
  const dn::GemmPlan g = op_plan<T>(p, w.cus);
  p.zero16 = w.zero;
  p.part = w.part;
  p.part_floats = w.part_floats;
  if (p.wscale)
    dn::gemm_fp8(p, g, s);
  else
    dn::gemm<T>(p, g, s);
}

// ---------------------------------------------------------------- packed sequences

// Rows of a tensor of heads: 16-byte aligned, at least `width` and a multiple of 16 bytes apart.
void check_heads(const char* who, int32_t dtype, const void* x, int64_t ld, int64_t width) {
  const int64_t vec = dtype == DN_BF16 ? 8 : 4;
  DN_CHECK(x, std::string(who) + ": null pointer");
  DN_CHECK(on(x, 16), std::string(who) + ": rows must be 16-byte aligned");
  DN_CHECK(ld >= width && ld % vec == 0 && ld <= (1 << 23),
           std::string(who) + ": row stride must cover the heads, be a multiple of 16 bytes and at most 2^23");
}

dn::Sequences sequences(const char* who, const dn_sequences* s) {
  DN_CHECK(s->n >= 1, std::string(who) + ": at least one sequence");
  DN_CHECK(s->q_start && s->kv_start && s->kv_len, std::string(who) + ": null pointer in the sequences");
  DN_CHECK(on(s->q_start, 4) && on(s->kv_start, 8) && on(s->kv_len, 4), std::string(who) + ": misaligned sequences");
  DN_CHECK(s->max_kv_len >= 1, std::string(who) + ": max_kv_len must be positive");
  dn::Sequences r;
  r.n = s->n;
  r.q_start = s->q_start;
  r.kv_start = reinterpret_cast<const long long*>(s->kv_start);
  r.kv_len = s->kv_len;
  return r;
}

dn::RotaryParams rotation(const char* who, int32_t dtype, int64_t T, int32_t head_dim, const dn_rotation* r) {
  DN_CHECK(is_dtype(dtype), std::string(who) + ": bad dtype");
  DN_CHECK(T >= 1 && T <= 0x7fffffff, std::string(who) + ": bad row count");
  DN_CHECK(head_dim >= 8 && head_dim <= DN_ROPE_MAX_DIM && head_dim % 8 == 0,
           std::string(who) + ": head_dim must be a multiple of 8, at most 256");
  DN_CHECK(r && r->table && r->pos, std::string(who) + ": null rotation, table or positions");
  DN_CHECK(on(r->table, 16) && on(r->pos, 4), std::string(who) + ": misaligned table or positions");
  DN_CHECK(r->n_axes >= 1 && r->n_axes <= DN_ROPE_MAX_AXES, std::string(who) + ": one to four axes");
  DN_CHECK(r->pairing == DN_ROPE_PAIRS || r->pairing == DN_ROPE_HALVES, std::string(who) + ": bad pairing");
  DN_CHECK(r->rot_dim >= 2 && r->rot_dim <= head_dim && r->rot_dim % 2 == 0,
           std::string(who) + ": rot_dim must be even, 2 .. head_dim");
  DN_CHECK(r->pairing == DN_ROPE_PAIRS || r->rot_dim % 8 == 0, std::string(who) + ": DN_ROPE_HALVES needs rot_dim % 8 == 0");
  dn::RotaryParams p;
  p.T = T;
  p.D = head_dim;
  p.table = static_cast<const dn::RopeEntry*>(r->table);
  p.pos = r->pos;
  p.n_axes = r->n_axes;
  p.half = r->rot_dim / 2;
  p.halves = r->pairing == DN_ROPE_HALVES;
  return p;
}

void run_rotary(int32_t dtype, const dn::RotaryParams& p, void* stream) {
  dtype == DN_BF16 ? dn::rotary<dn::bf16>(p, as_stream(stream)) : dn::rotary<float>(p, as_stream(stream));
}

void check_packed_sizes(const char* who, int32_t dtype, int64_t T, int32_t heads, int32_t kv_heads, int32_t head_dim) {
  DN_CHECK(is_dtype(dtype), std::string(who) + ": bad dtype");
  DN_CHECK(T >= 1 && T <= 0x7fffffff, std::string(who) + ": bad row count");
  DN_CHECK(heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0, std::string(who) + ": heads must be a multiple of kv_heads");
  DN_CHECK(heads <= 65535, std::string(who) + ": at most 65535 heads");
  DN_CHECK(dn::attention_packed_dim(head_dim), std::string(who) + ": head_dim must be 32, 64, 96 or 128");
  // a sequence's rows (tokens times the heads of a group) are counted in 32 bits
  DN_CHECK(T * (heads / kv_heads) <= 0x7fffffff - 65536, std::string(who) + ": too many rows");
}

}  // namespace

struct dn_handle {
  dn::Model* m = nullptr;
};
struct dn_vae {
  dn::Vae* v = nullptr;
};

extern "C" {

dn_status dn_weight_count(const dn_config* cfg, size_t* n_floats) {
  return guarded([&] {
    DN_CHECK(cfg && n_floats, "dn_weight_count: null pointer");
    const auto t = dn::weight_table(*cfg);
    *n_floats = t.empty() ? 0 : static_cast<size_t>(t.back().offset + t.back().numel);
  });
}

dn_status dn_weight_table(const dn_config* cfg, int64_t* numel, int32_t* fan_in, int32_t* kind, size_t capacity,
                          size_t* n_tensors) {
  return guarded([&] {
    DN_CHECK(cfg && n_tensors, "dn_weight_table: null pointer");
    const auto t = dn::weight_table(*cfg);
    DN_CHECK(capacity == 0 || capacity >= t.size(), "dn_weight_table: capacity too small");
    DN_CHECK(capacity == 0 || (numel && fan_in && kind), "dn_weight_table: null output array");
    if (capacity) {
      for (size_t i = 0; i < t.size(); ++i) {
        numel[i] = t[i].numel;
        fan_in[i] = t[i].fan_in;
        kind[i] = t[i].kind;
      }
    }
    *n_tensors = t.size();
  });
}

dn_status dn_create(const dn_config* cfg, const float* weights, size_t n_floats, int32_t weights_location,
                    dn_handle** out) {
  return guarded([&] {
    DN_CHECK(cfg && weights && out, "dn_create: null pointer");
    DN_CHECK(weights_location == DN_WEIGHTS_HOST || weights_location == DN_WEIGHTS_DEVICE,
             "dn_create: bad weights_location");
    dn::Model* m = dn::model_create(*cfg, weights, n_floats, weights_location == DN_WEIGHTS_DEVICE);
    dn_handle* h = new dn_handle();
    h->m = m;
    *out = h;
  });
}

dn_status dn_denoise(dn_handle* h, float* latent, const float* text_ctx, const int32_t* timesteps,
                     int32_t n_timesteps, int32_t start_step, int32_t n_steps, float cfg_scale, void* stream) {
  return guarded([&] {
    DN_CHECK(h && h->m, "dn_denoise: null handle");
    dn::model_denoise(h->m, latent, text_ctx, timesteps, n_timesteps, start_step, n_steps, cfg_scale,
                      as_stream(stream));
  });
}

dn_status dn_denoise_capture(dn_handle* h, float* latent, const float* text_ctx, const int32_t* timesteps,
                             int32_t n_timesteps, int32_t start_step, int32_t n_steps, float cfg_scale,
                             const int32_t* capture_at, int32_t n_capture, uint16_t* out_latents, void* stream) {
  return guarded([&] {
    DN_CHECK(h && h->m, "dn_denoise_capture: null handle");
    dn::model_denoise(h->m, latent, text_ctx, timesteps, n_timesteps, start_step, n_steps, cfg_scale,
                      as_stream(stream), capture_at, n_capture, out_latents);
  });
}

dn_status dn_unet_eps(dn_handle* h, const float* x, int32_t t, const float* text_ctx, float cfg_scale, float* out_raw,
                      float* out_guided, void* stream) {
  return guarded([&] {
    DN_CHECK(h && h->m, "dn_unet_eps: null handle");
    dn::model_unet_eps(h->m, x, t, text_ctx, cfg_scale, out_raw, out_guided, as_stream(stream));
  });
}

dn_status ac_lookup(const uint16_t* query_emb, const uint16_t* cache_embs, int64_t n, int32_t dim, int64_t* out_idx,
                    float* out_score) {
  return guarded([&] {
    DN_CHECK(query_emb && cache_embs && out_idx, "ac_lookup: null pointer");
    DN_CHECK(n >= 1, "ac_lookup: n must be >= 1");
    DN_CHECK(dim >= 1, "ac_lookup: dim must be >= 1");
    int dev = 0;
    DN_HIP(hipGetDevice(&dev));
    void* ws = nullptr;
    LookupRes* res = nullptr;
    lookup_state(dev, &ws, &res);
    res->idx = -1;
    res->score = 0.f;
    dn::lookup(query_emb, cache_embs, n, dim, ws, &res->idx, &res->score, nullptr);
    DN_HIP(hipStreamSynchronize(nullptr));
    // written by the device: read through volatile so the values set above are not reused
    const long long idx = *static_cast<volatile long long*>(&res->idx);
    const float score = *static_cast<volatile float*>(&res->score);
    DN_CHECK(idx >= 0 && idx < n, "ac_lookup: no row scored (zero query or zero-norm cache)");
    *out_idx = idx;
    if (out_score) *out_score = score;
  });
}

dn_status ac_lookup_batch(const uint16_t* query_embs, int32_t nq, const uint16_t* cache_embs, int64_t n, int32_t dim,
                          int64_t* out_idx, float* out_score) {
  return guarded([&] {
    lookup_batch_host(query_embs, nq, cache_embs, n, dim, out_idx, out_score, nullptr, nullptr, "ac_lookup_batch");
  });
}

dn_status ac_lookup_batch_k(const uint16_t* query_embs, int32_t nq, const uint16_t* cache_embs, int64_t n,
                            int32_t dim, const ac_k_table* table, int64_t* out_idx, float* out_score,
                            int32_t* out_k) {
  return guarded([&] {
    const dn::KTable kt = k_table(table);
    lookup_batch_host(query_embs, nq, cache_embs, n, dim, out_idx, out_score, &kt, out_k, "ac_lookup_batch_k");
  });
}

dn_status ac_lookup_batch_noalloc(const uint16_t* query_embs, int32_t nq, const uint16_t* cache_embs, int64_t n,
                                  int32_t dim, int64_t* out_idx, float* out_score, void* stream) {
  return guarded([&] {
    DN_CHECK(query_embs && cache_embs && out_idx, "ac_lookup_batch_noalloc: null pointer");
    DN_CHECK(nq >= 1, "ac_lookup_batch_noalloc: nq must be >= 1");
    DN_CHECK(n >= 1, "ac_lookup_batch_noalloc: n must be >= 1");
    DN_CHECK(dim >= 1, "ac_lookup_batch_noalloc: dim must be >= 1");
    const bool batched = dn::lookup_batch_supported(query_embs, cache_embs, n, dim);
    const size_t need = batched ? dn::lookup_batch_workspace_bytes() : dn::lookup_workspace_bytes();
    DN_CHECK(need <= kScratchWinnerBytes, "ac_lookup_batch_noalloc: scan needs " + std::to_string(need) +
                                              " bytes of scratch, the library holds " +
                                              std::to_string(kScratchWinnerBytes));
    DN_CHECK(batched || dim <= 16384, "ac_lookup_batch_noalloc: dim too large for the per-query scan");
    char* ws = static_cast<char*>(scratch_ptr());
    float* dummy = reinterpret_cast<float*>(ws + kScratchWinnerBytes);
    const hipStream_t s = as_stream(stream);
    long long* idx = reinterpret_cast<long long*>(out_idx);
    if (batched) {
      const int mq = dn::lookup_batch_max_queries();
      for (int j0 = 0; j0 < nq; j0 += mq) {
        const int m = nq - j0 < mq ? nq - j0 : mq;
        dn::lookup_batch(query_embs + (size_t)j0 * dim, m, cache_embs, n, dim, ws, idx + j0,
                         out_score ? out_score + j0 : dummy, s);
      }
    } else {
      for (int j = 0; j < nq; ++j)
        dn::lookup(query_embs + (size_t)j * dim, cache_embs, n, dim, ws, idx + j, out_score ? out_score + j : dummy,
                   s);
    }
  });
}

dn_status ac_fetch_latent(const uint16_t* cache_latents, int64_t n, int64_t numel, int64_t idx, float* latent,
                          void* stream) {
  return guarded([&] {
    DN_CHECK(cache_latents && latent, "ac_fetch_latent: null pointer");
    DN_CHECK(n >= 1 && numel >= 1, "ac_fetch_latent: empty cache");
    DN_CHECK(idx >= 0 && idx < n, "ac_fetch_latent: index out of range");
    dn::bf16_latent_to_f32(cache_latents + idx * numel, latent, numel, as_stream(stream));
  });
}

dn_status dn_mx_bytes(int32_t dtype, int64_t rows, int64_t cols, int64_t* bytes) {
  return guarded([&] {
    DN_CHECK(is_mx(dtype), "dn_mx_bytes: dtype must be DN_MXFP4 or DN_MXFP8");
    DN_CHECK(bytes, "dn_mx_bytes: null pointer");
    *bytes = dn::mx_bytes(dtype, rows, cols);
  });
}

dn_status dn_mx_quantize(int32_t dtype, int32_t x_dtype, const void* x, int64_t ldx, int64_t rows, int64_t cols, void* q,
                         void* stream) {
  return guarded([&] {
    check_mx("dn_mx_quantize", dtype, q, rows, cols, x, ldx, rows);
    store_rows("dn_mx_quantize", dtype, x_dtype, x, ldx, rows, cols, nullptr, rows, q, nullptr, stream);
  });
}

dn_status dn_mx_dequantize(int32_t dtype, const void* q, int64_t rows, int64_t cols, float* y, int64_t ldy, void* stream) {
  return guarded([&] {
    check_mx("dn_mx_dequantize", dtype, q, rows, cols, y, ldy, rows);
    DN_CHECK(on(y, 4), "dn_mx_dequantize: misaligned output");
    dn::mx_fetch(dtype, q, rows, cols, nullptr, rows, y, ldy, as_stream(stream));
  });
}

dn_status ac_mx_store_bytes(int64_t n_rows, int64_t n_slots, int64_t* bytes) {
  return guarded([&] {
    DN_CHECK(bytes, "ac_mx_store_bytes: null pointer");
    // as many slots as a table can have (dn_mx_bytes)
    DN_CHECK(n_rows >= 1 && n_slots >= 1 && n_slots <= (1ll << 46), "ac_mx_store_bytes: bad sizes");
    *bytes = static_cast<int64_t>(dn::mx_store_workspace(n_rows, n_slots));
  });
}

dn_status ac_mx_store(int32_t dtype, int32_t x_dtype, const void* x, int64_t ldx, int64_t n_rows, const int64_t* slots,
                      void* table, int64_t n_slots, int64_t dim, void* ws, void* stream) {
  return guarded([&] {
    check_mx("ac_mx_store", dtype, table, n_slots, dim, x, ldx, n_rows);
    DN_CHECK(slots && on(slots, 8), "ac_mx_store: null or misaligned slots");
    DN_CHECK((ws && reinterpret_cast<uintptr_t>(ws) % 4 == 0) || dn::mx_store_workspace(n_rows, n_slots) == 0,
             "ac_mx_store: this many rows need the workspace of ac_mx_store_bytes");
    store_rows("ac_mx_store", dtype, x_dtype, x, ldx, n_rows, dim, slots, n_slots, table, ws, stream);
  });
}

dn_status ac_mx_fetch(int32_t dtype, const void* table, int64_t n_slots, int64_t dim, const int64_t* idx, int64_t n_idx,
                      float* out, int64_t ldo, void* stream) {
  return guarded([&] {
    check_mx("ac_mx_fetch", dtype, table, n_slots, dim, out, ldo, n_idx);
    DN_CHECK(idx && on(idx, 8), "ac_mx_fetch: null or misaligned indices");
    DN_CHECK(on(out, 4), "ac_mx_fetch: misaligned output");
    dn::mx_fetch(dtype, table, n_slots, dim, reinterpret_cast<const long long*>(idx), n_idx, out, ldo, as_stream(stream));
  });
}

dn_status ac_mx_lookup_bytes(int32_t nq, int64_t n, int32_t dim, int64_t* bytes) {
  return guarded([&] {
    DN_CHECK(bytes, "ac_mx_lookup_bytes: null pointer");
    DN_CHECK(nq >= 1 && n >= 1 && dim >= 1, "ac_mx_lookup_bytes: bad sizes");
    *bytes = static_cast<int64_t>(dn::mx_lookup_workspace());
  });
}

dn_status ac_mx_lookup(int32_t dtype, const uint16_t* query_embs, int32_t nq, const void* table, int64_t n, int32_t dim,
                       const ac_k_table* levels, int64_t* out_idx, float* out_score, int32_t* out_k, void* ws, void* stream) {
  return guarded([&] {
    check_mx("ac_mx_lookup", dtype, table, n, dim, query_embs, dim, nq);
    DN_CHECK(out_idx && ws, "ac_mx_lookup: null pointer");
    DN_CHECK((levels != nullptr) == (out_k != nullptr), "ac_mx_lookup: a level table and a level output go together");
    DN_CHECK(on(ws, 16), "ac_mx_lookup: the workspace must be 16-byte aligned");
    DN_CHECK(on(query_embs, 2) && on(out_idx, 8) && on(out_score, 4) && on(out_k, 4), "ac_mx_lookup: misaligned queries or outputs");
    dn::KTable kt;
    if (levels) kt = k_table(levels);
    dn::mx_lookup(dtype, query_embs, nq, table, n, dim, ws, reinterpret_cast<long long*>(out_idx), out_score,
                  levels ? &kt : nullptr, out_k, as_stream(stream));
  });
}

dn_status dn_packed_weight_elems(int32_t dtype, int32_t N, int32_t K, int64_t* elems) {
  return guarded([&] {
    DN_CHECK(is_dtype_op(dtype), "dn_packed_weight_elems: bad dtype");
    DN_CHECK(elems, "dn_packed_weight_elems: null pointer");
    DN_CHECK(N >= 1 && K >= 1, "dn_packed_weight_elems: bad sizes");
    if (dtype == DN_FP8) {
      DN_CHECK(dn::gemm_fp8_layout(N, K), "dn_packed_weight_elems: DN_FP8 needs N % 32 == 0, K % 128 == 0");
      *elems = (int64_t)dn::gemm_fp8_code_bytes(N, K) + 4ll * N;
      return;
    }
    if (dtype == DN_MXFP4) {
      DN_CHECK(dn::gemm_mx4_layout(N, K), "dn_packed_weight_elems: DN_MXFP4 needs N % 32 == 0, K % 128 == 0, both at most 2^22");
      *elems = (int64_t)dn::gemm_mx4_bytes(N, K);
      return;
    }
    *elems = dtype == DN_BF16 && dn::gemm_frag_layout(N, K) ? (int64_t)dn::gemm_frag_elems(N, K) : (int64_t)N * K;
  });
}

dn_status dn_pack_weight(int32_t dtype, const void* w, int32_t N, int32_t K, void* out, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype_op(dtype), "dn_pack_weight: bad dtype");
    DN_CHECK(w && out, "dn_pack_weight: null pointer");
    if (dtype == DN_MXFP4) {
      DN_CHECK(dn::gemm_mx4_layout(N, K), "dn_pack_weight: DN_MXFP4 needs N % 32 == 0, K % 128 == 0, both at most 2^22");
      DN_CHECK(reinterpret_cast<uintptr_t>(out) % 16 == 0 && reinterpret_cast<uintptr_t>(w) % 4 == 0,
               "dn_pack_weight: DN_MXFP4 needs a 16-byte aligned output and a 4-byte aligned source");
      dn::PackParams p;
      p.dst = out;
      p.rows = p.src_rows = N;
      p.cols = p.src_cols = K;
      p.src = static_cast<const float*>(w);
      dn::pack_mx4(p, static_cast<unsigned char*>(out) + dn::gemm_mx4_code_bytes(N, K), as_stream(stream));
      return;
    }
    if (dtype == DN_FP8) {
      DN_CHECK(dn::gemm_fp8_layout(N, K), "dn_pack_weight: DN_FP8 needs N % 32 == 0, K % 128 == 0");
      dn::PackParams p;
      p.dst = out;
      p.rows = N;
      p.cols = K;
      p.ld_dst = K;
      p.src = static_cast<const float*>(w);
      p.src_rows = N;
      p.src_cols = K;
      dn::pack_fp8(p, reinterpret_cast<float*>(static_cast<char*>(out) + dn::gemm_fp8_code_bytes(N, K)),
                   as_stream(stream));
      return;
    }
    DN_CHECK(N >= 1 && K >= 1 && K % 16 == 0, "dn_pack_weight: bad sizes (K must be a multiple of 16)");
    if (dtype == DN_BF16 && dn::gemm_frag_layout(N, K)) {
      dn::to_frag(static_cast<const dn::bf16*>(w), N, K, K, static_cast<dn::bf16*>(out), as_stream(stream));
    } else {
      const size_t bytes = (size_t)N * K * (dtype == DN_BF16 ? 2 : 4);
      DN_HIP(hipMemcpyAsync(out, w, bytes, hipMemcpyDeviceToDevice, as_stream(stream)));
    }
  });
}

dn_status dn_op_linear(int32_t dtype, const void* x, const void* w, const float* bias, const void* resid,
                       int32_t resid_f32, void* y, int32_t y_f32, int64_t M, int32_t N, int32_t K, int32_t geglu,
                       void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype_op(dtype), "dn_op_linear: bad dtype");
    DN_CHECK(x && w && y, "dn_op_linear: null pointer");
    DN_CHECK(M >= 1 && M <= 0x7fffffff && N >= 1 && K >= 1, "dn_op_linear: bad sizes");
    DN_CHECK(!geglu || N % 32 == 0, "dn_op_linear: GEGLU needs N % 32 == 0");
    DN_CHECK(!(geglu && resid), "dn_op_linear: GEGLU takes no residual");
    if (dtype == DN_MXFP4) {
      DN_CHECK(N <= 0x3fffffff && dn::gemm_mx4_layout(geglu ? 2 * N : N, K),
               "dn_op_linear: DN_MXFP4 needs N % 32 == 0 and K % 128 == 0, N (GEGLU: 2N) and K at most 2^22");
      dn::GemmMx4Params q;
      q.a = x;
      q.b = w;
      q.M = static_cast<int>(M);
      q.N = geglu ? 2 * N : N;
      q.K = K;
      q.bias = bias;
      q.resid = resid;
      q.resid_f32 = resid_f32;
      q.out = y;
      q.out_f32 = y_f32;
      q.geglu = geglu;
      dn::gemm_mx4_check(q);
      dn::gemm_mx4(q, current_cus(), as_stream(stream));
      return;
    }
    dn::GemmParams p;
    p.a0 = x;
    p.c0 = K;
    p.lda0 = K;
    p.taps = 1;
    p.b = w;
    p.ldb = K;
    p.M = static_cast<int>(M);
    p.N = geglu ? 2 * N : N;
    p.K = K;
    p.bias = bias;
    p.resid = resid;
    p.ldr = N;
    p.resid_f32 = resid_f32;
    p.out = y;
    p.ldo = N;
    p.out_f32 = y_f32;
    p.n_store = N;
    p.geglu = geglu;
    if (dtype == DN_FP8) {
      const int Nw = geglu ? 2 * N : N;
      DN_CHECK(dn::gemm_fp8_layout(Nw, K), "dn_op_linear: DN_FP8 needs N % 32 == 0 and K % 128 == 0");
      p.wscale = reinterpret_cast<const float*>(static_cast<const char*>(w) + dn::gemm_fp8_code_bytes(Nw, K));
      p.out_fp8 = !y_f32 && geglu;
      op_gemm<dn::bf16>(p, as_stream(stream));
    } else if (dtype == DN_BF16) {
      op_gemm<dn::bf16>(p, as_stream(stream));
    } else {
      op_gemm<float>(p, as_stream(stream));
    }
  });
}

dn_status dn_op_conv3x3(int32_t dtype, const void* x, int32_t n, int32_t H, int32_t W, int32_t Cin, int32_t up,
                        int32_t stride, const void* w, const float* bias, const float* temb, const void* resid,
                        void* y, int32_t Cout, int32_t y_f32, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype(dtype), "dn_op_conv3x3: bad dtype");
    DN_CHECK(x && w && y, "dn_op_conv3x3: null pointer");
    DN_CHECK(n >= 1 && H >= 1 && W >= 1 && Cin >= 1 && Cout >= 1, "dn_op_conv3x3: bad sizes");
    DN_CHECK(up == 0 || up == 1, "dn_op_conv3x3: up must be 0 or 1");
    DN_CHECK(stride == 1 || stride == 2, "dn_op_conv3x3: stride must be 1 or 2");
    const int hl = up ? 2 * H : H, wl = up ? 2 * W : W;
    const int ho = (hl - 1) / stride + 1, wo = (wl - 1) / stride + 1;
    dn::GemmParams p;
    p.a0 = x;
    p.c0 = Cin;
    p.lda0 = Cin;
    p.taps = 9;
    p.in_h = H;
    p.in_w = W;
    p.up = up;
    p.out_h = ho;
    p.out_w = wo;
    p.stride = stride;
    p.b = w;
    p.ldb = 9 * Cin;
    p.M = n * ho * wo;
    p.N = Cout;
    p.K = 9 * Cin;
    p.bias = bias;
    p.rowvec = temb;
    p.rowvec_ld = Cout;
    p.rows_per_sample = ho * wo;
    p.resid = resid;
    p.ldr = Cout;
    p.out = y;
    p.ldo = Cout;
    p.out_f32 = y_f32;
    p.n_store = Cout;
    if (dtype == DN_BF16)
      op_gemm<dn::bf16>(p, as_stream(stream));
    else
      op_gemm<float>(p, as_stream(stream));
  });
}

dn_status dn_op_attention(int32_t dtype, const void* q, int32_t ldq, const void* k, int32_t ldk, const void* vt,
                          int32_t vt_ld, void* o, int32_t ldo, int32_t B, int32_t heads, int32_t Sq, int32_t Skv,
                          int32_t head_stride, float scale, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype(dtype), "dn_op_attention: bad dtype");
    DN_CHECK(q && k && vt && o, "dn_op_attention: null pointer");
    DN_CHECK(head_stride == 32 || head_stride == 64, "dn_op_attention: head_stride must be 32 or 64");
    DN_CHECK(B >= 1 && heads >= 1 && Sq >= 1 && Skv >= 1, "dn_op_attention: bad sizes");
    DN_CHECK(ldq >= heads * head_stride && ldk >= heads * head_stride && ldo >= heads * head_stride,
             "dn_op_attention: leading dimension smaller than heads * head_stride");
    DN_CHECK(vt_ld >= (Skv + 63) / 64 * 64, "dn_op_attention: vt_ld must cover Skv rounded up to 64");
    dn::AttnParams a;
    a.q = q;
    a.k = k;
    a.vt = vt;
    a.o = o;
    a.ldq = ldq;
    a.ldk = ldk;
    a.vt_ld = vt_ld;
    a.ldo = ldo;
    a.q_bs = (long long)Sq * ldq;
    a.k_bs = (long long)Skv * ldk;
    a.o_bs = (long long)Sq * ldo;
    a.B = B;
    a.heads = heads;
    a.Sq = Sq;
    a.Skv = Skv;
    a.scale_log2 = scale * 1.4426950408889634f;
    const int cus = current_cus();
    if (dtype == DN_BF16)
      dn::attention<dn::bf16>(a, head_stride, cus, as_stream(stream));
    else
      dn::attention<float>(a, head_stride, cus, as_stream(stream));
  });
}

dn_status dn_rope_table(const double* freqs, const int32_t* axis_dims, int32_t n_axes, void* table, void* stream) {
  return guarded([&] {
    DN_CHECK(freqs && axis_dims && table, "dn_rope_table: null pointer");
    DN_CHECK(on(table, 16), "dn_rope_table: the table must be 16-byte aligned");
    DN_CHECK(n_axes >= 1 && n_axes <= DN_ROPE_MAX_AXES, "dn_rope_table: one to four axes");
    dn::RopeTableParams p = {};
    int n = 0;
    for (int a = 0; a < n_axes; ++a) {
      DN_CHECK(axis_dims[a] >= 2 && axis_dims[a] % 2 == 0 && axis_dims[a] <= DN_ROPE_MAX_DIM - 2 * n,
               "dn_rope_table: axis dims must be even and at most 256 together");
      for (int j = 0; j < axis_dims[a] / 2; ++j, ++n) {
        DN_CHECK(std::isfinite(freqs[n]) && std::fabs(freqs[n]) <= 65536.0,
                 "dn_rope_table: frequencies must be finite, at most 65536");
        p.turn[n] = dn::rope_turn(freqs[n]);
        p.axis[n] = static_cast<unsigned char>(a);
      }
    }
    dn::rope_table(p, table, as_stream(stream));
  });
}

dn_status dn_op_rope(int32_t dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t T, int32_t heads,
                     int32_t head_dim, const dn_rotation* rot, void* stream) {
  return guarded([&] {
    dn::RotaryParams p = rotation("dn_op_rope", dtype, T, head_dim, rot);
    DN_CHECK(heads >= 1 && heads <= 65535, "dn_op_rope: bad head count");
    check_heads("dn_op_rope", dtype, x, ldx, (int64_t)heads * head_dim);
    check_heads("dn_op_rope", dtype, y, ldy, (int64_t)heads * head_dim);
    DN_CHECK(x != y || ldx == ldy, "dn_op_rope: in place needs one row stride");
    p.q = x;
    p.qo = y;
    p.ldq = ldx;
    p.ldqo = ldy;
    p.heads = heads;
    run_rotary(dtype, p, stream);
  });
}

dn_status dn_op_qk_norm_rope(int32_t dtype, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                             int64_t ldv, int64_t T, int32_t heads, int32_t kv_heads, int32_t head_dim,
                             const float* q_gain, const float* k_gain, float eps, const dn_rotation* rot,
                             const dn_sequences* seqs, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* v_out,
                             int64_t ldvo, int64_t kv_rows, void* stream) {
  return guarded([&] {
    const char* who = "dn_op_qk_norm_rope";
    dn::RotaryParams p = rotation(who, dtype, T, head_dim, rot);
    DN_CHECK(heads >= 1 && heads <= 65535 && kv_heads >= 1 && kv_heads <= 65535, "dn_op_qk_norm_rope: bad head counts");
    DN_CHECK(q_gain && k_gain && on(q_gain, 4) && on(k_gain, 4), "dn_op_qk_norm_rope: null or misaligned gains");
    DN_CHECK(eps >= 0.f && std::isfinite(eps), "dn_op_qk_norm_rope: eps must be finite and not negative");
    DN_CHECK((v == nullptr) == (v_out == nullptr), "dn_op_qk_norm_rope: values and their output go together");
    const int64_t wq = (int64_t)heads * head_dim, wk = (int64_t)kv_heads * head_dim;
    check_heads(who, dtype, q, ldq, wq);
    check_heads(who, dtype, q_out, ldqo, wq);
    check_heads(who, dtype, k, ldk, wk);
    check_heads(who, dtype, k_out, ldko, wk);
    if (v) {
      check_heads(who, dtype, v, ldv, wk);
      check_heads(who, dtype, v_out, ldvo, wk);
    }
    DN_CHECK(q != q_out || ldq == ldqo, "dn_op_qk_norm_rope: in place needs one row stride");
    if (seqs) {
      DN_CHECK(k != k_out && (!v || v != v_out), "dn_op_qk_norm_rope: with sequences keys and values are not written in place");
      DN_CHECK(kv_rows >= 1 && kv_rows <= (1ll << 40), "dn_op_qk_norm_rope: bad kv_rows");
      p.seqs = sequences(who, seqs);
      p.kv_rows = kv_rows;
    } else {
      DN_CHECK((k != k_out || ldk == ldko) && (!v || v != v_out || ldv == ldvo), "dn_op_qk_norm_rope: in place needs one row stride");
    }
    p.q = q, p.k = k, p.v = v, p.qo = q_out, p.ko = k_out, p.vo = v_out;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldqo = ldqo, p.ldko = ldko, p.ldvo = ldvo;
    p.heads = heads;
    p.kv_heads = kv_heads;
    p.v_heads = v ? kv_heads : 0;
    p.gq = q_gain;
    p.gk = k_gain;
    p.eps = eps;
    run_rotary(dtype, p, stream);
  });
}

dn_status dn_attention_packed_bytes(int32_t dtype, int64_t T, int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t n,
                                    int32_t max_kv_len, int64_t* bytes) {
  return guarded([&] {
    DN_CHECK(bytes, "dn_attention_packed_bytes: null pointer");
    check_packed_sizes("dn_attention_packed_bytes", dtype, T, heads, kv_heads, head_dim);
    DN_CHECK(n >= 1 && max_kv_len >= 1, "dn_attention_packed_bytes: bad sizes");
    *bytes = static_cast<int64_t>(
        dn::attention_packed_bytes(dtype == DN_BF16 ? 2 : 4, T, heads, kv_heads, head_dim, n, max_kv_len));
  });
}

dn_status dn_op_attention_packed(int32_t dtype, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                                 int64_t ldv, void* o, int64_t ldo, int64_t T, int64_t kv_rows, int32_t heads,
                                 int32_t kv_heads, int32_t head_dim, const dn_sequences* seqs, int32_t causal, float scale,
                                 void* ws, void* stream) {
  return guarded([&] {
    const char* who = "dn_op_attention_packed";
    check_packed_sizes(who, dtype, T, heads, kv_heads, head_dim);
    DN_CHECK(kv_rows >= 1 && kv_rows <= (1ll << 40), "dn_op_attention_packed: bad kv_rows");
    DN_CHECK(seqs, "dn_op_attention_packed: null sequences");
    DN_CHECK(causal == 0 || causal == 1, "dn_op_attention_packed: causal is 0 or 1");
    DN_CHECK(std::fabs(scale) <= 1e38f, "dn_op_attention_packed: the scale's magnitude is at most 1e38");
    const int64_t wq = (int64_t)heads * head_dim, wk = (int64_t)kv_heads * head_dim;
    check_heads(who, dtype, q, ldq, wq);
    check_heads(who, dtype, k, ldk, wk);
    check_heads(who, dtype, v, ldv, wk);
    check_heads(who, dtype, o, ldo, wq);
    DN_CHECK(o != q && o != k && o != v, "dn_op_attention_packed: the output is not written in place");
    dn::PackedAttnParams p;
    p.seqs = sequences(who, seqs);
    p.q = q, p.k = k, p.v = v, p.o = o;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv, p.ldo = ldo;
    p.T = T;
    p.kv_rows = kv_rows;
    p.heads = heads;
    p.kv_heads = kv_heads;
    p.max_kv = seqs->max_kv_len;
    p.causal = causal != 0;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.ws = ws;
    DN_CHECK(ws ? on(ws, 16)
                : dn::attention_packed_bytes(dtype == DN_BF16 ? 2 : 4, T, heads, kv_heads, head_dim, seqs->n, p.max_kv) == 0,
             "dn_op_attention_packed: the workspace of dn_attention_packed_bytes is needed, 16-byte aligned");
    dtype == DN_BF16 ? dn::attention_packed<dn::bf16>(p, head_dim, as_stream(stream))
                     : dn::attention_packed<float>(p, head_dim, as_stream(stream));
  });
}

dn_status dn_op_linear_vt(int32_t dtype, const void* x, const void* w, const float* bias, void* y, int64_t M,
                          int32_t N, int32_t K, int32_t vt_col0, void* vt, int32_t heads, int32_t head_stride,
                          int32_t seq, int32_t vt_ld, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype(dtype), "dn_op_linear_vt: bad dtype");
    DN_CHECK(x && w && y && vt, "dn_op_linear_vt: null pointer");
    DN_CHECK(M >= 1 && M <= 0x7fffffff && N >= 1 && K >= 1, "dn_op_linear_vt: bad sizes");
    DN_CHECK(vt_col0 >= 4 && vt_col0 % 4 == 0 && vt_col0 < N, "dn_op_linear_vt: vt_col0 must be in [4, N), % 4 == 0");
    DN_CHECK(head_stride >= 4 && head_stride % 4 == 0 && heads >= 1 && (N - vt_col0) == heads * head_stride,
             "dn_op_linear_vt: N - vt_col0 must equal heads * head_stride (a multiple of 4)");
    DN_CHECK(seq >= 1 && M % seq == 0 && vt_ld >= seq, "dn_op_linear_vt: rows must be whole sequences, vt_ld >= seq");
    dn::GemmParams p;
    p.a0 = x;
    p.c0 = K;
    p.lda0 = K;
    p.taps = 1;
    p.b = w;
    p.ldb = K;
    p.M = static_cast<int>(M);
    p.N = N;
    p.K = K;
    p.bias = bias;
    p.out = y;
    p.ldo = vt_col0;
    p.n_store = N;
    p.vt = vt;
    p.vt_col0 = vt_col0;
    p.vt_dp = head_stride;
    p.vt_heads = heads;
    p.vt_seq = seq;
    p.vt_ld = vt_ld;
    if (dtype == DN_BF16)
      op_gemm<dn::bf16>(p, as_stream(stream));
    else
      op_gemm<float>(p, as_stream(stream));
  });
}

dn_status dn_op_groupnorm(int32_t dtype, const void* x, void* y, int32_t n, int32_t HW, int32_t C, int32_t G,
                          const float* gamma, const float* beta, float eps, int32_t silu, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype(dtype), "dn_op_groupnorm: bad dtype");
    DN_CHECK(x && y && gamma && beta, "dn_op_groupnorm: null pointer");
    DN_CHECK(n >= 1 && HW >= 1 && C >= 1 && G >= 1 && C % G == 0, "dn_op_groupnorm: bad sizes");
    int dev = 0;
    DN_HIP(hipGetDevice(&dev));
    const size_t part = dn::groupnorm_workspace_floats(n, HW, C, G);
    float* ws = nullptr;
    {
      std::lock_guard<std::mutex> lk(g_op_mu);
      OpDev& d = op_dev_locked(dev);
      grow(&d.gn, &d.gn_floats, part + (size_t)2 * n * C);
      ws = d.gn;
    }
    dn::GroupNormParams p;
    p.cus = current_cus();
    p.x0 = x;
    p.c0 = C;
    p.n = n;
    p.HW = HW;
    p.G = G;
    p.gamma = gamma;
    p.beta = beta;
    p.eps = eps;
    p.silu = silu;
    p.y = y;
    p.partial = ws;
    p.stats = ws + part;
    if (dtype == DN_BF16)
      dn::groupnorm<dn::bf16>(p, as_stream(stream));
    else
      dn::groupnorm<float>(p, as_stream(stream));
  });
}

dn_status dn_op_layernorm(int32_t dtype, const float* x, void* y, int64_t M, int32_t C, const float* gamma,
                          const float* beta, float eps, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype_op(dtype), "dn_op_layernorm: bad dtype");
    DN_CHECK(x && y && gamma && beta, "dn_op_layernorm: null pointer");
    if (dtype == DN_MXFP4)
      dn::layernorm<dn::Mx4Row>(x, static_cast<dn::Mx4Row*>(y), M, C, gamma, beta, eps, as_stream(stream));
    else if (dtype == DN_FP8)
      dn::layernorm<uint8_t>(x, static_cast<uint8_t*>(y), M, C, gamma, beta, eps, as_stream(stream));
    else if (dtype == DN_BF16)
      dn::layernorm<dn::bf16>(x, static_cast<dn::bf16*>(y), M, C, gamma, beta, eps, as_stream(stream));
    else
      dn::layernorm<float>(x, static_cast<float*>(y), M, C, gamma, beta, eps, as_stream(stream));
  });
}

dn_status dn_op_layernorm_slabs(int32_t dtype, float* x, void* y, int64_t M, int32_t C, const float* gamma,
                                const float* beta, float eps, const float* slabs, int32_t nsplit, const float* bias,
                                int32_t resid, void* stream) {
  return guarded([&] {
    DN_CHECK(is_dtype(dtype), "dn_op_layernorm_slabs: bad dtype");
    DN_CHECK(x && y && gamma && beta && slabs, "dn_op_layernorm_slabs: null pointer");
    DN_CHECK(nsplit >= 1 && nsplit <= 8, "dn_op_layernorm_slabs: nsplit must be in [1, 8]");
    DN_CHECK(resid == 0 || resid == 1, "dn_op_layernorm_slabs: resid must be 0 or 1");
    if (dtype == DN_BF16)
      dn::layernorm_reduce<dn::bf16>(x, static_cast<dn::bf16*>(y), M, C, gamma, beta, eps, slabs, nsplit, bias,
                                     resid != 0, as_stream(stream));
    else
      dn::layernorm_reduce<float>(x, static_cast<float*>(y), M, C, gamma, beta, eps, slabs, nsplit, bias,
                                  resid != 0, as_stream(stream));
  });
}

dn_status dn_probe_mfma_rate(int32_t iters, double* tflops, double* clock_ghz) {
  return guarded([&] {
    DN_CHECK(tflops && clock_ghz, "dn_probe_mfma_rate: null pointer");
    DN_CHECK(iters >= 1 && iters <= (1 << 20), "dn_probe_mfma_rate: iters must be in [1, 2^20]");
    dn::mfma_rate(iters, tflops, clock_ghz);
  });
}

dn_status dn_vae_weight_count(const dn_vae_config* cfg, size_t* n_floats) {
  return guarded([&] {
    DN_CHECK(cfg && n_floats, "dn_vae_weight_count: null pointer");
    const auto t = dn::vae_weight_table(*cfg);
    *n_floats = static_cast<size_t>(t.back().offset + t.back().numel);
  });
}

dn_status dn_vae_weight_table(const dn_vae_config* cfg, int64_t* numel, int32_t* fan_in, int32_t* kind,
                              size_t capacity, size_t* n_tensors) {
  return guarded([&] {
    DN_CHECK(cfg && n_tensors, "dn_vae_weight_table: null pointer");
    const auto t = dn::vae_weight_table(*cfg);
    DN_CHECK(capacity == 0 || capacity >= t.size(), "dn_vae_weight_table: capacity too small");
    DN_CHECK(capacity == 0 || (numel && fan_in && kind), "dn_vae_weight_table: null output array");
    if (capacity)
      for (size_t i = 0; i < t.size(); ++i) {
        numel[i] = t[i].numel;
        fan_in[i] = t[i].fan_in;
        kind[i] = t[i].kind;
      }
    *n_tensors = t.size();
  });
}

dn_status dn_vae_create(const dn_vae_config* cfg, const float* weights, size_t n_floats, int32_t weights_location,
                        dn_vae** out) {
  return guarded([&] {
    DN_CHECK(cfg && weights && out, "dn_vae_create: null pointer");
    DN_CHECK(weights_location == DN_WEIGHTS_HOST || weights_location == DN_WEIGHTS_DEVICE,
             "dn_vae_create: bad weights_location");
    dn::Vae* v = dn::vae_create(*cfg, weights, n_floats, weights_location == DN_WEIGHTS_DEVICE);
    dn_vae* h = new dn_vae();
    h->v = v;
    *out = h;
  });
}

dn_status dn_vae_decode(dn_vae* h, const float* latent, float* image, void* stream) {
  return guarded([&] {
    DN_CHECK(h && h->v, "dn_vae_decode: null handle");
    dn::vae_decode(h->v, latent, image, as_stream(stream));
  });
}

void dn_vae_destroy(dn_vae* h) {
  if (!h) return;
  dn::vae_destroy(h->v);
  delete h;
}

void dn_destroy(dn_handle* h) {
  if (!h) return;
  dn::model_destroy(h->m);
  delete h;
}

const char* dn_last_error(void) { return g_last_error.c_str(); }

}  // extern "C"
