"""ctypes binding of ``libargus_dn.so`` (the C ABI in include/argus_dn.h).

Argument marshalling only: every step of the denoise loop and of the cache
lookup runs in the library's HIP kernels. PyTorch tensors serve as device
buffers (``data_ptr()``) and PyTorch streams as HIP streams. Importing this
module raises if the library has not been built: there is no fallback.
"""

import ctypes as C
import functools
import os
import struct

import numpy as np

from .workloads import DnConfig, VaeConfig

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libargus_dn.so")

DN_OK, DN_EINVAL, DN_ENOMEM, DN_EHIP, DN_EUNSUPPORTED = 0, -1, -2, -3, -4
DN_FP32, DN_BF16, DN_FP8, DN_MXFP4, DN_MXFP8, DN_FP16 = 0, 1, 2, 3, 4, 5
DN_WEIGHTS_HOST, DN_WEIGHTS_DEVICE = 0, 1
DN_ROPE_PAIRS, DN_ROPE_HALVES = 0, 1
DN_ROPE_TABLE_BYTES = 2048
ABI_VERSION = 1
MAX_LEVELS = 4

EXPORTED = ("dn_weight_count", "dn_weight_table", "dn_create", "dn_denoise", "dn_denoise_capture", "dn_unet_eps", "ac_lookup",
            "ac_lookup_batch", "ac_lookup_batch_k", "ac_lookup_batch_noalloc", "ac_fetch_latent", "dn_packed_weight_elems", "dn_pack_weight", "dn_op_linear", "dn_op_conv3x3",
            "dn_op_attention", "dn_op_groupnorm", "dn_op_layernorm", "dn_op_layernorm_slabs", "dn_op_linear_vt",
            "dn_probe_mfma_rate",
            "dn_destroy", "dn_last_error", "dn_vae_weight_count", "dn_vae_weight_table", "dn_vae_create",
            "dn_vae_decode", "dn_vae_destroy", "dn_mx_bytes", "dn_mx_quantize", "dn_mx_dequantize", "ac_mx_store_bytes",
            "ac_mx_store", "ac_mx_fetch", "ac_mx_lookup_bytes", "ac_mx_lookup", "dn_rope_table", "dn_op_rope", "dn_op_qk_norm_rope",
            "dn_attention_packed_bytes", "dn_op_attention_packed", "argus_oda", "argus_route", "argus_select_worker", "argus_last_error")


AC_MAX_K_LEVELS = 16


class _KTable(C.Structure):
    _fields_ = [("n_thresholds", C.c_int32), ("threshold", C.c_float * (AC_MAX_K_LEVELS - 1)),
                ("level", C.c_int32 * AC_MAX_K_LEVELS)]


class DnError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"[{code}] {msg}")
        self.code = code


class _Level(C.Structure):
    _fields_ = [("channels", C.c_int32), ("depth", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32)]


class _Config(C.Structure):
    _fields_ = [
        ("abi_version", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32),
        ("latent_c", C.c_int32), ("latent_h", C.c_int32), ("latent_w", C.c_int32),
        ("model_channels", C.c_int32), ("n_levels", C.c_int32), ("level", _Level * MAX_LEVELS),
        ("layers_per_block", C.c_int32), ("mid_depth", C.c_int32), ("tiny_topology", C.c_int32),
        ("ctx_len", C.c_int32), ("ctx_dim", C.c_int32), ("ff_mult", C.c_int32), ("gn_groups", C.c_int32),
        ("gn_eps", C.c_float), ("tx_gn_eps", C.c_float), ("ln_eps", C.c_float),
        ("n_train_steps", C.c_int32), ("beta_start", C.c_float), ("beta_end", C.c_float),
        ("beta_schedule", C.c_int32),
    ]


class _VaeConfig(C.Structure):
    _fields_ = [
        ("abi_version", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int32),
        ("latent_c", C.c_int32), ("latent_h", C.c_int32), ("latent_w", C.c_int32),
        ("n_levels", C.c_int32), ("channels", C.c_int32 * MAX_LEVELS), ("layers_per_block", C.c_int32),
        ("gn_groups", C.c_int32), ("gn_eps", C.c_float), ("scaling_factor", C.c_float), ("out_c", C.c_int32),
    ]


class _Sequences(C.Structure):
    _fields_ = [("n", C.c_int32), ("max_kv_len", C.c_int32), ("q_start", C.c_void_p), ("kv_start", C.c_void_p),
                ("kv_len", C.c_void_p)]


def _load():
    # One HIP runtime per process: PyTorch bundles its own libamdhip64 with the
    # same soname as ROCm's. Importing torch first makes the library bind to that
    # already-loaded runtime, so torch's streams and allocations are the library's.
    import torch  # noqa: F401
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with __graft_entry__.build() "
                          "(python -c 'import __graft_entry__ as g; g.build()')")
    lib = C.CDLL(_LIB_PATH)
    P, I32, I64, F32, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    sig = {
        "dn_weight_count": [C.POINTER(_Config), C.POINTER(SZ)],
        "dn_weight_table": [C.POINTER(_Config), P, P, P, SZ, C.POINTER(SZ)],
        "dn_create": [C.POINTER(_Config), P, SZ, I32, C.POINTER(P)],
        "dn_denoise": [P, P, P, P, I32, I32, I32, F32, P],
        "dn_denoise_capture": [P, P, P, P, I32, I32, I32, F32, P, I32, P, P],
        "dn_unet_eps": [P, P, I32, P, F32, P, P, P],
        "ac_lookup": [P, P, I64, I32, C.POINTER(I64), C.POINTER(F32)],
        "ac_lookup_batch": [P, I32, P, I64, I32, C.POINTER(I64), C.POINTER(F32)],
        "ac_lookup_batch_k": [P, I32, P, I64, I32, C.POINTER(_KTable), P, P, P],
        "ac_lookup_batch_noalloc": [P, I32, P, I64, I32, P, P, P],
        "ac_fetch_latent": [P, I64, I64, I64, P, P],
        "dn_mx_bytes": [I32, I64, I64, C.POINTER(I64)],
        "dn_mx_quantize": [I32, I32, P, I64, I64, I64, P, P],
        "dn_mx_dequantize": [I32, P, I64, I64, P, I64, P],
        "ac_mx_store_bytes": [I64, I64, C.POINTER(I64)],
        "ac_mx_store": [I32, I32, P, I64, I64, P, P, I64, I64, P, P],
        "ac_mx_fetch": [I32, P, I64, I64, P, I64, P, I64, P],
        "ac_mx_lookup_bytes": [I32, I64, I32, C.POINTER(I64)],
        "ac_mx_lookup": [I32, P, I32, P, I64, I32, C.POINTER(_KTable), P, P, P, P, P],
        "dn_rope_table": [P, P, I32, P, P],
        "dn_op_rope": [I32, P, I64, P, I64, I64, I32, I32, P, P],
        "dn_op_qk_norm_rope": [I32, P, I64, P, I64, P, I64, I64, I32, I32, I32, P, P, F32, P,
                               C.POINTER(_Sequences), P, I64, P, I64, P, I64, I64, P],
        "dn_attention_packed_bytes": [I32, I64, I32, I32, I32, I32, I32, C.POINTER(I64)],
        "dn_op_attention_packed": [I32, P, I64, P, I64, P, I64, P, I64, I64, I64, I32, I32, I32, C.POINTER(_Sequences), I32,
                                   F32, P, P],
        "dn_packed_weight_elems": [I32, I32, I32, C.POINTER(I64)],
        "dn_pack_weight": [I32, P, I32, I32, P, P],
        "dn_op_linear": [I32, P, P, P, P, I32, P, I32, I64, I32, I32, I32, P],
        "dn_op_conv3x3": [I32, P, I32, I32, I32, I32, I32, I32, P, P, P, P, P, I32, I32, P],
        "dn_op_attention": [I32, P, I32, P, I32, P, I32, P, I32, I32, I32, I32, I32, I32, F32, P],
        "dn_op_linear_vt": [I32, P, P, P, P, I64, I32, I32, I32, P, I32, I32, I32, I32, P],
        "dn_op_groupnorm": [I32, P, P, I32, I32, I32, I32, P, P, F32, I32, P],
        "dn_op_layernorm": [I32, P, P, I64, I32, P, P, F32, P],
        "dn_op_layernorm_slabs": [I32, P, P, I64, I32, P, P, F32, P, I32, P, I32, P],
        "dn_probe_mfma_rate": [I32, C.POINTER(C.c_double), C.POINTER(C.c_double)],
        "argus_oda": [P, P, I32, P],
        "argus_route": [P, I32, I32, C.c_double, C.POINTER(I32)],
        "argus_select_worker": [P, P, P, I32, I32, C.POINTER(I32)],
        "argus_last_error": [],
        "dn_vae_weight_count": [C.POINTER(_VaeConfig), C.POINTER(SZ)],
        "dn_vae_weight_table": [C.POINTER(_VaeConfig), P, P, P, SZ, C.POINTER(SZ)],
        "dn_vae_create": [C.POINTER(_VaeConfig), P, SZ, I32, C.POINTER(P)],
        "dn_vae_decode": [P, P, P, P],
        "dn_vae_destroy": [P],
        "dn_destroy": [P],
        "dn_last_error": [],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = C.c_int
    lib.dn_destroy.restype = None
    lib.dn_vae_destroy.restype = None
    lib.dn_last_error.restype = C.c_char_p
    lib.argus_last_error.restype = C.c_char_p
    return lib


lib = _load()


def _check(code):
    if code != DN_OK:
        raise DnError(code, lib.dn_last_error().decode())


def _ptr(t):
    """Device (or host numpy) address of a buffer; None -> NULL."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


@functools.lru_cache(maxsize=None)
def _raw_stream():
    """Function that gives the current stream's handle. torch.cuda.current_stream() builds an object first,
    2.8 us of a call whose launch takes 3."""
    import torch
    device, raw = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if device is None or raw is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    torch.cuda.init()
    return lambda: raw(device())


def _stream(stream):
    if stream is None:
        return _raw_stream()()
    return getattr(stream, "cuda_stream", stream)


def _new(shape, dtype, device, stream):
    """A new tensor for a call on `stream` (None: the current one), of the memory that is free in that stream's order: of the
    current stream's, work that is still to come there may hold it."""
    import torch
    if stream is None or device.type != "cuda":
        return torch.empty(shape, device=device, dtype=dtype)
    with torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(stream, device)):
        return torch.empty(shape, device=device, dtype=dtype)


@functools.lru_cache(maxsize=None)
def _current_device():
    import torch
    return getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _stream_on(device, stream, name):
    """The stream of a call whose tensors all lie on GPU device (-1: they do not)."""
    if device < 0 or device != _current_device()():
        raise ValueError(f"{name}: all tensors must lie on the current GPU")
    return _stream(stream)


def to_c_config(cfg: DnConfig) -> _Config:
    c = _Config()
    c.abi_version = ABI_VERSION
    c.dtype = cfg.dtype
    c.batch = cfg.batch
    c.latent_c, c.latent_h, c.latent_w = cfg.latent_c, cfg.latent_h, cfg.latent_w
    c.model_channels = cfg.model_channels
    c.n_levels = len(cfg.levels)
    for i, lv in enumerate(cfg.levels):
        c.level[i] = _Level(*lv)
    c.layers_per_block = cfg.layers_per_block
    c.mid_depth = cfg.mid_depth
    c.tiny_topology = cfg.tiny_topology
    c.ctx_len, c.ctx_dim, c.ff_mult, c.gn_groups = cfg.ctx_len, cfg.ctx_dim, cfg.ff_mult, cfg.gn_groups
    c.gn_eps, c.tx_gn_eps, c.ln_eps = cfg.gn_eps, cfg.tx_gn_eps, cfg.ln_eps
    c.n_train_steps = cfg.n_train_steps
    c.beta_start, c.beta_end = cfg.beta_start, cfg.beta_end
    c.beta_schedule = cfg.beta_schedule
    return c


def weight_count(cfg):
    n = C.c_size_t()
    _check(lib.dn_weight_count(C.byref(to_c_config(cfg)), C.byref(n)))
    return n.value


def weight_table(cfg):
    """[(numel, fan_in, kind)] with kind as in the C header (0 w, 1 b, 2 scale, 3 shift)."""
    c = to_c_config(cfg)
    n = C.c_size_t()
    _check(lib.dn_weight_table(C.byref(c), None, None, None, 0, C.byref(n)))
    numel = np.zeros(n.value, np.int64)
    fan = np.zeros(n.value, np.int32)
    kind = np.zeros(n.value, np.int32)
    _check(lib.dn_weight_table(C.byref(c), numel.ctypes.data, fan.ctypes.data, kind.ctypes.data, n.value,
                               C.byref(n)))
    return list(zip(numel.tolist(), fan.tolist(), kind.tolist()))


class Denoiser:
    """Owns a dn_handle. ``weights``: fp32 numpy array (host) or CUDA tensor (device)."""

    def __init__(self, cfg: DnConfig, weights):
        self.cfg = cfg
        self._h = C.c_void_p()
        on_dev = not isinstance(weights, np.ndarray)
        if on_dev:
            n = weights.numel()
        else:
            weights = np.ascontiguousarray(weights, dtype=np.float32)
            n = weights.size
        _check(lib.dn_create(C.byref(to_c_config(cfg)), _ptr(weights), n,
                             DN_WEIGHTS_DEVICE if on_dev else DN_WEIGHTS_HOST, C.byref(self._h)))

    def close(self):
        if self._h:
            lib.dn_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def denoise(self, latent, text_ctx, timesteps, start_step, n_steps, cfg_scale, stream=None):
        ts = np.ascontiguousarray(timesteps, dtype=np.int32)
        _check(lib.dn_denoise(self._h, _ptr(latent), _ptr(text_ctx), ts.ctypes.data, ts.size, start_step, n_steps,
                              cfg_scale, _stream(stream)))

    def denoise_capture(self, latent, text_ctx, timesteps, start_step, n_steps, cfg_scale, capture_at, out_latents,
                        stream=None):
        """dn_denoise that also writes the latent after each iteration count in capture_at
        (bf16) to out_latents [len(capture_at), B, C, H, W] (a bf16 CUDA tensor)."""
        ts = np.ascontiguousarray(timesteps, dtype=np.int32)
        cap = np.ascontiguousarray(capture_at, dtype=np.int32)
        _check(lib.dn_denoise_capture(self._h, _ptr(latent), _ptr(text_ctx), ts.ctypes.data, ts.size, start_step,
                                      n_steps, cfg_scale, cap.ctypes.data if cap.size else None, cap.size,
                                      _ptr(out_latents), _stream(stream)))

    def unet_eps(self, x, t, text_ctx, cfg_scale, out_raw, out_guided=None, stream=None):
        _check(lib.dn_unet_eps(self._h, _ptr(x), int(t), _ptr(text_ctx), cfg_scale, _ptr(out_raw),
                               _ptr(out_guided), _stream(stream)))


def to_c_vae_config(cfg: VaeConfig) -> _VaeConfig:
    c = _VaeConfig()
    c.abi_version = ABI_VERSION
    c.dtype, c.batch = cfg.dtype, cfg.batch
    c.latent_c, c.latent_h, c.latent_w = cfg.latent_c, cfg.latent_h, cfg.latent_w
    c.n_levels = len(cfg.block_channels)
    for i, ch in enumerate(cfg.block_channels):
        c.channels[i] = ch
    c.layers_per_block, c.gn_groups, c.gn_eps = cfg.layers_per_block, cfg.gn_groups, cfg.gn_eps
    c.scaling_factor, c.out_c = cfg.scaling_factor, cfg.out_c
    return c


def vae_weight_table(cfg):
    """[(numel, fan_in, kind)] of the decoder's canonical blob."""
    c = to_c_vae_config(cfg)
    n = C.c_size_t()
    _check(lib.dn_vae_weight_table(C.byref(c), None, None, None, 0, C.byref(n)))
    numel = np.zeros(n.value, np.int64)
    fan = np.zeros(n.value, np.int32)
    kind = np.zeros(n.value, np.int32)
    _check(lib.dn_vae_weight_table(C.byref(c), numel.ctypes.data, fan.ctypes.data, kind.ctypes.data, n.value,
                                   C.byref(n)))
    return list(zip(numel.tolist(), fan.tolist(), kind.tolist()))


class Decoder:
    """Owns a dn_vae. ``weights``: fp32 numpy array (host) or CUDA tensor (device)."""

    def __init__(self, cfg: VaeConfig, weights):
        self.cfg = cfg
        self._h = C.c_void_p()
        on_dev = not isinstance(weights, np.ndarray)
        if on_dev:
            n = weights.numel()
        else:
            weights = np.ascontiguousarray(weights, dtype=np.float32)
            n = weights.size
        _check(lib.dn_vae_create(C.byref(to_c_vae_config(cfg)), _ptr(weights), n,
                                 DN_WEIGHTS_DEVICE if on_dev else DN_WEIGHTS_HOST, C.byref(self._h)))

    def decode(self, latent, image, stream=None):
        _check(lib.dn_vae_decode(self._h, _ptr(latent), _ptr(image), _stream(stream)))

    def close(self):
        if self._h:
            lib.dn_vae_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def ac_lookup(query, cache):
    """(index, cosine) of the nearest cache row; query [dim], cache [n, dim] fp16 CUDA tensors."""
    idx = C.c_int64(-7)
    score = C.c_float()
    n, dim = (cache.shape[0], cache.shape[1]) if cache.dim() == 2 else (cache.shape[0], 1)
    _check(lib.ac_lookup(_ptr(query), _ptr(cache), n, dim, C.byref(idx), C.byref(score)))
    return idx.value, score.value


def ac_lookup_raw(query_ptr, cache_ptr, n, dim):
    idx = C.c_int64(-7)
    score = C.c_float()
    code = lib.ac_lookup(query_ptr, cache_ptr, n, dim, C.byref(idx), C.byref(score))
    return code, idx.value, score.value


def ac_lookup_batch(queries, cache):
    """(indices, cosines) of the nearest cache row for every query: queries [nq, dim],
    cache [n, dim] fp16 CUDA tensors. Lists of length nq; index -1 for a zero query."""
    nq, dim = queries.shape
    n = cache.shape[0]
    if cache.shape[1] != dim:
        raise ValueError("ac_lookup_batch: query and cache widths differ")
    idx = (C.c_int64 * nq)()
    score = (C.c_float * nq)()
    _check(lib.ac_lookup_batch(_ptr(queries), nq, _ptr(cache), n, dim, idx, score))
    return list(idx), list(score)


def k_table(thresholds, levels):
    """ac_k_table from thresholds [L] and levels [L + 1] (no checks: the library checks)."""
    t = _KTable()
    t.n_thresholds = len(thresholds)
    for i, v in enumerate(thresholds):
        t.threshold[i] = v
    for i, v in enumerate(levels):
        t.level[i] = v
    return t


def ac_lookup_batch_k(queries, cache, thresholds, levels):
    """(indices, cosines, levels K) for every query: ac_lookup_batch plus the approximation
    level chosen from the retrieved cosine by the threshold table (thresholds [L],
    levels [L + 1])."""
    nq, dim = queries.shape
    if cache.shape[1] != dim:
        raise ValueError("ac_lookup_batch_k: query and cache widths differ")
    if len(thresholds) >= AC_MAX_K_LEVELS or len(levels) > AC_MAX_K_LEVELS:
        raise ValueError("ac_lookup_batch_k: at most 15 thresholds")
    idx = (C.c_int64 * nq)()
    score = (C.c_float * nq)()
    k = (C.c_int32 * nq)()
    tab = k_table(thresholds, levels)
    _check(lib.ac_lookup_batch_k(_ptr(queries), nq, _ptr(cache), cache.shape[0], dim, C.byref(tab), idx, score, k))
    return list(idx), list(score), list(k)


def ac_lookup_batch_noalloc(queries, cache, out_idx, out_score=None, stream=None):
    """ac_lookup_batch on a stream with device outputs and no allocation in the library:
    queries [nq, dim], cache [n, dim] fp16 CUDA tensors; out_idx int64 [nq] and out_score
    float32 [nq] (or None) CUDA tensors receive the results."""
    nq, dim = queries.shape
    if cache.shape[1] != dim:
        raise ValueError("ac_lookup_batch_noalloc: query and cache widths differ")
    _check(lib.ac_lookup_batch_noalloc(_ptr(queries), nq, _ptr(cache), cache.shape[0], dim, _ptr(out_idx),
                                       _ptr(out_score), _stream(stream)))


def ac_fetch_latent(cache_latents, idx, latent, stream=None):
    n = cache_latents.shape[0]
    numel = cache_latents[0].numel()
    _check(lib.ac_fetch_latent(_ptr(cache_latents), n, numel, idx, _ptr(latent), _stream(stream)))


# ----------------------------------------------------------------------------- microscaled rows

# Sizes are functions of their arguments; calls check buffers against them each time.
@functools.lru_cache(maxsize=1024)
def mx_bytes(dtype, rows, cols):
    """Bytes of an MX buffer (DN_MXFP4 or DN_MXFP8) of `rows` rows of `cols` values."""
    n = C.c_int64()
    _check(lib.dn_mx_bytes(dtype, rows, cols, C.byref(n)))
    return n.value


@functools.lru_cache(maxsize=None)
def _row_types():
    import torch
    return {torch.float32: DN_FP32, torch.bfloat16: DN_BF16, torch.float16: DN_FP16}


@functools.lru_cache(maxsize=None)
def _int64():
    import torch
    return torch.int64


@functools.lru_cache(maxsize=None)
def _lookup_types():
    import torch
    return torch.int64, torch.float32, torch.int32


def _rows(x, name):
    """(dtype, row stride, rows, columns) of a row source: a 2-D tensor whose rows are dense."""
    if x.dim() != 2:
        raise ValueError(f"{name}: a 2-D tensor with dense rows is needed")
    (rows, cols), (ld, step) = x.shape, x.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{name}: a 2-D tensor with dense rows is needed")
    dt = _row_types().get(x.dtype)
    if dt is None:
        raise ValueError(f"{name}: rows must be float32, bfloat16 or float16")
    return dt, max(ld, cols) if rows == 1 else ld, rows, cols


def _buffer(t, need, name):
    """Checks a caller's byte buffer (uint8, dense) against the bytes a call accesses."""
    if t.nbytes < need or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous buffer of at least {need} bytes is needed")


def _index(t, name):
    if t.dtype is not _int64() or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{name}: a dense 1-D int64 tensor is needed")


def mx_quantize(dtype, x, q=None, stream=None):
    """Rows x [rows, cols] (float32, bfloat16 or float16, any row stride) -> an MX buffer (uint8
    tensor of mx_bytes bytes; `q` or a new one)."""
    import torch
    xt, ldx, rows, cols = _rows(x, "mx_quantize")
    need = mx_bytes(dtype, rows, cols)
    if q is None:
        q = _new(need, torch.uint8, x.device, stream)
    _buffer(q, need, "mx_quantize")
    _check(lib.dn_mx_quantize(dtype, xt, _ptr(x), ldx, rows, cols, _ptr(q), _stream(stream)))
    return q


def mx_dequantize(dtype, q, rows, cols, y=None, stream=None):
    """The fp32 values [rows, cols] an MX buffer stands for (into `y` or a new tensor)."""
    import torch
    _buffer(q, mx_bytes(dtype, rows, cols), "mx_dequantize")
    if y is None:
        y = _new((rows, cols), torch.float32, q.device, stream)
    yt, ldy, r, c = _rows(y, "mx_dequantize")
    if yt != DN_FP32 or (r, c) != (rows, cols):
        raise ValueError("mx_dequantize: y must be float32 [rows, cols]")
    _check(lib.dn_mx_dequantize(dtype, _ptr(q), rows, cols, _ptr(y), ldy, _stream(stream)))
    return y


@functools.lru_cache(maxsize=1024)
def ac_mx_store_bytes(n_rows, n_slots):
    """Workspace bytes of ac_mx_store (0: none is needed)."""
    n = C.c_int64()
    _check(lib.ac_mx_store_bytes(n_rows, n_slots, C.byref(n)))
    return n.value


def ac_mx_store(dtype, x, slots, table, n_slots, ws=None, stream=None):
    """Quantises row j of x [n, dim] into slot slots[j] (int64 CUDA tensor [n]) of an MX table of
    n_slots slots (uint8, mx_bytes(dtype, n_slots, dim)); ws: uint8, ac_mx_store_bytes(n, n_slots)."""
    xt, ldx, n, dim = _rows(x, "ac_mx_store")
    _index(slots, "ac_mx_store")
    if slots.shape[0] != n:
        raise ValueError("ac_mx_store: one slot per row is needed")
    _buffer(table, mx_bytes(dtype, n_slots, dim), "ac_mx_store")
    need = ac_mx_store_bytes(n, n_slots)
    if ws is not None:
        _buffer(ws, need, "ac_mx_store workspace")
    _check(lib.ac_mx_store(dtype, xt, _ptr(x), ldx, n, _ptr(slots), _ptr(table), n_slots, dim,
                           _ptr(ws) if need else None, _stream(stream)))


def ac_mx_fetch(dtype, table, n_slots, idx, out, stream=None):
    """Row j of out [n, dim] (float32) <- slot idx[j] (int64 CUDA tensor [n]) of an MX table; rows whose
    index lies outside the table (the -1 of a lookup) are left as they are."""
    ot, ldo, n, dim = _rows(out, "ac_mx_fetch")
    _index(idx, "ac_mx_fetch")
    if ot != DN_FP32 or idx.shape[0] != n:
        raise ValueError("ac_mx_fetch: out must be float32 with one row per index")
    _buffer(table, mx_bytes(dtype, n_slots, dim), "ac_mx_fetch")
    _check(lib.ac_mx_fetch(dtype, _ptr(table), n_slots, dim, _ptr(idx), n, _ptr(out), ldo, _stream(stream)))


@functools.lru_cache(maxsize=1024)
def ac_mx_lookup_bytes(nq, n, dim):
    """Workspace bytes of ac_mx_lookup."""
    b = C.c_int64()
    _check(lib.ac_mx_lookup_bytes(nq, n, dim, C.byref(b)))
    return b.value


def ac_mx_lookup(dtype, queries, table, n, ws, out_idx, out_score=None, out_k=None, thresholds=None, levels=None,
                 stream=None):
    """The nearest row of an MX table of n embeddings for every query [nq, dim] (float16, dense): out_idx
    int64, out_score float32 or None, and with a threshold table out_k int32 (CUDA tensors [nq])."""
    qt, ldq, nq, dim = _rows(queries, "ac_mx_lookup")
    if qt != DN_FP16 or ldq != dim:
        raise ValueError("ac_mx_lookup: queries must be dense float16 rows")
    _buffer(table, mx_bytes(dtype, n, dim), "ac_mx_lookup")
    _buffer(ws, ac_mx_lookup_bytes(nq, n, dim), "ac_mx_lookup workspace")
    _index(out_idx, "ac_mx_lookup")
    for t, kind, name in zip((out_idx, out_score, out_k), _lookup_types(), ("out_idx", "out_score", "out_k")):
        if t is not None and (t.numel() < nq or t.dtype is not kind or not t.is_contiguous()):
            raise ValueError(f"ac_mx_lookup: {name} must be dense with one {kind} per query")
    tab = None
    if thresholds is not None:
        if levels is None or len(thresholds) >= AC_MAX_K_LEVELS or len(levels) != len(thresholds) + 1:
            raise ValueError("ac_mx_lookup: at most 15 thresholds, and one level more than thresholds")
        tab = C.byref(k_table(thresholds, levels))
    _check(lib.ac_mx_lookup(dtype, _ptr(queries), nq, _ptr(table), n, dim, tab, _ptr(out_idx), _ptr(out_score),
                            _ptr(out_k), _ptr(ws), _stream(stream)))


# ----------------------------------------------------------------------------- packed sequences

@functools.lru_cache(maxsize=None)
def _head_types():
    import torch
    return {torch.float32: DN_FP32, torch.bfloat16: DN_BF16}


@functools.lru_cache(maxsize=None)
def _plain_types():
    import torch
    return torch.int32, torch.float32


def _heads(x, name):
    """(address, row stride, dtype, shape) of a tensor of heads: [rows, heads, head_dim] with dense heads side by
    side (a slice of a wider projection output is one)."""
    shape, stride = x.shape, x.stride()
    if len(shape) != 3:
        raise ValueError(f"{name}: a tensor [rows, heads, head_dim] is needed")
    dim = shape[2]
    if (stride[2] != 1 and dim > 1) or (stride[1] != dim and shape[1] > 1):
        raise ValueError(f"{name}: the heads of a row must be dense, side by side")
    dt = _head_types().get(x.dtype)
    if dt is None:
        raise ValueError(f"{name}: heads must be float32 or bfloat16")
    # the stride of a single row (one token of a long projection) says nothing
    return x.data_ptr(), shape[1] * dim if shape[0] == 1 else stride[0], dt, shape


def _dense(t, dtype, shape, name):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a dense {dtype} tensor {list(shape)} is needed")
    return t.data_ptr()


class Sequences:
    """The sequences of a packed batch: q_start int32 [n + 1], kv_start int64 [n], kv_len int32 [n] (CUDA tensors, read
    when the work runs; kept until then), and a bound of kv_len the caller knows."""

    def __init__(self, q_start, kv_start, kv_len, max_kv_len):
        import torch
        n = kv_len.shape[0] if kv_len.dim() == 1 else -1
        _dense(kv_len, torch.int32, (n,), "Sequences: kv_len")
        _dense(kv_start, torch.int64, (n,), "Sequences: kv_start")
        _dense(q_start, torch.int32, (n + 1,), "Sequences: q_start")
        self.n, self.max_kv_len = n, int(max_kv_len)
        self.device = kv_len.get_device()
        if not self.device == kv_start.get_device() == q_start.get_device():
            raise ValueError("Sequences: tensors of one device are needed")
        self._keep = (q_start, kv_start, kv_len)
        self._c = _Sequences(n, self.max_kv_len, _ptr(q_start), _ptr(kv_start), _ptr(kv_len))
        self.ref = C.byref(self._c)


def rope_freqs(axis_dims, theta=10000.0, per_axis=True):
    """Frequencies of every rotated pair in axis order: theta^(-2 i / d), over the dims d of its own axis (per_axis)
    or of all axes together."""
    total, out = sum(axis_dims), []
    for d in axis_dims:
        for j in range(d // 2):
            out.append(float(theta) ** (-2.0 * j / d if per_axis else -2.0 * len(out) / total))
    return out


class RopeTable:
    """A rotation table on the GPU (dn_rope_table), filled on `stream`: calls on other streams come after that, and it is kept
    until they have finished."""

    def __init__(self, axis_dims, freqs, device, stream=None):
        import torch
        self.axis_dims = tuple(int(d) for d in axis_dims)
        dims = np.ascontiguousarray(self.axis_dims, dtype=np.int32)
        f = np.ascontiguousarray(freqs, dtype=np.float64)
        if dims.ndim != 1 or f.shape != (sum(self.axis_dims) // 2,):
            raise ValueError("rope_table: one frequency per rotated pair is needed")
        self.rot_dim, self.n_axes = sum(self.axis_dims), len(self.axis_dims)
        self.data = _new(DN_ROPE_TABLE_BYTES, torch.uint8, torch.device(device), stream)
        self.address, self.device = self.data.data_ptr(), self.data.get_device()
        _check(lib.dn_rope_table(f.ctypes.data, dims.ctypes.data, self.n_axes, self.address,
                                 _stream_on(self.device, stream, "rope_table")))


def rope_table(axis_dims, theta=10000.0, per_axis=True, freqs=None, device="cuda", stream=None):
    """The table of a rotation over axes of axis_dims rotated values each (time, height, width, ...); freqs: radians per
    position of every pair (default rope_freqs)."""
    return RopeTable(axis_dims, rope_freqs(axis_dims, theta, per_axis) if freqs is None else freqs, device, stream)


# dn_rotation as bytes: a fifth of the time that a ctypes structure takes, in a call of 5 us
_rotation_bytes = struct.Struct("@PPiii4x").pack


def _rotation(table, pos, rows, pairing, name):
    return _rotation_bytes(table.address, _dense(pos, _plain_types()[0], (rows, table.n_axes), f"{name}: pos"), table.n_axes,
                           table.rot_dim, pairing)


def op_rope(x, pos, table, y=None, pairing=DN_ROPE_PAIRS, stream=None):
    """Rotates the heads of x [rows, heads, head_dim] to pos int32 [rows, axes] (into y, a new tensor, or x itself)."""
    src, ldx, dt, shape = _heads(x, "op_rope")
    if y is None:
        y = _new(shape, x.dtype, x.device, stream)
    dst, ldy, yt, y_shape = _heads(y, "op_rope: y")
    if yt != dt or y_shape != shape:
        raise ValueError("op_rope: y must have the type and shape of x")
    rows, heads, dim = shape
    turn = _rotation(table, pos, rows, pairing, "op_rope")
    dev = x.get_device()
    on = _stream_on(dev if dev == y.get_device() == pos.get_device() == table.device else -1, stream, "op_rope")
    _check(lib.dn_op_rope(dt, src, ldx, dst, ldy, rows, heads, dim, turn, on))
    return y


def op_qk_norm_rope(q, k, q_gain, k_gain, eps, pos, table, q_out, k_out, v=None, v_out=None, seqs=None,
                    pairing=DN_ROPE_PAIRS, stream=None):
    """RMS norm and rotation of every head of q and k [rows, heads, head_dim] into q_out and k_out, v copied to v_out;
    with seqs (Sequences) k_out and v_out are caches whose rows the sequences own."""
    name = "op_qk_norm_rope"
    pq, ldq, dt, shape = _heads(q, name)
    pk, ldk, kt, k_shape = _heads(k, name)
    pqo, ldqo, qot, qo_shape = _heads(q_out, name)
    pko, ldko, kot, ko_shape = _heads(k_out, name)
    rows, heads, dim = shape
    if kt != dt or qot != dt or kot != dt or k_shape[0] != rows or k_shape[2] != dim or qo_shape != shape:
        raise ValueError(f"{name}: types, rows and head widths of q, k and their outputs must agree")
    if (ko_shape[1:] if seqs is not None else ko_shape) != (k_shape[1:] if seqs is not None else k_shape):
        raise ValueError(f"{name}: k_out must have the heads of k, and its rows where there are no sequences")
    pv = pvo = None
    ldv = ldvo = 0
    if (v is None) != (v_out is None):
        raise ValueError(f"{name}: values and their output go together")
    if v is not None:
        pv, ldv, vt, v_shape = _heads(v, name)
        pvo, ldvo, vot, vo_shape = _heads(v_out, name)
        if vt != dt or vot != dt or v_shape != k_shape or vo_shape != ko_shape:
            raise ValueError(f"{name}: values must have the type and shape of the keys, and so must their output")
    f32 = _plain_types()[1]
    pqg = _dense(q_gain, f32, (dim,), "op_qk_norm_rope: q_gain")
    pkg = _dense(k_gain, f32, (dim,), "op_qk_norm_rope: k_gain")
    turn = _rotation(table, pos, rows, pairing, name)
    dev = q.get_device()
    one = (dev == k.get_device() == q_out.get_device() == k_out.get_device() == q_gain.get_device() == k_gain.get_device()
           == pos.get_device() == table.device and (v is None or dev == v.get_device() == v_out.get_device())
           and (seqs is None or dev == seqs.device))
    on = _stream_on(dev if one else -1, stream, name)
    _check(lib.dn_op_qk_norm_rope(dt, pq, ldq, pk, ldk, pv, ldv, rows, heads, k_shape[1], dim, pqg, pkg, eps, turn,
                                  None if seqs is None else seqs.ref, pqo, ldqo, pko, ldko, pvo, ldvo, ko_shape[0], on))


@functools.lru_cache(maxsize=1024)
def _attention_packed_bytes(dtype, rows, heads, kv_heads, dim, n, max_kv_len):
    b = C.c_int64()
    _check(lib.dn_attention_packed_bytes(dtype, rows, heads, kv_heads, dim, n, max_kv_len, C.byref(b)))
    return b.value


def attention_packed_bytes(q, k, seqs):
    """Workspace bytes of op_attention_packed for tensors like q and k (0: none is needed)."""
    _, _, dt, (rows, heads, dim) = _heads(q, "attention_packed_bytes: q")
    return _attention_packed_bytes(dt, rows, heads, k.shape[1], dim, seqs.n, seqs.max_kv_len)


def op_attention_packed(q, k, v, o, seqs, causal=True, scale=None, ws=None, stream=None):
    """Attention of packed sequences: q, o [rows, heads, head_dim], k, v [kv_rows, kv_heads, head_dim]; scale: default
    head_dim^-1/2; ws: uint8, attention_packed_bytes."""
    name = "op_attention_packed"
    pq, ldq, dt, shape = _heads(q, name)
    pk, ldk, kt, k_shape = _heads(k, name)
    pv, ldv, vt, v_shape = _heads(v, name)
    po, ldo, ot, o_shape = _heads(o, name)
    rows, heads, dim = shape
    kv_rows, kv_heads, k_dim = k_shape
    if kt != dt or vt != dt or ot != dt or o_shape != shape or v_shape != k_shape or k_dim != dim:
        raise ValueError(f"{name}: types and shapes of q, k, v and o must agree")
    need = _attention_packed_bytes(dt, rows, heads, kv_heads, dim, seqs.n, seqs.max_kv_len)
    if ws is not None:
        _buffer(ws, need, name)
    dev = q.get_device()
    one = dev == k.get_device() == v.get_device() == o.get_device() == seqs.device and (ws is None or dev == ws.get_device())
    on = _stream_on(dev if one else -1, stream, name)
    _check(lib.dn_op_attention_packed(dt, pq, ldq, pk, ldk, pv, ldv, po, ldo, rows, kv_rows, heads, kv_heads, dim, seqs.ref,
                                      1 if causal else 0, dim ** -0.5 if scale is None else scale,
                                      ws.data_ptr() if need and ws is not None else None, on))


def packed_weight_elems(dtype, N, K):
    n = C.c_int64()
    _check(lib.dn_packed_weight_elems(dtype, N, K, C.byref(n)))
    return n.value


def pack_weight(dtype, w, N, K, stream=None):
    """Row-major device weight [N][K] (dtype elements; fp32 for DN_FP8 and DN_MXFP4) -> a new tensor in
    the GEMM's packed layout (uint8 for those two: codes, then the scales)."""
    import torch
    out = _new(packed_weight_elems(dtype, N, K), torch.uint8 if dtype in (DN_FP8, DN_MXFP4) else w.dtype, w.device, stream)
    _check(lib.dn_pack_weight(dtype, _ptr(w), N, K, _ptr(out), _stream(stream)))
    return out


def op_linear(dtype, x, w, bias, y, M, N, K, resid=None, resid_f32=False, y_f32=False, geglu=False, stream=None):
    _check(lib.dn_op_linear(dtype, _ptr(x), _ptr(w), _ptr(bias), _ptr(resid), int(resid_f32), _ptr(y), int(y_f32),
                            M, N, K, int(geglu), _stream(stream)))


def op_conv3x3(dtype, x, n, H, W, Cin, w, bias, y, Cout, up=0, stride=1, temb=None, resid=None, y_f32=False,
               stream=None):
    _check(lib.dn_op_conv3x3(dtype, _ptr(x), n, H, W, Cin, up, stride, _ptr(w), _ptr(bias), _ptr(temb),
                             _ptr(resid), _ptr(y), Cout, int(y_f32), _stream(stream)))


def op_attention(dtype, q, ldq, k, ldk, vt, vt_ld, o, ldo, B, heads, Sq, Skv, head_stride, scale, stream=None):
    _check(lib.dn_op_attention(dtype, _ptr(q), ldq, _ptr(k), ldk, _ptr(vt), vt_ld, _ptr(o), ldo, B, heads, Sq, Skv,
                               head_stride, scale, _stream(stream)))


def op_linear_vt(dtype, x, w, bias, y, M, N, K, vt_col0, vt, heads, head_stride, seq, vt_ld, stream=None):
    _check(lib.dn_op_linear_vt(dtype, _ptr(x), _ptr(w), _ptr(bias), _ptr(y), M, N, K, vt_col0, _ptr(vt), heads,
                               head_stride, seq, vt_ld, _stream(stream)))


def op_groupnorm(dtype, x, y, n, HW, Cc, G, gamma, beta, eps, silu, stream=None):
    _check(lib.dn_op_groupnorm(dtype, _ptr(x), _ptr(y), n, HW, Cc, G, _ptr(gamma), _ptr(beta), eps, int(silu),
                               _stream(stream)))


def op_layernorm(dtype, x, y, M, Cc, gamma, beta, eps, stream=None):
    _check(lib.dn_op_layernorm(dtype, _ptr(x), _ptr(y), M, Cc, _ptr(gamma), _ptr(beta), eps, _stream(stream)))


def op_layernorm_slabs(dtype, x, y, M, Cc, gamma, beta, eps, slabs, nsplit, bias=None, resid=True, stream=None):
    _check(lib.dn_op_layernorm_slabs(dtype, _ptr(x), _ptr(y), M, Cc, _ptr(gamma), _ptr(beta), eps, _ptr(slabs), nsplit,
                                     _ptr(bias), int(resid), _stream(stream)))


def probe_mfma_rate(iters=4000):
    """(TFLOP/s, GHz): the bf16 matrix-core rate the device sustains and its clock
    meanwhile (dn_probe_mfma_rate; a measurement, not a step of the method)."""
    tf, ghz = C.c_double(0.0), C.c_double(0.0)
    _check(lib.dn_probe_mfma_rate(iters, C.byref(tf), C.byref(ghz)))
    return tf.value, ghz.value


# ----------------------------------------------------------------------------- routing control plane (host)

def _check_ctl(code):
    if code != DN_OK:
        raise DnError(code, lib.argus_last_error().decode())


def oda(H, F):
    """PASM [n, n] (numpy fp64) from the demand histogram H and the load split F."""
    H = np.ascontiguousarray(H, dtype=np.float64)
    F = np.ascontiguousarray(F, dtype=np.float64)
    if H.shape != F.shape or H.ndim != 1:
        raise ValueError("oda: H and F must be 1-D of the same length")
    out = np.zeros((H.size, H.size), np.float64)
    _check_ctl(lib.argus_oda(H.ctypes.data, F.ctypes.data, H.size, out.ctypes.data))
    return out


def route(pasm, level, u):
    pasm = np.ascontiguousarray(pasm, dtype=np.float64)
    out = C.c_int32()
    _check_ctl(lib.argus_route(pasm.ctypes.data, pasm.shape[0], level, u, C.byref(out)))
    return out.value


def select_worker(queue_len, t_proc, worker_level, level):
    q = np.ascontiguousarray(queue_len, dtype=np.int32)
    t = np.ascontiguousarray(t_proc, dtype=np.float64)
    lv = np.ascontiguousarray(worker_level, dtype=np.int32)
    out = C.c_int32()
    _check_ctl(lib.argus_select_worker(q.ctypes.data, t.ctypes.data, lv.ctypes.data, q.size, level, C.byref(out)))
    return out.value
