"""Performance cases of the microscaled (MX) operators.

An MX row holds its values in blocks of 32: one power-of-two scale per block (E8M0) and a code
per value, E2M1 (4 bits) or E4M3 (8 bits). Three users of the format are measured:

- `cache`: rows are quantised into slots of a cache as they are written (ac_mx_store) and read
  back as fp32 (ac_mx_fetch): intermediate latents, prompt embeddings;
- `lookup`: the nearest-prompt search over embeddings held in such a cache (ac_mx_lookup);
- `linear`, `mlp`: the 4-bit product (dn_mx_quantize and dn_op_linear), and the feed-forward of
  a transformer block made of it (dn_op_layernorm, GEGLU layer, output layer with the residual).

Each case is a dict of plain values. `prepare` makes what a program holds before the call, `run`
is one pass: with `own` the library's calls, without it the same in elementary torch operations.
`exact` is the definition in 64-bit floating point, written apart from both.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 32
MX4, MX8 = "mxfp4", "mxfp8"
EMAX = {MX4: 2, MX8: 8}            # exponent of the largest code: 6 = 1.5 * 2^2, 448 = 1.75 * 2^8
TOP = {MX4: 6.0, MX8: 448.0}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}

# approximation levels by the retrieved cosine
THRESHOLDS = [0.775, 0.825, 0.875, 0.925]
LEVELS = [5, 10, 15, 20, 25]


def listed():
    return [
        # The intermediate states of one 1024 x 1024 image at its five cache iterations, written
        # by a worker as it captures them and read back by later prompts.
        {"name": "cache_states_5", "kind": "cache", "fmt": MX4, "src": "bf16", "rows": 5, "cols": 4 * 128 * 128, "slots": 64},
        # The smallest call: one fp32 state of a 200 x 168 pixel image (25 x 21: a ragged last block).
        {"name": "cache_state_ragged", "kind": "cache", "fmt": MX8, "src": "fp32", "rows": 1, "cols": 4 * 25 * 21, "slots": 16},
        # A batch of queued requests resumes: 64 states, 8-bit cache.
        {"name": "cache_states_64", "kind": "cache", "fmt": MX8, "src": "bf16", "rows": 64, "cols": 4 * 128 * 128, "slots": 256},
        # The embedding table is built from 100,000 prompts (the largest call).
        {"name": "cache_embeddings", "kind": "cache", "fmt": MX4, "src": "fp16", "rows": 100000, "cols": 768, "slots": 100000},
        # One request against the 100,000-prompt table.
        {"name": "lookup_one", "kind": "lookup", "fmt": MX4, "nq": 1, "n": 100000, "dim": 768},
        # 64 queued requests against the same table.
        {"name": "lookup_batch", "kind": "lookup", "fmt": MX4, "nq": 64, "n": 100000, "dim": 768},
        # A young 8-bit cache with odd sizes: 9 requests, 4,097 prompts, 500-wide embeddings.
        {"name": "lookup_ragged", "kind": "lookup", "fmt": MX8, "nq": 9, "n": 4097, "dim": 500},
        # One row through a square layer: latency.
        {"name": "linear_one", "kind": "linear", "m": 1, "n": 1280, "k": 1280, "resid": True, "y": "fp32"},
        # The output layer of a feed-forward at 992 x 992 pixels: 2 x 961 rows, residual stream in fp32.
        {"name": "linear_ragged", "kind": "linear", "m": 1922, "n": 1280, "k": 5120, "resid": True, "y": "fp32"},
        # A GEGLU-wide layer over four images' 64 x 64 tokens: the largest product.
        {"name": "linear_large", "kind": "linear", "m": 32768, "n": 5120, "k": 640, "resid": False, "y": "bf16"},
        # The feed-forward of a 32 x 32 block (1280 wide), 60 times an iteration.
        {"name": "mlp_32x32", "kind": "mlp", "m": 2048, "c": 1280},
        # The same at 64 x 64 (640 wide).
        {"name": "mlp_64x64", "kind": "mlp", "m": 8192, "c": 640},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["cache", "cache", "lookup", "lookup", "linear", "linear", "mlp"])
    if kind == "cache":
        rows = _log_int(rng, 1, 20000)
        cols = _log_int(rng, 32, min(4 * 128 * 128, 60000000 // rows))
        return {"kind": kind, "fmt": rng.choice([MX4, MX8]), "src": rng.choice(["fp32", "bf16", "fp16"]), "rows": rows,
                "cols": cols, "slots": rows + rng.randint(0, 100)}
    if kind == "lookup":
        return {"kind": kind, "fmt": rng.choice([MX4, MX8]), "nq": rng.choice([1, _log_int(rng, 2, 64)]),
                "n": _log_int(rng, 100, 100000), "dim": rng.choice([256, 512, 768, 768, rng.randint(64, 768)])}
    if kind == "mlp":
        c, f = rng.choice([(1280, 1), (640, 2), (640, 1)])
        return {"kind": kind, "m": 2 * f * f * rng.randint(16, 32) * rng.randint(16, 32), "c": c}
    n, k = 32 * _log_int(rng, 1, 160), 128 * _log_int(rng, 1, 40)
    return {"kind": kind, "m": _log_int(rng, 1, min(32768, 100000000000 // (n * k))), "n": n, "k": k,
            "resid": rng.random() < 0.5, "y": rng.choice(["fp32", "bf16"])}


# ----------------------------------------------------------------------------- inputs

def _dev():
    return torch.device("cuda:0")


def _gen(seed, salt=0):
    return torch.Generator(device=_dev()).manual_seed(1000003 * (seed + 1) + salt)


def _normal(g, *shape, std=1.0, mean=0.0):
    return torch.empty(shape, device=_dev(), dtype=torch.float32).normal_(mean, std, generator=g)


def _interleave(w):
    """GEGLU weights or bias [2 n, ...] (values, then gates) in 32-row blocks of each."""
    n = w.shape[0] // 2
    return torch.stack([w[:n].view(n // 32, 32, *w.shape[1:]), w[n:].view(n // 32, 32, *w.shape[1:])],
                       1).reshape(2 * n, *w.shape[1:]).contiguous()


def _inputs(case, seed):
    """The inputs both forms and `exact` start from."""
    g = _gen(seed, 17)
    if case["kind"] == "cache":
        # states and embeddings are near normal, each row with its own spread
        r, c = case["rows"], case["cols"]
        x = _normal(g, r, c).mul_(torch.empty(r, 1, device=_dev()).uniform_(0.5, 2.0, generator=g))
        x = x.to(TYPES[case["src"]])
        slots = torch.randperm(case["slots"], device=_dev(), generator=g)[:r].contiguous()
        idx = slots[torch.randperm(r, device=_dev(), generator=g)].contiguous()
        return {"x": x, "slots": slots, "idx": idx}
    if case["kind"] == "lookup":
        e = _normal(g, case["n"], case["dim"])
        e = (e / e.norm(dim=1, keepdim=True)).half()
        at = torch.randint(0, case["n"], (case["nq"],), device=_dev(), generator=g)
        # similar prompts: cosines around the middle of a level's range
        mid = torch.randint(0, 5, (case["nq"],), device=_dev(), generator=g).float() * 0.05 + 0.75
        cos = mid + torch.empty(case["nq"], device=_dev()).uniform_(-0.015, 0.015, generator=g)
        u = _normal(g, case["nq"], case["dim"])
        c = _decode(*_encode(e[at].float(), case["fmt"]), case["fmt"], case["dim"]).double()
        c = c / c.norm(dim=1, keepdim=True)
        u = u.double() - (u.double() * c).sum(1, keepdim=True) * c
        u = u / u.norm(dim=1, keepdim=True)
        q = cos.double()[:, None] * c + (1 - cos.double() ** 2).sqrt()[:, None] * u
        return {"emb": e, "q": q.half()}
    if case["kind"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"x": _normal(g, m, k).bfloat16(), "w": _normal(g, n, k, std=k ** -0.5), "b": _normal(g, n, std=0.1),
                "r": _normal(g, m, n) if case["resid"] else None}
    m, c = case["m"], case["c"]
    return {"x": _normal(g, m, c, std=2.0), "g": _normal(g, c, std=0.1, mean=1.0), "beta": _normal(g, c, std=0.1),
            "w1": _normal(g, 8 * c, c, std=c ** -0.5), "b1": _normal(g, 8 * c, std=0.1),
            "w2": _normal(g, c, 4 * c, std=(4 * c) ** -0.5), "b2": _normal(g, c, std=0.1)}


def prepare(case, seed):
    s = {"case": case, "in": _inputs(case, seed)}
    i, kind = s["in"], case["kind"]
    if own:
        from paper_2511_06724_amd import dn
        s["dn"] = dn
        s["fmt"] = {MX4: dn.DN_MXFP4, MX8: dn.DN_MXFP8}[case.get("fmt", MX4)]
        if kind == "cache":
            s["table"] = torch.zeros(dn.mx_bytes(s["fmt"], case["slots"], case["cols"]), device=_dev(), dtype=torch.uint8)
            s["ws"] = torch.empty(dn.ac_mx_store_bytes(case["rows"], case["slots"]), device=_dev(), dtype=torch.uint8)
            s["out"] = torch.empty(case["rows"], case["cols"], device=_dev())
        elif kind == "lookup":
            s["table"] = dn.mx_quantize(s["fmt"], i["emb"])
            nq = case["nq"]
            s["ws"] = torch.empty(dn.ac_mx_lookup_bytes(nq, case["n"], case["dim"]), device=_dev(), dtype=torch.uint8)
            s["out"] = (torch.empty(nq, device=_dev(), dtype=torch.int64), torch.empty(nq, device=_dev()),
                        torch.empty(nq, device=_dev(), dtype=torch.int32))
        elif kind == "linear":
            s["xq"] = torch.empty(dn.mx_bytes(s["fmt"], case["m"], case["k"]), device=_dev(), dtype=torch.uint8)
            s["w"] = dn.pack_weight(s["fmt"], i["w"], case["n"], case["k"])
            s["out"] = torch.empty(case["m"], case["n"], device=_dev(), dtype=TYPES[case["y"]])
        else:
            m, c = case["m"], case["c"]
            s["a"] = torch.empty(dn.mx_bytes(s["fmt"], m, c), device=_dev(), dtype=torch.uint8)
            s["h"] = torch.empty(dn.mx_bytes(s["fmt"], m, 4 * c), device=_dev(), dtype=torch.uint8)
            s["w1"], s["b1"] = dn.pack_weight(s["fmt"], _interleave(i["w1"]), 8 * c, c), _interleave(i["b1"])
            s["w2"] = dn.pack_weight(s["fmt"], i["w2"], c, 4 * c)
            s["out"] = torch.empty(m, c, device=_dev(), dtype=torch.bfloat16)
        return s
    if kind == "cache":
        blocks = -(-case["cols"] // BLOCK)
        s["codes"] = torch.zeros(case["slots"], blocks * BLOCK, device=_dev(), dtype=torch.uint8)
        s["scales"] = torch.zeros(case["slots"], blocks, device=_dev(), dtype=torch.uint8)
    elif kind == "lookup":
        s["codes"], s["scales"] = _encode(i["emb"].float(), case["fmt"])
    elif kind == "linear":
        s["w"] = _encode(i["w"], MX4)
    else:
        s["w1"], s["w2"] = _encode(i["w1"], MX4), _encode(i["w2"], MX4)
    return s


# ----------------------------------------------------------------------------- the plain form

def _pow2(e):
    """2^e exactly (a power function may round), for integer e in [-1022, 1023]."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _encode(x, fmt):
    """Rows x [r, c] fp32 -> (codes [r, blocks * 32], scales [r, blocks]), both uint8 (one code a byte)."""
    r, c = x.shape
    blocks = -(-c // BLOCK)
    if c % BLOCK:
        x = torch.cat([x, x.new_zeros(r, blocks * BLOCK - c)], 1)
    codes = torch.empty(r, blocks * BLOCK, device=x.device, dtype=torch.uint8)
    scales = torch.empty(r, blocks, device=x.device, dtype=torch.uint8)
    step = max(1, (1 << 24) // (blocks * BLOCK))
    for a in range(0, r, step):
        v = x[a:a + step].reshape(-1, blocks, BLOCK)
        amax = v.abs().amax(2)
        e = torch.frexp(amax)[1] - 1                       # floor(log2 amax)
        s = torch.where(amax > 0, e - EMAX[fmt] + 127, torch.zeros_like(e)).clamp(0, 254)
        s = torch.where(torch.isfinite(amax), s, torch.full_like(s, 255))
        t = v.double() * _pow2(127 - s)[:, :, None]
        m = t.abs().clamp(max=TOP[fmt])
        if fmt == MX4:
            q = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
            m = torch.round(m / q) * q                     # nearest, ties to the even multiple
            code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4))
        else:
            # the quantum: 2^(e - 3) in [2^e, 2^(e + 1)), that of the least exponent -6 below
            ex = torch.frexp(m.clamp(min=2.0 ** -6))[1] - 1
            m = torch.round(m * _pow2(3 - ex)) * _pow2(ex - 3)
            ex = torch.frexp(m.clamp(min=2.0 ** -6))[1] - 1
            code = (ex + 6) * 8 + m * _pow2(3 - ex)        # below 2^-6 the second term is under 8
        code = torch.where(s[:, :, None] < 255, code, torch.zeros_like(code))
        sign = torch.signbit(t).to(torch.uint8) * (8 if fmt == MX4 else 128)
        codes[a:a + step] = (code.to(torch.uint8) + sign).reshape(-1, blocks * BLOCK)
        scales[a:a + step] = s.to(torch.uint8)
    return codes, scales


_TABLES = {}


def _decode(codes, scales, fmt, cols):
    """The fp32 values of (codes, scales), first `cols` of every row."""
    if fmt not in _TABLES:
        if fmt == MX4:
            pos = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
        else:
            pos = [m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)]
        _TABLES[fmt] = torch.tensor(pos + [-v for v in pos], dtype=torch.float32)
    values = _TABLES[fmt].to(codes.device)[codes.int()]
    scale = _pow2(scales.int() - 127)
    scale = torch.where(scales < 255, scale, torch.full_like(scale, float("nan"))).float()
    r, blocks = scales.shape
    return (values.view(r, blocks, BLOCK) * scale[:, :, None]).reshape(r, blocks * BLOCK)[:, :cols]


def _gelu(x):
    return 0.5 * x * (1 + torch.erf(x * 0.70710678118654752))


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    case, i = s["case"], s["in"]
    if case["kind"] == "cache":
        codes, scales = _encode(i["x"].float(), case["fmt"])
        s["codes"][i["slots"]] = codes
        s["scales"][i["slots"]] = scales
        return _decode(s["codes"][i["idx"]], s["scales"][i["idx"]], case["fmt"], case["cols"])
    if case["kind"] == "lookup":
        c = _decode(s["codes"], s["scales"], case["fmt"], case["dim"])
        q = i["q"].float()
        score = (q @ c.t()) / c.norm(dim=1) / q.norm(dim=1, keepdim=True)
        best, idx = score.max(dim=1)
        first = (score == best[:, None]).to(torch.uint8).argmax(dim=1)     # ties to the lowest row
        j = (best[:, None] >= torch.tensor(THRESHOLDS, device=best.device, dtype=torch.float32)).sum(1)
        return first, best, torch.tensor(LEVELS, device=best.device, dtype=torch.int32)[j]
    if case["kind"] == "linear":
        x = _decode(*_encode(i["x"].float(), MX4), MX4, case["k"])
        y = x @ _decode(*s["w"], MX4, case["k"]).t() + i["b"]
        if i["r"] is not None:
            y = y + i["r"]
        return y.to(TYPES[case["y"]])
    c = case["c"]
    x = i["x"]
    d = x - x.mean(1, keepdim=True)
    a = d * torch.rsqrt((d * d).mean(1, keepdim=True) + 1e-5) * i["g"] + i["beta"]
    a = _decode(*_encode(a, MX4), MX4, c)
    u = a @ _decode(*s["w1"], MX4, c).t() + i["b1"]
    h = u[:, :4 * c] * _gelu(u[:, 4 * c:])
    h = _decode(*_encode(h, MX4), MX4, 4 * c)
    return (h @ _decode(*s["w2"], MX4, 4 * c).t() + i["b2"] + x).bfloat16()


# ----------------------------------------------------------------------------- the library's calls

def _run_own(s):
    case, i, dn = s["case"], s["in"], s["dn"]
    if case["kind"] == "cache":
        dn.ac_mx_store(s["fmt"], i["x"], i["slots"], s["table"], case["slots"], s["ws"])
        dn.ac_mx_fetch(s["fmt"], s["table"], case["slots"], i["idx"], s["out"])
        return s["out"]
    if case["kind"] == "lookup":
        dn.ac_mx_lookup(s["fmt"], i["q"], s["table"], case["n"], s["ws"], *s["out"], THRESHOLDS, LEVELS)
        return s["out"]
    if case["kind"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        dn.mx_quantize(s["fmt"], i["x"], s["xq"])
        dn.op_linear(s["fmt"], s["xq"], s["w"], i["b"], s["out"], m, n, k, resid=i["r"], resid_f32=True,
                     y_f32=case["y"] == "fp32")
        return s["out"]
    m, c = case["m"], case["c"]
    dn.op_layernorm(s["fmt"], i["x"], s["a"], m, c, i["g"], i["beta"], 1e-5)
    dn.op_linear(s["fmt"], s["a"], s["w1"], s["b1"], s["h"], m, 4 * c, c, geglu=True)
    dn.op_linear(s["fmt"], s["h"], s["w2"], i["b2"], s["out"], m, c, 4 * c, resid=i["x"], resid_f32=True)
    return s["out"]


# ----------------------------------------------------------------------------- what a pass cannot do without

def _mx(rows, cols, fmt):
    """Bytes of an MX buffer."""
    blocks = -(-cols // BLOCK)
    return rows * blocks * (BLOCK // 2 + 1 if fmt == MX4 else BLOCK + 1)


def work(case):
    if case["kind"] == "cache":
        e = case["rows"] * case["cols"]
        src = 4 if case["src"] == "fp32" else 2
        return {"bytes": e * (src + 4) + 2 * _mx(case["rows"], case["cols"], case["fmt"]) + 16 * case["rows"], "flops": 0}
    if case["kind"] == "lookup":
        nq, n, d = case["nq"], case["n"], case["dim"]
        return {"bytes": _mx(n, d, case["fmt"]) + 2 * nq * d + 16 * nq, "flops": 2 * nq * n * d}
    if case["kind"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = m * n * ((4 if case["y"] == "fp32" else 2) + (4 if case["resid"] else 0))
        return {"bytes": 2 * m * k + _mx(n, k, MX4) + out + 4 * n, "flops": 2 * m * n * k}
    m, c = case["m"], case["c"]
    return {"bytes": m * c * (4 + 2) + _mx(8 * c, c, MX4) + _mx(c, 4 * c, MX4), "flops": 2 * m * c * 12 * c}


# ----------------------------------------------------------------------------- 64 bits

def _bounds(values):
    """Where a magnitude rounds up to the next of the ascending `values`: the midpoint, which
    itself goes to the neighbour of even index."""
    mids = [(a + b) / 2 for a, b in zip(values, values[1:])]
    return [m if k % 2 else float(np.nextafter(m, np.inf)) for k, m in enumerate(mids)]


def _quantised(x, fmt):
    """The values an MX row stands for, by search among the format's magnitudes (64 bits)."""
    if fmt == MX4:
        values = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        values = [math.ldexp(m, -9) for m in range(8)] + [math.ldexp(8 + m, e) for e in range(-9, 6) for m in range(8)]
        values = values[:127]                                             # the last would be 480
    bounds = torch.tensor(_bounds(values), device=x.device, dtype=torch.float64)
    grid = torch.tensor(values, device=x.device, dtype=torch.float64)
    powers = torch.tensor([2.0 ** k for k in range(-150, 129)], device=x.device, dtype=torch.float64)
    r, c = x.shape
    out = torch.empty(r, c, device=x.device, dtype=torch.float64)
    pad = -c % BLOCK
    step = max(1, (1 << 24) // (c + pad))
    for a in range(0, r, step):
        v = torch.nn.functional.pad(x[a:a + step].double(), (0, pad)).unflatten(1, (-1, BLOCK))
        top = v.abs().amax(2, keepdim=True)
        # the exponent of the largest magnitude, by search among exact powers of two
        log = torch.bucketize(top, powers, right=True) - 1 - 150
        log = (log - math.floor(math.log2(values[-1]))).clamp(min=-127)
        scale = powers[log + 150]
        n = torch.bucketize((v / scale).abs(), bounds, right=True)
        out[a:a + step] = (torch.sign(v) * grid[n] * scale).flatten(1)[:, :c]
    return out


def exact(case, seed):
    i = _inputs(case, seed)
    if case["kind"] == "cache":
        order = torch.empty(case["slots"], device=_dev(), dtype=torch.int64)
        order[i["slots"]] = torch.arange(case["rows"], device=_dev())
        return _quantised(i["x"], case["fmt"])[order[i["idx"]]]
    if case["kind"] == "lookup":
        c = _quantised(i["emb"], case["fmt"])
        q = i["q"].double()
        cos = torch.nn.functional.normalize(q) @ torch.nn.functional.normalize(c).t()
        best, idx = cos.max(1)
        level = torch.full((case["nq"],), LEVELS[0], device=_dev(), dtype=torch.int32)
        for t, k in zip(THRESHOLDS, LEVELS[1:]):
            level[best >= t] = k
        return idx, best, level
    if case["kind"] == "linear":
        y = torch.addmm(i["b"].double(), _quantised(i["x"], MX4), _quantised(i["w"], MX4).t())
        return y if i["r"] is None else y + i["r"]
    x, c = i["x"].double(), case["c"]
    a = torch.nn.functional.layer_norm(x, (c,), i["g"].double(), i["beta"].double(), 1e-5)
    u = torch.addmm(i["b1"].double(), _quantised(a, MX4), _quantised(i["w1"], MX4).t())
    h = u[:, :4 * c] * torch.nn.functional.gelu(u[:, 4 * c:])
    return torch.addmm(i["b2"].double(), _quantised(h, MX4), _quantised(i["w2"], MX4).t()) + x
