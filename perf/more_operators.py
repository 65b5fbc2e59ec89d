"""Performance cases of the rotated, grouped-head attention layer over packed sequences.

Three operators that follow one another between a transformer's input projection and its output
projection, where positions enter by rotation and requests of different lengths are packed:

- `rope`: rotary positions with one to four axes (time, height, width of an image or video token)
  on every head of a row (dn_op_rope);
- `qkn`: the RMS norm of every query and key head and the rotation in one pass, the new keys and
  values going to their rows of a cache where there is one (dn_op_qk_norm_rope);
- `attn`: attention of packed sequences over their keys and values, causal or not, several query
  heads per key head, from whole prompts to one token per sequence over a long cache
  (dn_op_attention_packed).

Each case is a dict of plain values. `prepare` makes what a program holds before the call, `run`
is one pass: with `own` the library's calls, without it the same in elementary torch operations.
`exact` is the definition in 64-bit floating point, written apart from both.
"""

import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # One new token of each of four requests, 32 heads, three position axes: latency.
        {"name": "rope_token", "kind": "rope", "type": "bf16", "rows": 4, "heads": 32, "dim": 128, "axes": "32,48,48",
         "pairing": "halves", "per_axis": False, "theta": 1e6, "grid": "1x2x2"},
        # The image tokens of a 64 x 64 level (640 wide), both guidance rows: rows and columns.
        {"name": "rope_image", "kind": "rope", "type": "bf16", "rows": 2 * 64 * 64, "heads": 10, "dim": 64, "axes": "32,32",
         "pairing": "pairs", "per_axis": True, "theta": 1e4, "grid": "1x64x64"},
        # A video of 21 latent frames of 30 x 52 tokens in fp32.
        {"name": "rope_video", "kind": "rope", "type": "fp32", "rows": 21 * 30 * 52, "heads": 20, "dim": 128,
         "axes": "44,42,42", "pairing": "pairs", "per_axis": True, "theta": 1e4, "grid": "21x30x52"},
        # One decoding step of 48 requests far into their contexts, grouped heads, into the cache.
        {"name": "qkn_decode", "kind": "qkn", "type": "bf16", "n": 48, "q_lo": 1, "q_hi": 1, "kv_hi": 1024, "lens": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "axes": "128", "pairing": "halves", "per_axis": True, "theta": 1e6,
         "far": 1000000, "cache": True},
        # Packed prompts of 1 to 231 tokens in fp32, an 80-wide head of which 64 dims are rotated.
        {"name": "qkn_prompts", "kind": "qkn", "type": "fp32", "n": 64, "q_lo": 1, "q_hi": 231, "kv_hi": 0, "lens": 2,
         "heads": 20, "kv_heads": 4, "dim": 80, "axes": "16,24,24", "pairing": "pairs", "per_axis": True, "theta": 1e4,
         "far": 0, "cache": True},
        # The same video's tokens in bf16, as many key heads as query heads, no cache.
        {"name": "qkn_video", "kind": "qkn", "type": "bf16", "n": 1, "q_lo": 21 * 30 * 52, "q_hi": 21 * 30 * 52, "kv_hi": 0,
         "lens": 3, "heads": 20, "kv_heads": 20, "dim": 128, "axes": "16,56,56", "pairing": "pairs", "per_axis": True,
         "theta": 1e4, "far": 0, "cache": False},
        # One token over the 77 of a prompt: the smallest call.
        {"name": "attn_token", "kind": "attn", "type": "bf16", "n": 1, "q_lo": 1, "q_hi": 1, "kv_lo": 77, "kv_hi": 77,
         "lens": 4, "heads": 20, "kv_heads": 20, "dim": 64, "causal": True},
        # One decoding step of 32 requests whose contexts have one token to 65,536.
        {"name": "attn_decode", "kind": "attn", "type": "bf16", "n": 32, "q_lo": 1, "q_hi": 1, "kv_lo": 1, "kv_hi": 65536,
         "lens": 5, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True},
        # 64 packed prompts of 1 to 300 tokens through a causal text encoder, 20 heads of 64.
        {"name": "attn_prompts", "kind": "attn", "type": "bf16", "n": 64, "q_lo": 1, "q_hi": 300, "kv_lo": 0, "kv_hi": 0,
         "lens": 6, "heads": 20, "kv_heads": 20, "dim": 64, "causal": True},
        # Four long prompts, grouped heads: the largest call.
        {"name": "attn_prefill", "kind": "attn", "type": "bf16", "n": 4, "q_lo": 7000, "q_hi": 16000, "kv_lo": 0, "kv_hi": 0,
         "lens": 7, "heads": 32, "kv_heads": 8, "dim": 128, "causal": True},
        # Joint attention of two images' 64 x 64 tokens and their 77 prompt tokens, every token to all.
        {"name": "attn_image", "kind": "attn", "type": "bf16", "n": 2, "q_lo": 4173, "q_hi": 4173, "kv_lo": 0, "kv_hi": 0,
         "lens": 8, "heads": 20, "kv_heads": 20, "dim": 128, "causal": False},
        # Chunks of 1 to 200 new tokens behind up to 1,500 cached ones in fp32, five query heads a key head.
        {"name": "attn_chunks_fp32", "kind": "attn", "type": "fp32", "n": 7, "q_lo": 1, "q_hi": 200, "kv_lo": 200,
         "kv_hi": 1500, "lens": 9, "heads": 10, "kv_heads": 2, "dim": 64, "causal": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotation(rng, dim):
    pairing = rng.choice(["pairs", "halves"])
    step = 16 if pairing == "halves" else 2            # dims rotated in all
    rot = dim if rng.random() < 0.6 else step * rng.randint(1, dim // step)
    n = rng.randint(1, min(4, rot // 2))
    cuts = sorted(rng.sample(range(1, rot // 2), n - 1)) if n > 1 else []
    axes = [2 * (b - a) for a, b in zip([0] + cuts, cuts + [rot // 2])]
    return {"axes": ",".join(map(str, axes)), "pairing": pairing, "per_axis": rng.random() < 0.5,
            "theta": rng.choice([1e4, 5e5, 1e6])}


def draw(rng):
    kind = rng.choice(["rope", "qkn", "attn", "attn"])
    case = {"kind": kind, "type": rng.choice(["bf16", "bf16", "fp32"])}
    if kind == "rope":
        case["dim"] = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        case["heads"] = _log_int(rng, 1, 40)
        t, h, w = (_log_int(rng, 1, hi) for hi in (21, 64, 64))
        most = 80000000 // (case["dim"] * case["heads"])
        case["rows"] = min(t * h * w + rng.randint(0, 3), most)
        case["grid"] = f"{t}x{h}x{w}"
        case.update(_draw_rotation(rng, case["dim"]))
        return case
    case["lens"] = rng.randrange(1 << 30)
    group = rng.choice([1, 1, 2, 4, 5, 8])
    case["kv_heads"] = _log_int(rng, 1, 20 if group < 4 else 8)
    case["heads"] = group * case["kv_heads"]
    if kind == "qkn":
        case["dim"] = rng.choice([64, 64, 80, 96, 128, 128, 256])
        case["n"] = _log_int(rng, 1, 64)
        width = (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        case["q_lo"], case["q_hi"] = 1, rng.choice([1, _log_int(rng, 2, max(2, min(4096, 120000000 // (width * case["n"]))))])
        case["cache"] = rng.random() < 0.7
        case["kv_hi"] = rng.choice([0, 512]) if case["cache"] else 0
        case["far"] = rng.choice([0, 30000, 1000000])
        case.update(_draw_rotation(rng, case["dim"]))
        return case
    case["dim"] = rng.choice([32, 64, 64, 96, 128, 128])
    case["causal"] = rng.random() < 0.7
    per_key = 2 * case["kv_heads"] * case["dim"] * BYTES[case["type"]]
    if rng.random() < 0.5:     # a few new tokens behind a cache
        case["n"] = _log_int(rng, 1, 64)
        case["q_lo"], case["q_hi"] = 1, rng.choice([1, 1, rng.randint(2, 8)])
        case["kv_lo"] = case["q_hi"]
        case["kv_hi"] = _log_int(rng, 16, max(16, min(65536, 1000000000 // (case["n"] * per_key))))
    else:                      # whole prompts, or chunks of them behind a cache
        case["n"] = _log_int(rng, 1, 64)
        flops = 1e12 if case["type"] == "bf16" else 1e11
        longest = math.sqrt(flops / (4 * case["heads"] * case["dim"] * case["n"]))
        case["q_lo"], case["q_hi"] = 1, _log_int(rng, 16, max(16, min(12000, int(longest))))
        case["kv_lo"], case["kv_hi"] = rng.choice([(0, 0), (0, 0), (case["q_hi"], 2 * case["q_hi"])])
    return case


# ----------------------------------------------------------------------------- lengths

def _spread(rng, lo, hi):
    """A length in [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, _log_int(rng, lo, hi))) if hi > lo else lo


def _lengths(case):
    """(new tokens, keys) of every sequence; the keys include the new tokens."""
    rng = random.Random(case["lens"])
    q = [_spread(rng, case["q_lo"], case["q_hi"]) for _ in range(case["n"])]
    if not case["kv_hi"]:
        return q, list(q)
    lo = case.get("kv_lo", case["q_hi"])
    return q, [max(a, _spread(rng, lo, max(lo, case["kv_hi"]))) for a in q]


def _starts(case, kv):
    """First cache row of every sequence and the rows of the cache: whole prompts are packed, a
    sequence that grows has room behind it."""
    at, starts = 0, []
    for n in kv:
        starts.append(at)
        at += n if not case["kv_hi"] else -(-(n + 1) // 16) * 16
    return starts, at


# ----------------------------------------------------------------------------- inputs

def _dev():
    return torch.device("cuda:0")


def _gen(seed, salt=0):
    return torch.Generator(device=_dev()).manual_seed(1000003 * (seed + 1) + salt)


def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.empty(shape, device=_dev(), dtype=torch.float32).normal_(mean, std, generator=g).to(dtype)


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def _inputs(case, seed):
    """The inputs both forms and `exact` start from."""
    g, dtype, dim = _gen(seed, 29), TYPES[case["type"]], case["dim"]
    rng = random.Random(seed)
    if case["kind"] == "rope":
        x = _normal(g, case["rows"], case["heads"], dim, dtype=dtype)
        t, h, w = (int(a) for a in case["grid"].split("x"))
        at = torch.arange(case["rows"], device=_dev())
        grid = [at // (h * w) % t, at // w % h, at % w, at]
        n = len(_axes(case))
        axes = {1: [3], 2: [1, 2], 3: [0, 1, 2], 4: [0, 1, 2, 3]}[n]
        pos = torch.stack([grid[a] + rng.randint(0, 500) for a in axes], 1).to(torch.int32).contiguous()
        return {"x": x, "pos": pos}
    q_len, kv_len = _lengths(case)
    starts, rows = _starts(case, kv_len)
    total, heads, kv_heads = sum(q_len), case["heads"], case["kv_heads"]
    q_start = [0]
    for n in q_len:
        q_start.append(q_start[-1] + n)
    out = {"q_len": q_len, "kv_len": kv_len, "starts": starts, "q_start": q_start, "rows": rows}
    if case["kind"] == "attn":
        # queries after a norm with a gain: logits of about two standard deviations
        out["q"] = _normal(g, total, heads, dim, std=2.0, dtype=dtype)
        out["k"] = _normal(g, rows, kv_heads, dim, dtype=dtype)
        out["v"] = _normal(g, rows, kv_heads, dim, dtype=dtype)
        return out
    # the output of one projection for queries, keys and values
    qkv = _normal(g, total, heads + 2 * kv_heads, dim, std=2.0, dtype=dtype)
    out["q"], out["k"], out["v"] = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    out["gq"], out["gk"] = _normal(g, dim, std=0.2, mean=1.0), _normal(g, dim, std=0.2, mean=1.0)
    first = [m - n + rng.randint(0, case["far"]) for n, m in zip(q_len, kv_len)]
    pos = torch.cat([torch.arange(a, a + n) for a, n in zip(first, q_len)])
    n_axes = len(_axes(case))
    pos = torch.stack([pos, pos // 52 % 30, pos % 52, pos // 7][:n_axes], 1)
    out["pos"] = pos.to(torch.int32).to(_dev())
    if case["cache"]:
        out["kc"] = _normal(g, rows, kv_heads, dim, dtype=dtype)
        out["vc"] = _normal(g, rows, kv_heads, dim, dtype=dtype)
        out["at"] = torch.cat([torch.arange(s + m - n, s + m) for s, n, m in zip(starts, q_len, kv_len)]).to(_dev())
    return out


def prepare(case, seed):
    s = {"case": case, "in": _inputs(case, seed)}
    i = s["in"]
    if own:
        from paper_2511_06724_amd import dn
        s["dn"] = dn
        if case["kind"] != "attn":
            s["rope"] = dn.rope_table(_axes(case), case["theta"], per_axis=case["per_axis"], device=_dev())
            s["pairing"] = {"pairs": dn.DN_ROPE_PAIRS, "halves": dn.DN_ROPE_HALVES}[case["pairing"]]
        if case["kind"] == "rope":
            s["out"] = torch.empty_like(i["x"])
            return s
        s["seqs"] = dn.Sequences(torch.tensor(i["q_start"], device=_dev(), dtype=torch.int32),
                                 torch.tensor(i["starts"], device=_dev(), dtype=torch.int64),
                                 torch.tensor(i["kv_len"], device=_dev(), dtype=torch.int32), max(i["kv_len"]))
        s["out"] = torch.empty_like(i["q"], memory_format=torch.contiguous_format)
        if case["kind"] == "attn":
            s["ws"] = torch.empty(dn.attention_packed_bytes(i["q"], i["k"], s["seqs"]), device=_dev(), dtype=torch.uint8)
        elif not case["cache"]:
            s["k_out"] = torch.empty_like(i["k"], memory_format=torch.contiguous_format)
        return s
    if case["kind"] != "attn":
        s["freq"] = _frequencies(case)
    return s


# ----------------------------------------------------------------------------- the plain form

def _frequencies(case):
    """(radians per position, axis) of every rotated pair, in 64 bits."""
    axes = _axes(case)
    total, freq, axis = sum(axes), [], []
    for a, d in enumerate(axes):
        for j in range(d // 2):
            i, n = (j, d) if case["per_axis"] else (len(freq), total)
            freq.append(case["theta"] ** (-2.0 * i / n))
            axis.append(a)
    return (torch.tensor(freq, device=_dev(), dtype=torch.float64), torch.tensor(axis, device=_dev()))


def _rotate(case, x, pos, freq):
    """Rotated heads x [rows, heads, dim] in 32 bits; the angles are taken in 64."""
    f, axis = freq
    angle = pos.double()[:, axis] * f
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = f.numel()
    y = x.clone()
    if case["pairing"] == "pairs":
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, a * sin + b * cos
    return y


def _norm(x, gain):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain


def _attend(case, i):
    """Attention sequence by sequence, a block of queries at a time: scores, softmax, values."""
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group, scale = heads // kv_heads, dim ** -0.5
    out = torch.empty_like(i["q"])
    for s, (n, m) in enumerate(zip(i["q_len"], i["kv_len"])):
        a, b = i["q_start"][s], i["starts"][s]
        k = i["k"][b:b + m].float().permute(1, 2, 0).contiguous()              # [kv_heads, dim, m]
        v = i["v"][b:b + m].float().permute(1, 0, 2).contiguous()              # [kv_heads, m, dim]
        step = max(1, min(n, 1000000000 // (heads * m)))
        for c in range(0, n, step):
            e = min(n, c + step)
            q = i["q"][a + c:a + e].float().view(e - c, kv_heads, group, dim).permute(1, 2, 0, 3)
            p = torch.matmul(q.reshape(kv_heads, group * (e - c), dim), k) * scale
            p = p.view(kv_heads, group, e - c, m)
            if case["causal"]:
                last = torch.arange(c, e, device=p.device) + (m - n)
                p = p.masked_fill(torch.arange(m, device=p.device)[None] > last[:, None], float("-inf"))
            p = torch.exp(p - p.amax(-1, keepdim=True))
            l = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(kv_heads, group * (e - c), m), v).view(kv_heads, group, e - c, dim) / l
            out[a + c:a + e] = o.permute(2, 0, 1, 3).reshape(e - c, heads, dim).to(out.dtype)
    return out


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    case, i = s["case"], s["in"]
    if case["kind"] == "rope":
        return _rotate(case, i["x"].float(), i["pos"], s["freq"]).to(i["x"].dtype)
    if case["kind"] == "attn":
        return _attend(case, i)
    dtype = i["q"].dtype
    q = _rotate(case, _norm(i["q"].float(), i["gq"]), i["pos"], s["freq"]).to(dtype)
    k = _rotate(case, _norm(i["k"].float(), i["gk"]), i["pos"], s["freq"]).to(dtype)
    if not case["cache"]:
        return q, k
    i["kc"][i["at"]] = k
    i["vc"][i["at"]] = i["v"]
    return q, i["kc"], i["vc"]


# ----------------------------------------------------------------------------- the library's calls

def _run_own(s):
    case, i, dn = s["case"], s["in"], s["dn"]
    if case["kind"] == "rope":
        dn.op_rope(i["x"], i["pos"], s["rope"], s["out"], pairing=s["pairing"])
        return s["out"]
    if case["kind"] == "attn":
        dn.op_attention_packed(i["q"], i["k"], i["v"], s["out"], s["seqs"], causal=case["causal"],
                               scale=case["dim"] ** -0.5, ws=s["ws"])
        return s["out"]
    if not case["cache"]:
        dn.op_qk_norm_rope(i["q"], i["k"], i["gq"], i["gk"], EPS, i["pos"], s["rope"], s["out"], s["k_out"],
                           pairing=s["pairing"])
        return s["out"], s["k_out"]
    dn.op_qk_norm_rope(i["q"], i["k"], i["gq"], i["gk"], EPS, i["pos"], s["rope"], s["out"], i["kc"], v=i["v"],
                       v_out=i["vc"], seqs=s["seqs"], pairing=s["pairing"])
    return s["out"], i["kc"], i["vc"]


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e, dim = BYTES[case["type"]], case["dim"]
    if case["kind"] == "rope":
        n = case["rows"] * case["heads"] * dim
        return {"bytes": 2 * e * n + 4 * len(_axes(case)) * case["rows"], "flops": 3 * n}
    q, kv = _lengths(case)
    total, heads, kv_heads = sum(q), case["heads"], case["kv_heads"]
    if case["kind"] == "qkn":
        n = total * (heads + kv_heads) * dim
        moved = n + (total * kv_heads * dim if case["cache"] else 0)
        return {"bytes": 2 * e * moved + 4 * len(_axes(case)) * total + 8 * dim, "flops": 7 * n}
    # a query attends the keys up to its own position, or all
    pairs = sum(n * m - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(q, kv))
    return {"bytes": e * dim * 2 * (total * heads + sum(kv) * kv_heads), "flops": 4 * pairs * heads * dim}


# ----------------------------------------------------------------------------- 64 bits

def _turned(case, x, pos):
    """The rotation as a product of complex numbers."""
    axes, parts, first = _axes(case), [], 0
    half = sum(axes) // 2
    for a, d in enumerate(axes):
        j = torch.arange(d // 2, device=x.device, dtype=torch.float64)
        power = j / (d // 2) if case["per_axis"] else (j + first) / half
        parts.append(pos[:, a:a + 1].double() * torch.exp(-power * math.log(case["theta"])))
        first += d // 2
    angle = torch.cat(parts, 1)[:, None]
    turn = torch.polar(torch.ones_like(angle), angle)
    head, tail = x[..., :2 * half], x[..., 2 * half:]
    if case["pairing"] == "pairs":
        z = torch.view_as_complex(head.contiguous().unflatten(-1, (half, 2))) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), tail], -1)
    z = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * turn
    return torch.cat([z.real, z.imag, tail], -1)


def exact(case, seed):
    i = _inputs(case, seed)
    if case["kind"] == "rope":
        return _turned(case, i["x"].double(), i["pos"])
    if case["kind"] == "qkn":
        heads = []
        for x, gain in ((i["q"].double(), i["gq"].double()), (i["k"].double(), i["gk"].double())):
            size = (x.square().sum(-1, keepdim=True) / case["dim"] + EPS).sqrt()
            heads.append(_turned(case, x / size * gain, i["pos"]))
        if not case["cache"]:
            return tuple(heads)
        kc, vc = i["kc"].double(), i["vc"].double()
        return heads[0], kc.index_copy(0, i["at"], heads[1]), vc.index_copy(0, i["at"], i["v"].double())
    q, k, v = i["q"], i["k"], i["v"]
    group = case["heads"] // case["kv_heads"]
    out = torch.empty(q.shape, device=q.device, dtype=torch.float64)
    for s in range(case["n"]):
        n, m, a, b = i["q_len"][s], i["kv_len"][s], i["q_start"][s], i["starts"][s]
        rows = max(1, 200000000 // m)
        for h in range(case["heads"]):
            kh, vh = k[b:b + m, h // group].double(), v[b:b + m, h // group].double()
            for c in range(0, n, rows):
                e = min(n, c + rows)
                logits = q[a + c:a + e, h].double() @ kh.t() / math.sqrt(case["dim"])
                if case["causal"]:
                    logits += torch.full((e - c, m), float("-inf"), device=q.device, dtype=torch.float64).triu(m - n + c + 1)
                out[a + c:a + e, h] = torch.softmax(logits, -1) @ vh
    return out
