"""dn::attention_packed_plan of the built library (how a packed attention call is run), and batches for ways of running it."""

import ctypes as C

from paper_2511_06724_amd import dn

JOIN_NONE, JOIN_ROWS, JOIN_UNITS = range(3)


class Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("waves", "most", "shares", "join", "split")]


_plan = getattr(dn.lib, "_ZN2dn21attention_packed_planEiixiiiix")
_plan.argtypes = [C.c_int, C.c_int, C.c_longlong] + [C.c_int] * 4 + [C.c_longlong]
_plan.restype = Plan


def plan(dtype, dim, rows, heads, kv_heads, n, max_kv, kv_rows):
    return _plan(2 if dtype == dn.DN_BF16 else 4, dim, rows, heads, kv_heads, n, max_kv, kv_rows)


def way(p):
    """What tells one kernel of a call from another: "tiles" of so many waves, "whole" units, or how divided ones are joined."""
    return f"tiles {p.waves}" if p.waves else ("whole", "rows", "units")[p.join]


# (new tokens, keys, heads, key heads, how it is run) of batches whose keys are divided, at every head width and type: parts
# joined by units' workgroups and by rows' waves, of few long sequences, many short ones, one of several units a key head.
DIVIDED = [([1, 1, 2], [5000, 20, 1300], 8, 2, ("units",)),
           ([2, 1, 0, 3] * 11, [900, 333, 70, 1200] * 11, 8, 2, ("rows",)),
           ([130], [3000], 8, 1, ("rows", "units"))]
# Prompts, chunks and single tokens behind long contexts in one call.
MIXED = [([1, 700, 1, 1, 2], [6000, 700, 5000, 20, 3000], 8, 2, 128), ([1, 1, 300, 40], [4000, 1, 2500, 40], 4, 4, 64),
         ([5] * 16, [64 * (i * i + 1) for i in range(16)], 16, 2, 96), ([1, 90, 1], [2000, 90, 900], 3, 1, 32)]


def batch_way(dtype, dim, q_len, kv_len, heads, kv_heads, behind=2):
    """How a batch of the GPU tests is run: its key rows lie up to three apart."""
    n, rows = len(q_len), sum(kv_len) + 2
    ways = {way(plan(dtype, dim, sum(q_len) + behind, heads, kv_heads, n, max(max(kv_len), 1), r)) for r in (rows, rows + 3 * n)}
    assert len(ways) == 1
    return ways.pop()
