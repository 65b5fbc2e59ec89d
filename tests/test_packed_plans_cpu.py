"""How packed attention calls are run (dn::attention_packed_plan, a host function of the library): the batches of the GPU tests
reach every kernel, and a plan's workgroups fit its workspace."""

import pytest

from paper_2511_06724_amd import dn
from tests.packed_plans import DIVIDED, JOIN_ROWS, MIXED, batch_way, plan
from tests.test_gpu_packed import LENGTHS, WAYS

TYPES = (dn.DN_FP32, dn.DN_BF16)
DIMS = (32, 64, 96, 128)


def ways_of(dtype, dim):
    tiles = {"tiles 4"} if dtype == dn.DN_FP32 else {"tiles 2", "tiles 6" if dim == 96 else "tiles 4"} | ({"tiles 8"} if dim == 128 else set())
    return tiles | {"whole", "rows", "units"}


def test_gpu_batches_reach_every_kernel():
    have = {(w[0], w[1], batch_way(*w)) for w in WAYS}
    have |= {(t, d, batch_way(t, d, *b[:4])) for t in TYPES for d in DIMS for b in DIVIDED}
    have |= {(t, b[4], batch_way(t, b[4], *b[:4])) for t in TYPES for b in MIXED}
    have |= {(t, d, batch_way(t, d, *b, hq, hk)) for t in TYPES for hq, hk, d in ((2, 2, 64), (8, 2, 128), (3, 3, 32), (8, 1, 96)) for b in LENGTHS}
    assert have == {(t, d, w) for t in TYPES for d in DIMS for w in ways_of(t, d)}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_divided_batches(dtype, dim):
    for b in DIVIDED:
        assert batch_way(dtype, dim, *b[:4]) in b[4]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_plans_fit_their_workspace_and_launches(dtype, dim):
    """The workspace is for the most shares, whatever the rows of the keys; the launched ones are no more."""
    elem = 2 if dtype == dn.DN_BF16 else 4
    for heads, kv_heads in ((1, 1), (8, 1), (32, 8), (20, 20), (65535, 65535), (65535, 1)):
        for n in (1, 7, 64, 5000):
            for rows in (1, 64, 1000, 100000):
                if rows * (heads // kv_heads) > 2 ** 31 - 65537:
                    continue
                for max_kv in (1, 256, 257, 1024, 1025, 65536, 2 ** 31 - 1):
                    most = plan(dtype, dim, rows, heads, kv_heads, n, max_kv, 0).most
                    for kv_rows in (1, 1000, 10 ** 6, 2 ** 32):
                        p = plan(dtype, dim, rows, heads, kv_heads, n, max_kv, kv_rows)
                        assert p.most == most and p.waves in (0, 2, 4, 6, 8) and (most == 0 or p.waves == 0)
                        assert (1 <= p.shares <= most <= (2048 if dim * elem <= 64 else 1024) if most else p.shares == p.join == 0)
                        assert 1 <= p.split <= 8 and (p.split == 1 or p.join == JOIN_ROWS)
