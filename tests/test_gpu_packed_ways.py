"""Attention of packed sequences in the ways of running it that depend on the head width, the division of the keys and the mix of
a call's sequences, against the fp64 oracle (tolerances as in test_gpu_packed)."""

import numpy as np
import pytest
import torch

from paper_2511_06724_amd import dn
from tests.gpu_util import announce, host
from tests.packed_plans import DIVIDED, MIXED, batch_way
from tests.test_gpu_packed import TYPES, Batch, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("batch", range(len(DIVIDED)))
def test_divided_keys(batch, dim, dtype, causal):
    q_len, kv_len, hq, hk, ways = DIVIDED[batch]
    announce(f"divided {dtype} {dim} {q_len[:4]} {kv_len[:4]} {causal} {batch_way(dtype, dim, q_len, kv_len, hq, hk)}")
    b = Batch(q_len, kv_len, hq, hk, dim, dtype, seed=batch)
    first = b.run(causal).clone()
    b.check(causal, rows=np.array([0, 1, 2, 31, 32, 63, 64, 100, 129]))
    assert torch.equal(b.run(causal), first)
    # what is not finite in the last key of the last sequence is seen by no other sequence and no earlier row
    at = b.start[-1] + kv_len[-1] - 1
    b.v[at] = float("nan")
    b.k[at] = float("inf")
    b.run(causal)
    last = b.total - 1
    assert torch.isnan(b.o[last]).all()
    b.v[at] = b.k[at] = 0.0
    for s, (rows, ref, tol) in enumerate(b.expect(causal, rows=np.array([0, 1, 31, 100]))):
        keep = np.ones(len(rows), bool) if s < len(q_len) - 1 else (rows < last) & causal
        close(host(b.o)[rows[keep]], ref[keep], tol[keep])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch", range(len(MIXED)))
def test_prompts_and_tokens_in_one_call(batch, dtype, causal):
    q_len, kv_len, hq, hk, dim = MIXED[batch]
    announce(f"mixed {dtype} {dim} {q_len[:5]} {kv_len[:5]} {causal} {batch_way(dtype, dim, q_len, kv_len, hq, hk)}")
    b = Batch(q_len, kv_len, hq, hk, dim, dtype, seed=batch)
    first = b.run(causal).clone()
    b.check(causal, rows=np.array([0, 1, 4, 31, 39, 89, 127, 128, 255, 299, 698, 699]))
    assert torch.equal(b.run(causal), first)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bound", [1, 100, 100000])
@pytest.mark.parametrize("q_len,kv_len,hq,hk,dim", [([1, 5], [3000, 777], 8, 2, 96), ([300, 1], [900, 1500], 2, 2, 64), ([40, 90], [400, 90], 2, 1, 32),
                                                    ([600] * 4, [600, 700, 800, 1200], 8, 8, 128)])
def test_a_bound_that_is_too_small_or_too_large(q_len, kv_len, hq, hk, dim, bound, dtype):
    b = Batch(q_len, kv_len, hq, hk, dim, dtype, max_kv=bound)
    b.run(True)
    b.check(True, rows=np.array([0, 1, 4, 39, 40, 89, 128, 299, 599]))
