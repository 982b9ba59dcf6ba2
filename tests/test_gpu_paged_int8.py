"""Attention over an INT8 cache where the scales, or the size of the queries, make the products hard to hold."""
import numpy as np
import pytest

import paged_reference as ref
from test_gpu_paged_bounds import _serve, _workspace

pytestmark = pytest.mark.gpu

# requests of up to 16 rows per key/value head (4 query heads each here) and of more: one tile of 128 rows, and two
LENGTHS = [([1, 1, 1], [2, 7, 40]), ([3, 4], [33, 5]), ([20], [33]), ([150], [150])]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,total", LENGTHS)
def test_keys_of_equal_score_weigh_the_same_under_large_queries(new, total, dim):
    """All queries are 20 + 1/64 in every feature and every key of a head is a permutation of the same codes, so that all
    scores of a head are equal.  Products and their sums are whole multiples of 1/64 below 2^24 / 64, exact in FP32 in any
    order: the weights are equal to the last bit, and y is the mean of the values seen.  Bound: 2^-11 of y for its FP16
    rounding, 2^-11 for the weights' (the same for all of them), and n + 8 roundings of 2^-24 on sums below n max|v|,
    divided by the n weights."""
    d = ref.attention_inputs(8, 2, dim, 16, "int8", new, total, seed=dim + sum(total))
    rng = np.random.default_rng(5)
    base = rng.integers(-128, 128, (2, dim)).astype(np.int8)
    assert (1281 * np.abs(base.astype(np.int64)).sum(1) < 2**24).all()
    d["q"][:] = np.float16(20 + 1 / 64)
    d["k"][:] = rng.permuted(np.broadcast_to(base[None, :, None], d["k"].shape), axis=3)
    d["ks"][:], d["vs"][:] = np.float32(0.125), np.float32(2.0 ** -6)
    got = _serve(d, workspace=_workspace(d))
    for b, length in enumerate(total):
        j = np.arange(length)
        v = d["v"][d["table"][b, j // 16], :, j % 16].astype(np.float64) * 2.0 ** -6       # [keys, kv_heads, dim]
        for i in range(new[b]):
            n = length - new[b] + i + 1
            want = v[:n].mean(0).repeat(4, 0)
            bound = 2.0 ** -10 * np.abs(want) + (n + 8) * 2.0 ** -24 * np.abs(v[:n]).max() + 2.0 ** -25
            off = np.abs(got[d["q_start"][b] + i] - want)
            assert (off <= bound).all(), f"request {b}, row {i}: {off.max()}"
