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


FEW = [([2], [20], 0), ([4, 1], [30, 7], 0), ([3], [200], 0), ([3], [60], 16), ([4], [300], 1)]


def _far_larger_scale_on_an_unseen_key(new, total, window, seed):
    """Value scales in [2^-15, 2^-14), but 2^22 times that at the newest key of every request and, with a window, at the
    oldest that its first row sees: the first rows see the one, the last rows the other, the rows between neither."""
    d = ref.attention_inputs(8, 2, 128, 16, "int8", new, total, window=window, seed=seed)
    d["vs"][:] = np.random.default_rng(seed).uniform(0.5, 1.0, d["vs"].shape) * 2.0 ** -14
    for b, (n, length) in enumerate(zip(new, total)):
        for at in {length - 1, max(0, length - n + 1 - window) if window else length - 1}:
            d["vs"][d["table"][b, at // 16], :, at % 16] *= np.float32(2.0 ** 22)
    return d


@pytest.mark.parametrize("new,total,window", FEW)
def test_a_value_that_a_row_does_not_see_leaves_its_weights_alone(new, total, window):
    d = _far_larger_scale_on_an_unseen_key(new, total, window, seed=sum(total))
    y, bound = ref.attention(d)
    off = np.abs(_serve(d, workspace=_workspace(d)) - y)
    assert (off <= bound).all(), f"rows {np.unique(np.argwhere(off > bound)[:, 0])}"


def _far_larger_scale_on_a_key_of_little_weight(new, total, heavy):
    """One key with nearly all of the weight and a small value scale; all other keys weigh 2^-28 of it and have value scales
    2^22 times as large, so that their products with the values are small beside its own.  (inputs, y, bound): the weights
    are rounded to FP16, 2^-11 of each, or half of FP16's smallest step, 2^-25 of the largest product of weight and scale,
    which is at least half of the unit that they are taken in, for codes up to 128; 2^-11 for the result; 2^-10 for the rest
    (scores of up to 20 in FP32)."""
    d = ref.attention_inputs(8, 2, 128, 16, "int8", new, total, seed=sum(total))
    d["q"][:] = 1
    d["k"][:] = 0
    d["ks"][:] = np.float32(28 * np.log(2) / (128 ** 0.5 * 100))
    d["vs"][:] = np.float32(2.0 ** 8)
    y, bound = np.zeros(d["q"].shape), np.zeros(d["q"].shape)
    for b, length in enumerate(total):
        page = d["table"][b, heavy // 16]
        d["k"][page, :, heavy % 16], d["vs"][page, :, heavy % 16] = 100, np.float32(1.37 * 2.0 ** -14)
        j = np.arange(length)
        ids = d["table"][b, j // 16]
        v, scale = d["v"][ids, :, j % 16].astype(np.float64), d["vs"][ids, :, j % 16].astype(np.float64)
        for i in range(new[b]):
            n = length - new[b] + i + 1
            w = np.where(j[:n] == heavy, 1.0, 2.0 ** -28) / (1 + (n - 1) * 2.0 ** -28)
            p = w[:, None] * scale[:n]                                                        # [keys, kv_heads]
            row = d["q_start"][b] + i
            y[row] = np.einsum("jh,jhd->hd", p, v[:n]).repeat(4, 0)
            bound[row] = (2.0 ** -9 * np.einsum("jh,jhd->hd", p, np.abs(v[:n])) + (n * 2.0 ** -24 * 128 * p.max(0))[:, None]).repeat(4, 0) + 2.0 ** -25
    return d, y, bound


@pytest.mark.parametrize("new,total,heavy", [([1, 1], [30, 90], 3), ([3], [50], 40), ([2], [500], 17)])
def test_weights_keep_their_bits_beside_a_far_larger_value_scale(new, total, heavy):
    d, y, bound = _far_larger_scale_on_a_key_of_little_weight(new, total, heavy)
    assert (np.abs(_serve(d, workspace=_workspace(d)) - y) <= bound).all()


# The same for requests of more rows: one tile of 128, two, several.  Up to 128 keys are seen, which half a step of FP16,
# 2^-25 under a largest weight of 2^7 at least, adds up to 2^-25 of the largest product over.
MANY = [([5], [20], 0), ([20, 3], [100, 7], 0), ([40, 2], [100, 20], 0), ([100], [128], 0), ([5], [200], 16), ([300], [400], 50), ([70], [60], 1)]


@pytest.mark.parametrize("new,total,window", MANY)
def test_a_value_that_a_row_does_not_see_leaves_its_weights_alone_in_long_chunks(new, total, window):
    d = _far_larger_scale_on_an_unseen_key(new, total, window, seed=sum(total))
    y, bound = ref.attention(d)
    off = np.abs(_serve(d, workspace=_workspace(d)) - y)
    assert (off <= bound).all(), f"rows {np.unique(np.argwhere(off > bound)[:, 0])}"


@pytest.mark.parametrize("new,total,heavy", [([5], [50], 3), ([20], [120], 40), ([40], [300], 17), ([200], [700], 450)])
def test_weights_keep_their_bits_beside_a_far_larger_value_scale_in_long_chunks(new, total, heavy):
    d, y, bound = _far_larger_scale_on_a_key_of_little_weight(new, total, heavy)
    assert (np.abs(_serve(d, workspace=_workspace(d)) - y) <= bound).all()
