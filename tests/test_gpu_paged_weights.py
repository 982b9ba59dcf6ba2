"""Attention over the paged cache where most of a row's answer comes from keys of very small weight, or from none."""
import numpy as np
import pytest

import paged_reference as ref
from test_gpu_paged_bounds import _serve, _workspace

pytestmark = pytest.mark.gpu

LENGTHS = [([1, 1], [3000, 500]), ([3], [2000]), ([20], [3000]), ([100], [2500])]


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("heavy", [5, 300])
@pytest.mark.parametrize("new,total", LENGTHS)
def test_many_keys_of_very_small_weight_add_up(new, total, heavy, cache):
    """One key has value 0 and 2^26.4 times the weight of every other: the answer is the others' sum.  Bound: 2^-9 of it for
    the FP16 roundings of weights and result and for scores of up to 27 in FP32; FP16's smallest step under weights of up to
    2^7 at least, 2^-32 of the largest weight, from every key; half of the result's smallest step."""
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total))
    rng = np.random.default_rng(9)
    d["q"][:] = 1
    at = [(d["table"][b, heavy // 16], heavy % 16) for b in range(len(new))]
    if cache == "f16":
        d["k"][:], d["v"][:] = 0, rng.uniform(32, 64, d["v"].shape).astype(np.float16)
        for page, off in at:
            d["k"][page, :, off], d["v"][page, :, off] = np.float16(26.4 * np.log(2) / 128 ** 0.5), 0
    else:
        d["k"][:], d["v"][:] = 0, rng.integers(64, 128, d["v"].shape)
        d["ks"][:], d["vs"][:] = np.float32(26.4 * np.log(2) / 128 ** 0.5 / 100), np.float32(0.5)
        for page, off in at:
            d["k"][page, :, off], d["v"][page, :, off] = 100, 0
    y, _ = ref.attention(d)
    got = _serve(d, workspace=_workspace(d))
    assert (y > 2e-4).all()                    # the input is what it is meant to be
    for b, length in enumerate(total):
        rows = slice(d["q_start"][b], d["q_start"][b + 1])
        assert (np.abs(got[rows] - y[rows]) <= 2.0 ** -9 * y[rows] + length * 2.0 ** -32 * 64 + 2.0 ** -25).all()


@pytest.mark.parametrize("new,total", [([1, 3], [300, 40]), ([20], [300]), ([100], [250])])
def test_value_scales_of_zero_give_zero(new, total):
    d = ref.attention_inputs(8, 2, 128, 16, "int8", new, total, seed=1)
    d["vs"][:] = 0                       # as vectors of zeros leave them, whatever the codes
    assert (_serve(d, workspace=_workspace(d)) == 0).all()
    d["ks"][:] = 0
    assert (_serve(d) == 0).all()
