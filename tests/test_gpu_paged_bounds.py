"""Attention over the paged cache at the ends of what its arguments may be: bounds far above the lengths, windows of any
size, workspaces cut short."""
import numpy as np
import pytest

import paged_reference as ref
from test_gpu_paged_attention import _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("max_kv", [2**31 - 1, 2**32, 1 << 40, 2**62])
@pytest.mark.parametrize("new,total", [([1], [1000]), ([3, 1], [700, 40]), ([70], [900]), ([40, 2], [300, 500])])
def test_a_bound_of_the_cached_tokens_may_be_anything(new, total, max_kv, cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total))
    _check(d, workspace=False, max_kv=max_kv)
    assert np.array_equal(_run(d, workspace=False, max_kv=max_kv).cpu().numpy(), _run(d, workspace=False).cpu().numpy())
