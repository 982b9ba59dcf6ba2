"""Attention over the paged cache at the ends of what its arguments may be: bounds far above the lengths, windows of any
size, workspaces cut short."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq
from test_gpu_paged_attention import DEV, _check, _run, _t

pytestmark = pytest.mark.gpu


def _serve(d, max_q=None, max_kv=None, workspace=None, window=None):
    """One call over the inputs `d`; the workspace is the caller's."""
    out = torch.full(d["q"].shape, float("nan"), dtype=torch.float16, device=DEV)
    pq.pq_paged_attention(_t(d["q"]), pq.PagedKV(_t(d["k"]), _t(d["v"]), _t(d["ks"]), _t(d["vs"])), _t(d["table"]),
                          _t(d["q_start"]), _t(d["kv_len"]), int(np.diff(d["q_start"]).max()) if max_q is None else max_q,
                          int(d["kv_len"].max()) if max_kv is None else max_kv,
                          window=d["window"] if window is None else window, out=out, workspace=workspace)
    assert pq.pq_device_status() == 0
    return out.cpu().numpy().astype(np.float64)


def _workspace(d, max_q=None, max_kv=None, **more):
    kv_heads, _, dim = d["k"].shape[1:]
    n = pq.pq_attention_workspace_bytes(len(d["kv_len"]), d["q"].shape[0], int(np.diff(d["q_start"]).max()) if max_q is None else max_q,
                                        int(d["kv_len"].max()) if max_kv is None else max_kv, d["q"].shape[1], kv_heads, dim, **more)
    return pq.pq_workspace_init(torch.empty((n,), dtype=torch.uint8, device=DEV)) if n else None


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("max_kv", [2**31 - 1, 2**32, 1 << 40, 2**62])
@pytest.mark.parametrize("new,total", [([1], [1000]), ([3, 1], [700, 40]), ([70], [900]), ([40, 2], [300, 500])])
def test_a_bound_of_the_cached_tokens_may_be_anything(new, total, max_kv, cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total))
    _check(d, workspace=False, max_kv=max_kv)
    assert np.array_equal(_run(d, workspace=False, max_kv=max_kv).cpu().numpy(), _run(d, workspace=False).cpu().numpy())


@pytest.mark.parametrize("max_q", [2**31, 1 << 40, 2**61, 2**62, 2**63 - 1])
@pytest.mark.parametrize("new,total", [([40, 2], [300, 500]), ([70], [900]), ([1, 3], [50, 60])])
def test_a_bound_of_the_rows_may_be_anything(new, total, max_q):
    d = ref.attention_inputs(8, 2, 128, 16, "f16", new, total, seed=sum(total))
    y, bound = ref.attention(d)
    for workspace in (_workspace(d, max_q=max_q), None):
        assert (np.abs(_serve(d, max_q=max_q, workspace=workspace) - y) <= bound).all()


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 64, 2**30, 301])
@pytest.mark.parametrize("new,total", [([200], [100]), ([300, 3], [7, 1]), ([4, 2], [2, 300]), ([70], [300])])
def test_a_window_as_long_as_anything_is_none(new, total, window, cache):
    """Also where the chunk is longer than what is cached, so that its first rows stand before the first key."""
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(new))
    y, bound = ref.attention(d)
    for workspace in (_workspace(d), None):
        assert (np.abs(_serve(d, window=window, workspace=workspace) - y) <= bound).all()


def _split(d, share=1.0, window=0):
    """One call with `share` of the workspace that the query asks for at this window."""
    full = _workspace(d, window=window)
    header = 65536
    pq.pq_workspace_init(full)
    return _serve(d, window=window, workspace=full[: header + int((full.numel() - header) * share)] if share < 1 else full)


@pytest.mark.parametrize("heads,kv_heads,dim,new,total,window", [
    (32, 8, 128, [300], [4300], 4096), (32, 8, 128, [150, 150], [3000, 3000], 2048), (32, 32, 64, [1, 1, 1], [1300] * 3, 1024),
    (8, 2, 128, [3], [2600], 1500)])
def test_the_workspace_for_a_window_is_all_that_the_call_uses(heads, kv_heads, dim, new, total, window):
    d = ref.attention_inputs(heads, kv_heads, dim, 16, "f16", new, total, window=window, seed=sum(total))
    y, bound = ref.attention(d)
    a = _split(d, window=window)
    assert (np.abs(a - y) <= bound).all()
    room = pq.pq_workspace_init(torch.empty((1 << 28,), dtype=torch.uint8, device=DEV))
    assert np.array_equal(a, _serve(d, workspace=room))            # the same parts as with any amount of room


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("new,total", [([1], [5000]), ([3, 1], [4100, 700]), ([3], [2500])])
def test_a_workspace_cut_short_still_serves_few_rows(new, total, cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total))
    y, bound = ref.attention(d)
    for share in (0.5, 0.2, 0.02):
        assert (np.abs(_split(d, share) - y) <= bound).all()


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("new,total", [([1], [5000]), ([3, 1], [4100, 700]), ([70], [6000]), ([2, 40], [3000, 2000])])
def test_a_bound_of_the_cached_tokens_that_is_too_small_costs_speed_only(new, total, cache):
    """With parts all the same: the last one takes the keys that are left."""
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total))
    y, bound = ref.attention(d)
    for hint in (1500, 700, 200):
        assert (np.abs(_serve(d, max_kv=hint, workspace=_workspace(d)) - y) <= bound).all()
