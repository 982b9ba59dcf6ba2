"""The served attention block of the example against the same layer computed densely, request by request."""
import os
import sys

import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq
from paper_2512_23367_b200 import synth

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paged_attention_layer as example  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dense(layer, x, int8):
    """Attention of one request's tokens in 64 bits from the layer's own q, k, v: (y, bound)."""
    T = x.shape[0]
    q, k, v = (t.view(T, -1, layer.dim).cpu().numpy() for t in layer.project(x))
    d = {"q": q, "table": np.zeros((1, 1), np.int32), "q_start": np.array([0, T]), "kv_len": np.array([T]), "window": 0, "ks": None, "vs": None}
    if int8:
        (d["k"], d["ks"]), (d["v"], d["vs"]) = ((c.swapaxes(0, 1)[None], s.swapaxes(0, 1)[None]) for c, s in (ref.quantize(k), ref.quantize(v)))
    else:
        d["k"], d["v"] = (t.swapaxes(0, 1)[None] for t in (k, v))     # one page of T tokens
    return ref.attention(d)


@pytest.mark.parametrize("cache", ["f16", "int8"])
def test_served_in_chunks_and_tokens_as_computed_at_once(cache):
    prompts, decoded, page = [150, 3, 37], 4, 16
    layer = example.PagedAttentionLayer(8, 2, 64, 3, pages=sum(-(-(p + decoded) // page) for p in prompts), page=page, width=12,
                                        cache=torch.int8 if cache == "int8" else torch.float16)
    inputs = [torch.from_numpy(synth.activations(p + decoded, 512, seed=i)).to(DEV) * 0.1 for i, p in enumerate(prompts)]
    seen = []
    attend, pq.pq_paged_attention = pq.pq_paged_attention, lambda *a, **k: seen.append(attend(*a, **k)) or seen[-1]
    try:
        out = example.serve(layer, inputs, prompts, chunk=64)
    finally:
        pq.pq_paged_attention = attend
    assert pq.pq_device_status() == 0
    assert int(layer.free_head) == layer.cache.pages                # every page handed out, none twice
    assert sorted(layer.table[b, c].item() for b, p in enumerate(prompts) for c in range(-(-(p + decoded) // page))) == list(range(layer.cache.pages))
    # the attention outputs of the steps, request by request
    news, done = [], [0] * 3
    while any(d < len(x) for d, x in zip(done, inputs)):
        news.append([min(64, p - d) if d < p else min(1, len(x) - d) for d, p, x in zip(done, prompts, inputs)])
        done = [d + n for d, n in zip(done, news[-1])]
    assert [sum(n) for n in news] == [len(y) for y in seen]
    for b, x in enumerate(inputs):
        got = torch.cat([torch.split(y, n)[b] for y, n in zip(seen, news)])
        y, bound = _dense(layer, x, cache == "int8")
        assert (np.abs(got.view(len(x), 8, 64).cpu().numpy() - y) <= bound).all()
        assert torch.equal(out[b], pq.pq_linear_w8a8(got.contiguous(), *layer.o, 512))


def test_the_example_runs_as_a_command():
    import subprocess
    for cache in ("f16", "int8"):
        r = subprocess.run([sys.executable, example.__file__, "--cache", cache], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0 and "status 0 finite True" in r.stdout, r.stdout + r.stderr


def _inputs(new, seed):
    return torch.from_numpy(synth.activations(sum(new), 512, seed=seed)).to(DEV)


def test_the_workspace_is_kept_from_step_to_step():
    layer = example.PagedAttentionLayer(8, 2, 64, 2, pages=130, page=16, width=64)
    layer.step(_inputs([900, 100], 1), [900, 100])
    seen = []
    for i in range(12):
        layer.step(_inputs([1, 1], 2 + i), [1, 1])
        seen.append((layer.workspace.data_ptr(), layer.workspace.numel()))
    sizes = [n for _, n in seen]
    assert sizes == sorted(sizes) and len(set(seen)) == len(set(sizes)) <= 2
    assert pq.pq_device_status() == 0


def test_a_step_that_the_pages_do_not_hold_is_refused():
    layer = example.PagedAttentionLayer(8, 2, 64, 2, pages=6, page=16, width=4)
    layer.step(_inputs([40, 10], 1), [40, 10])                   # 3 + 1 pages
    for new in ([20, 30], [30, 1]):                              # 4 + 3 pages, 5 columns
        with pytest.raises(ValueError, match="pages"):
            layer.step(_inputs(new, 2), new)
        assert layer.lengths == [40, 10]
    y = layer.step(_inputs([20, 7], 3), [20, 7])                 # 4 + 2
    assert torch.isfinite(y).all() and int(layer.free_head) == 6 and pq.pq_device_status() == 0
