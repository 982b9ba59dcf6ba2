"""The served latent attention block of the example: its steps against the 64-bit form, its two forms against each other."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2512_23367_b200 as pq
from paper_2512_23367_b200 import synth

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import latent_attention_layer as example  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(sizes, hidden):
    return [torch.from_numpy(synth.activations(n, hidden, seed=i)).to(DEV) * 0.1 for i, n in enumerate(sizes)]


@pytest.mark.parametrize("latent", [512, 256])
def test_served_in_chunks_and_tokens(latent, monkeypatch):
    """Every attention of the run, in either form, is that of its own operands over the cache as it stands."""
    prompts, decoded, page, hidden, heads = [150, 3, 37], 4, 16, 512, 6
    layer = example.LatentAttentionLayer(heads, hidden, latent, 3, pages=sum(-(-(p + decoded) // page) for p in prompts), page=page, width=12)
    seen = {"absorbed": 0, "expanded": 0}

    def absorbed(q, cache, table, q_start, kv_len, scale, **more):
        y = real_absorbed(q, cache, table, q_start, kv_len, scale, **more)
        n = lambda t: t.cpu().numpy()  # noqa: E731
        d = dict(q=n(q), data=n(cache.data), table=n(table), q_start=n(q_start), kv_len=n(kv_len), latent=latent)
        want, bound = ref.latent_attention(d, scale)
        assert (np.abs(n(y) - want) <= bound).all()
        seen["absorbed"] += 1
        return y

    def expanded(q, kv, rope, q_start, kv_start, max_q, scale, **more):
        y = real_expanded(q, kv, rope, q_start, kv_start, max_q, scale, **more)
        n = lambda t: t.cpu().numpy()  # noqa: E731
        d = dict(q=n(q).reshape(len(q), -1), kv=n(kv).reshape(len(kv), -1), k_rope=n(rope), heads=heads, q_start=n(q_start), kv_start=n(kv_start))
        want, bound = ref.expanded_attention(d, scale)
        assert (np.abs(n(y) - want) <= bound).all()
        seen["expanded"] += 1
        return y

    real_absorbed, real_expanded = pq.pq_latent_attention, pq.pq_expanded_attention
    monkeypatch.setattr(pq, "pq_latent_attention", absorbed)
    monkeypatch.setattr(pq, "pq_expanded_attention", expanded)
    out = example.serve(layer, _inputs([p + decoded for p in prompts], hidden), prompts, chunk=64)
    assert pq.pq_device_status() == 0 and int(layer.free_head) == layer.cache.pages and [len(y) for y in out] == [154, 7, 41]
    assert seen["absorbed"] > 0 and seen["expanded"] > 0
    # the cache holds the turned keys of all positions: as if appended at once
    for b, x in enumerate(_inputs([p + decoded for p in prompts], hidden)):
        n = len(x)
        slots = layer.table[b, torch.arange(n, device=DEV) // page].long() * page + torch.arange(n, device=DEV) % page
        c, rope = pq.pq_latent_read(layer.cache, slots)
        ckr = pq.pq_gemm_w8a8_group(*pq.pq_quantize_act(x), layer.in_proj)[1]
        turned = pq.pq_rotate(ckr[:, None, latent:], torch.arange(n, dtype=torch.int32, device=DEV), layer.rotary)[:, 0]
        assert torch.equal(c, ckr[:, :latent]) and torch.equal(rope, turned)


def test_both_forms_serve_the_same_step():
    """A decode step in the one form and in the other: the expanded form quantizes the latents for its W8A8 linear (half a code of
    127.5 of a vector's largest value), the absorbed one takes them as they are; the outputs stay within that."""
    outs = []
    for last in (False, True):
        layer = example.LatentAttentionLayer(16, 512, 512, 2, pages=20, page=64, width=10)
        xs = _inputs([300, 90], 512)
        layer.step(torch.cat([xs[0][:-1], xs[1][:-1]]), [299, 89], expanded=True)
        seen = []
        real, pq.pq_linear_w8a8 = pq.pq_linear_w8a8, lambda x, *a, **k: seen.append(x) or real(x, *a, **k)
        try:
            layer.step(torch.cat([xs[0][-1:], xs[1][-1:]]), [1, 1], expanded=last)
        finally:
            pq.pq_linear_w8a8 = real
        outs.append(seen[-1].double())                     # what goes into the output linear
    assert (outs[0] - outs[1]).norm() <= 0.03 * outs[0].norm() and pq.pq_device_status() == 0


def test_the_example_runs_as_a_command():
    r = subprocess.run([sys.executable, example.__file__], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "status 0 finite True" in r.stdout, r.stdout + r.stderr


def test_a_step_that_the_pages_do_not_hold_is_refused():
    layer = example.LatentAttentionLayer(2, 512, 256, 2, pages=6, page=16, width=4)
    x = _inputs([50, 7], 512)
    layer.step(x[0], [40, 10], expanded=True)                    # 3 + 1 pages
    with pytest.raises(ValueError, match="pages"):
        layer.step(x[0], [20, 30], expanded=True)
    assert layer.lengths == [40, 10]
    y = layer.step(x[1][:2], [1, 1], expanded=False)
    assert torch.isfinite(y).all() and pq.pq_device_status() == 0
