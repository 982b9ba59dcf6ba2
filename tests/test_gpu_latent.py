"""Latent attention, absorbed form, against the softmax in 64 bits; the products per head."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PQ_ERR_TIMEOUT = 6
WAIT_NONE = 0xFFFFFFFF


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Call:
    def __init__(self, d, scale, workspace=True):
        self.q, self.table, self.starts, self.lengths = (_t(d[k]) for k in ("q", "table", "q_start", "kv_len"))
        self.cache, self.scale = pq.LatentKV(_t(d["data"])), scale
        self.ws = pq.pq_latent_workspace(DEV) if workspace else None
        self.out = torch.full((*d["q"].shape[:2], d["latent"]), float("nan"), dtype=torch.float16, device=DEV)

    def __call__(self):
        return pq.pq_latent_attention(self.q, self.cache, self.table, self.starts, self.lengths, self.scale, out=self.out, workspace=self.ws)


def _check(d, scale=None, workspace=True):
    scale = (d["latent"] + 64) ** -0.5 if scale is None else scale
    call = Call(d, scale, workspace)
    got = call().cpu().numpy().astype(np.float64)
    assert pq.pq_device_status() == 0
    y, bound = ref.latent_attention(d, scale)
    rows = ~np.isnan(y[:, 0, 0])
    assert (np.abs(got - y)[rows] <= bound[rows]).all()
    assert np.isnan(got[~rows]).all()                       # rows outside every request are left as they were
    return call


CASES = {
    "one_token_one_head": (1, [1], [1], 16), "one_token": (16, [1], [130], 16), "a_step": (16, [1] * 9, [5, 64, 65, 127, 128, 129, 1000, 1, 63], 64),
    "odd_heads": (20, [1, 3, 2], [300, 77, 2], 48), "all_heads": (128, [1, 1, 2], [500, 70, 129], 64), "more_heads": (200, [2], [90], 32),
    "drafts": (32, [4, 4, 1, 7], [900, 4, 65, 2000], 16), "a_chunk": (8, [150], [400], 128), "a_prompt": (3, [129, 1, 64], [129, 1, 64], 16),
    "empty_requests": (16, [0, 2, 0, 1, 0], [0, 50, 77, 3, 0], 16), "long": (16, [1], [9000], 64), "heads_past_a_tile": (48, [5], [333], 16),
}


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("kind", list(CASES))
def test_latent_attention(kind, latent):
    heads, new, total, page = CASES[kind]
    _check(ref.latent_inputs(heads, latent, page, new, total, seed=len(kind), gap=3))


@pytest.mark.parametrize("kind", ["a_step", "all_heads", "drafts", "a_chunk", "long"])
def test_without_a_workspace(kind):
    heads, new, total, page = CASES[kind]
    _check(ref.latent_inputs(heads, 512, page, new, total, seed=3), workspace=False)


def test_rows_that_see_nothing_give_zero():
    """Requests longer than their cached tokens, and lengths of zero."""
    d = ref.latent_inputs(4, 512, 16, [5, 3, 40], [2, 0, 30], seed=1)
    out = _check(d).out
    assert (out[:3] == 0).all() and (out[5:8] == 0).all() and (out[8:18] == 0).all() and (out[18] != 0).any()


def test_lost_pages_read_as_zeros_and_the_tables_end_hides_tokens():
    _check(ref.latent_inputs(16, 512, 16, [1, 2], [200, 90], seed=2, lost=[(0, 0), (0, 5), (0, 11), (1, 2)]))
    _check(ref.latent_inputs(16, 512, 16, [1, 70], [500, 300], seed=2, width=9))


@pytest.mark.parametrize("scale", [0.0, -0.03, 0.2])
def test_scales(scale):
    _check(ref.latent_inputs(16, 512, 16, [1, 3], [300, 100], seed=4), scale)


def test_large_scores_move_the_reference():
    """Scores that grow along the request by far more than a weight's range, and a row whose one token outweighs all."""
    d = ref.latent_inputs(16, 512, 64, [2, 1], [1500, 700], seed=6)
    j = np.arange(1500)
    ids = d["table"][0, j // 64]
    d["data"][ids, j % 64, 0] = (j / 100).astype(np.float16)
    d["q"][:2, :, 0] = 30
    d["data"][d["table"][1, 3], 7, 1] = 60
    d["q"][2, :, 1] = 40
    _check(d, 0.05)


def test_what_a_masked_place_holds_does_not_reach_a_row():
    """Infinities and NaN in pages behind a request's length, in other requests' pages and in rows between requests."""
    d = ref.latent_inputs(16, 512, 16, [1, 1], [37, 61], seed=8)
    for fill in (np.inf, -np.inf, np.nan, -65504):
        e = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in d.items()}
        e["data"][d["table"][0, 2], 5:] = fill
        e["data"][d["table"][1, 3], 13:] = fill
        _check(e)


def test_calls_in_a_row_give_the_same_bits():
    for kind in ("a_step", "all_heads", "drafts", "long"):
        heads, new, total, page = CASES[kind]
        call = Call(ref.latent_inputs(heads, 512, page, new, total, seed=1), 0.04)
        good = call().clone()
        assert sum(not torch.equal(call(), good) for _ in range(40)) == 0
    assert pq.pq_device_status() == 0


@pytest.mark.parametrize("kind", ["a_step", "all_heads", "long"])
def test_a_wait_that_runs_out_is_reported_and_leaves_everything_usable(kind):
    heads, new, total, page = CASES[kind]
    call = Call(ref.latent_inputs(heads, 512, page, new, total, seed=1), 0.04)
    good = call().clone()
    assert pq.pq_device_status() == 0
    for limit in (WAIT_NONE, 1, 16, 256):
        pq.pq_set_wait_limit(limit)
        try:
            got = call().clone()
            status = pq.pq_device_status()
        finally:
            pq.pq_set_wait_limit(0)
        if limit == WAIT_NONE:
            assert status == PQ_ERR_TIMEOUT
        else:
            assert status in (0, PQ_ERR_TIMEOUT)
            if status == 0:
                assert torch.equal(got, good)
        pq.pq_workspace_init(call.ws)
        assert torch.equal(call(), good) and pq.pq_device_status() == 0


def test_two_streams_with_a_workspace_each_and_a_graph():
    calls = [Call(ref.latent_inputs(16, 512, 16, [1] * 5, [700, 30, 400, 64, 999], seed=s), 0.04) for s in (1, 2)]
    good = [c().clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                c()
    torch.cuda.synchronize()
    assert all(torch.equal(c.out, g) for c, g in zip(calls, good))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls[0]()
    calls[0].q.copy_(calls[1].q)
    fresh = calls[0]().clone()
    calls[0].out.zero_()
    graph.replay()
    assert torch.equal(calls[0].out, fresh) and pq.pq_device_status() == 0


@pytest.mark.parametrize("T,heads,K,N", [(1, 1, 64, 128), (1, 32, 128, 512), (17, 5, 512, 128), (64, 16, 512, 128), (65, 3, 320, 256), (130, 4, 128, 512),
                                         (200, 2, 256, 1024), (16, 128, 128, 512)])
def test_head_linear(T, heads, K, N):
    """Against the product in 64 bits: half a step of FP16 of the result, K FP32 roundings (truncations at worst, 2^-23 each) of the
    sum of magnitudes."""
    rng = np.random.default_rng(T + K)
    x, w = rng.standard_normal((T, heads, K)).astype(np.float16), (rng.standard_normal((heads, N, K)) / K ** 0.5).astype(np.float16)
    got = pq.pq_head_linear(_t(x), _t(w)).cpu().numpy().astype(np.float64)
    want = np.einsum("thk,hnk->thn", x.astype(np.float64), w.astype(np.float64))
    most = np.einsum("thk,hnk->thn", np.abs(x).astype(np.float64), np.abs(w).astype(np.float64))
    assert (np.abs(got - want) <= 2.0 ** -11 * np.abs(want) + K * 2.0 ** -23 * most + 2.0 ** -25).all() and pq.pq_device_status() == 0


def test_head_linear_of_slices():
    """Queries' first part out of whole heads into the latent queries' first part; values of a wider output."""
    rng = np.random.default_rng(2)
    x, w = _t(rng.standard_normal((21, 6, 192)).astype(np.float16)), _t(rng.standard_normal((6, 512, 128)).astype(np.float16) / 12)
    out = torch.full((21, 6, 576), 5.0, dtype=torch.float16, device=DEV)
    pq.pq_head_linear(x[..., :128], w, out=out[..., :512])
    assert torch.equal(out[..., :512], pq.pq_head_linear(x[..., :128].contiguous(), w)) and (out[..., 512:] == 5).all()
    assert pq.pq_head_linear(x[:0, :, :128], w).shape == (0, 6, 512)
    pq.pq_set_wait_limit(WAIT_NONE)
    try:
        pq.pq_head_linear(x[..., :128], w)
        assert pq.pq_device_status() == PQ_ERR_TIMEOUT
    finally:
        pq.pq_set_wait_limit(0)
    assert torch.equal(out[..., :512], pq.pq_head_linear(x[..., :128], w)) and pq.pq_device_status() == 0
