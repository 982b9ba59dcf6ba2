"""Latent attention, expanded form, against the softmax in 64 bits."""
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
        h = d["heads"]
        self.q, self.kv, self.rope = _t(d["q"])[:, : h * 192].unflatten(1, (h, 192)), _t(d["kv"])[:, : h * 256].unflatten(1, (h, 256)), _t(d["k_rope"])[:, :64]
        self.starts, self.kv_starts, self.scale = _t(d["q_start"]), _t(d["kv_start"]), scale
        self.max_q = int(np.diff(d["q_start"]).max())
        self.ws = pq.pq_latent_workspace(DEV) if workspace else None
        self.out = torch.full((len(d["q"]), h, 128), float("nan"), dtype=torch.float16, device=DEV)

    def __call__(self):
        return pq.pq_expanded_attention(self.q, self.kv, self.rope, self.starts, self.kv_starts, self.max_q, self.scale, out=self.out, workspace=self.ws)


def _check(d, scale=192 ** -0.5, workspace=True):
    call = Call(d, scale, workspace)
    got = call().cpu().numpy().astype(np.float64)
    assert pq.pq_device_status() == 0
    y, bound = ref.expanded_attention(d, scale)
    rows = ~np.isnan(y[:, 0, 0])
    assert (np.abs(got - y)[rows] <= bound[rows]).all()
    assert np.isnan(got[~rows]).all()
    return call


CASES = {
    "one_token": (1, [1], [1]), "one_more": (3, [1], [81]), "a_prompt": (2, [300], [300]), "prompts": (3, [80, 1, 128, 129, 256, 257], [80, 1, 128, 129, 256, 257]),
    "chunks": (2, [100, 300, 5], [500, 340, 1000]), "wide": (16, [40, 3], [50, 200]), "empty": (4, [0, 7, 0, 2], [5, 7, 0, 300]), "long": (2, [2], [9000]),
    "many": (40, [30] * 6, [40] * 6), "turns": (148, [520], [520]),
}


@pytest.mark.parametrize("kind", list(CASES))
def test_expanded_attention(kind):
    heads, new, total = CASES[kind]
    _check(ref.expanded_inputs(heads, new, total, seed=len(kind), gap=3))


@pytest.mark.parametrize("kind", ["prompts", "chunks", "long", "many"])
def test_without_a_workspace(kind):
    heads, new, total = CASES[kind]
    _check(ref.expanded_inputs(heads, new, total, seed=2), workspace=False)


def test_slices_of_wider_matrices():
    _check(ref.expanded_inputs(3, [50, 200], [90, 200], seed=3, stride=24))


def test_rows_that_see_nothing_give_zero():
    out = _check(ref.expanded_inputs(4, [5, 3, 200], [2, 0, 30], seed=1)).out
    assert (out[:3] == 0).all() and (out[5:8] == 0).all() and (out[8:178] == 0).all() and (out[178] != 0).any()
    out = _check(ref.expanded_inputs(4, [5, 3], [0, 0], seed=1)).out             # no keys at all
    assert (out == 0).all()


@pytest.mark.parametrize("scale", [0.0, -0.05, 0.3])
def test_scales(scale):
    _check(ref.expanded_inputs(2, [150, 20], [150, 300], seed=4), scale)


def test_large_scores_move_the_reference():
    d = ref.expanded_inputs(2, [200, 100], [700, 900], seed=5)
    d["kv"][:700, 0] = (np.arange(700) / 20).astype(np.float16)
    d["q"][:200, 0] = 40
    d["k_rope"][700 + 333, 5] = 90
    d["q"][200:, 128 + 5] = 50
    _check(d, 0.05)


def test_what_other_requests_hold_does_not_reach_a_row():
    """Keys behind a request's own are the next request's: infinities and NaN there change nothing."""
    d = ref.expanded_inputs(2, [30, 40], [50, 60], seed=6)
    good = Call(d, 0.07)().clone()
    for fill in (np.inf, np.nan):
        e = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in d.items()}
        e["kv"][50:], e["k_rope"][50:] = fill, fill
        assert torch.equal(Call(e, 0.07)()[:30], good[:30])
        assert pq.pq_device_status() == 0


def test_calls_in_a_row_give_the_same_bits():
    for kind in ("prompts", "chunks", "long", "turns"):
        heads, new, total = CASES[kind]
        call = Call(ref.expanded_inputs(heads, new, total, seed=1), 0.07)
        good = call().clone()
        assert sum(not torch.equal(call(), good) for _ in range(40)) == 0
    assert pq.pq_device_status() == 0


@pytest.mark.parametrize("kind", ["prompts", "many", "long", "turns"])
def test_a_wait_that_runs_out_is_reported_and_leaves_everything_usable(kind):
    heads, new, total = CASES[kind]
    call = Call(ref.expanded_inputs(heads, new, total, seed=1), 0.07)
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


def test_one_workspace_serves_both_forms_in_turn():
    d, e = ref.expanded_inputs(4, [100], [900], seed=7), ref.latent_inputs(16, 512, 16, [1, 1], [800, 300], seed=7)
    first = Call(d, 0.07)
    want = first().clone()
    q, table, starts, lengths = (_t(e[k]) for k in ("q", "table", "q_start", "kv_len"))
    cache = pq.LatentKV(_t(e["data"]))
    absorbed = lambda ws: pq.pq_latent_attention(q, cache, table, starts, lengths, 0.04, workspace=ws)  # noqa: E731
    other = absorbed(pq.pq_latent_workspace(DEV))
    for _ in range(5):
        assert torch.equal(absorbed(first.ws), other) and torch.equal(first(), want)
