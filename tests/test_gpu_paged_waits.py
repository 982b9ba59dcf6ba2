"""The attention tile kernel's waits: a wait that runs out ends in PQ_ERR_TIMEOUT and leaves everything usable (the poll
bound is lowered, nothing is broken), and calls in a row give the same bits -- a stage that is announced before all of
it is written shows as a result that differs now and then."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PQ_ERR_TIMEOUT = 6
WAIT_NONE = 0xFFFFFFFF

CASES = {"two_tiles": (32, 8, 128, [300], [511]), "one_tile": (16, 1, 128, [5, 3], [700, 90]), "dim_64": (4, 4, 64, [300, 20], [300, 433]),
         "split_keys": (8, 2, 128, [70], [6000])}


def _call(kind, cache):
    heads, kv_heads, dim, new, total = CASES[kind]
    d = ref.attention_inputs(heads, kv_heads, dim, 48, cache, new, total, seed=len(kind))
    t = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    kv = pq.PagedKV(t(d["k"]), t(d["v"]), t(d["ks"]), t(d["vs"]))
    q, table, starts, lengths = t(d["q"]), t(d["table"]), t(d["q_start"]), t(d["kv_len"])
    ws = pq.pq_attention_workspace(q, kv, len(new), max(new), max(total))
    call = lambda: pq.pq_paged_attention(q, kv, table, starts, lengths, max(new), max(total), workspace=ws)  # noqa: E731
    return d, call, (lambda: ws is not None and pq.pq_workspace_init(ws))


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("kind", list(CASES))
def test_a_wait_that_runs_out_is_reported_and_leaves_everything_usable(kind, cache):
    d, call, reinit = _call(kind, cache)
    good = call().clone()
    assert pq.pq_device_status() == 0
    y, bound = ref.attention(d)
    assert (np.abs(good.cpu().numpy() - y) <= bound).all()
    for limit in (WAIT_NONE, 1, 16, 256):
        pq.pq_set_wait_limit(limit)
        try:
            got = call().clone()
            status = pq.pq_device_status()        # synchronizes
        finally:
            pq.pq_set_wait_limit(0)
        if limit == WAIT_NONE:
            assert status == PQ_ERR_TIMEOUT
        else:
            assert status in (0, PQ_ERR_TIMEOUT)
            if status == 0:
                assert torch.equal(got, good)     # nothing ran out: the result is the normal one
        reinit()                                   # a caller's workspace is prepared again after a give-up
        assert torch.equal(call(), good)
        assert pq.pq_device_status() == 0


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("kind", list(CASES))
def test_calls_in_a_row_give_the_same_bits(kind, cache):
    _, call, _ = _call(kind, cache)
    good = call().clone()
    assert sum(not torch.equal(call(), good) for _ in range(60)) == 0
    assert pq.pq_device_status() == 0
