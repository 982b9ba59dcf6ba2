"""The products per head where calls are out of the ordinary."""
import pytest
import torch

import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PQ_ERR_TIMEOUT = 6
WAIT_NONE = 0xFFFFFFFF


def _operands(T, heads, K, N, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *s: torch.empty(s, dtype=torch.float16, device=DEV).normal_(generator=gen)  # noqa: E731
    return rand(T, heads, K), rand(heads, N, K) * K ** -0.5


def _check(y, x, w):
    """Half a step of FP16 of the result, K FP32 roundings (truncations at worst, 2^-23 each) of the sum of magnitudes."""
    x, w, K = x.double().transpose(0, 1), w.double().transpose(1, 2), x.shape[2]
    want, most = (x @ w).transpose(0, 1), (x.abs() @ w.abs()).transpose(0, 1)
    assert ((y.double() - want).abs() <= 2.0 ** -11 * want.abs() + K * 2.0 ** -23 * most + 2.0 ** -25).all()


@pytest.mark.parametrize("T,heads,K,N", [(1, 32, 128, 512), (64, 128, 512, 128), (200, 16, 256, 256)])
def test_a_wait_that_runs_out_anywhere_is_reported_and_leaves_everything_usable(T, heads, K, N):
    """Bounds of a few polls, at which some of the warps that store the results have had theirs and others not."""
    x, w = _operands(T, heads, K, N)
    good = pq.pq_head_linear(x, w)
    assert pq.pq_device_status() == 0
    _check(good, x, w)
    for limit in (WAIT_NONE, 1, 2, 3, 4, 6, 8, 16, 64, 256):
        for _ in range(5):
            pq.pq_set_wait_limit(limit)
            try:
                got = pq.pq_head_linear(x, w)
                status = pq.pq_device_status()
            finally:
                pq.pq_set_wait_limit(0)
            assert status == PQ_ERR_TIMEOUT if limit == WAIT_NONE else status in (0, PQ_ERR_TIMEOUT)
            assert status != 0 or torch.equal(got, good)
        assert torch.equal(pq.pq_head_linear(x, w), good) and pq.pq_device_status() == 0


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("T,heads,K,N", [(1, 8, 128, 512), (64, 128, 512, 128), (16, 128, 128, 512)])
def test_weights_may_be_written_by_the_launch_right_before(T, heads, K, N, captured):
    """Matrices that a kernel of this library (which lets the next launch begin early; a rotation by nothing is a copy) or one of
    torch's leaves, another one's at every call."""
    x, w = _operands(T, heads, K, N)
    sources = [w, _operands(T, heads, K, N, 1)[1], _operands(T, heads, K, N, 2)[1]]
    good = [pq.pq_head_linear(x, s) for s in sources]
    for g, s in zip(good, sources):
        _check(g, x, s)
    room, out = torch.zeros_like(w), [torch.zeros_like(good[0]) for _ in range(30)]
    rotary, pos = pq.Rotary(16, device=DEV), torch.zeros(heads * N, dtype=torch.int32, device=DEV)

    def run():
        for i, y in enumerate(out):
            if i % 5 == 4:
                room.copy_(sources[i % 3])
            else:
                pq.pq_rotate(sources[i % 3].view(-1, 1, K), pos, rotary, out=room.view(-1, 1, K))
            pq.pq_head_linear(x, room, out=y)

    if captured:
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        for y in out:
            y.zero_()
        graph.replay()
    else:
        torch.cuda.synchronize()
        run()
    assert all(torch.equal(y, good[i % 3]) for i, y in enumerate(out)) and pq.pq_device_status() == 0


def test_more_tokens_than_a_grids_outer_dimensions_hold():
    """65536 batches of 128 tokens and a ragged one, of one head."""
    T, w = 65536 * 128 + 77, _operands(1, 1, 64, 128)[1]
    gen = torch.Generator(DEV).manual_seed(3)
    x = torch.empty((T, 1, 64), dtype=torch.float16, device=DEV).normal_(generator=gen)
    y = pq.pq_head_linear(x, w)
    assert pq.pq_device_status() == 0
    for t0 in range(0, T, 1 << 20):
        _check(y[t0: t0 + (1 << 20)], x[t0: t0 + (1 << 20)], w)
