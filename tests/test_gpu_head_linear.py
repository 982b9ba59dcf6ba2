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
