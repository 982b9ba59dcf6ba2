"""Refusals of the latent calls at the ends of what they take."""
import pytest

import paper_2512_23367_b200 as pq
from test_latent_abi import ALIGN, LIMIT, SHAPE, _latent

FAR = 1 << 38   # elements: a tensor map holds strides below 2^40 bytes


@pytest.mark.parametrize("out", [8, 24, 18])
def test_outputs_off_a_16_byte_boundary(out):
    assert pq.lib().pq_latent_attention(16, 4, _latent(), 16, 4, 16, 16, 2, 3, 0.1, out, None, 0, None) == ALIGN
    assert pq.lib().pq_expanded_attention(16, 768, 4, 16, 1024, 16, 64, 9, 16, 16, 2, 3, 2, 0.1, out, None, 0, None) == ALIGN
    assert pq.lib().pq_head_linear(16, 512, 128, 16, 4, 512, 128, 3, out, 2048, 512, None) == ALIGN


def test_strides_beyond_a_tensor_map():
    def expanded(qs=768, kvs=1024, krs=64):
        return pq.lib().pq_expanded_attention(None, qs, 4, None, kvs, None, krs, 0, None, None, 0, 3, 2, 0.1, None, None, 0, None)

    assert expanded() == 0
    assert expanded(qs=FAR) == SHAPE and expanded(kvs=FAR) == SHAPE and expanded(krs=FAR) == SHAPE
    assert expanded(qs=FAR - 8) == 0 and expanded(kvs=FAR - 8) == 0 and expanded(krs=FAR - 8) == 0

    def head(xs, xhs):
        return pq.lib().pq_head_linear(None, xs, xhs, None, 4, 512, 128, 2, None, 2048, 512, None)

    assert head(FAR, 128) == SHAPE and head(512, FAR) == SHAPE


def test_requests_and_rows():
    def calls(requests, heads, tokens):
        return {pq.lib().pq_latent_attention(None, heads, _latent(), None, 4, None, None, requests, tokens, 0.1, None, None, 0, None),
                pq.lib().pq_expanded_attention(None, heads * 192, heads, None, heads * 256, None, 64, 0, None, None, requests, tokens, 2, 0.1, None, None, 0, None)}

    assert calls(4096, 8, 0) == {0} and calls(4097, 8, 0) == {LIMIT}
    assert calls(0, 8, (1 << 28) - 1) == {0} and calls(0, 8, 1 << 28) == {SHAPE}
