"""Refusals of the paged cache calls: argument errors come back before anything touches a device."""
import ctypes
import types

import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq
from paper_2512_23367_b200 import binding

NULL, SHAPE, ALIGN, LIMIT = 1, 2, 3, 7


_KEEP = []    # the structs whose addresses the calls below are given


def _cache(**change):
    a = dict(k=16, v=16, k_scale=None, v_scale=None, pages=4, heads=2, page=16, dim=64, type=0) | change
    _KEEP.append(binding._KVCache(**a))
    return ctypes.addressof(_KEEP[-1])


def test_cache_geometry():
    L = pq.lib()
    read = lambda c: L.pq_kv_read(c, 16, 1, 16, 16, None)  # noqa: E731
    assert read(None) == NULL
    assert read(_cache(k=None)) == NULL
    assert read(_cache(type=1)) == NULL                       # INT8 without scales
    assert read(_cache(type=2)) == SHAPE
    assert read(_cache(dim=96)) == SHAPE
    assert read(_cache(page=8)) == SHAPE and read(_cache(page=24)) == SHAPE and read(_cache(page=2048)) == SHAPE
    assert read(_cache(heads=0)) == SHAPE and read(_cache(heads=1025)) == SHAPE
    assert read(_cache(pages=0)) == SHAPE
    assert read(_cache(pages=1 << 26, heads=2, page=16)) == SHAPE       # 2^31 vectors
    assert read(_cache(v=24)) == ALIGN
    assert read(_cache(type=1, k_scale=16, v_scale=20)) == ALIGN


def test_block_tables_refuses():
    L = pq.lib()

    def call(kv=16, new=16, requests=2, table=16, width=4, free=16, count=8, head=16, page=16, tokens=3, q=16, total=32,
             slots=16, pos=16, nxt=32):
        return L.pq_block_tables(kv, new, requests, table, width, free, count, head, page, tokens, q, total, slots, pos, nxt, None)

    assert call(requests=-1) == SHAPE and call(tokens=-1) == SHAPE and call(width=0) == SHAPE and call(count=-1) == SHAPE
    assert call(tokens=1 << 31) == SHAPE
    assert call(page=0) == SHAPE and call(page=20) == SHAPE
    assert call(requests=4097) == LIMIT
    assert call(kv=None) == NULL and call(head=None) == NULL and call(free=None) == NULL and call(slots=None) == NULL
    assert call(nxt=16) == SHAPE and call(total=16) == SHAPE       # in place


def test_append_and_read_refuse():
    L = pq.lib()
    c = _cache()
    assert L.pq_kv_append(c, 16, 127, 16, 128, 16, 1, None) == SHAPE      # stride below the row
    assert L.pq_kv_append(c, 16, 132, 16, 128, 16, 1, None) == SHAPE      # stride % 8
    assert L.pq_kv_append(c, 16, 128, 16, 128, 16, -1, None) == SHAPE
    assert L.pq_kv_append(c, None, 128, 16, 128, 16, 1, None) == NULL
    assert L.pq_kv_append(c, 16, 128, 8, 128, 16, 1, None) == ALIGN
    assert L.pq_kv_append(c, None, 128, None, 128, None, 0, None) == 0    # nothing to do
    assert L.pq_kv_read(c, 16, 1, 16, None, None) == NULL
    assert L.pq_kv_read(c, 16, 1, 8, 16, None) == ALIGN
    assert L.pq_kv_read(c, None, 0, None, None, None) == 0


def test_attention_refuses():
    L = pq.lib()

    def call(q=16, stride=256, heads=4, c=None, table=16, width=4, qs=16, kl=16, requests=2, tokens=3, max_q=2, max_kv=9,
             scale=0.1, window=0, out=16, ws=None, ws_bytes=0):
        return L.pq_paged_attention(q, stride, heads, _cache() if c is None else c, table, width, qs, kl, requests, tokens,
                                    max_q, max_kv, scale, window, out, ws, ws_bytes, None)

    assert call(c=_cache(dim=80)) == SHAPE
    assert call(heads=3) == SHAPE and call(heads=0) == SHAPE and call(heads=130, stride=130 * 64) == SHAPE   # group of 65
    assert call(stride=248) == SHAPE and call(stride=260) == SHAPE
    assert call(width=0) == SHAPE and call(max_q=-1) == SHAPE and call(max_kv=-1) == SHAPE and call(window=-1) == SHAPE
    assert call(scale=float("nan")) == SHAPE and call(scale=float("inf")) == SHAPE
    assert call(requests=-1) == SHAPE and call(tokens=-2) == SHAPE and call(requests=4097) == LIMIT
    assert call(q=None) == NULL and call(kl=None) == NULL and call(out=None) == NULL
    assert call(q=8) == ALIGN and call(ws=128, ws_bytes=1 << 20) == ALIGN
    assert call(requests=0, qs=None, kl=None, table=None) == 0 and call(tokens=0) == 0       # nothing to do


def test_binding_measures_every_operand():
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    k = f16(4, 2, 16, 64)
    with pytest.raises(ValueError, match="CUDA"):
        pq.PagedKV(k, k)
    with pytest.raises(ValueError, match="4-D"):
        pq.PagedKV(k[0], k[0])
    with pytest.raises(ValueError, match="v: expected"):
        pq.PagedKV(k, k[:2])
    with pytest.raises(TypeError):
        pq.PagedKV(k.float(), k.float())
    with pytest.raises(ValueError, match="k_scale"):
        pq.PagedKV(k.to(torch.int8), k.to(torch.int8))
    with pytest.raises(ValueError, match="v_scale: expected 128"):
        pq.PagedKV(k.to(torch.int8), k.to(torch.int8), torch.zeros(4, 2, 16), torch.zeros(4, 2, 15))
    with pytest.raises(ValueError, match="contiguous"):
        pq.PagedKV(k.transpose(0, 1), k.transpose(0, 1))
    with pytest.raises(ValueError, match="new_len: expected 2"):
        pq.pq_block_tables(i32(2), i32(3), i32(2, 4), i32(5), i32(1), 16, 3)
    with pytest.raises(TypeError):
        pq.pq_block_tables(i32(2), i32(2).long(), i32(2, 4), i32(5), i32(1), 16, 3)
    with pytest.raises(ValueError, match="block_table: expected"):
        pq.pq_block_tables(i32(2), i32(2), i32(3, 4), i32(5), i32(1), 16, 3)
    with pytest.raises(ValueError, match="tokens"):
        pq.pq_block_tables(i32(2), i32(2), i32(2, 4), i32(5), i32(1), 16)
    with pytest.raises(ValueError, match="pos: expected 3"):
        pq.PagedStep(i32(3), i32(2), i32(3).long(), i32(2), i32(1))
    with pytest.raises(ValueError, match="CUDA"):
        pq.PagedStep(i32(3), i32(2), i32(3).long(), i32(3), i32(1))
    step = types.SimpleNamespace(requests=2, tokens=3, device=-1)
    with pytest.raises(ValueError, match="step: made for 2 requests and 3 tokens"):
        pq.pq_block_tables(i32(3), i32(3), i32(3, 4), i32(5), i32(1), 16, step=step)
    with pytest.raises(ValueError, match="step: made for"):
        pq.pq_block_tables(i32(2), i32(2), i32(2, 4), i32(5), i32(1), 16, 4, step=step)
    with pytest.raises(ValueError, match="CUDA"):
        pq.pq_block_tables(i32(2), i32(2), i32(2, 4), i32(5), i32(1), 16, 3)

    Fake = types.SimpleNamespace(heads=2, dim=64, page=16, pages=4, device=-1, _ref=0)   # no call gets as far as its memory
    with pytest.raises(ValueError, match="k: expected rows"):
        pq.pq_kv_append(Fake, f16(3, 1, 64), f16(3, 2, 64), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="k: expected rows"):
        pq.pq_kv_append(Fake, f16(2, 3, 64).transpose(0, 1), f16(3, 2, 64), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="v: expected 3 rows"):
        pq.pq_kv_append(Fake, f16(3, 2, 64), f16(2, 128), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="slots: expected 3"):
        pq.pq_kv_append(Fake, f16(3, 2, 64), f16(3, 128), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        pq.pq_kv_append(Fake, f16(3, 2, 64), f16(3, 128), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        pq.pq_paged_attention(torch.zeros(3, 4, 64), Fake, i32(2, 4), i32(3), i32(2), 2, 9)
    with pytest.raises(ValueError, match="q_start: expected 3"):
        pq.pq_paged_attention(f16(3, 4, 64), Fake, i32(2, 4), i32(2), i32(2), 2, 9)
    with pytest.raises(ValueError, match="block_table: expected"):
        pq.pq_paged_attention(f16(3, 4, 64), Fake, i32(3, 4), i32(3), i32(2), 2, 9)
    with pytest.raises(ValueError, match="out: expected"):
        pq.pq_paged_attention(f16(3, 4, 64), Fake, i32(2, 4), i32(3), i32(2), 2, 9, out=f16(3, 4, 63))
    with pytest.raises(ValueError, match="CUDA"):
        pq.pq_paged_attention(f16(3, 4, 64), Fake, i32(2, 4), i32(3), i32(2), 2, 9)


def test_the_plain_attention_is_the_softmax_by_hand():
    """The reference itself, on a case small enough to write out: two keys of scores 0 and ln 3."""
    d = ref.attention_inputs(1, 1, 64, 16, "f16", [2], [2], seed=1)
    i = d["table"][0, 0]
    d["q"][:] = 0
    d["q"][:, 0, 0] = 1
    d["k"][i, 0, :2] = 0
    d["k"][i, 0, 1, 0] = 1
    d["v"][i, 0, 0], d["v"][i, 0, 1] = 4, 8
    y, _ = ref.attention(d, scale=np.log(3.0))
    assert np.allclose(y[0, 0], 4) and np.allclose(y[1, 0], (4 + 3 * 8) / 4)


def test_the_plain_block_tables_by_hand():
    table, q_start, total, slots, pos, head = ref.block_tables(
        np.array([15, 0]), np.array([2, 1]), np.array([[9, -1], [-1, -1]], np.int32), np.array([5, 6, 7]), 1, 16, 4)
    assert table.tolist() == [[9, 6], [7, -1]] and q_start.tolist() == [0, 2, 3] and total.tolist() == [17, 1]
    assert slots.tolist() == [9 * 16 + 15, 6 * 16, 7 * 16, -1] and pos.tolist() == [15, 16, 0, -1] and head == 3


def test_workspace_query_takes_bounds_of_any_size():
    size = pq.pq_attention_workspace_bytes
    assert size(1, 300, 300, 8192, 32, 8, 128) > 65536
    for max_q in (301, 2**31, 2**61, 2**62, 2**63 - 1):         # no request has more rows than the step
        assert size(1, 300, max_q, 8192, 32, 8, 128) == size(1, 300, 300, 8192, 32, 8, 128)
    for max_kv in (2**31 - 1, 2**40, 2**63 - 1):
        assert size(1, 300, 300, max_kv, 32, 8, 128) == size(1, 300, 300, 2**30, 32, 8, 128)
    assert size(1, 2**31, 300, 8192, 32, 8, 128) == 0


def test_workspace_query_refuses_what_the_call_refuses():
    size = pq.pq_attention_workspace_bytes
    assert size(1, 100, 100, 9000, 64, 1, 64) > 0
    for heads, kv_heads in ((65, 1), (129, 1), (100000, 1), (4096, 2048), (3, 2), (0, 1), (4, 0)):   # groups of 65 and more, ...
        assert size(1, 100, 100, 9000, heads, kv_heads, 64) == 0
    assert size(1, 100, 100, 9000, 8, 2, 80) == 0 and size(4097, 5000, 2, 9000, 8, 2, 64) == 0


def test_workspace_query_knows_the_window():
    size = lambda window: pq.pq_attention_workspace_bytes(1, 300, 300, 4300, 32, 8, 128, window=window)  # noqa: E731
    part = 2 * 128 * (128 + 2) * 4                   # 40 units of 256 rows, in 3 parts without a window, in 4 with this one
    assert size(0) == 65536 + 40 * 3 * part and size(4096) == 65536 + 40 * 4 * part
    assert size(1) == 0 and size(2**31 - 1) == size(0) and size(-1) == 0
    L = pq.lib()
    assert L.pq_attention_workspace_bytes(1, 300, 300, 4300, 32, 8, 128, 148) == size(0)


def test_workspace_query_leaves_out_the_kernel_that_a_call_does_not_use():
    """More than 16 query heads per key/value head: every request is the tile kernel's, whose parts are of one size."""
    part = 2 * 128 * (64 + 2) * 4
    for heads in (17, 32, 64):
        for max_kv in (300, 1000, 200_000):
            n = pq.pq_attention_workspace_bytes(3, 3, 1, max_kv, heads, 1, 64)
            assert n == 0 or (n - 65536) % (3 * part) == 0
    assert (pq.pq_attention_workspace_bytes(3, 3, 1, 1000, 16, 1, 64) - 65536) % (16 * (64 + 2) * 4) == 0


def test_sizes_beyond_32_bits_are_refused_not_cut():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    Fake = types.SimpleNamespace(heads=2, dim=64, page=16, pages=4, device=-1, _ref=0)
    q = torch.zeros((3, 4, 64), dtype=torch.float16)
    for window in (2**32 + 5, 2**31, -2**31 - 1):
        with pytest.raises(ValueError, match="window: .* 32 bits"):
            pq.pq_paged_attention(q, Fake, i32(2, 4), i32(3), i32(2), 2, 9, window=window)
        with pytest.raises(ValueError, match="window: .* 32 bits"):
            pq.pq_attention_workspace_bytes(1, 300, 300, 4300, 32, 8, 128, window=window)
    with pytest.raises(ValueError, match="page: .* 32 bits"):
        pq.pq_block_tables(i32(2), i32(2), i32(2, 4), i32(5), i32(1), 2**32 + 16, 3)
    with pytest.raises(ValueError, match="heads: .* 32 bits"):
        pq.pq_attention_workspace_bytes(1, 300, 300, 4300, 2**32 + 32, 8, 128)
