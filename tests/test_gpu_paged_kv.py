"""Block tables, slot map, cache append and read-back against their plain forms: whole numbers and codes bit for bit."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _tables_case(requests, page, new_max, cached_max, seed, spare=8, narrow=0):
    rng = np.random.default_rng(seed)
    kv = rng.integers(0, cached_max + 1, requests).astype(np.int32)
    new = rng.integers(0, new_max + 1, requests).astype(np.int32)
    have, want = -(-kv // page), -(-(kv + new) // page)
    width = max(int(want.max(initial=1)) - narrow, 1)
    pages = int(want.sum()) + spare
    order = rng.permutation(max(pages, 1)).astype(np.int32)
    table = rng.integers(-3, 1 << 20, (requests, width)).astype(np.int32)
    at = 0
    for b in range(requests):
        m = min(int(have[b]), width)
        table[b, :m] = order[at:at + m]
        at += m
    return kv, new, table, order[: max(pages + min(spare, 0), 0)], at


def _check_tables(kv, new, table, free, head, page, tokens, step=None):
    want = ref.block_tables(kv, new, table, free, head, page, tokens)
    dev_table = _t(table)
    step = pq.pq_block_tables(_t(kv), _t(new), dev_table, _t(free), _t(np.array([head], np.int32)), page, tokens, step=step)
    got = (dev_table, step.q_start, step.kv_len, step.slots, step.pos, step.free_head)
    for g, w, name in zip(got, want, ("table", "q_start", "kv_len", "slots", "pos", "free_head")):
        assert np.array_equal(g.cpu().numpy().ravel(), np.asarray(w).ravel()), name


@pytest.mark.parametrize("requests,page,new_max,cached_max", [
    (1, 16, 1, 0), (1, 16, 0, 5), (3, 16, 33, 40), (8, 64, 1, 3000), (255, 48, 3, 500), (256, 16, 2, 100), (257, 32, 5, 70),
    (1000, 16, 40, 300), (4096, 128, 3, 900), (7, 1024, 3000, 2000), (64, 16, 700, 10)])
def test_block_tables(requests, page, new_max, cached_max):
    kv, new, table, free, head = _tables_case(requests, page, new_max, cached_max, requests + page)
    for extra in (0, 37):      # rows beyond the step's own
        _check_tables(kv, new, table, free, head, page, int(new.sum()) + extra)


def test_block_tables_without_requests_or_tokens():
    none = np.zeros(0, np.int32)
    _check_tables(none, none, np.zeros((0, 3), np.int32), np.arange(4, dtype=np.int32), 2, 16, 5)
    _check_tables(none, none, np.zeros((0, 3), np.int32), none, 0, 16, 0)
    kv = np.array([0, 17, 64], np.int32)
    _check_tables(kv, np.zeros(3, np.int32), np.full((3, 4), 7, np.int32), np.arange(9, dtype=np.int32), 1, 16, 0)


def test_block_tables_when_pages_or_columns_or_rows_run_out():
    kv, new, table, free, head = _tables_case(20, 16, 50, 60, 5, spare=-7)         # the free list is 7 pages short
    _check_tables(kv, new, table, free, head, 16, int(new.sum()))
    kv, new, table, free, head = _tables_case(20, 16, 50, 60, 6, narrow=2)         # tables two columns too narrow
    _check_tables(kv, new, table, free, head, 16, int(new.sum()))
    kv, new, table, free, head = _tables_case(20, 16, 50, 60, 7)                   # fewer rows than new tokens
    _check_tables(kv, new, table, free, head, 16, int(new.sum()) - 21)
    kv, new, table, free, head = _tables_case(20, 16, 50, 60, 8)                   # negative lengths count as 0
    kv[3], new[4], new[5] = -9, -1, -1000
    _check_tables(kv, new, table, free, head, 16, int(np.maximum(new, 0).sum()))


def test_block_tables_fills_the_buffers_it_is_given():
    kv, new, table, free, head = _tables_case(12, 16, 9, 90, 9)
    step = pq.PagedStep.empty(12, int(new.sum()), DEV)
    for _ in range(2):
        _check_tables(kv, new, table, free, head, 16, None or int(new.sum()), step=step)


def _slots(rng, tokens, pages, page, skip=True):
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    if skip and tokens > 2:
        slots[1], slots[tokens // 2] = -1, pages * page      # skipped rows
    return slots


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("tokens,heads,dim,page,wide", [
    (1, 1, 64, 16, False), (3, 1, 128, 16, True), (5, 5, 64, 48, False), (64, 8, 128, 16, True), (33, 7, 128, 32, False),
    (130, 32, 128, 64, True), (17, 40, 64, 16, False), (300, 2, 64, 1024, True)])
def test_append_and_read(cache, tokens, heads, dim, page, wide):
    rng = np.random.default_rng(tokens + heads)
    pages = -(-tokens // page) + 2
    slots = _slots(rng, tokens, pages, page)
    k, v = (rng.standard_normal((tokens, heads, dim)).astype(np.float16) for _ in range(2))
    k[0, 0] = 0                                   # a vector of zeros: scale 0, codes 0
    v[-1, -1, :] = np.float16(-3.0)               # every value the minimum: code -128
    shape = (pages, heads, page, dim)
    if cache == "f16":
        kv = pq.PagedKV(*(_t(np.full(shape, 7, np.float16)) for _ in "kv"))
    else:
        kv = pq.PagedKV(*(_t(np.full(shape, 7, np.int8)) for _ in "kv"), *(_t(np.full(shape[:3], 9, np.float32)) for _ in "kv"))
    if wide:   # slices of one wide matrix, as a fused q/k/v linear leaves them
        both = _t(np.concatenate([np.ones((tokens, 8), np.float16), k.reshape(tokens, -1), v.reshape(tokens, -1)], 1))
        tk, tv = both[:, 8: 8 + heads * dim], both[:, 8 + heads * dim:]
    else:
        tk, tv = _t(k), _t(v)
    pq.pq_kv_append(kv, tk, tv, _t(slots))
    live = (slots >= 0) & (slots < pages * page)
    at, off = slots[live] // page, slots[live] % page
    read = pq.pq_kv_read(kv, _t(slots))
    for x, got, got_scale, back in ((k, kv.k, kv.k_scale, read[0]), (v, kv.v, kv.v_scale, read[1])):
        if cache == "f16":
            want = np.full(shape, 7, np.float16)
            want[at, :, off] = x[live]
            values = x
        else:
            codes, scales = ref.quantize(x)
            want, want_scale = np.full(shape, 7, np.int8), np.full(shape[:3], 9, np.float32)
            want[at, :, off], want_scale[at, :, off] = codes[live], scales[live]
            assert np.array_equal(got_scale.cpu().numpy(), want_scale)
            values = (codes.astype(np.float32) * scales[..., None]).astype(np.float16)
        assert np.array_equal(got.cpu().numpy(), want)
        assert np.array_equal(back.cpu().numpy(), np.where(live[:, None, None], values, np.float16(0)))


def test_append_codes_are_those_of_the_activation_quantizer():
    x = torch.randn((50, 1, 128), dtype=torch.float16, device=DEV)
    kv = pq.PagedKV.empty(4, 1, 16, 128, torch.int8, DEV)
    pq.pq_kv_append(kv, x, x, torch.arange(50, device=DEV))
    q, s = pq.pq_quantize_act(x.view(50, 128))
    assert torch.equal(kv.k.view(-1, 128)[:50], q) and torch.equal(kv.v_scale.view(-1)[:50], s)


def test_append_of_no_tokens_and_beyond_32_bit_offsets():
    kv = pq.PagedKV.empty(2, 1, 16, 64, torch.float16, DEV)
    none = torch.empty((0, 1, 64), dtype=torch.float16, device=DEV)
    pq.pq_kv_append(kv, none, none, torch.empty((0,), dtype=torch.int64, device=DEV))
    assert pq.pq_kv_read(kv, torch.empty((0,), dtype=torch.int64, device=DEV))[0].shape == (0, 1, 64)
    pages, heads, page, dim = 140_000, 8, 16, 128       # 2.3e9 values per tensor
    big = pq.PagedKV(*(torch.empty((pages, heads, page, dim), dtype=torch.int8, device=DEV) for _ in "kv"),
                     *(torch.empty((pages, heads, page), dtype=torch.float32, device=DEV) for _ in "kv"))
    x = torch.randn((2, heads, dim), dtype=torch.float16, device=DEV)
    slots = torch.tensor([pages * page - 1, 131_072 * page + 5], device=DEV)
    pq.pq_kv_append(big, x, -x, slots)
    codes, scales = ref.quantize(x.cpu().numpy())
    for i, s in enumerate(slots.tolist()):
        assert np.array_equal(big.k[s // page, :, s % page].cpu().numpy(), codes[i])
        assert np.array_equal(big.v_scale[s // page, :, s % page].cpu().numpy(), scales[i])
    back = pq.pq_kv_read(big, slots)[0]
    assert np.array_equal(back.cpu().numpy(), (codes.astype(np.float32) * scales[..., None]).astype(np.float16))
