"""Attention over the paged cache against the plain 64-bit form, with everything that must not be read poisoned."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _t(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _run(d, workspace=True, wide=False, scale=None, max_kv=None):
    cache = pq.PagedKV(_t(d["k"]), _t(d["v"]), _t(d["ks"]), _t(d["vs"]))
    q = _t(d["q"])
    T, heads, dim = q.shape
    if wide:     # rows of a wider matrix
        q = torch.cat([q.view(T, -1), torch.full((T, 24), float("nan"), dtype=torch.float16, device=DEV)], 1)[:, : heads * dim]
    n = np.diff(d["q_start"])
    max_q, max_kv = int(n.max(initial=0)), int(d["kv_len"].max(initial=0)) if max_kv is None else max_kv
    ws = pq.pq_attention_workspace(q, cache, len(n), max_q, max_kv) if workspace else None
    out = torch.full((T, heads, dim), float("nan"), dtype=torch.float16, device=DEV)
    pq.pq_paged_attention(q, cache, _t(d["table"]), _t(d["q_start"]), _t(d["kv_len"]), max_q, max_kv, scale=scale,
                          window=d["window"], out=out, workspace=ws)
    assert pq.pq_device_status() == 0
    return out


def _check(d, **more):
    y, bound = ref.attention(d, scale=more.get("scale"))
    got = _run(d, **more).cpu().numpy().astype(np.float64)
    off = np.abs(got - y)
    assert np.isfinite(got).all(), f"{np.argwhere(~np.isfinite(got))[:4]}"
    bad = np.argwhere(off > bound)
    assert len(bad) == 0, f"{len(bad)} values off, first {bad[:4].tolist()}: {off[tuple(bad[0])]} > {bound[tuple(bad[0])]}"


HEADS = [(32, 8, 128), (4, 4, 64), (7, 1, 128), (6, 2, 64), (16, 1, 128), (40, 1, 64), (64, 1, 128)]


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("page,total", [(16, [1, 2, 15, 16, 17, 33]), (48, [47, 48, 49, 500]), (64, [64, 1000, 3]),
                                        (1024, [130, 1025])])
def test_one_token_per_request(heads, kv_heads, dim, page, total, cache):
    _check(ref.attention_inputs(heads, kv_heads, dim, page, cache, [1] * len(total), total, seed=page + heads))


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS[:5])
@pytest.mark.parametrize("page,new,cached", [
    (16, [2, 5, 3], [0, 100, 31]), (32, [9, 1, 16, 4], [7, 640, 0, 255]), (16, [17, 40, 1], [500, 3, 77]),
    (64, [130, 1, 257], [0, 300, 129]), (128, [128, 127, 129], [128, 1, 0]), (48, [300], [211])])
def test_chunks(heads, kv_heads, dim, page, new, cached, cache):
    total = [n + c for n, c in zip(new, cached)]
    _check(ref.attention_inputs(heads, kv_heads, dim, page, cache, new, total, seed=page + sum(new)), wide=True)


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window", [1, 16, 100, 128, 1000])
def test_sliding_window_reads_no_page_before_it(window, dim, cache):
    new, total = [1, 5, 140, 260], [700, 333, 400, 260]
    _check(ref.attention_inputs(8, 2, dim, 16, cache, new, total, window=window, seed=window))
    _check(ref.attention_inputs(8, 2, dim, 64, cache, [1, 1, 2], [130, 129, 1], window=window, seed=window + 1))


@pytest.mark.parametrize("cache", ["f16", "int8"])
def test_rows_without_a_key_give_zero(cache):
    # requests of no rows, of no keys, and shorter than their own chunk (the first rows stand before the first key)
    for new, total in (([1, 0, 3, 2], [0, 5, 1, 2]), ([200, 1, 150], [40, 9, 0])):
        d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=3)
        _check(d)
        out = _run(d).cpu().numpy()
        t = d["q_start"][2] if new[2] == 150 else 0
        assert (out[t] == 0).all()


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("heads,kv_heads,dim,new,total", [
    (4, 1, 128, [1], [5000]), (8, 8, 64, [1, 1], [4097, 12]), (32, 8, 128, [1], [999]), (16, 1, 128, [3], [9001]),
    (8, 2, 128, [70], [6000]), (4, 1, 64, [300, 2], [4000, 2500])])
def test_keys_split_over_the_machine(heads, kv_heads, dim, new, total, cache):
    d = ref.attention_inputs(heads, kv_heads, dim, 16, cache, new, total, seed=sum(total))
    _check(d)                      # with a workspace
    _check(d, workspace=False)
    _check(d, max_kv=1)            # a hint that is too small costs speed only
    a, b = _run(d), _run(d)
    assert torch.equal(a, b)       # parts are joined in a fixed order


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("new", [[1, 1, 1], [150, 3, 20]])
def test_scores_of_every_size(new, cache):
    total = [400, 300, 129]
    d = ref.attention_inputs(8, 2, 128, 32, cache, new, total, seed=11, spread=3.0)   # one key takes most of the weight
    _check(d)
    _check(d, scale=0.0)           # all keys alike
    _check(d, scale=-0.05)
    # a maximum that keeps growing along the keys, far beyond the first tile's
    d = ref.attention_inputs(8, 2, 128, 32, cache, new, total, seed=12)
    if cache == "f16":
        d["q"][:] = np.float16(0.25)
        for b, length in enumerate(total):
            for j in range(length):
                d["k"][d["table"][b, j // 32], :, j % 32] = np.float16(j / 32)
    else:
        d["q"][:] = np.float16(0.25)
        for b, length in enumerate(total):
            for j in range(length):
                i = d["table"][b, j // 32]
                d["k"][i, :, j % 32], d["ks"][i, :, j % 32] = 100, np.float32(j / 3200)
    _check(d)
    _check(d, scale=-0.088)        # ... and one that is largest at the first key


@pytest.mark.parametrize("cache", ["f16", "int8"])
def test_values_of_very_different_size(cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, [1, 3, 200], [300, 500, 333], seed=21)
    if cache == "f16":
        small = (d["k"][..., :1] > 0)
        d["v"] = np.where(small, d["v"] * np.float16(2.0 ** -10), d["v"] * np.float16(256)).astype(np.float16)
    else:
        rng = np.random.default_rng(2)
        d["vs"] = (d["vs"] * 2.0 ** rng.integers(-12, 12, d["vs"].shape)).astype(np.float32)
    _check(d)


@pytest.mark.parametrize("cache", ["f16", "int8"])
def test_pages_outside_the_cache_read_as_zeros_and_short_tables_end_the_keys(cache):
    lost = [(0, 0), (0, 2), (1, 1), (2, 4), (2, 9)]
    _check(ref.attention_inputs(8, 2, 128, 16, cache, [1, 4, 150], [60, 100, 200], seed=31, lost=lost))
    d = ref.attention_inputs(8, 2, 128, 16, cache, [1, 4, 150], [60, 100, 200], seed=32)
    d["table"] = np.ascontiguousarray(d["table"][:, :5])       # 80 keys of each at most
    _check(d)


def test_rows_outside_every_request_are_left_as_they_are():
    for new in ([2, 1], [140, 20]):
        d = ref.attention_inputs(8, 2, 128, 16, "f16", new, [50, 30] if new[0] == 2 else [150, 30], seed=41)
        n = sum(new)
        d["q"] = np.concatenate([np.full((3, 8, 128), np.nan, np.float16), d["q"], np.full((5, 8, 128), np.nan, np.float16)])
        d["q_start"] = d["q_start"] + 3
        out = _run(d).cpu().numpy()
        assert np.isnan(out[:3]).all() and np.isnan(out[3 + n:]).all()
        y, bound = ref.attention(d)
        assert (np.abs(out[3: 3 + n] - y[3: 3 + n]) <= bound[3: 3 + n]).all()


@pytest.mark.parametrize("cache", ["f16", "int8"])
def test_on_a_side_stream_and_captured_in_a_graph(cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, [1, 1, 90], [700, 31, 400], seed=51)
    y, bound = ref.attention(d)
    cachet = pq.PagedKV(_t(d["k"]), _t(d["v"]), _t(d["ks"]), _t(d["vs"]))
    q, table, qs, kl = _t(d["q"]), _t(d["table"]), _t(d["q_start"]), _t(d["kv_len"])
    ws = pq.pq_attention_workspace(q, cachet, 3, 90, 700)
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pq.pq_paged_attention(q, cachet, table, qs, kl, 90, 700, out=out, workspace=ws)
    side.synchronize()
    first = out.cpu().numpy()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pq.pq_paged_attention(q, cachet, table, qs, kl, 90, 700, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), first)
    assert (np.abs(first - y) <= bound).all()


def test_offsets_beyond_32_bits():
    pages, heads, page, dim = 140_000, 8, 16, 128       # 2.3e9 values per tensor
    d = ref.attention_inputs(16, heads, dim, page, "f16", [1, 130], [100, 130], seed=61)
    used = d["k"].shape[0]
    k, v = (torch.zeros((pages, heads, page, dim), dtype=torch.float16, device=DEV) for _ in "kv")
    move = np.arange(used) + pages - used               # the pages at the very end of the cache
    k[move[0]:], v[move[0]:] = _t(d["k"]), _t(d["v"])
    table = np.where((d["table"] >= 0) & (d["table"] < used), d["table"] + pages - used, d["table"]).astype(np.int32)
    out = pq.pq_paged_attention(_t(d["q"]), pq.PagedKV(k, v), _t(table), _t(d["q_start"]), _t(d["kv_len"]), 130, 130)
    y, bound = ref.attention(d)
    assert (np.abs(out.cpu().numpy() - y) <= bound).all()


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("heads,kv_heads,dim,new,total,window", [
    (32, 8, 64, [1220], [2720], 0),                  # 160 units, the last 12 in parts
    (16, 8, 64, [1250, 3, 1190], [1700, 900, 2500], 0),
    (32, 8, 64, [1220], [2720], 1300)])
def test_units_of_the_last_wave_in_parts(heads, kv_heads, dim, new, total, window, cache):
    d = ref.attention_inputs(heads, kv_heads, dim, 32, cache, new, total, window=window, seed=sum(total))
    _check(d)
    _check(d, workspace=False)                       # every unit whole


def test_a_workspace_too_small_for_all_parts_still_serves():
    d = ref.attention_inputs(8, 2, 128, 16, "f16", [70], [6000], seed=77)
    y, bound = ref.attention(d)
    cache = pq.PagedKV(_t(d["k"]), _t(d["v"]))
    q, table, qs, kl = _t(d["q"]), _t(d["table"]), _t(d["q_start"]), _t(d["kv_len"])
    full = pq.pq_attention_workspace(q, cache, 1, 70, 6000)
    for share in (2, 5, 50):
        ws = full[: 65536 + (full.numel() - 65536) // share]
        out = pq.pq_paged_attention(q, cache, table, qs, kl, 70, 6000, workspace=ws)
        assert (np.abs(out.cpu().numpy() - y) <= bound).all()
        assert pq.pq_device_status() == 0


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("new,total", [([5, 1], [90, 33]), ([40, 3], [40, 17]), ([300], [400])])
def test_a_key_that_is_not_a_number_reaches_only_the_rows_that_see_it(new, total, cache):
    d = ref.attention_inputs(8, 2, 128, 16, cache, new, total, seed=sum(total) + 1)
    y, bound = ref.attention(d)
    at = total[0] - 1                                # the first request's newest key
    page, off = d["table"][0][at // 16], at % 16
    if cache == "f16":
        d["k"][page, :, off] = np.nan
    else:
        d["ks"][page, :, off] = np.nan
    got = _run(d).cpu().numpy().astype(np.float64)
    hit = new[0] - 1
    assert np.isnan(got[hit]).all()
    rest = np.arange(sum(new)) != hit
    assert (np.abs(got - y)[rest] <= bound[rest]).all()
