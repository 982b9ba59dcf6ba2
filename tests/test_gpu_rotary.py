"""Rotary positions by themselves and on the way into the paged caches, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paged_reference as paged
import paper_2512_23367_b200 as pq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALED = {"none": {}, "bands": dict(factor=16.0, original=4096.0), "waves": dict(factor=8.0, original=8192.0, low=1.0, high=4.0)}


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _rand(rng, *shape):
    return rng.standard_normal(shape).astype(np.float16)


def _rotary(dim, layout, scaling="none", base=10000.0, **more):
    return pq.Rotary(dim, base, layout, scaling, device=DEV, **SCALED[scaling], **more), ref.frequencies(dim, base, scaling, **SCALED[scaling])


def _close(got, want, x, dim, amplitude):
    return (np.abs(got.astype(np.float64) - want) <= ref.rotation_bound(x, dim, amplitude)).all()


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("scaling", list(SCALED))
@pytest.mark.parametrize("T,heads,width,dim", [(1, 40, 128, 128), (3, 1, 16, 16), (65, 5, 96, 32), (300, 7, 192, 192), (2, 3, 256, 256), (1000, 33, 64, 48),
                                               (4099, 16, 128, 64)])
def test_rotate(T, heads, width, dim, scaling, layout):
    rng = np.random.default_rng(T + dim)
    rot, (freq, amp) = _rotary(dim, layout, scaling)
    x, pos = _rand(rng, T, heads, width), rng.integers(0, 200000, T).astype(np.int32)
    got = pq.pq_rotate(_t(x), _t(pos), rot).cpu().numpy()
    assert _close(got, ref.rotate(x, pos, freq, layout, amp), x, dim, amp)
    assert np.array_equal(got[..., dim:], x[..., dim:])


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_positions_of_any_size(layout):
    """The angle is exact modulo a turn wherever the position lies; in FP32 radians it would be off by up to 256."""
    rng = np.random.default_rng(5)
    rot, _ = _rotary(64, layout)
    pos = np.array([0, 1, 2**20 + 1, 2**24 + 1, 2**31 - 1, -1, -2**31], np.int32)
    x = _rand(rng, len(pos), 2, 64)
    # exact turns from the integers themselves, as 64-bit fractions
    freq = rot.freq.cpu().numpy().view(np.uint64)
    turns = np.array([[((int(p) * int(f)) % 2**64) / 2.0**64 for f in freq] for p in pos])
    got = pq.pq_rotate(_t(x), _t(pos), rot).cpu().numpy()
    want = np.concatenate([ref.rotate(x[i: i + 1], np.array([1.0]), 2 * np.pi * turns[i], layout) for i in range(len(pos))])
    assert _close(got, want, x, 64, 1.0)


def test_slices_in_place_and_out_of_place():
    """The end of every head of a wider matrix turned into the end of another's heads; in place; amplitude."""
    rng = np.random.default_rng(7)
    rot, (freq, _) = _rotary(64, "pairs", amplitude=0.5)
    T, heads = 37, 6
    x, pos = _rand(rng, T, heads, 192), np.arange(T, dtype=np.int32) * 911
    want = ref.rotate(x[..., 128:], pos, freq, "pairs", 0.5)
    wide, out = _t(x), torch.full((T, heads, 576), 7.0, dtype=torch.float16, device=DEV)
    pq.pq_rotate(wide[..., 128:], _t(pos), rot, out=out[..., 512:])
    assert _close(out[..., 512:].cpu().numpy(), want, x[..., 128:], 64, 0.5) and (out[..., :512] == 7).all()
    assert np.array_equal(wide.cpu().numpy(), x)
    pq.pq_rotate(wide[..., 128:], _t(pos), rot, out=wide[..., 128:])
    assert torch.equal(wide[..., 128:], out[..., 512:]) and np.array_equal(wide[..., :128].cpu().numpy(), x[..., :128])
    # heads first: rows of one head lie together
    first = _t(x.transpose(1, 0, 2))
    got = pq.pq_rotate(first.transpose(0, 1)[..., 128:], _t(pos), rot)
    assert torch.equal(got, out[..., 512:])


@pytest.mark.parametrize("cache", ["f16", "int8"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,heads,kv_heads,width,dim,page", [(1, 8, 2, 128, 128, 16), (70, 32, 8, 128, 64, 48), (333, 5, 5, 64, 64, 16), (3, 0, 3, 64, 32, 64),
                                                             (2500, 4, 1, 128, 128, 32)])
def test_append_rotated(T, heads, kv_heads, width, dim, page, layout, cache):
    rng = np.random.default_rng(T + heads)
    rot, (freq, amp) = _rotary(dim, layout, "bands")
    qkv, pos = _rand(rng, T, heads + 2 * kv_heads, width), rng.integers(0, 100000, T).astype(np.int32)
    pages = -(-T // page) + 2
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    skipped = rng.random(T) < 0.1
    slots[skipped] = np.where(rng.random(skipped.sum()) < 0.5, -1, pages * page)
    kv = pq.PagedKV.empty(pages, kv_heads, page, width, torch.float16 if cache == "f16" else torch.int8, DEV)
    x = _t(qkv)
    q, k, v = x[:, :heads], x[:, heads: heads + kv_heads], x[:, heads + kv_heads:]
    got = pq.pq_kv_append_rotated(kv, k, v, _t(slots), _t(pos), rot, **({"q": q} if heads else {}))
    assert np.array_equal(x.cpu().numpy(), qkv)
    if heads:
        assert _close(got.cpu().numpy(), ref.rotate(qkv[:, :heads], pos, freq, layout, amp), qkv[:, :heads], dim, amp)
    turned = ref.rotate(qkv[:, heads: heads + kv_heads], pos, freq, layout, amp)
    kk, vv = (t.cpu().numpy() for t in pq.pq_kv_read(kv, _t(slots)))
    values = qkv[:, heads + kv_heads:]
    assert not kk[skipped].any() and not vv[skipped].any()
    if cache == "f16":
        assert _close(kk[~skipped], turned[~skipped], qkv[~skipped, heads: heads + kv_heads], dim, amp)
        assert np.array_equal(vv[~skipped], values[~skipped])
        untouched = np.ones(pages * page, bool)
        untouched[slots[~skipped]] = False
        assert not kv.k.transpose(1, 2).reshape(pages * page, -1).cpu().numpy()[untouched].any()
        return
    # the value is within half a step of the code, one code's rounding of the FP32 rotation, and the FP16 of the read-back
    for got8, want in ((kk, turned), (vv, values.astype(np.float64))):
        step = np.abs(want).max(-1, keepdims=True) / 127.5
        # 127.5 / 127.5 rounds to 128, which the codes' range holds only below zero: there the error is a whole half step of 127.5
        bound = step * (0.5 + 1e-3) + np.abs(want) * 2.0 ** -11 + 2.0 ** -25 + 8 * 2.0 ** -24 * step * 255
        assert (np.abs(got8 - want)[~skipped] <= bound[~skipped]).all()
    codes, scales = paged.quantize(values)                   # values are not turned: bit for bit as pq_kv_append
    at, off = slots[~skipped] // page, slots[~skipped] % page
    assert np.array_equal(kv.v.cpu().numpy()[at, :, off], codes[~skipped]) and np.array_equal(kv.v_scale.cpu().numpy()[at, :, off], scales[~skipped])


def test_append_rotated_by_nothing_is_append():
    """Position 0 turns nothing: codes, scales and FP16 values are pq_kv_append's, bit for bit, zero vectors too."""
    rng = np.random.default_rng(11)
    k, v = _rand(rng, 50, 4, 128), _rand(rng, 50, 4, 128)
    k[3], v[4] = 0, 0
    rot, _ = _rotary(128, "half")
    slots = _t(rng.permutation(64)[:50].astype(np.int64))
    for dtype in (torch.float16, torch.int8):
        a, b = (pq.PagedKV.empty(4, 4, 16, 128, dtype, DEV) for _ in range(2))
        pq.pq_kv_append(a, _t(k), _t(v), slots)
        pq.pq_kv_append_rotated(b, _t(k), _t(v), slots, torch.zeros(50, dtype=torch.int32, device=DEV), rot)
        assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
        if dtype == torch.int8:
            assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)


@pytest.mark.parametrize("latent,heads,T,page", [(512, 16, 1, 16), (512, 3, 100, 48), (256, 0, 7, 64), (256, 20, 1500, 32)])
def test_latent_append_and_read(latent, heads, T, page):
    rng = np.random.default_rng(T)
    rot, (freq, amp) = _rotary(64, "pairs", "waves")
    both, q, pos = _rand(rng, T, latent + 64), _rand(rng, T, max(heads, 1), 192), rng.integers(0, 60000, T).astype(np.int32)
    pages = -(-T // page) + 1
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    skip = np.zeros(T, bool)
    if T > 1:
        skip[T // 2] = True
        slots[skip] = -7
    cache = pq.LatentKV.empty(pages, page, latent, DEV)
    cache.data.fill_(3.0)
    x, qd = _t(both), _t(q)
    out = torch.zeros((T, heads, latent + 64), dtype=torch.float16, device=DEV)[..., latent:] if heads else None
    got = pq.pq_latent_append(cache, x[:, :latent], x[:, latent:], _t(slots), _t(pos), rot, **({"q": qd[..., 128:], "out": out} if heads else {}))
    if heads:
        assert got is out and _close(out.cpu().numpy(), ref.rotate(q[..., 128:], pos, freq, "pairs", amp), q[..., 128:], 64, amp)
    want = ref.rotate(both[:, None, latent:], pos, freq, "pairs", amp)[:, 0]
    flat = cache.data.view(pages * page, -1).cpu().numpy()
    assert np.array_equal(flat[slots[~skip], :latent], both[~skip, :latent]) and _close(flat[slots[~skip], latent:], want[~skip], both[~skip, latent:], 64, amp)
    rest = np.setdiff1d(np.arange(pages * page), slots[~skip])
    assert (flat[rest] == 3).all()
    c, k = (t.cpu().numpy() for t in pq.pq_latent_read(cache, _t(slots)))
    assert np.array_equal(c[~skip], flat[slots[~skip], :latent]) and np.array_equal(k[~skip], flat[slots[~skip], latent:]) and not c[skip].any() and not k[skip].any()


def test_no_rows_and_other_streams():
    rot, _ = _rotary(64, "half")
    empty = torch.empty((0, 4, 64), dtype=torch.float16, device=DEV)
    assert pq.pq_rotate(empty, torch.empty(0, dtype=torch.int32, device=DEV), rot).shape == (0, 4, 64)
    x, pos = torch.randn((2000, 8, 64), device=DEV).half(), torch.arange(2000, dtype=torch.int32, device=DEV)
    good = pq.pq_rotate(x, pos, rot)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = pq.pq_rotate(x, pos, rot)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(good, other)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(x)
    with torch.cuda.graph(graph):
        pq.pq_rotate(x, pos, rot, out=out)
    x.neg_()
    graph.replay()
    assert torch.equal(out, -good)
