"""Refusals of the rotary and latent calls, and what of them runs without a GPU."""
import ctypes
import types

import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2512_23367_b200 as pq
from paper_2512_23367_b200 import binding

NULL, SHAPE, ALIGN, LIMIT = 1, 2, 3, 7
_KEEP = []    # the structs whose addresses the calls below are given


def _kept(struct, **fields):
    _KEEP.append(struct(**fields))
    return ctypes.addressof(_KEEP[-1])


def _rotary(**change):
    return _kept(binding._Rotary, **(dict(freq=16, dim=64, layout=0, amplitude=1.0) | change))


def _kv(**change):
    return _kept(binding._KVCache, **(dict(k=16, v=16, k_scale=None, v_scale=None, pages=4, heads=2, page=16, dim=64, type=0) | change))


def _latent(**change):
    return _kept(binding._LatentCache, **(dict(data=16, pages=4, page=16, latent=512) | change))


@pytest.mark.parametrize("dim", [16, 64, 128, 256])
@pytest.mark.parametrize("scaling,args", [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                          ("bands", dict(factor=16.0, original=4096.0, low=1.0, high=32.0)),
                                          ("waves", dict(factor=8.0, original=8192.0, low=1.0, high=4.0))])
def test_frequencies_are_the_formulas(dim, scaling, args):
    """Turns in units of 2^-64: off by the 2^-62 turn that a double holds of them, and by 64-bit roundings of the formula."""
    freq, amplitude = (ctypes.c_uint64 * (dim // 2))(), ctypes.c_float()
    a = dict(factor=1.0, original=0.0, low=1.0, high=32.0) | args
    assert pq.lib().pq_rotary_frequencies(dim, 500000.0, pq.Rotary.SCALINGS[scaling], a["factor"], a["original"], a["low"], a["high"],
                                          ctypes.addressof(freq), ctypes.addressof(amplitude)) == 0
    want, most = ref.frequencies(dim, 500000.0, scaling, **args)
    got = np.array([int(f) / 2.0 ** 64 for f in freq]) * 2 * np.pi
    assert (np.abs(got - want) <= want * 1e-14 + 2.0 ** -59).all()
    assert amplitude.value == np.float32(most)


def test_frequencies_refuse():
    out, amp = (ctypes.c_uint64 * 128)(), ctypes.c_float()

    def call(dim=64, base=1e4, scaling=0, factor=1.0, original=0.0, low=1.0, high=32.0, freq=ctypes.addressof(out)):
        return pq.lib().pq_rotary_frequencies(dim, base, scaling, factor, original, low, high, freq, ctypes.addressof(amp))

    assert call() == 0 and call(freq=None) == NULL
    assert call(dim=8) == SHAPE and call(dim=24) == SHAPE and call(dim=272) == SHAPE
    assert call(base=1.0) == SHAPE and call(base=float("nan")) == SHAPE and call(base=float("inf")) == SHAPE
    assert call(scaling=5) == SHAPE and call(scaling=-1) == SHAPE
    assert call(scaling=1, factor=0.5) == SHAPE and call(scaling=1, factor=float("nan")) == SHAPE
    assert call(scaling=3, factor=2.0, original=0.0) == SHAPE and call(scaling=4, factor=2.0, original=4096.0, low=4.0, high=4.0) == SHAPE
    assert call(scaling=3, factor=2.0, original=4096.0, low=0.0) == SHAPE


def test_rotate_refuses():
    def call(r=None, x=16, xs=512, xhs=128, heads=4, width=128, pos=16, tokens=3, out=16, os=512, ohs=128):
        return pq.lib().pq_rotate(_rotary() if r is None else r, x, xs, xhs, heads, width, pos, tokens, out, os, ohs, None)

    assert pq.lib().pq_rotate(None, 16, 512, 128, 4, 128, 16, 3, 16, 512, 128, None) == NULL
    assert call(r=_rotary(freq=None)) == NULL and call(r=_rotary(freq=12)) == ALIGN
    assert call(r=_rotary(dim=144)) == SHAPE and call(r=_rotary(dim=40)) == SHAPE and call(r=_rotary(layout=2)) == SHAPE
    assert call(r=_rotary(amplitude=0.0)) == SHAPE and call(r=_rotary(amplitude=float("nan"))) == SHAPE and call(r=_rotary(amplitude=1e6)) == SHAPE
    assert call(width=120) == SHAPE and call(width=1040) == SHAPE and call(heads=0) == SHAPE and call(heads=1025) == SHAPE
    assert call(tokens=-1) == SHAPE and call(tokens=1 << 31) == SHAPE
    assert call(xs=516) == SHAPE and call(xhs=124) == SHAPE and call(xhs=120) == SHAPE and call(xs=-512) == SHAPE
    assert call(os=64) == SHAPE and call(os=0) == SHAPE
    assert call(x=None) == NULL and call(out=None) == NULL and call(pos=None) == NULL and call(x=8) == ALIGN
    assert call(tokens=0, x=None, out=None, pos=None) == 0


def test_appends_refuse():
    def kv(c=None, r=None, k=16, ks=128, v=16, vs=128, slots=16, pos=16, tokens=3, q=16, qs=128, qhs=64, heads=2, out=16, os=128, ohs=64):
        return pq.lib().pq_kv_append_rotated(_kv() if c is None else c, _rotary() if r is None else r, k, ks, v, vs, slots, pos, tokens, q, qs,
                                             qhs, heads, out, os, ohs, None)

    assert kv(c=_kv(dim=96)) == SHAPE and kv(r=_rotary(dim=128)) == SHAPE and kv(ks=120) == SHAPE and kv(vs=132) == SHAPE
    assert kv(heads=-1) == SHAPE and kv(heads=1025) == SHAPE and kv(qhs=56) == SHAPE and kv(os=48) == SHAPE
    assert kv(k=None) == NULL and kv(slots=None) == NULL and kv(pos=None) == NULL and kv(q=None) == NULL and kv(out=None) == NULL
    assert kv(k=8) == ALIGN and kv(q=8) == ALIGN
    assert kv(tokens=0, k=None, v=None, slots=None, pos=None, q=None, out=None) == 0

    def latent(c=None, r=None, v=16, vs=576, k=16, ks=576, slots=16, pos=16, tokens=3, q=16, qs=192, qhs=192, heads=1, out=16, os=64, ohs=64):
        return pq.lib().pq_latent_append(_latent() if c is None else c, _rotary() if r is None else r, v, vs, k, ks, slots, pos, tokens, q, qs, qhs,
                                         heads, out, os, ohs, None)

    assert latent(c=_latent(data=None)) == NULL and latent(c=_latent(latent=384)) == SHAPE and latent(c=_latent(page=24)) == SHAPE
    assert latent(c=_latent(page=2048)) == SHAPE and latent(c=_latent(pages=0)) == SHAPE and latent(c=_latent(pages=1 << 27)) == SHAPE
    assert latent(c=_latent(data=8)) == ALIGN and latent(r=_rotary(dim=128)) == SHAPE
    assert latent(vs=504) == SHAPE and latent(ks=56) == SHAPE and latent(vs=580) == SHAPE and latent(tokens=-1) == SHAPE
    assert latent(v=None) == NULL and latent(k=None) == NULL and latent(slots=None) == NULL and latent(pos=None) == NULL
    assert latent(tokens=0, v=None, k=None, slots=None, pos=None, q=None, out=None) == 0
    assert pq.lib().pq_latent_read(_latent(), None, 1, 16, 16, None) == NULL and pq.lib().pq_latent_read(_latent(), 16, -1, 16, 16, None) == SHAPE
    assert pq.lib().pq_latent_read(_latent(), 16, 1, 8, 16, None) == ALIGN and pq.lib().pq_latent_read(_latent(), None, 0, None, None, None) == 0


def test_head_linear_refuses():
    def call(x=16, xs=512, xhs=128, w=16, heads=4, N=512, K=128, tokens=3, y=16, ys=2048, yhs=512):
        return pq.lib().pq_head_linear(x, xs, xhs, w, heads, N, K, tokens, y, ys, yhs, None)

    assert call(heads=0) == SHAPE and call(heads=1025) == SHAPE and call(N=64) == SHAPE and call(N=192) == SHAPE and call(N=1152) == SHAPE
    assert call(K=32) == SHAPE and call(K=96) == SHAPE and call(K=576) == SHAPE and call(tokens=-1) == SHAPE
    assert call(xhs=120) == SHAPE and call(xs=96) == SHAPE and call(xs=516) == SHAPE and call(yhs=504) == SHAPE and call(ys=0) == SHAPE
    assert call(x=None) == NULL and call(w=None) == NULL and call(y=None) == NULL and call(w=8) == ALIGN
    assert call(tokens=0, x=None, w=None, y=None) == 0


def test_attentions_refuse():
    def latent(q=16, heads=4, c=None, table=16, width=4, qs=16, kl=16, requests=2, tokens=3, scale=0.1, out=16, ws=None, n=0):
        return pq.lib().pq_latent_attention(q, heads, _latent() if c is None else c, table, width, qs, kl, requests, tokens, scale, out, ws, n, None)

    assert latent(c=_latent(latent=128)) == SHAPE and latent(heads=0) == SHAPE and latent(heads=1025) == SHAPE
    assert latent(tokens=1 << 30) == SHAPE and latent(tokens=1 << 62) == SHAPE and latent(tokens=-1) == SHAPE and latent(requests=-1) == SHAPE
    assert latent(width=0) == SHAPE and latent(scale=float("nan")) == SHAPE and latent(requests=4097) == LIMIT
    assert latent(q=None) == NULL and latent(table=None) == NULL and latent(qs=None) == NULL and latent(kl=None) == NULL and latent(out=None) == NULL
    assert latent(q=8) == ALIGN and latent(ws=128, n=1 << 20) == ALIGN
    assert latent(requests=0, q=None, table=None, qs=None, kl=None, out=None) == 0 and latent(tokens=0, q=None, out=None) == 0

    def expanded(q=16, qs=768, heads=4, kv=16, kvs=1024, kr=16, krs=64, keys=9, starts=16, ks=16, requests=2, tokens=3, max_q=2, scale=0.1,
                 out=16, ws=None, n=0):
        return pq.lib().pq_expanded_attention(q, qs, heads, kv, kvs, kr, krs, keys, starts, ks, requests, tokens, max_q, scale, out, ws, n, None)

    assert expanded(heads=0) == SHAPE and expanded(qs=760) == SHAPE and expanded(kvs=1016) == SHAPE and expanded(krs=56) == SHAPE
    assert expanded(qs=772) == SHAPE and expanded(keys=-1) == SHAPE and expanded(keys=1 << 31) == SHAPE and expanded(max_q=-1) == SHAPE
    assert expanded(scale=float("inf")) == SHAPE and expanded(tokens=1 << 40) == SHAPE and expanded(requests=4097) == LIMIT
    assert expanded(q=None) == NULL and expanded(kv=None) == NULL and expanded(kr=None) == NULL and expanded(ks=None) == NULL and expanded(out=None) == NULL
    assert expanded(kv=8) == ALIGN and expanded(ws=128, n=1 << 20) == ALIGN
    assert expanded(requests=0, q=None) == 0 and expanded(tokens=0, q=None) == 0


def test_workspace_holds_two_parts_of_every_multiprocessor():
    size = pq.lib().pq_latent_workspace_bytes
    assert size(0) == 0 and size(-5) == 0
    assert size(148) >= 65536 + 148 * 2 * max(64 * 514, 256 * 130) * 4 and size(148) < 64 << 20


def test_binding_measures_every_operand():
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    i64 = lambda *s: torch.zeros(s, dtype=torch.int64)  # noqa: E731
    with pytest.raises(ValueError, match="layout"):
        pq.Rotary(64, layout="other")
    with pytest.raises(ValueError, match="scaling"):
        pq.Rotary(64, scaling="other")
    with pytest.raises(pq.PQError):
        pq.Rotary(40, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        pq.Rotary(64, device="cpu")
    with pytest.raises(ValueError, match="dim: .* 32 bits"):
        pq.Rotary(2**32 + 64, device="cpu")
    for shape, what in (((4, 16), "3-D"), ((4, 16, 500), "512")):
        with pytest.raises(ValueError, match=what):
            pq.LatentKV(f16(*shape))
    with pytest.raises(ValueError, match="CUDA"):
        pq.LatentKV(f16(4, 16, 576))
    with pytest.raises(TypeError):
        pq.LatentKV(torch.zeros(4, 16, 576))
    rot = types.SimpleNamespace(dim=64, device=-1, freq=i64(32), _ref=0)          # no call gets as far as its memory
    with pytest.raises(ValueError, match="x: expected"):
        pq.pq_rotate(f16(3, 128), i32(3), rot)
    with pytest.raises(ValueError, match="x: expected"):
        pq.pq_rotate(f16(3, 128, 2).transpose(1, 2), i32(3), rot)
    with pytest.raises(ValueError, match="out: expected"):
        pq.pq_rotate(f16(3, 2, 128), i32(3), rot, out=f16(3, 2, 64))
    with pytest.raises(ValueError, match="out: expected 3 rows"):
        pq.pq_rotate(f16(3, 2, 128), i32(3), rot, out=f16(4, 2, 128))
    with pytest.raises(ValueError, match="pos: expected 3"):
        pq.pq_rotate(f16(3, 2, 128), i32(4), rot)
    with pytest.raises(TypeError):
        pq.pq_rotate(f16(3, 2, 128), i64(3), rot)
    with pytest.raises(ValueError, match="CUDA"):
        pq.pq_rotate(f16(3, 2, 128), i32(3), rot)
    kv = types.SimpleNamespace(heads=2, dim=64, page=16, pages=4, device=-1, _ref=0)
    with pytest.raises(ValueError, match="q: expected 3 rows"):
        pq.pq_kv_append_rotated(kv, f16(3, 2, 64), f16(3, 128), i64(3), i32(3), rot, q=f16(4, 8, 64))
    with pytest.raises(ValueError, match="out: there are no queries"):
        pq.pq_kv_append_rotated(kv, f16(3, 2, 64), f16(3, 128), i64(3), i32(3), rot, out=f16(3, 8, 64))
    with pytest.raises(ValueError, match="rotary: expected 16"):
        pq.pq_kv_append_rotated(kv, f16(3, 2, 64), f16(3, 128), i64(3), i32(3), types.SimpleNamespace(dim=32, freq=i64(15), _ref=0))
    lat = types.SimpleNamespace(latent=512, page=16, pages=4, device=-1, _ref=0)
    with pytest.raises(ValueError, match="c: expected rows of 512"):
        pq.pq_latent_append(lat, f16(3, 511), f16(3, 64), i64(3), i32(3), rot)
    with pytest.raises(ValueError, match="k_rope: expected 3 rows"):
        pq.pq_latent_append(lat, f16(3, 512), f16(2, 64), i64(3), i32(3), rot)
    with pytest.raises(ValueError, match="slots: expected 3"):
        pq.pq_latent_append(lat, f16(3, 512), f16(3, 64), i64(2), i32(3), rot)
    with pytest.raises(ValueError, match="w: expected"):
        pq.pq_head_linear(f16(3, 4, 128), f16(4, 512, 64))
    with pytest.raises(ValueError, match="w: expected"):
        pq.pq_head_linear(f16(3, 4, 128), f16(2, 512, 256))
    with pytest.raises(ValueError, match="out: expected"):
        pq.pq_head_linear(f16(3, 4, 128), f16(4, 512, 128), out=f16(3, 4, 256))
    with pytest.raises(ValueError, match="q: expected 6912"):
        pq.pq_latent_attention(f16(3, 4, 512), lat, i32(2, 4), i32(3), i32(2), 0.1)
    with pytest.raises(ValueError, match="q_start: expected 3"):
        pq.pq_latent_attention(f16(3, 4, 576), lat, i32(2, 4), i32(2), i32(2), 0.1)
    with pytest.raises(ValueError, match="out: expected"):
        pq.pq_latent_attention(f16(3, 4, 576), lat, i32(2, 4), i32(3), i32(2), 0.1, out=f16(3, 4, 576))
    with pytest.raises(ValueError, match="CUDA"):
        pq.pq_latent_attention(f16(3, 4, 576), lat, i32(2, 4), i32(3), i32(2), 0.1)
    with pytest.raises(ValueError, match="kv: expected rows of 1024"):
        pq.pq_expanded_attention(f16(3, 4, 192), f16(9, 4, 192), f16(9, 64), i32(3), i32(3), 2, 0.1)
    with pytest.raises(ValueError, match="k_rope: expected 9 rows"):
        pq.pq_expanded_attention(f16(3, 4, 192), f16(9, 4, 256), f16(8, 64), i32(3), i32(3), 2, 0.1)
    with pytest.raises(ValueError, match="kv_start: expected 3"):
        pq.pq_expanded_attention(f16(3, 4, 192), f16(9, 4, 256), f16(9, 64), i32(3), i32(4), 2, 0.1)


def test_the_plain_rotation_turns_a_quarter():
    x = np.arange(32.0).reshape(1, 1, 32)
    quarter = np.full(8, np.pi / 2)
    y = ref.rotate(x, np.array([1]), quarter, "half")
    assert np.allclose(y[0, 0, :8], -x[0, 0, 8:16]) and np.allclose(y[0, 0, 8:16], x[0, 0, :8]) and (y[0, 0, 16:] == x[0, 0, 16:]).all()
    y = ref.rotate(x, np.array([1]), quarter, "pairs")
    assert np.allclose(y[0, 0, 0:16:2], -x[0, 0, 1:16:2]) and np.allclose(y[0, 0, 1:16:2], x[0, 0, 0:16:2])


def test_the_two_plain_forms_of_latent_attention_are_one():
    """Absorbed queries over the latents give the latents that the expanded form's values are made of."""
    rng = np.random.default_rng(3)
    heads, latent, L, n = 3, 256, 21, 4
    up = rng.standard_normal((heads, 256, latent)) / 16                      # a head's keys, then its values, out of a latent
    c, rope = rng.standard_normal((L, latent)), rng.standard_normal((L, 64))
    q = rng.standard_normal((n, heads, 192))
    d = dict(q=np.concatenate([np.einsum("thk,hkc->thc", q[..., :128], up[:, :128]), q[..., 128:]], -1), latent=latent, table=np.zeros((1, 1), int),
             data=np.concatenate([c, rope], -1)[None], q_start=np.array([0, n]), kv_len=np.array([L]))
    absorbed = np.einsum("thc,hvc->thv", ref.latent_attention(d, 0.07)[0], up[:, 128:])
    e = dict(q=q.reshape(n, -1), kv=np.einsum("lc,hkc->lhk", c, up).reshape(L, -1), k_rope=rope, heads=heads, q_start=np.array([0, n]),
             kv_start=np.array([0, L]))
    assert np.allclose(ref.expanded_attention(e, 0.07)[0], absorbed, atol=1e-12)


def test_one_heads_strides_are_not_looked_at():
    assert pq.lib().pq_rotate(_rotary(), 16, 128, 3, 1, 128, None, 0, 16, 128, -5, None) == 0
    assert pq.lib().pq_rotate(_rotary(), 16, 128, 3, 2, 128, None, 0, 16, 128, 128, None) == SHAPE
    assert pq.lib().pq_head_linear(16, 128, 3, 16, 1, 512, 128, 0, 16, 512, -5, None) == 0


def test_a_tables_width_is_bounded_by_its_tokens():
    """Steps round up to whole tokens of 64 in 32 bits."""
    def call(width, page):
        return pq.lib().pq_latent_attention(16, 4, _latent(page=page), None, width, None, None, 0, 3, 0.1, None, None, 0, None)

    assert call(1 << 26, 16) == 0 and call((1 << 26) + 1, 16) == LIMIT
    assert call(1 << 20, 1024) == 0 and call((1 << 20) + 1, 1024) == LIMIT and call(0x7fffffff, 16) == LIMIT


def test_empty_operands_have_rows_of_any_stride():
    """An empty tensor's strides say nothing about its rows."""
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    assert binding._strided_rows(f16(64, 0).t(), 64, "x") == (0, 64)
    assert binding._head_rows(f16(128, 2, 0).permute(2, 1, 0), 2, 128, "x")[:3] == (0, 2, 128)
    with pytest.raises(ValueError, match="x: expected"):
        binding._strided_rows(f16(64, 3).t(), 64, "x")
    with pytest.raises(ValueError, match="x: expected"):
        binding._head_rows(f16(128, 2, 3).permute(2, 1, 0), 2, 128, "x")


def test_heads_and_widths_are_not_cut_to_32_bits():
    """A view of 2^32 + 1 heads takes no memory, and 2^32 + 1 cut to 32 bits would be one head."""
    x = torch.zeros(128, dtype=torch.float16).expand(1, 2**32 + 1, 128)
    with pytest.raises(ValueError, match="x's heads: .* 32 bits"):
        binding._head_rows(x, None, None, "x")
