"""Latent attention by the norm of a row's error: a key that is left out, or counted twice, where a request's keys are cut between
multiprocessors moves many values by less than the bound on each of them, but all of them at once."""
import numpy as np
import pytest

import latent_reference as ref
import paper_2512_23367_b200 as pq

ABSORBED = {   # heads, latent, new, total, page
    "long": (16, 512, [1], [9000], 64), "long_256": (16, 256, [2], [9000], 16), "all_heads": (128, 512, [1, 1, 2], [1500, 700, 1290], 64),
    "drafts": (32, 512, [4, 4, 1, 7], [2900, 4, 650, 2000], 16), "a_chunk": (8, 512, [150], [1400], 128),
}
EXPANDED = {"long": (8, [2], [9000]), "chunks": (4, [100, 300, 5], [1500, 1340, 1000]), "a_prompt": (2, [700], [700])}


def _inputs(form, kind):
    if form == "absorbed":
        heads, latent, new, total, page = ABSORBED[kind]
        return ref.latent_inputs(heads, latent, page, new, total, seed=11), (latent + 64) ** -0.5
    heads, new, total = EXPANDED[kind]
    return ref.expanded_inputs(heads, new, total, seed=11), 192 ** -0.5


def _requests(d):
    """(queries [n, heads, width], keys and values as functions of the head) of every request."""
    starts = d["q_start"].astype(int)
    for b in range(len(starts) - 1):
        t0, t1 = starts[b: b + 2]
        if "data" in d:
            page, L = d["data"].shape[1], int(d["kv_len"][b])
            c = d["data"][d["table"][b, : -(-L // page)].astype(int)].reshape(-1, d["data"].shape[2])[:L].astype(np.float64)
            yield d["q"][t0:t1].astype(np.float64), lambda h, c=c: (c, c[:, : d["latent"]])
        else:
            k0, k1 = (int(x) for x in d["kv_start"][b: b + 2])
            heads = d["heads"]
            kv = d["kv"][k0:k1, : heads * 256].reshape(k1 - k0, heads, 256).astype(np.float64)
            rope = d["k_rope"][k0:k1, :64].astype(np.float64)
            yield (d["q"][t0:t1, : heads * 192].reshape(t1 - t0, heads, 192).astype(np.float64),
                   lambda h, kv=kv, rope=rope: (np.concatenate([kv[:, h, :128], rope], 1), kv[:, h, 128:]))


def _exact(d, scale, without=()):
    """(y, bound on the norm of a row's error [rows, heads], y with each of the keys `without` left out of its sums).
    The roundings of the weights to FP16, 2^-11 of each at most, have nothing to do with each other, and neither have the FP32
    errors of the scores (within 2^-23 of the sum of magnitudes for each of `width` products and 64 steps more): the squares of w_j |v_j|
    times them add up.  (At most: a rounding's mean square is a third of that, and a norm over 128 values and more is within a fifth
    of its mean.)  A common factor, which the sum of the weights may have, counts as the score's.  2^-11 of the result's own norm for its
    rounding, 2^-25 of each value for subnormal ones, 2^-32 of the largest weight for each weight below FP16's normal range."""
    y, bounds, mutants = [], [], [[] for _ in without]
    for q, of_head in _requests(d):
        n, heads, width = q.shape
        one, bound, missing = [], [], [[] for _ in without]
        for h in range(heads):
            k, v = of_head(h)
            L = len(k)
            s, seen = q[:, h] @ k.T * scale, np.arange(L)[None] <= np.arange(L - n, L)[:, None]
            sums = (np.abs(q[:, h]) @ np.abs(k.T)).max(1) * abs(scale)
            yh, w = ref.softmax_sum(s, seen, v)
            size = (v * v).sum(1)
            spread = np.sqrt((w * w) @ size + (w * w).sum(1) * (yh * yh).sum(1))
            one.append(yh)
            bound.append(2.0 ** -11 * np.sqrt((yh * yh).sum(1)) + (2.0 ** -11 + (width + 64) * 2.0 ** -23 * sums) * spread +
                         2.0 ** -32 * w.max(1) * np.sqrt(seen @ size) + 2.0 ** -25 * v.shape[1] ** 0.5)
            for m, j in zip(missing, without):
                m.append((yh - w[:, j, None] * v[j]) / (1 - w[:, j, None]))
        y.append(np.stack(one, 1)), bounds.append(np.stack(bound, 1))
        for m, x in zip(mutants, missing):
            m.append(np.stack(x, 1))
    return np.concatenate(y), np.concatenate(bounds), [np.concatenate(m) for m in mutants]


def _holds(got, y, bound):
    return (np.sqrt(((got - y) ** 2).sum(2)) <= bound).all()


@pytest.mark.parametrize("form,kind", [("absorbed", "long"), ("absorbed", "long_256"), ("expanded", "long")])
def test_a_key_left_out_at_a_seam_is_seen(form, kind):
    """The mistake planted in the plain form: the last key of a step, or the first one of the next, of any seam.  The plain form with its
    results rounded to FP16 holds the bound."""
    d, scale = _inputs(form, kind)
    keys = [key for step in (64, 80) for seam in range(step * 3, 9000, step * 7) for key in (seam - 1, seam)]
    y, bound, mutants = _exact(d, scale, keys)
    assert _holds(y.astype(np.float16).astype(np.float64), y, bound)
    assert [key for key, m in zip(keys, mutants) if _holds(m, y, bound)] == []


@pytest.mark.gpu
@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("form,kind", [("absorbed", k) for k in ABSORBED] + [("expanded", k) for k in EXPANDED])
def test_rows_hold_the_bound_on_their_norm(form, kind, workspace):
    from test_gpu_expanded import Call as Expanded
    from test_gpu_latent import Call as Absorbed
    d, scale = _inputs(form, kind)
    got = (Absorbed if form == "absorbed" else Expanded)(d, scale, workspace)().cpu().numpy().astype(np.float64)
    assert pq.pq_device_status() == 0
    assert _holds(got, *_exact(d, scale)[:2])


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["absorbed", "expanded"])
@pytest.mark.parametrize("heavy", [5, 300])
@pytest.mark.parametrize("new,total", [([1, 1], [3000, 500]), ([3], [2000]), ([20], [3000]), ([200], [2500])])
def test_many_keys_of_very_small_weight_add_up(new, total, heavy, form):
    """One key has value 0 and 2^26.4 times the weight of every other: the answer is the others' sum.  Bound: 2^-9 of it for
    the FP16 roundings of weights and result and for scores of up to 19 out of 64 products in FP32; FP16's smallest step under weights of
    up to 2^7 at least, 2^-32 of the largest weight, from every key; half of the result's smallest step."""
    from test_gpu_expanded import Call as Expanded
    from test_gpu_latent import Call as Absorbed
    rng = np.random.default_rng(9)
    if form == "absorbed":
        scale, d = 0.125, ref.latent_inputs(16, 512, 16, new, total, seed=1)
        d["q"][..., :512], d["q"][..., 512:] = 0, 1
        d["data"][..., :512], d["data"][..., 512:] = rng.uniform(32, 64, d["data"][..., :512].shape), 0
        for b in range(len(new)):
            page, off = d["table"][b, heavy // 16], heavy % 16
            d["data"][page, off, :512], d["data"][page, off, 512:] = 0, 26.4 * np.log(2) / (64 * scale)
        call, y = Absorbed(d, scale), ref.latent_attention(d, scale)[0]
    else:
        scale, d = 192 ** -0.5, ref.expanded_inputs(3, new, total, seed=1)
        d["q"].reshape(-1, 3, 192)[..., :128], d["q"].reshape(-1, 3, 192)[..., 128:] = 0, 1
        kv = d["kv"].reshape(-1, 3, 256)
        kv[..., :128], kv[..., 128:], d["k_rope"][:] = 0, rng.uniform(32, 64, kv[..., 128:].shape), 0
        for first in d["kv_start"][:-1]:
            kv[first + heavy], d["k_rope"][first + heavy] = 0, 26.4 * np.log(2) / (64 * scale)
        call, y = Expanded(d, scale), ref.expanded_attention(d, scale)[0]
    assert (y > 2e-4).all()                    # the input is what it is meant to be
    got = call().cpu().numpy().astype(np.float64)
    assert pq.pq_device_status() == 0
    for b, length in enumerate(total):
        rows = slice(d["q_start"][b], d["q_start"][b + 1])
        assert (np.abs(got[rows] - y[rows]) <= 2.0 ** -9 * y[rows] + length * 2.0 ** -32 * 64 + 2.0 ** -25).all()
