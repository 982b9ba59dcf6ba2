"""Plain 64-bit forms of rotary positions and of latent attention (numpy, one request and one head at a time), and inputs
for their tests.  What an operator must not look at is poisoned: cache rows beyond a request's length and rows between
requests hold NaN, table entries that no token needs rubbish page ids."""
import math

import numpy as np

ROPE = 64


def frequencies(dim, base=10000.0, scaling="none", factor=1.0, original=0.0, low=1.0, high=32.0):
    """(radians per position [dim / 2], amplitude), as the header states them."""
    out = []
    if scaling == "base":
        base *= factor ** (dim / (dim - 2))
    for i in range(dim // 2):
        f = base ** (-2 * i / dim)
        turns = original * f / (2 * math.pi)          # over the original length
        share = {"linear": 1.0, "waves": 1 - (turns - low) / (high - low)}.get(scaling, 0.0)
        if scaling == "bands":
            at = lambda r: dim * math.log(original / (r * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), dim - 1)
            share = (i - first) / max(last - first, 0.001)
        share = min(max(share, 0.0), 1.0)
        out.append(f / factor * share + f * (1 - share))
    return np.array(out), 0.1 * math.log(factor) + 1 if scaling == "bands" else 1.0


def rotate(x, pos, freq, layout, amplitude=1.0):
    """x [T, heads, width] in 64 bits, its first 2 len(freq) values turned."""
    x, half = x.astype(np.float64).copy(), len(freq)
    angle = pos.astype(np.float64)[:, None] * freq
    c, s = (f(angle)[:, None] * amplitude for f in (np.cos, np.sin))
    a, b = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    p, q = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = p * c - q * s, q * c + p * s
    return x


def rotation_bound(x, dim, amplitude):
    """On |computed - exact| of an FP16 result: half a step of FP16 (2^-11 relative, 2^-25 absolute below the normal range) of
    a value of at most amplitude (|a| + |b|), and in FP32 the angle (2^-24 pi absolute at most), cosine and sine (2 units), their
    product with the amplitude and the two products of a pair (2^-24 each): 8 * 2^-24 of the same sum."""
    x = np.abs(x.astype(np.float64))
    most = x.copy()
    half = dim // 2
    for a, b in ((slice(0, half), slice(half, dim)), (slice(0, dim, 2), slice(1, dim, 2))):   # of either layout
        both = amplitude * (x[..., a] + x[..., b])
        most[..., a], most[..., b] = np.maximum(most[..., a], both), np.maximum(most[..., b], both)
    return most * (2.0 ** -11 + 8 * 2.0 ** -24) + 2.0 ** -25


def softmax_sum(s, seen, v):
    """(sum of weights x values, weights), rows that see nothing 0."""
    s = np.where(seen, s, -np.inf)
    top = s.max(1, keepdims=True)
    w = np.exp(s - np.where(np.isfinite(top), top, 0))
    total = w.sum(1, keepdims=True)
    w = w / np.where(total > 0, total, 1)
    return w @ v, w


def attention_bound(w, v, sums, width):
    """On |computed - y|, `sums` the largest sum of |scale q k| of each row [rows, 1].  Weights and the result are rounded to
    FP16: 2^-11 each of sum |w v|.  A score is a sum of `width` products in FP32, at worst truncated (2^-23 of the sum of
    magnitudes each), then scaled and taken to a power (within 64 such steps): its error moves a weight and the sum of
    weights.  Weights below FP16's normal range: half a step of 2^-24 where the largest is 2^7 at least.  2^-25: a subnormal
    result."""
    at = w @ np.abs(v)
    keys = (w > 0).sum(1, keepdims=True)
    return at * (2.0 ** -10 + 2 * (width + 64) * 2.0 ** -23 * sums) + 2.0 ** -32 * keys * w.max(1, keepdims=True) * np.abs(v).max(initial=0) + 2.0 ** -25


def latent_inputs(heads, latent, page, new, total, seed=0, spread=1.0, width=None, lost=(), gap=0):
    """total[b] cached tokens of request b with its own new[b] (it may be shorter than the chunk).  lost: (request, column)
    entries set to an id outside the cache.  gap: rows of the step behind the last request."""
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in total]
    width = max(max(used), 1) if width is None else width
    pages = sum(used) + 2
    table = rng.integers(-5, 1 << 30, (len(new), width)).astype(np.int32)
    ids = iter(rng.permutation(pages))
    data = np.full((pages, page, latent + ROPE), np.nan, np.float16)
    for b, length in enumerate(total):
        for col in range(used[b]):
            i = next(ids)
            if col < width:
                table[b, col] = i
            data[i, : min(page, length - col * page)] = rng.standard_normal((min(page, length - col * page), latent + ROPE))
    for b, col in lost:
        table[b, col] = [-1, pages, 1 << 30][col % 3]
    q = (rng.standard_normal((sum(new) + gap, heads, latent + ROPE)) * spread).astype(np.float16)
    return dict(q=q, data=data, table=table, q_start=np.concatenate([[0], np.cumsum(new)]).astype(np.int32),
                kv_len=np.array(total, np.int32), latent=latent)


def latent_attention(d, scale):
    """(y, bound); rows outside every request are NaN in y."""
    q, table, latent = d["q"].astype(np.float64), d["table"], d["latent"]
    T, heads, wide = q.shape
    pages, page, _ = d["data"].shape
    y, bound = np.full((T, heads, latent), np.nan), np.zeros((T, heads, latent))
    for b, length in enumerate(int(n) for n in d["kv_len"]):
        t0, t1 = (int(t) for t in d["q_start"][b: b + 2])
        j = np.arange(min(max(length, 0), table.shape[1] * page))
        ids = table[b, j // page].astype(np.int64)
        there = (ids >= 0) & (ids < pages)
        c = np.where(there[:, None], d["data"][np.where(there, ids, 0), j % page].astype(np.float64), 0.0)
        seen = j[None] <= np.arange(length - (t1 - t0), length)[:, None]
        for h in range(heads):
            if len(j) == 0:
                y[t0:t1, h] = 0
                continue
            sums = (np.abs(q[t0:t1, h]) @ np.abs(c.T)).max(1, keepdims=True) * abs(scale)
            y[t0:t1, h], w = softmax_sum(q[t0:t1, h] @ c.T * scale, seen, c[:, :latent])
            bound[t0:t1, h] = attention_bound(w, c[:, :latent], sums, wide)
    return y, bound


def expanded_inputs(heads, new, total, seed=0, spread=1.0, gap=0, stride=0):
    """Ragged q, kv, k_rope; gap: rows behind the last request; stride: unused values at the end of every row."""
    rng = np.random.default_rng(seed)
    rand = lambda n, m: np.concatenate([rng.standard_normal((n, m)), np.full((n, stride), np.nan)], 1).astype(np.float16)  # noqa: E731
    T, S = sum(new), sum(max(n, 0) for n in total)
    d = dict(q=rand(T + gap, heads * 192) * np.float16(spread), kv=rand(S + gap, heads * 256), k_rope=rand(S + gap, ROPE), heads=heads,
             q_start=np.concatenate([[0], np.cumsum(new)]).astype(np.int32), kv_start=np.concatenate([[0], np.cumsum(total)]).astype(np.int32))
    d["kv"][S:], d["k_rope"][S:] = np.nan, np.nan
    return d


def expanded_attention(d, scale):
    heads = d["heads"]
    T = d["q"].shape[0]
    q, kv = d["q"][:, : heads * 192].reshape(T, heads, 192).astype(np.float64), d["kv"][:, : heads * 256].reshape(-1, heads, 256).astype(np.float64)
    rope = d["k_rope"][:, :ROPE].astype(np.float64)
    y, bound = np.full((T, heads, 128), np.nan), np.zeros((T, heads, 128))
    for b in range(len(d["q_start"]) - 1):
        t0, t1, k0, k1 = (int(x) for x in (*d["q_start"][b: b + 2], *d["kv_start"][b: b + 2]))
        seen = np.arange(k1 - k0)[None] <= np.arange(k1 - k0 - (t1 - t0), k1 - k0)[:, None]
        for h in range(heads):
            if k1 == k0:
                y[t0:t1, h] = 0
                continue
            k, v = np.concatenate([kv[k0:k1, h, :128], rope[k0:k1]], 1), kv[k0:k1, h, 128:]
            sums = (np.abs(q[t0:t1, h]) @ np.abs(k.T)).max(1, keepdims=True) * abs(scale)
            y[t0:t1, h], w = softmax_sum(q[t0:t1, h] @ k.T * scale, seen, v)
            bound[t0:t1, h] = attention_bound(w, v, sums, 192)
    return y, bound
