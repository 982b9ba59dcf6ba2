"""Plain 64-bit forms of the paged cache operators (numpy, one request and one head at a time), and inputs for their
tests.  Everything that an operator must not look at is poisoned: cache slots beyond a request's length hold NaN (f16)
or NaN scales (int8), table entries that no visible key needs hold rubbish page ids."""
import numpy as np


def block_tables(kv_len, new_len, table, free_list, head, page, tokens):
    kv_len, new_len = np.maximum(kv_len, 0).astype(np.int64), np.maximum(new_len, 0).astype(np.int64)
    table = table.copy()
    width = table.shape[1]
    q_start = np.concatenate([[0], np.cumsum(new_len)])
    slots, pos = np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int64)
    take, t = head, 0
    for b in range(len(kv_len)):
        have, want = -(-kv_len[b] // page), -(-(kv_len[b] + new_len[b]) // page)
        fresh = {}
        for col in range(have, want):
            fresh[col] = free_list[take] if 0 <= take < len(free_list) else -1
            take += 1
            begins = q_start[b] + max(col * page - kv_len[b], 0)
            if col < width and begins < tokens:
                table[b, col] = fresh[col]
        for p in range(kv_len[b], kv_len[b] + new_len[b]):
            if t >= tokens:
                break
            col = p // page
            at = -1 if col >= width else (table[b, col] if col < have else fresh[col])
            slots[t] = -1 if at < 0 else at * page + p % page
            pos[t] = p
            t += 1
    return table, q_start, kv_len + new_len, slots, pos, take


def quantize(x):
    """Eq. 1-2 per vector in binary32, as the activation quantizer states it: (codes, scales)."""
    x = x.astype(np.float32)
    a = np.abs(x).max(-1)
    with np.errstate(divide="ignore"):
        f = np.where(a > 0, np.float32(127.5) / a, np.float32(0)).astype(np.float32)
    return np.clip(np.rint(x * f[..., None]), -128, 127).astype(np.int8), (a / np.float32(127.5)).astype(np.float32)


def attention_inputs(heads, kv_heads, dim, page, cache, new, total, window=0, seed=0, spread=1.0, width=None, lost=()):
    """numpy inputs; `total[b]` cached tokens of request b with its own new[b] (it may be shorter than the chunk).
    lost: (request, column) table entries set to an id outside the cache although their keys are visible."""
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in total]
    width = max(max(used), 1) if width is None else width
    pages = sum(used) + 2
    table = rng.integers(-5, 1 << 30, (len(new), width)).astype(np.int32)
    ids = iter(rng.permutation(pages))
    shape = (pages, kv_heads, page, dim)
    if cache == "f16":
        k, v = np.full(shape, np.nan, np.float16), np.full(shape, np.nan, np.float16)
        ks = vs = None
    else:
        k, v = (rng.integers(-128, 128, shape).astype(np.int8) for _ in range(2))
        ks, vs = np.full(shape[:3], np.nan, np.float32), np.full(shape[:3], np.nan, np.float32)
    for b, (n, length) in enumerate(zip(new, total)):
        lowest = max(0, length - n + 1 - window) if window else 0   # what the first row of the chunk still sees
        for col in range(lowest // page, used[b]):
            i = table[b, col] = next(ids)
            inside = slice(lowest - col * page if col == lowest // page else 0, min(page, length - col * page))
            m = inside.stop - inside.start
            if cache == "f16":
                k[i, :, inside] = rng.standard_normal((kv_heads, m, dim)) * spread
                v[i, :, inside] = rng.standard_normal((kv_heads, m, dim))
            else:
                ks[i, :, inside] = rng.uniform(0.25, 1.0, (kv_heads, m)) * spread / 64
                vs[i, :, inside] = 2.0 ** rng.uniform(-9, -5, (kv_heads, m))
    for b, col in lost:
        table[b, col] = [-1, pages, 1 << 30][col % 3]
    q = rng.standard_normal((sum(new), heads, dim)).astype(np.float16)
    return dict(q=q, k=k, v=v, ks=ks, vs=vs, table=table, q_start=np.concatenate([[0], np.cumsum(new)]).astype(np.int32),
                kv_len=np.array(total, np.int32), window=window)


def attention(d, scale=None):
    """(y, bound on |computed - y|) in 64 bits.  The bound: 2^-11 of the sum of |weights x values| each for the FP16
    rounding of the weights and of the result, twice 2^-11 for scores summed in FP32 (dim + 8 roundings of 2^-24 on
    |scale q k| sums below 64) that move a weight and the sum of weights, and half the smallest FP16 step, 2^-25, of
    the largest value per key, for weights that round in FP16's subnormal range (largest weight >= 1); 2^-24 for a
    subnormal result."""
    q, table, window = d["q"].astype(np.float64), d["table"], d["window"]
    T, heads, dim = q.shape
    pages, kv_heads, page, _ = d["k"].shape
    scale = dim ** -0.5 if scale is None else scale
    y, bound = np.zeros((T, heads, dim)), np.full((T, heads, dim), 2.0 ** -24)
    for b, length in enumerate(d["kv_len"]):
        t0, t1 = d["q_start"][b], d["q_start"][b + 1]
        n = t1 - t0
        length = int(length)
        lowest = max(0, length - n + 1 - window) if window else 0
        j = np.arange(lowest, min(length, table.shape[1] * page))
        if n == 0 or len(j) == 0:
            continue
        ids = table[b, j // page].astype(np.int64)
        there = (ids >= 0) & (ids < pages)
        ids = np.where(there, ids, 0)
        last = np.arange(length - n, length)[:, None]
        seen = (j[None] <= last) & ((j[None] > last - window) if window else True)
        for hk in range(kv_heads):
            k, v = (d[x][ids, hk, j % page].astype(np.float64) for x in "kv")
            if d["ks"] is not None:
                k, v = (x * d[s][ids, hk, j % page].astype(np.float64)[:, None] for x, s in ((k, "ks"), (v, "vs")))
            k, v = (np.where(there[:, None], x, 0.0) for x in (k, v))
            for h in range(hk * heads // kv_heads, (hk + 1) * heads // kv_heads):
                s = np.where(seen, q[t0:t1, h] @ k.T * scale, -np.inf)
                assert (np.abs(q[t0:t1, h]) @ np.abs(k.T) * abs(scale)).max() < 64   # what the bound assumes
                top = s.max(1, keepdims=True)
                w = np.exp(s - np.where(np.isfinite(top), top, 0))
                total = w.sum(1, keepdims=True)
                some = total[:, 0] > 0
                w = w / np.where(total > 0, total, 1)
                y[t0:t1, h] = w @ v
                bound[t0:t1, h] += 2.0 ** -9 * (w @ np.abs(v)) + (some * 2.0 ** -25)[:, None] * np.where(
                    seen[..., None], np.abs(v).max(-1)[None, :, None], 0).sum(1) / np.where(total > 0, total, 1)
    return y, bound
