"""What is measured of the paged key/value cache: cases, inputs, the operators' plain forms and exact values.

Four operators stand between the q/k/v linears of a decoder layer and its output linear:

  tables     block tables, slot map and positions of a step, from the requests' lengths
  append     the step's keys and values written into the paged cache (FP16, or INT8 with a scale per token and head);
             an INT8 cache is read back, so that the values that its codes stand for come out
  attention  the step's queries over the paged cache: one token per request, a few, or a long chunk

`own` selects the package's kernels; otherwise the plain forms below run, elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    # 32 query heads of 128 over 8 key/value heads are the 4096-wide decoder layer, 16 heads of 128 without sharing
    # and 32 heads of 64 the 2048-wide one.
    layer = {"op": "attention", "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "cache": "f16", "window": 0}
    return [
        # the start of a decode step of a small server: latency
        {"name": "tables_8_decoding", "op": "tables", "requests": 8, "new": 1, "cached": 2000, "ragged": True, "page": 16},
        # a large server's step in which many prompts begin
        {"name": "tables_512_prompts", "op": "tables", "requests": 512, "new": 128, "cached": 4000, "ragged": True, "page": 16},
        # one decode step's new tokens of 64 requests: latency
        {"name": "append_64_f16", "op": "append", "tokens": 64, "kv_heads": 8, "dim": 128, "page": 16, "cache": "f16"},
        # a long prompt into the 8-bit cache
        {"name": "append_8192_int8", "op": "append", "tokens": 8192, "kv_heads": 8, "dim": 128, "page": 64, "cache": "int8"},
        # one user, an early token: latency
        {**layer, "name": "decode_1x1000", "requests": 1, "new": 1, "cached": 999, "ragged": False},
        # one decode step of a busy server, lengths as they come
        {**layer, "name": "decode_64_ragged", "requests": 64, "new": 1, "cached": 8191, "ragged": True},
        # the same load from the 8-bit cache
        {**layer, "name": "decode_64_int8", "requests": 64, "new": 1, "cached": 8191, "ragged": True, "page": 64, "cache": "int8"},
        # few requests with very long contexts: the keys have to be split over the machine
        {**layer, "name": "decode_3x131072", "requests": 3, "new": 1, "cached": 131071, "ragged": False},
        # drafted tokens of the 2048-wide layer, a sliding window, no sharing of heads
        {**layer, "name": "draft_5_window", "requests": 48, "new": 5, "cached": 6000, "ragged": True, "heads": 32,
         "kv_heads": 32, "dim": 64, "window": 1024},
        # a whole prompt
        {**layer, "name": "prompt_4096", "requests": 1, "new": 4096, "cached": 0, "ragged": False},
        # the next chunk of a long prompt: the largest
        {**layer, "name": "chunk_2048_of_18432", "requests": 1, "new": 2048, "cached": 16384, "ragged": False, "page": 64},
        # ragged chunks of several prompts over the 8-bit cache
        {**layer, "name": "chunks_6_int8", "requests": 6, "new": 700, "cached": 5000, "ragged": True, "page": 32, "cache": "int8"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    kind = rng.choice(["tables", "append", "decode", "decode", "draft", "chunk", "chunk"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    cache = rng.choice(["f16", "int8"])
    if kind == "tables":
        return {"op": "tables", "requests": _log(rng, 1, 1024), "new": _log(rng, 1, 256), "cached": _log(rng, 16, 8000),
                "ragged": True, "page": page}
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (32, 32, 128), (16, 16, 128), (32, 32, 64), (32, 4, 64),
                                       (40, 8, 128), (28, 4, 128), (16, 1, 128)])
    if kind == "append":
        return {"op": "append", "tokens": _log(rng, 1, 8192), "kv_heads": kv_heads, "dim": dim, "page": page, "cache": cache}
    case = {"op": "attention", "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "cache": cache,
            "window": rng.choice([0, 0, 0, _log(rng, 32, 4096)]), "ragged": rng.random() < 0.7}
    if kind == "chunk":
        case["new"] = _log(rng, 17, 2048)
        case["requests"] = _log(rng, 1, max(1, min(8, 4096 // case["new"])))
    else:
        case["new"] = 1 if kind == "decode" else rng.randint(2, 16)
        case["requests"] = _log(rng, 1, 128)
    # the plain form's scores and its gathered keys stay below those of the largest listed cases
    most = min(131071, int(1.2e9 / (case["requests"] * heads * case["new"])), int(3.9e8 / (case["requests"] * kv_heads * dim)))
    if kind == "chunk":
        most = min(most, 16384)
    case["cached"] = _log(rng, 16, max(17, most - case["new"]))
    return case


def _lengths(case):
    """(new, cached) of every request, from the case alone."""
    n = case["requests"]
    if not case["ragged"]:
        return [case["new"]] * n, [case["cached"]] * n
    rng = random.Random("%d %d %d" % (n, case["new"], case["cached"]))
    new = [rng.randint(1, case["new"]) for _ in range(n)]
    cached = [rng.randint(case["cached"] // 8, case["cached"]) for _ in range(n)]
    new[0], cached[-1] = case["new"], case["cached"]
    return new, cached


def _visible(case):
    """(query, key) pairs that the mask leaves, and the keys that have to be read."""
    pairs = keys = 0
    w = case["window"]
    for n, c in zip(*_lengths(case)):
        lo = max(0, c + 1 - w) if w else 0
        keys += c + n - lo
        full = n * (c + 1) + n * (n - 1) // 2
        if w:  # query i sees min(w, c + 1 + i) keys
            k = max(0, min(n, w - c))  # queries that the window does not cut
            full = k * (c + 1) + k * (k - 1) // 2 + (n - k) * w
        pairs += full
    return pairs, keys


def work(case):
    if case["op"] == "tables":
        new, cached = _lengths(case)
        p = case["page"]
        fresh = sum(-(-(c + n) // p) - -(-c // p) for n, c in zip(new, cached))
        return {"bytes": 16 * len(new) + 8 * fresh + 12 * sum(new), "flops": 0}
    elt = 2 if case["cache"] == "f16" else 1
    vec = case["kv_heads"] * (case["dim"] * elt + (0 if elt == 2 else 4))
    if case["op"] == "append":
        row = case["kv_heads"] * case["dim"] * 2
        again = 0 if elt == 2 else vec + row  # the read-back of the 8-bit cache
        return {"bytes": case["tokens"] * (8 + 2 * (row + vec + again)), "flops": 0}
    pairs, keys = _visible(case)
    rows = sum(_lengths(case)[0]) * case["heads"] * case["dim"]
    return {"bytes": 2 * vec * keys + 4 * rows, "flops": 4 * case["dim"] * case["heads"] * pairs}


# --------------------------------------------------------------------------------------------------- inputs

def _cache(case, pages, gen, filled):
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    s = {}
    for name in ("k", "v"):
        if not filled:
            s[name] = torch.zeros(shape, dtype=torch.float16 if case["cache"] == "f16" else torch.int8, device=DEV)
            s[name + "_scale"] = None if case["cache"] == "f16" else torch.zeros(shape[:3], device=DEV)
        elif case["cache"] == "f16":
            s[name] = torch.empty(shape, dtype=torch.float16, device=DEV).normal_(generator=gen)
            s[name + "_scale"] = None
        else:  # codes of rows whose largest value takes the end of the range, as the quantizer leaves them
            s[name] = torch.randint(-127, 128, shape, dtype=torch.int8, device=DEV, generator=gen)
            s[name + "_scale"] = torch.empty(shape[:3], device=DEV).uniform_(0.01, 0.03, generator=gen)
    return s


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *shape: torch.empty(shape, dtype=torch.float16, device=DEV).normal_(generator=gen)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    page = case["page"]
    s = {"op": case["op"], "page": page}
    if case["op"] == "append":
        # slots of a chunk: whole pages in random order
        t = case["tokens"]
        pages = -(-t // page) + 3
        order = torch.randperm(pages, generator=gen, device=DEV)
        tok = torch.arange(t, device=DEV)
        s["slots"] = order[tok // page] * page + tok % page
        s["new_k"], s["new_v"] = (rand(t, case["kv_heads"], case["dim"]) for _ in "kv")
        return s | _cache(case, pages, gen, filled=False)
    new, cached = _lengths(case)
    have = [-(-c // page) for c in cached]
    want = [-(-(c + n) // page) for n, c in zip(new, cached)]
    width = max(want)
    if case["op"] == "tables":
        pages = sum(want) + 64
        order = torch.randperm(pages, generator=gen, device=DEV).int()
        used = sum(have)
        table = torch.zeros((len(new), width), dtype=torch.int32, device=DEV)
        mask = torch.arange(width, device=DEV)[None] < ints(have)[:, None]
        table[mask] = order[:used]
        return s | {"kv_len": ints(cached), "new_len": ints(new), "table": table, "free_list": order, "free_head": ints([used]),
                    "tokens": sum(new)}
    pages = sum(want)
    table = torch.zeros((len(new), width), dtype=torch.int32, device=DEV)
    mask = torch.arange(width, device=DEV)[None] < ints(want)[:, None]
    table[mask] = torch.randperm(pages, generator=gen, device=DEV).int()
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s |= {"table": table, "q_start": ints(start), "kv_len": ints([n + c for n, c in zip(new, cached)]), "max_q": max(new),
          "max_kv": max(n + c for n, c in zip(new, cached)), "window": case["window"],
          "q": rand(start[-1], case["heads"], case["dim"])}
    return s | _cache(case, pages, gen, filled=True)


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_tables(s):
    kv, new, page, head = s["kv_len"].long(), s["new_len"].long(), s["page"], s["free_head"].long()
    start = torch.cat([torch.zeros_like(head), new.cumsum(0)])
    have, want = (kv + page - 1) // page, (kv + new + page - 1) // page
    first = (want - have).cumsum(0) - (want - have)
    col = torch.arange(s["table"].shape[1], device=DEV)[None]
    fresh = (col >= have[:, None]) & (col < want[:, None])
    take = head + first[:, None] + col - have[:, None]
    there = take < s["free_list"].shape[0]
    ids = torch.where(there, s["free_list"].long()[torch.where(fresh & there, take, 0)], -1)
    table = torch.where(fresh, ids, s["table"].long())
    tok = torch.arange(s["tokens"], device=DEV)
    req = (tok[:, None] >= start[None, 1:]).sum(1)
    pos = kv[req] + tok - start[req]
    at = table[req, pos // page]
    slots = torch.where(at >= 0, at * page + pos % page, -1)
    return table.int(), start.int(), (kv + new).int(), slots, pos.int(), (head + (want - have).sum()).int()


def _plain_append(s):
    at, off = s["slots"] // s["page"], s["slots"] % s["page"]
    if s["k_scale"] is None:
        s["k"][at, :, off] = s["new_k"]
        s["v"][at, :, off] = s["new_v"]
        return s["k"], s["v"]

    def one(codes, scales, new):
        x = new.float()
        most = x.abs().amax(-1)
        r = torch.where(most > 0, 127.5 / most, 0.0)
        codes[at, :, off] = (x * r[..., None]).round().clamp(-128, 127).to(torch.int8)
        scales[at, :, off] = most / 127.5
        return (codes[at, :, off].float() * scales[at, :, off][..., None]).half()

    return one(s["k"], s["k_scale"], s["new_k"]), one(s["v"], s["v_scale"], s["new_v"])


def _plain_attention(s):
    q, table, start, kv = s["q"], s["table"], s["q_start"].long(), s["kv_len"].long()
    b, hk, dim = table.shape[0], s["k"].shape[1], q.shape[2]
    g, width = q.shape[1] // hk, table.shape[1] * s["page"]
    n = start[1:] - start[:-1]

    def gathered(codes, scales):
        x = codes[table.long()].float()
        if scales is not None:
            x = x * scales[table.long()][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(b, hk, width, dim)

    i = torch.arange(s["max_q"], device=DEV)
    inside = i[None] < n[:, None]
    rows = torch.where(inside, start[:-1, None] + i[None], 0)
    x = q[rows].float().view(b, -1, hk, g, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dim)
    score = (x @ gathered(s["k"], s["k_scale"]).transpose(2, 3)) * (1 / math.sqrt(dim))
    last = (kv - n)[:, None] + i[None]
    j = torch.arange(width, device=DEV)
    seen = j[None, None] <= last[..., None]
    if s["window"]:
        seen = seen & (j[None, None] > last[..., None] - s["window"])
    score = score.view(b, hk, g, -1, width).masked_fill(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    e = (score - torch.where(most == -math.inf, 0.0, most)).exp_()
    total = e.sum(-1, keepdim=True)
    out = e.view(b, hk, -1, width) @ gathered(s["v"], s["v_scale"])
    out = out.view(b, hk, g, -1, dim) / torch.where(total == 0, 1.0, total)
    return out.permute(0, 3, 1, 2, 4).reshape(b, -1, hk * g, dim)[inside].half()


# --------------------------------------------------------------------------------------------- a pass, exact

def run(s):
    if not own:
        return {"tables": _plain_tables, "append": _plain_append, "attention": _plain_attention}[s["op"]](s)
    import paper_2512_23367_b200 as pq
    # Objects and buffers that a user's program keeps from step to step: the cache with its geometry, the step's
    # outputs, the workspace.
    if s["op"] == "tables":
        if "step" not in s:
            s["step"] = pq.PagedStep.empty(s["kv_len"].shape[0], s["tokens"], DEV)
        step = pq.pq_block_tables(s["kv_len"], s["new_len"], s["table"], s["free_list"], s["free_head"], s["page"], step=s["step"])
        return (s["table"], step.q_start, step.kv_len, step.slots, step.pos, step.free_head)
    if "cache" not in s:
        s["cache"] = pq.PagedKV(s["k"], s["v"], s["k_scale"], s["v_scale"])
    cache = s["cache"]
    if s["op"] == "append":
        pq.pq_kv_append(cache, s["new_k"], s["new_v"], s["slots"])
        return (s["k"], s["v"]) if s["k_scale"] is None else pq.pq_kv_read(cache, s["slots"])
    if "out" not in s:
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = pq.pq_attention_workspace(s["q"], cache, s["table"].shape[0], s["max_q"], s["max_kv"])
    return pq.pq_paged_attention(s["q"], cache, s["table"], s["q_start"], s["kv_len"], s["max_q"], s["max_kv"],
                                 window=s["window"], out=s["out"], workspace=s["workspace"])


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "tables":
        return None  # whole numbers
    if case["op"] == "append":
        page, out = s["page"], []
        for name in ("k", "v"):
            x = s["new_" + name].double()
            if case["cache"] == "int8":
                most = x.abs().amax(-1, keepdim=True)
                out.append(torch.clamp(torch.round(x * (127.5 / most)), -128, 127) * (most / 127.5))
            else:
                flat = s[name].double().transpose(1, 2).reshape(-1, *x.shape[1:])
                flat[s["slots"]] = x
                out.append(flat.view(-1, page, *x.shape[1:]).transpose(1, 2))
        return tuple(out)
    start, kv = s["q_start"].tolist(), s["kv_len"].tolist()
    hk, g = case["kv_heads"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, length in enumerate(kv):
        n = start[b + 1] - start[b]
        pages = s["table"][b, : -(-length // s["page"])].long()
        j = torch.arange(length, device=DEV)
        last = torch.arange(length - n, length, device=DEV)[:, None]
        gone = (j > last) | (j <= last - (case["window"] or length + 1))
        for h in range(hk):
            k, v = (s[x][pages, h].reshape(-1, case["dim"])[:length].double() for x in "kv")
            if case["cache"] == "int8":
                k, v = (y * s[x + "_scale"][pages, h].reshape(-1)[:length, None].double() for x, y in (("k", k), ("v", v)))
            for r in range(h * g, h * g + g):
                w = s["q"][start[b]: start[b + 1], r].double() @ k.T / math.sqrt(case["dim"])
                out[start[b]: start[b + 1], r] = w.masked_fill(gone, -math.inf).softmax(-1) @ v
    return out
