"""What is measured of rotary positions and of latent attention: cases, inputs, plain forms and exact values.

Five operators, in the order in which a decoder layer calls them between its linears:

  rotate     queries and keys turned by their positions: whole heads or a part, two layouts, scaled for long contexts
  append     the same on the way into a paged cache: keys and values in FP16 or INT8 with the queries rotated beside
             them, or one latent vector and one rotary key a token (an INT8 cache is read back as the values it holds)
  absorb     one matrix a head: the products that move the keys' and values' expansion to queries and results
  latent     attention over the paged latent cache, queries in the latent space: decode steps and drafts
  expanded   attention over keys and values expanded per head, with one rotary key a token: prompts and their chunks

`own` selects the package's kernels; otherwise the plain forms below run, elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
ROPE, NOPE, VALUE = 64, 128, 128   # of latent attention: rotary values of a head, the others, values of a head


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    turn = {"layout": "half", "scaling": "none", "far": 8191, "dim": 128}
    return [
        # queries and keys of one decoding user (32 + 8 heads of 128): latency
        {**turn, "name": "rotate_1", "op": "rotate", "tokens": 1, "heads": 40, "width": 128},
        # a chunk of a long prompt, half of each head turned, frequencies stretched in bands
        {"name": "rotate_8192_part", "op": "rotate", "tokens": 8192, "heads": 40, "width": 128, "dim": 64, "layout": "pairs",
         "scaling": "bands", "far": 131071},
        # one decode step of 64 requests into the FP16 cache
        {**turn, "name": "append_64_f16", "op": "append", "tokens": 64, "heads": 32, "kv_heads": 8, "width": 128, "page": 16,
         "cache": "f16"},
        # a long prompt into the 8-bit cache, frequencies stretched by wavelength
        {**turn, "name": "append_8192_int8", "op": "append", "tokens": 8192, "heads": 32, "kv_heads": 8, "width": 128, "page": 64,
         "cache": "int8", "scaling": "waves", "far": 65535},
        # chunks of prompts into the latent cache
        {"name": "append_4000_latent", "op": "append", "tokens": 4000, "heads": 32, "kv_heads": 1, "width": 512, "page": 64,
         "cache": "latent", "layout": "pairs", "scaling": "bands", "far": 65535, "dim": ROPE},
        # queries of one user into the latent space: latency
        {"name": "absorb_1", "op": "absorb", "tokens": 1, "heads": 32, "in": NOPE, "out": 512},
        # results of a busy decode step out of it
        {"name": "absorb_64_out", "op": "absorb", "tokens": 64, "heads": 128, "in": 512, "out": VALUE},
        # one user, an early token, the heads of one of eight devices: latency
        {"name": "latent_1x1000", "op": "latent", "requests": 1, "new": 1, "cached": 999, "ragged": False, "heads": 16,
         "latent": 512, "page": 64},
        # one decode step of a busy server, all heads
        {"name": "latent_64_ragged", "op": "latent", "requests": 64, "new": 1, "cached": 8191, "ragged": True, "heads": 128,
         "latent": 512, "page": 64},
        # drafted tokens over long contexts, small pages
        {"name": "latent_drafts", "op": "latent", "requests": 7, "new": 4, "cached": 30000, "ragged": True, "heads": 32,
         "latent": 512, "page": 16},
        # a whole prompt
        {"name": "expanded_4096", "op": "expanded", "requests": 1, "new": 4096, "cached": 0, "ragged": False, "heads": 32},
        # ragged chunks of several prompts
        {"name": "expanded_chunks", "op": "expanded", "requests": 5, "new": 700, "cached": 5000, "ragged": True, "heads": 16},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["rotate", "append", "append", "absorb", "latent", "latent", "expanded"])
    turn = {"layout": rng.choice(["half", "pairs"]), "scaling": rng.choice(["none", "linear", "base", "bands", "waves"]),
            "far": _log(rng, 1000, 1000000)}
    page = rng.choice([16, 16, 32, 48, 64, 128])
    if op == "rotate":
        width = rng.choice([64, 64, 96, 128, 128, 192])
        return {"op": op, **turn, "tokens": _log(rng, 1, 8192), "heads": rng.choice([1, 5, 8, 16, 24]), "width": width,
                "dim": rng.choice([32, 64, width])}
    if op == "append":
        cache = rng.choice(["f16", "int8", "latent"])
        heads, kv_heads, width = rng.choice([(32, 8, 128), (32, 32, 64), (28, 4, 128), (16, 16, 128), (32, 4, 64)])
        if cache == "latent":
            return {"op": op, **turn, "tokens": _log(rng, 1, 8192), "heads": rng.choice([16, 20, 32]), "kv_heads": 1,
                    "width": rng.choice([256, 512]), "page": page, "cache": cache, "dim": ROPE}
        return {"op": op, **turn, "tokens": _log(rng, 1, 8192), "heads": heads, "kv_heads": kv_heads, "width": width, "page": page,
                "cache": cache, "dim": rng.choice([width, width, width // 2])}
    heads = rng.choice([16, 20, 32, 64, 128])
    if op == "absorb":
        shape = rng.choice([(NOPE, 512), (512, VALUE), (NOPE, 256), (256, VALUE)])
        return {"op": op, "tokens": _log(rng, 1, 256), "heads": heads, "in": shape[0], "out": shape[1]}
    if op == "latent":
        new = rng.choice([1, 1, 1, rng.randint(2, 8)])
        n, latent = _log(rng, 1, 96), rng.choice([512, 512, 256])
        # the plain form's gathered keys and its scores stay below those of the largest listed cases
        most = min(131071, int(1.6e8 / (n * (latent + ROPE))), int(3.6e7 / (n * new * heads)))
        return {"op": op, "requests": n, "new": new, "cached": _log(rng, 8, max(16, most)), "ragged": rng.random() < 0.7,
                "heads": heads, "latent": latent, "page": page}
    heads = rng.choice([8, 16, 16, 20, 32])
    new = _log(rng, 1, 4096)
    n = _log(rng, 1, max(1, min(8, 4096 // new)))
    most = min(16384, int(2.6e8 / (n * heads * new)) - new, int(2.5e8 / (n * heads * (NOPE + ROPE))) - new)
    return {"op": op, "requests": n, "new": new, "cached": rng.choice([0, _log(rng, 8, max(8, most))]) if most >= 8 else 0,
            "ragged": rng.random() < 0.7, "heads": heads}


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


def work(case):
    op, rows = case["op"], case.get("tokens", 0) * case["heads"]
    if op == "rotate":
        return {"bytes": 4 * rows * case["width"] + 4 * case["tokens"], "flops": 3 * rows * case["dim"]}
    if op == "append":
        t, w = case["tokens"], case["kv_heads"] * case["width"]
        if case["cache"] == "latent":
            return {"bytes": 12 * t + 4 * rows * ROPE + 4 * t * (w + ROPE), "flops": 3 * (rows + t) * ROPE}
        vec = w * 2 if case["cache"] == "f16" else w + 4 * case["kv_heads"]
        again = 0 if case["cache"] == "f16" else vec + 2 * w   # the read-back of the 8-bit cache
        return {"bytes": 12 * t + 4 * rows * case["width"] + 2 * t * (2 * w + vec + again),
                "flops": 3 * (rows + t * case["kv_heads"]) * case["dim"]}
    if op == "absorb":
        return {"bytes": 2 * case["heads"] * case["in"] * case["out"] + 2 * rows * (case["in"] + case["out"]),
                "flops": 2 * rows * case["in"] * case["out"]}
    new, cached = _lengths(case)
    pairs = case["heads"] * sum(n * (c + 1) + n * (n - 1) // 2 for n, c in zip(new, cached))
    keys, rows = sum(new) + sum(cached), sum(new) * case["heads"]
    if op == "latent":
        wide = case["latent"] + ROPE
        return {"bytes": 2 * keys * wide + 2 * rows * (wide + case["latent"]), "flops": 2 * pairs * (wide + case["latent"])}
    return {"bytes": 2 * keys * (case["heads"] * (NOPE + VALUE) + ROPE) + 2 * rows * (NOPE + ROPE + VALUE),
            "flops": 2 * pairs * (NOPE + ROPE + VALUE)}


# --------------------------------------------------------------------------------------------------- inputs

SCALINGS = {"none": {}, "linear": {"factor": 4.0}, "base": {"factor": 8.0},
            "bands": {"factor": 16.0, "original": 8192, "low": 1.0, "high": 32.0},
            "waves": {"factor": 8.0, "original": 8192, "low": 1.0, "high": 4.0}}
BASE = 500000.0


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    rand = lambda *shape: torch.empty(shape, dtype=torch.float16, device=DEV).normal_(generator=gen)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    op, heads = case["op"], case["heads"]
    s = {"op": op, "case": dict(case)}
    if op in ("rotate", "append"):
        t, width = case["tokens"], case["width"]
        # tokens of a few prompts, each a run of positions
        run = torch.arange(t, device=DEV) % max(1, -(-t // 3))
        s["pos"] = (run + torch.randint(0, max(1, case["far"] - t), (1,), device=DEV, generator=gen)).int()
        if op == "rotate":
            return s | {"x": rand(t, heads, width)}
        page, kv_heads = case["page"], case["kv_heads"]
        pages = -(-t // page) + 3
        order = torch.randperm(pages, generator=gen, device=DEV)
        tok = torch.arange(t, device=DEV)
        s["slots"] = order[tok // page] * page + tok % page
        if case["cache"] == "latent":
            # latent and rotary key come out of one linear, the queries' rotary part is the end of every head
            both = rand(t, width + ROPE)
            return s | {"c": both[:, :width], "k_rope": both[:, width:], "q": rand(t, heads, NOPE + ROPE)[..., NOPE:],
                        "data": torch.zeros((pages, page, width + ROPE), dtype=torch.float16, device=DEV)}
        qkv = rand(t, heads + 2 * kv_heads, width)   # one linear's output
        s |= {"q": qkv[:, :heads], "new_k": qkv[:, heads: heads + kv_heads], "new_v": qkv[:, heads + kv_heads:]}
        shape = (pages, kv_heads, page, width)
        for name in ("k", "v"):
            s[name] = torch.zeros(shape, dtype=torch.float16 if case["cache"] == "f16" else torch.int8, device=DEV)
            s[name + "_scale"] = None if case["cache"] == "f16" else torch.zeros(shape[:3], device=DEV)
        return s
    if op == "absorb":
        return s | {"x": rand(case["tokens"], heads, case["in"]), "w": rand(heads, case["out"], case["in"]) * case["in"] ** -0.5}
    new, cached = _lengths(case)
    total = [n + c for n, c in zip(new, cached)]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s |= {"q_start": ints(start), "max_q": max(new), "max_kv": max(total), "scale": (NOPE + ROPE) ** -0.5}
    if op == "expanded":
        starts = [0]
        for n in total:
            starts.append(starts[-1] + n)
        return s | {"q": rand(start[-1], heads, NOPE + ROPE), "kv": rand(starts[-1], heads, NOPE + VALUE),
                    "k_rope": rand(starts[-1], ROPE), "kv_start": ints(starts)}
    page, wide = case["page"], case["latent"] + ROPE
    want = [-(-n // page) for n in total]
    table = torch.zeros((len(new), max(want)), dtype=torch.int32, device=DEV)
    table[torch.arange(max(want), device=DEV)[None] < ints(want)[:, None]] = torch.randperm(sum(want), generator=gen, device=DEV).int()
    # queries such that the scores spread by about 1.5, as those of expanded heads do
    return s | {"q": rand(start[-1], heads, wide) * (1.5 * ((NOPE + ROPE) / wide) ** 0.5), "data": rand(sum(want), page, wide),
                "table": table, "kv_len": ints(total)}


# ------------------------------------------------------------------------------------------------ plain forms

def _frequencies(case):
    """Radians a position, in 64 bits, and the factor of cosine and sine."""
    dim, kind, set_ = case["dim"], case["scaling"], SCALINGS[case["scaling"]]
    i = torch.arange(dim // 2, dtype=torch.float64, device=DEV)
    base, factor = BASE, set_.get("factor", 1.0)
    if kind == "base":
        base = BASE * factor ** (dim / (dim - 2))
    f = base ** (-2 * i / dim)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "bands":   # of the pairs, by the turns that they make over the original length
        at = lambda turns: dim * math.log(set_["original"] / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(at(set_["high"])), 0), min(math.ceil(at(set_["low"])), dim - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    if kind == "waves":   # by the wavelength's share of the original length
        keep = ((set_["original"] * f / (2 * math.pi) - set_["low"]) / (set_["high"] - set_["low"])).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _plain_turned(x, pos, case):
    """x [T, heads, width] in 32 bits with the first `dim` values of each head turned; angles in 64 bits."""
    f, amplitude = _frequencies(case)
    angle = pos.double()[:, None] * f
    c, s = (angle.cos() * amplitude).float()[:, None], (angle.sin() * amplitude).float()[:, None]
    x, dim = x.float(), case["dim"]
    y = x.clone()
    a, b = ((slice(0, dim // 2), slice(dim // 2, dim)) if case["layout"] == "half" else (slice(0, dim, 2), slice(1, dim, 2)))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def _plain_append(s):
    case = s["case"]
    page = case["page"]
    at, off = s["slots"] // page, s["slots"] % page
    q = _plain_turned(s["q"], s["pos"], case).half()
    if case["cache"] == "latent":
        width = case["width"]
        s["data"][at, off, :width] = s["c"]
        s["data"][at, off, width:] = _plain_turned(s["k_rope"][:, None], s["pos"], case)[:, 0].half()
        return q, s["data"]
    k, v = _plain_turned(s["new_k"], s["pos"], case), s["new_v"].float()
    if case["cache"] == "f16":
        s["k"][at, :, off], s["v"][at, :, off] = k.half(), v.half()
        return q, s["k"], s["v"]

    def one(codes, scales, x):
        most = x.abs().amax(-1)
        r = torch.where(most > 0, 127.5 / most, 0.0)
        codes[at, :, off] = (x * r[..., None]).round().clamp(-128, 127).to(torch.int8)
        scales[at, :, off] = most / 127.5
        return (codes[at, :, off].float() * scales[at, :, off][..., None]).half()

    return q, one(s["k"], s["k_scale"], k), one(s["v"], s["v_scale"], v)


def _rows_of(s):
    """Rows of every request, padded to the longest: indexes [requests, max_q] and which of them there are."""
    start = s["q_start"].long()
    i = torch.arange(s["max_q"], device=DEV)
    inside = i[None] < (start[1:] - start[:-1])[:, None]
    return torch.where(inside, start[:-1, None] + i[None], 0), inside, start[1:] - start[:-1]


def _softmax(score, seen):
    score = score.masked_fill_(~seen, -math.inf)
    most = score.amax(-1, keepdim=True)
    e = (score - torch.where(most == -math.inf, 0.0, most)).exp_()
    total = e.sum(-1, keepdim=True)
    return e, torch.where(total == 0, 1.0, total)


def _plain_latent(s):
    q, heads, latent = s["q"], s["case"]["heads"], s["case"]["latent"]
    rows, inside, n = _rows_of(s)
    b, width = rows.shape[0], s["table"].shape[1] * s["case"]["page"]
    keys = s["data"][s["table"].long()].view(b, width, -1).float()
    x = q[rows].float()                                               # [b, max_q, heads, wide]
    score = (x.view(b, -1, x.shape[-1]) @ keys.transpose(1, 2)) * s["scale"]
    last = (s["kv_len"].long() - n)[:, None] + torch.arange(s["max_q"], device=DEV)[None]
    seen = torch.arange(width, device=DEV)[None, None] <= last[..., None]
    e, total = _softmax(score.view(b, -1, heads, width), seen[:, :, None])
    out = (e.view(b, -1, width) @ keys[..., :latent]).view(b, -1, heads, latent) / total
    return out[inside].half()


def _plain_expanded(s):
    rows, inside, n = _rows_of(s)
    starts = s["kv_start"].long()
    length = starts[1:] - starts[:-1]
    j = torch.arange(s["max_kv"], device=DEV)
    at = torch.where(j[None] < length[:, None], starts[:-1, None] + j[None], 0)
    heads = s["case"]["heads"]
    q = s["q"][rows].float().transpose(1, 2)                          # [b, heads, max_q, 192]
    kv = s["kv"][at].float().transpose(1, 2)
    k = torch.cat([kv[..., :NOPE], s["k_rope"][at].float()[:, None].expand(-1, heads, -1, -1)], -1)
    score = (q @ k.transpose(2, 3)) * s["scale"]
    last = (length - n)[:, None] + torch.arange(s["max_q"], device=DEV)[None]
    e, total = _softmax(score, (j[None, None] <= last[..., None])[:, None])
    out = (e @ kv[..., NOPE:]) / total
    return out.transpose(1, 2)[inside].half()


# --------------------------------------------------------------------------------------------- a pass, exact

def run(s):
    op = s["op"]
    if not own:
        if op == "rotate":
            return _plain_turned(s["x"], s["pos"], s["case"]).half()
        if op == "absorb":
            return torch.matmul(s["x"].float().transpose(0, 1), s["w"].float().transpose(1, 2)).transpose(0, 1).half()
        return {"append": _plain_append, "latent": _plain_latent, "expanded": _plain_expanded}[op](s)
    import paper_2512_23367_b200 as pq
    # Objects and buffers that a user's program keeps from step to step: frequencies, the cache, outputs, the workspace.
    case = s["case"]
    if op in ("rotate", "append") and "rotary" not in s:
        s["rotary"] = pq.Rotary(case["dim"], base=BASE, layout=case["layout"], scaling=case["scaling"], device=DEV,
                                **SCALINGS[case["scaling"]])
    if op == "append":
        if "cache" not in s:
            s["cache"] = (pq.LatentKV(s["data"]) if case["cache"] == "latent" else
                          pq.PagedKV(s["k"], s["v"], s["k_scale"], s["v_scale"]))
            s["out"] = torch.empty(s["q"].shape, dtype=torch.float16, device=DEV)
        if case["cache"] == "latent":
            return pq.pq_latent_append(s["cache"], s["c"], s["k_rope"], s["slots"], s["pos"], s["rotary"], q=s["q"], out=s["out"]), s["data"]
        q = pq.pq_kv_append_rotated(s["cache"], s["new_k"], s["new_v"], s["slots"], s["pos"], s["rotary"], q=s["q"], out=s["out"])
        return (q, s["k"], s["v"]) if case["cache"] == "f16" else (q, *pq.pq_kv_read(s["cache"], s["slots"]))
    if op in ("latent", "expanded") and "workspace" not in s:
        s["workspace"] = pq.pq_latent_workspace(DEV)
        s["cache"] = pq.LatentKV(s["data"]) if op == "latent" else None
    if "out" not in s:
        x = s["x"] if "x" in s else s["q"]
        wide = {"rotate": case.get("width"), "absorb": case.get("out"), "latent": case.get("latent"), "expanded": VALUE}[op]
        s["out"] = torch.empty((*x.shape[:2], wide), dtype=torch.float16, device=DEV)
    if op == "rotate":
        return pq.pq_rotate(s["x"], s["pos"], s["rotary"], out=s["out"])
    if op == "absorb":
        return pq.pq_head_linear(s["x"], s["w"], out=s["out"])
    if op == "latent":
        return pq.pq_latent_attention(s["q"], s["cache"], s["table"], s["q_start"], s["kv_len"], s["scale"], out=s["out"],
                                      workspace=s["workspace"])
    return pq.pq_expanded_attention(s["q"], s["kv"], s["k_rope"], s["q_start"], s["kv_start"], s["max_q"], s["scale"], out=s["out"],
                                    workspace=s["workspace"])


def _exact_turned(x, pos, case):
    """Each pair as a complex number times e^(i angle)."""
    f, amplitude = _frequencies(case)
    x, dim = x.double(), case["dim"]
    turned = x[..., :dim].unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else x[..., :dim].unflatten(-1, (-1, 2))
    z = torch.view_as_complex(turned.contiguous()) * torch.polar(torch.full_like(f, amplitude).expand(len(pos), -1), pos.double()[:, None] * f)[:, None]
    y = torch.view_as_real(z)
    y = y.transpose(-1, -2) if case["layout"] == "half" else y
    return torch.cat([y.flatten(-2), x[..., dim:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotate":
        return _exact_turned(s["x"], s["pos"], case)
    if op == "append":
        page, q = case["page"], _exact_turned(s["q"], s["pos"], case)
        if case["cache"] == "latent":
            flat = s["data"].double().flatten(0, 1)
            flat[s["slots"]] = torch.cat([s["c"].double(), _exact_turned(s["k_rope"][:, None], s["pos"], case)[:, 0]], -1)
            return q, flat.view(s["data"].shape)
        out = [q]
        for name, x in (("k", _exact_turned(s["new_k"], s["pos"], case)), ("v", s["new_v"].double())):
            if case["cache"] == "int8":
                most = x.abs().amax(-1, keepdim=True)
                out.append(torch.clamp(torch.round(x * (127.5 / most)), -128, 127) * (most / 127.5))
            else:
                flat = s[name].double().transpose(1, 2).reshape(-1, *x.shape[1:])
                flat[s["slots"]] = x
                out.append(flat.view(-1, page, *x.shape[1:]).transpose(1, 2))
        return tuple(out)
    if op == "absorb":
        return torch.einsum("thk,hnk->thn", s["x"].double(), s["w"].double())
    start, heads = s["q_start"].tolist(), case["heads"]
    wide = case["latent"] if op == "latent" else VALUE
    out = torch.zeros((start[-1], heads, wide), dtype=torch.float64, device=DEV)
    lengths = s["kv_len"].tolist() if op == "latent" else (s["kv_start"][1:] - s["kv_start"][:-1]).tolist()
    first = 0
    for b, length in enumerate(lengths):
        n = start[b + 1] - start[b]
        gone = torch.arange(length, device=DEV)[None] > torch.arange(length - n, length, device=DEV)[:, None]
        if op == "latent":
            c = s["data"][s["table"][b, : -(-length // case["page"])].long()].flatten(0, 1)[:length].double()
        for h in range(heads):
            if op == "latent":
                k, v = c, c[:, :wide]
            else:
                kv = s["kv"][first: first + length, h].double()
                k, v = torch.cat([kv[:, :NOPE], s["k_rope"][first: first + length].double()], -1), kv[:, NOPE:]
            w = s["q"][start[b]: start[b + 1], h].double() @ k.T * s["scale"]
            out[start[b]: start[b + 1], h] = w.masked_fill(gone, -math.inf).softmax(-1) @ v
        first += length
    return out
