"""The latent attention block of a W8A8 decoder layer as a server runs it: prompts in the expanded form, then one token at a
time in the absorbed form, over one paged cache of latent vectors.

Per step: the step's tokens are quantized once and multiplied with the weights of the queries and of the latents in one grouped
launch; `pq_block_tables` gives each new token its slot; `pq_latent_append` writes latent vectors and turned rotary keys and turns
the queries' rotary part.  A step of prompts reads its requests' latents (`pq_latent_read`), multiplies them out per head
in one W8A8 linear and attends with `pq_expanded_attention`; a decode step takes its queries into the latent space
(`pq_head_linear`), attends over the cache with `pq_latent_attention` and brings the results back.  The output linear follows.

    python examples/latent_attention_layer.py
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_23367_b200 as pq  # noqa: E402
from paper_2512_23367_b200 import synth  # noqa: E402

NOPE, ROPE, VALUE = 128, 64, 128


class LatentAttentionLayer:
    """Weights, cache and page bookkeeping of one layer.  The keys' and values' expansion is held twice: as a W8A8 linear for
    prompts, and per head in FP16, dequantized from the same codes, for decode steps."""

    def __init__(self, heads: int, hidden: int, latent: int, requests: int, pages: int, width: int, page: int = 64, seed: int = 0,
                 device: str = "cuda:0"):
        self.heads, self.hidden, self.latent, self.device = heads, hidden, latent, device
        w = lambda n, k, s: torch.from_numpy(synth.weights(n, k, seed + s)).to(device)  # noqa: E731
        sizes = (heads * (NOPE + ROPE), latent + ROPE)
        self.in_proj = [(*pq.pq_pack_w8(w(n, hidden, i)), n) for i, n in enumerate(sizes)]
        self.expand_n = heads * (NOPE + VALUE)
        self.expand = pq.pq_pack_w8(w(self.expand_n, latent, 2))
        codes = pq.pq_unpack_w8(self.expand[0], self.expand_n, latent)
        each = (codes.float() * self.expand[1][:, None]).half().view(heads, NOPE + VALUE, latent)
        self.absorb_q = each[:, :NOPE].transpose(1, 2).contiguous()      # [heads, latent, 128]: queries into the latent space
        self.absorb_v = each[:, NOPE:].contiguous()                      # [heads, 128, latent]: results out of it
        self.o = pq.pq_pack_w8(w(hidden, heads * VALUE, 3))
        self.rotary = pq.Rotary(ROPE, layout="pairs", scaling="bands", factor=8.0, original=4096, device=device)
        self.scale = (NOPE + ROPE) ** -0.5
        self.cache = pq.LatentKV.empty(pages, page, latent, device)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.table, self.kv_len, self.free_head = i32(requests, width), i32(requests), i32(1)
        self.free_list = torch.arange(pages, dtype=torch.int32, device=device)   # pages are handed out in this order
        self.workspace = pq.pq_latent_workspace(device)
        self.lengths = [0] * requests      # the scheduler's own copy of kv_len: it chose the chunks

    def step(self, x: torch.Tensor, new: list[int], expanded: bool) -> torch.Tensor:
        """x f16 [sum(new), hidden]: new[b] tokens of request b, one request after the other -> f16 of the same shape."""
        if sum(new) != x.shape[0] or len(new) != len(self.lengths):
            raise ValueError("new: one number of tokens per request, x their rows")
        lengths = [a + b for a, b in zip(self.lengths, new)]
        columns = [-(-n // self.cache.page) for n in lengths]
        if max(columns) > self.table.shape[1] or sum(columns) > self.cache.pages:
            raise ValueError(f"{sum(columns)} pages, {max(columns)} for one request: the cache has {self.cache.pages}, "
                             f"a table row {self.table.shape[1]}")
        self.lengths = lengths
        T, heads = x.shape[0], self.heads
        new_len = torch.tensor(new, dtype=torch.int32, device=self.device)
        step = pq.pq_block_tables(self.kv_len, new_len, self.table, self.free_list, self.free_head, self.cache.page, T)
        q, ckr = pq.pq_gemm_w8a8_group(*pq.pq_quantize_act(x), self.in_proj)
        q = q.view(T, heads, NOPE + ROPE)
        c, k_rope = ckr[:, : self.latent], ckr[:, self.latent:]
        if expanded:
            y = self._expanded(q, c, k_rope, step, new)
        else:
            y = self._absorbed(q, c, k_rope, step)
        self.kv_len, self.free_head = step.kv_len, step.free_head
        return pq.pq_linear_w8a8(y.view(T, heads * VALUE), *self.o, self.hidden)

    def _expanded(self, q, c, k_rope, step, new):
        pq.pq_latent_append(self.cache, c, k_rope, step.slots, step.pos, self.rotary, q=q[..., NOPE:], out=q[..., NOPE:])
        # every cached token of the requests that have rows in this step, in order
        wanted = [n if m else 0 for n, m in zip(self.lengths, new)]
        kv_start = torch.tensor(np.concatenate([[0], np.cumsum(wanted)]), dtype=torch.int32, device=self.device)
        slots = torch.cat([self.table[b, torch.arange(n, device=self.device) // self.cache.page].long() * self.cache.page +
                           torch.arange(n, device=self.device) % self.cache.page for b, n in enumerate(wanted)])
        latents, rope = pq.pq_latent_read(self.cache, slots)
        kv = pq.pq_linear_w8a8(latents, *self.expand, self.expand_n).view(-1, self.heads, NOPE + VALUE)
        return pq.pq_expanded_attention(q, kv, rope, step.q_start, kv_start, max(new), self.scale, workspace=self.workspace)

    def _absorbed(self, q, c, k_rope, step):
        latent_q = torch.empty((q.shape[0], self.heads, self.latent + ROPE), dtype=torch.float16, device=self.device)
        pq.pq_head_linear(q[..., :NOPE], self.absorb_q, out=latent_q[..., : self.latent])
        pq.pq_latent_append(self.cache, c, k_rope, step.slots, step.pos, self.rotary, q=q[..., NOPE:], out=latent_q[..., self.latent:])
        y = pq.pq_latent_attention(latent_q, self.cache, self.table, step.q_start, step.kv_len, self.scale, workspace=self.workspace)
        return pq.pq_head_linear(y, self.absorb_v)


def serve(layer: LatentAttentionLayer, inputs: list[torch.Tensor], prompts: list[int], chunk: int) -> list[torch.Tensor]:
    """Runs every request's tokens (inputs[b] f16 [T_b, hidden]) through the layer: the first prompts[b] in chunks of `chunk`, the
    rest one per step.  A step that takes part of a prompt uses the expanded form.  Returns the outputs per request."""
    done, out = [0] * len(inputs), [[] for _ in inputs]
    while any(d < len(x) for d, x in zip(done, inputs)):
        new = [min(chunk, p - d) if d < p else min(1, len(x) - d) for d, p, x in zip(done, prompts, inputs)]
        y = layer.step(torch.cat([x[d: d + n] for d, n, x in zip(done, new, inputs)]), new, expanded=max(new) > 1)
        for b, part in enumerate(torch.split(y, new)):
            out[b].append(part)
        done = [d + n for d, n in zip(done, new)]
    return [torch.cat(o) for o in out]


def main() -> None:
    argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter).parse_args()
    prompts, decoded, page = [700, 33, 260, 5], 20, 64
    layer = LatentAttentionLayer(16, 2048, 512, len(prompts), pages=sum(-(-(p + decoded) // page) for p in prompts), page=page,
                                 width=-(-(max(prompts) + decoded) // page))
    inputs = [torch.from_numpy(synth.activations(p + decoded, 2048, seed=i)).to(layer.device) for i, p in enumerate(prompts)]
    out = serve(layer, inputs, prompts, chunk=256)
    print("lengths", [len(y) for y in out], "pages used", int(layer.free_head), "of", layer.cache.pages,
          "status", pq.pq_device_status(), "finite", bool(np.isfinite(torch.cat(out).cpu().numpy()).all()))


if __name__ == "__main__":
    main()
