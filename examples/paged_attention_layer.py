"""The attention block of a W8A8 decoder layer as a server runs it: requests of different lengths, their prompts taken in
chunks, then one token at a time, over a paged key/value cache.

Per step: the step's tokens are quantized once and multiplied with the q, k and v weights in one grouped launch;
`pq_block_tables` gives each new token its slot; `pq_kv_append` writes the keys and values (FP16, or INT8 by the same
per-vector rule as the activations); `pq_paged_attention` attends over the cache; the output linear follows in one call.

    python examples/paged_attention_layer.py [--cache int8]
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


class PagedAttentionLayer:
    """Weights, cache and page bookkeeping of one layer.  hidden = heads * dim."""

    def __init__(self, heads: int, kv_heads: int, dim: int, requests: int, pages: int, width: int, page: int = 16,
                 cache: torch.dtype = torch.float16, seed: int = 0, device: str = "cuda:0"):
        self.heads, self.kv_heads, self.dim, self.device = heads, kv_heads, dim, device
        self.sms = torch.cuda.get_device_properties(device).multi_processor_count
        hidden, kv = heads * dim, kv_heads * dim
        w = lambda n, k, s: torch.from_numpy(synth.weights(n, k, seed + s)).to(device)  # noqa: E731
        self.qkv = [(*pq.pq_pack_w8(w(n, hidden, i)), n) for i, n in enumerate((hidden, kv, kv))]
        self.o = pq.pq_pack_w8(w(hidden, hidden, 3))
        self.cache = pq.PagedKV.empty(pages, kv_heads, page, dim, cache, device)
        i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.table = i32(requests, width)
        self.kv_len = i32(requests)
        self.free_list = torch.arange(pages, dtype=torch.int32, device=device)   # pages are handed out in this order
        self.free_head = i32(1)
        self.lengths = [0] * requests      # the scheduler's own copy of kv_len: it chose the chunks
        self.workspace = None              # of the attention; kept from step to step, made anew when a step wants more

    def project(self, x: torch.Tensor) -> list[torch.Tensor]:
        """x f16 [T, hidden] -> q [T, heads * dim], k, v [T, kv_heads * dim]."""
        return pq.pq_gemm_w8a8_group(*pq.pq_quantize_act(x), self.qkv)

    def step(self, x: torch.Tensor, new: list[int]) -> torch.Tensor:
        """x f16 [sum(new), hidden]: new[b] tokens of request b, one request after the other -> f16 of the same shape."""
        if sum(new) != x.shape[0] or len(new) != len(self.lengths):
            raise ValueError("new: one number of tokens per request, x their rows")
        lengths = [a + b for a, b in zip(self.lengths, new)]
        columns = [-(-n // self.cache.page) for n in lengths]
        if max(columns) > self.table.shape[1] or sum(columns) > self.cache.pages:
            raise ValueError(f"{sum(columns)} pages, {max(columns)} for one request: the cache has {self.cache.pages}, "
                             f"a table row {self.table.shape[1]}")
        self.lengths = lengths
        new_len = torch.tensor(new, dtype=torch.int32, device=self.device)
        step = pq.pq_block_tables(self.kv_len, new_len, self.table, self.free_list, self.free_head, self.cache.page, x.shape[0])
        q, k, v = self.project(x)
        pq.pq_kv_append(self.cache, k, v, step.slots)
        max_q, max_kv = max(new), max(self.lengths)
        room = pq.pq_attention_workspace_bytes(len(new), x.shape[0], max_q, max_kv, self.heads, self.kv_heads, self.dim, self.sms)
        if room > (0 if self.workspace is None else self.workspace.numel()):
            self.workspace = pq.pq_workspace_init(torch.empty((room,), dtype=torch.uint8, device=self.device))
        y = pq.pq_paged_attention(q, self.cache, self.table, step.q_start, step.kv_len, max_q, max_kv, workspace=self.workspace)
        self.kv_len, self.free_head = step.kv_len, step.free_head
        return pq.pq_linear_w8a8(y, *self.o, self.heads * self.dim)


def serve(layer: PagedAttentionLayer, inputs: list[torch.Tensor], prompts: list[int], chunk: int) -> list[torch.Tensor]:
    """Runs every request's tokens (inputs[b] f16 [T_b, hidden]) through the layer: the first prompts[b] in chunks of
    `chunk`, the rest one per step, as a continuous batch (a request decodes while another's prompt is still going in).
    Returns the outputs per request."""
    done, out = [0] * len(inputs), [[] for _ in inputs]
    while any(d < len(x) for d, x in zip(done, inputs)):
        new = [min(chunk, p - d) if d < p else min(1, len(x) - d) for d, p, x in zip(done, prompts, inputs)]
        y = layer.step(torch.cat([x[d: d + n] for d, n, x in zip(done, new, inputs)]), new)
        for b, part in enumerate(torch.split(y, new)):
            out[b].append(part)
        done = [d + n for d, n in zip(done, new)]
    return [torch.cat(o) for o in out]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=("f16", "int8"), default="f16")
    a = ap.parse_args()
    prompts, decoded, page = [700, 33, 260, 5], 20, 16
    layer = PagedAttentionLayer(16, 4, 128, len(prompts), pages=sum(-(-(p + decoded) // page) for p in prompts), page=page,
                                width=-(-(max(prompts) + decoded) // page), cache=torch.int8 if a.cache == "int8" else torch.float16)
    inputs = [torch.from_numpy(synth.activations(p + decoded, 2048, seed=i)).to(layer.device) for i, p in enumerate(prompts)]
    out = serve(layer, inputs, prompts, chunk=256)
    print("lengths", [len(y) for y in out], "pages used", int(layer.free_head), "of", layer.cache.pages,
          "status", pq.pq_device_status(), "finite", bool(np.isfinite(torch.cat(out).cpu().numpy()).all()))


if __name__ == "__main__":
    main()
