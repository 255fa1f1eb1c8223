"""A decoder layer's attention on packed weights: prompts, then single tokens.

The {q, k, v} projections and o_proj are q-bit weights (sss_quantize).  Each step of
the loop takes the requests' new tokens through

    sss_page_plan      pages, positions and slots from the requests' lengths
    sss_gemm_multi     q, k, v = x W^T (sss_gemv for the single tokens of a decode step)
    sss_qk_norm_rope   heads normalised and rotated; keys and values into the cache
    sss_attention      over the paged cache
    sss_gemm           o_proj (sss_gemv for single tokens)

without reading anything back.  At the end the same tokens go through the layer as
whole packed prompts, without a cache, and the two results are compared.

    python examples/attention_step.py [--layer llama3_8b] [--q 4] [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_08779_gb300 import inputs, sss  # noqa: E402

# (query heads, key/value heads, head dimension, hidden size, normalised heads)
LAYERS = {"llama3_8b": (32, 8, 128, 4096, False), "qwen3_32b": (64, 8, 128, 5120, True),
          "small": (8, 2, 64, 512, True)}


class AttentionLayer:
    """Packed projections, the heads' norm and rotation, and a paged cache."""

    def __init__(self, heads, kv_heads, dim, hidden, norm, q, pages, page_size, max_pos, seed=1):
        self.heads, self.dim, self.page_size = heads, dim, page_size

        def packed(n, k, i):
            w = inputs.student_t_weights_cuda(n, k, seed + i)
            return sss.sss_quantize(w, q, 32, sss.GRID_SIGNED_SYM)

        self.qkv = [packed(n * dim, hidden, i) for i, n in enumerate((heads, kv_heads, kv_heads))]
        self.o = packed(hidden, heads * dim, 3)
        angle = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * (
            500000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) * 2 / dim))
        weights = [torch.linspace(0.5, 1.5, dim, device="cuda") for _ in range(2)] if norm else [None, None]
        self.rope = sss.Rope(angle.cos().float(), angle.sin().float(), sss.ROPE_HALF, *weights)
        self.cache = sss.empty_kv_cache(pages, page_size, kv_heads, dim)
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda")

    def project(self, x):
        """The three projections of bf16 x [tokens, hidden], fp32."""
        if x.shape[0] <= 16:
            return [sss.sss_gemv(w, x) for w in self.qkv]
        return sss.sss_gemm_multi(self.qkv, x)

    def output(self, a):
        """o_proj of the attention's rows [tokens, heads, dim], fp32."""
        a = a.view(a.shape[0], -1)
        return sss.sss_gemv(self.o, a) if a.shape[0] <= 16 else sss.sss_gemm(self.o, a)

    def step(self, x, past, fresh, table, max_q, max_kv, status):
        """The layer's output for the new tokens x of requests that hold `past` tokens
        and bring `fresh` (device int32 [batch]); table is updated."""
        batch, tokens = past.numel(), x.shape[0]
        cu_q, kv_len, used = (torch.empty(n, dtype=torch.int32, device="cuda")
                              for n in (batch + 1, batch, 1))
        positions, slots = (torch.empty(tokens, dtype=torch.int32, device="cuda") for _ in range(2))
        sss.sss_page_plan(past, fresh, self.page_size, self.free, table, cu_q, kv_len, positions,
                          slots, used, dev_status=status)
        q, k, v = self.project(x)
        qr = sss.sss_qk_norm_rope(q, k, v, self.rope, positions, self.cache, slots=slots,
                                  dev_status=status)
        a = sss.sss_attention(qr, self.cache, cu_q, kv_len, max_q, max_kv, block_table=table,
                              dev_status=status)
        return self.output(a)

    def whole(self, x, lengths, status):
        """The same for whole prompts, packed, without the cache."""
        cu = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
        positions = torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lengths])
        q, k, v = self.project(x)
        kv = [torch.empty((x.shape[0], self.cache.k.shape[1], self.dim), dtype=torch.bfloat16,
                          device="cuda") for _ in range(2)]
        packed = sss.KVCache(*kv)
        qr = sss.sss_qk_norm_rope(q, k, v, self.rope, positions, packed, dev_status=status)
        a = sss.sss_attention(qr, packed, cu, None, max(lengths), max(lengths), dev_status=status)
        return self.output(a)


def run(layer="llama3_8b", q=4, prompts=(512, 77, 200, 9), steps=8, page_size=16, seed=5):
    """Serves the prompts and `steps` single tokens of each.  Returns the largest
    difference between what the steps gave and whole prompts give, relative to the
    largest value, and the status word."""
    heads, kv_heads, dim, hidden, norm = LAYERS[layer]
    batch = len(prompts)
    total = [n + steps for n in prompts]
    pages = sum(-(-n // page_size) for n in total)
    net = AttentionLayer(heads, kv_heads, dim, hidden, norm, q, pages, page_size, max(total))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # the requests' activations, request by request
    xs = [inputs.normal_bf16_cuda((n, hidden), seed + i) for i, n in enumerate(total)]
    table = torch.full((batch, -(-max(total) // page_size)), -1, dtype=torch.int32, device="cuda")
    past = torch.zeros(batch, dtype=torch.int32, device="cuda")
    outs = [[] for _ in prompts]
    held = list(prompts)  # (the host knows the lengths: the bounds and the shapes)
    fresh = list(prompts)
    for step in range(steps + 1):
        f = torch.tensor(fresh, dtype=torch.int32, device="cuda")
        x = torch.cat([xs[b][held[b] - fresh[b]:held[b]] for b in range(batch)])
        y = net.step(x, past, f, table, max(fresh), max(held), status)
        for b, part in enumerate(y.split(fresh)):
            outs[b].append(part)
        past += f
        # (the pages taken, from the lengths that the host knows as well)
        net.free = net.free[sum(-(-h // page_size) - -(-(h - n) // page_size)
                                for h, n in zip(held, fresh)):]
        fresh = [1] * batch
        held = [n + 1 for n in held]
    got = torch.cat([torch.cat(o) for o in outs])
    want = net.whole(torch.cat(xs), total, status)
    torch.cuda.synchronize()
    return float((got - want).abs().max() / want.abs().max()), int(status)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--layer", choices=sorted(LAYERS), default="llama3_8b")
    p.add_argument("--q", type=int, choices=(2, 3, 4), default=4)
    p.add_argument("--steps", type=int, default=8)
    a = p.parse_args()
    diff, status = run(a.layer, a.q, steps=a.steps)
    print(f"{a.layer} q={a.q}: steps against whole prompts differ by {diff:.2e} of the largest value, "
          f"status {status}")


if __name__ == "__main__":
    main()
