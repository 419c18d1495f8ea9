"""A few answers generated token by token through a quantized attention block: what the key-value cache and its attention are for.

Per step and layer: the RMSNorm feeds the activation quantizer, the fused QKV projection (Q K V columns of one product) runs on
4-bit operands, the new keys and values go from its rows straight into the cache's pages, every new token attends to its own
sequence, and the output projection closes the block.  The prompts' keys and values come from the same projection, and are read
back once, as attention over a cached prefix would.  Weights and inputs are random.

    python examples/decode_cache.py [--fmt nvfp4|int4|bf16] [--steps 8]

The last line compares the block's attention with the same attention over an unquantized cache of the same tokens.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_09503_amd import pq  # noqa: E402

DEV = "cuda"


class Linear:
    """y = x W^T on 4-bit operands (INT4, groups of 64)."""

    def __init__(self, n_out, n_in, rng):
        w = (torch.randn(n_out, n_in, generator=rng, device=DEV) * n_in ** -0.5).to(torch.bfloat16)
        codes, scales = pq.alloc_quantized(pq.FMT_INT4, 64, n_out, n_in, DEV)
        pq.pq_quantize_weights(pq.FMT_INT4, 64, w, None, codes, scales, torch.empty(1, device=DEV))
        self.operand, self.shape = pq.pq_pack_operand(pq.FMT_INT4, 64, codes, scales), (n_out, n_in)

    def __call__(self, operand, rows):
        y = torch.empty((rows, self.shape[0]), dtype=torch.bfloat16, device=DEV)
        pq.pq_qgemm_packed(pq.FMT_INT4, 64, operand, None, self.operand, None, y, rows, *self.shape)
        return y


class Sequences:
    """Which pages hold which tokens: pages are handed out as sequences grow."""

    def __init__(self, seqs, page, max_len):
        per = (max_len + page - 1) // page
        self.page, self.free = page, torch.randperm(seqs * per, generator=torch.Generator().manual_seed(1)).tolist()
        self.pages, self.max_len = seqs * per, max_len
        self.table = torch.full((seqs, per), -1, dtype=torch.int32)
        self.lengths = torch.zeros(seqs, dtype=torch.int32)

    def append(self, b, n):
        """slots of n new tokens of sequence b"""
        first = int(self.lengths[b])
        for i in range((first + self.page - 1) // self.page, (first + n + self.page - 1) // self.page):
            self.table[b, i] = self.free.pop()
        pos = torch.arange(first, first + n)
        self.lengths[b] += n
        return self.table[b].long()[pos // self.page] * self.page + pos % self.page


def run(fmt="int4", steps=8, seqs=4, hidden=512, q_heads=8, kv_heads=2, head_dim=64, page=32, prompt=70):
    """(largest difference of the attention's outputs from the unquantized cache's, over their root mean square; the last hidden states)"""
    rng = torch.Generator(device=DEV).manual_seed(0)
    qkv = Linear((q_heads + 2 * kv_heads) * head_dim, hidden, rng)
    proj = Linear(hidden, q_heads * head_dim, rng)
    gamma = torch.ones(hidden, dtype=torch.bfloat16, device=DEV)
    place = Sequences(seqs, page, prompt + seqs + steps)
    fmt, group = {"nvfp4": (pq.FMT_NVFP4, 16), "int4": (pq.FMT_INT4, 64), "bf16": (pq.FMT_BF16, 0)}[fmt]

    def project(x):
        operand = pq.pq_norm_quantize_act_packed(pq.NORM_RMS, pq.FMT_INT4, 64, x, 1e-6, None, gamma=gamma)
        rows = qkv(operand, x.shape[0])
        split = [q_heads * head_dim, kv_heads * head_dim, kv_heads * head_dim]
        return [t.unflatten(1, (-1, head_dim)) for t in rows.split(split, 1)]

    # the prompts, of different lengths: their keys and values fill the cache
    lens = [prompt - 9 * b for b in range(seqs)]
    x = torch.randn(sum(lens), hidden, generator=rng, device=DEV).to(torch.bfloat16)
    _, k, v = project(x)
    ts = [torch.empty(1, device=DEV) for _ in range(2)] if fmt == pq.FMT_NVFP4 else [None, None]
    for t, s in zip((k, v), ts):
        if s is not None:                                        # a static tensor scale with room for what comes
            pq.pq_dynamic_tensor_scale(t.flatten(1), s)
            s.mul_(1.5)
    cache = pq.alloc_kv_cache(fmt, group, kv_heads, head_dim, page, place.pages, *ts)
    plain = pq.alloc_kv_cache(pq.FMT_BF16, 0, kv_heads, head_dim, page, place.pages)
    slots = torch.cat([place.append(b, n) for b, n in enumerate(lens)]).to(DEV)
    for c in (cache, plain):
        pq.pq_kv_write(c, k, v, slots)
    prefix_k, prefix_v = pq.pq_kv_read(cache, slots)
    assert prefix_k.shape == k.shape and prefix_v.shape == v.shape

    workspaces = [pq.pq_attn_decode_workspace(c, seqs, q_heads, place.max_len) for c in (cache, plain)]
    x, worst = torch.randn(seqs, hidden, generator=rng, device=DEV).to(torch.bfloat16), 0.0
    for _ in range(steps):
        q, k, v = project(x)
        slots = torch.cat([place.append(b, 1) for b in range(seqs)]).to(DEV)
        table, lengths = place.table.to(DEV), place.lengths.to(DEV)
        o = []
        for c, ws in zip((cache, plain), workspaces):
            pq.pq_kv_write(c, k, v, slots)
            o.append(pq.pq_attn_decode(c, q, table, lengths, place.max_len, head_dim ** -0.5, workspace=ws).flatten(1))
        worst = max(worst, float((o[0].float() - o[1].float()).abs().max() / o[1].float().square().mean().sqrt()))
        x = x + proj(pq.pq_quantize_act_packed(pq.FMT_INT4, 64, o[0], None), seqs)
    return worst, x


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--fmt", default="int4", choices=["nvfp4", "int4", "bf16"])
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    worst, x = run(a.fmt, a.steps)
    print("%d steps, hidden states of %d sequences; attention off by up to %.3f of its root mean square from the unquantized cache's"
          % (a.steps, x.shape[0], worst))
