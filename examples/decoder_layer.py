"""One Llama-style decoder layer on the library's operators: a prompt in chunks, then tokens
one by one.

    python examples/decoder_layer.py [--kind bf16|int8|int4] [--window W --sinks F]

The linears are outlier-aware INT4 (fq_w4a16_outlier_matmul), K and V go into a paged cache
(fq_kv_cache_write), attention reads it there (fq_paged_attention), and each norm is fused
with the residual sum before it (fq_gated_residual_norm).  Rotary embedding and the
activation are plain torch here.  Weights are random; the last lines compare the outputs
with the layer in 32-bit torch on the same dequantised weights.
"""

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_15531_amd as fq  # noqa: E402

HIDDEN, HEADS, KV_HEADS, DIM, FFN = 1024, 8, 2, 128, 2816
EPS = 1e-5


class Linear:
    """An outlier-aware INT4 linear, quantised from a dense fp32 weight [K][N]."""

    def __init__(self, W, frac=0.01):
        K, N = W.shape
        q = fq.fq_quantize_outlier_aware(W, frac)
        host = fq.fq_pack_tile_coo(K, N, q.k, q.n, q.v)
        dev = lambda a, t: torch.from_numpy(a.view(t).copy()).cuda()   # noqa: E731
        self.args = (dev(q.Wq, np.int32), dev(q.scales, np.int16).view(torch.float16), dev(q.zeros, np.int32),
                     fq.TileCOODevice(host))
        # the weight it stands for, for the comparison
        codes = (q.Wq[:, None, :] >> (4 * np.arange(8, dtype=np.uint32))[None, :, None]) & 15
        zeros = (q.zeros[:, :, None] >> (4 * np.arange(8, dtype=np.uint32))) & 15
        g = np.arange(K) // q.group
        dense = q.scales.view(np.float16)[g].astype(np.float32) * \
            (codes.reshape(K, N).astype(np.float32) - zeros.reshape(-1, N)[g].astype(np.float32))
        dense[q.k, q.n] = (q.v.astype(np.uint32) << 16).view(np.float32)
        self.dense = torch.from_numpy(dense).cuda()

    def __call__(self, x):
        return fq.fq_w4a16_outlier_matmul(x, *self.args)


def rotate(x, positions):
    """Rotary embedding of x [tokens][heads][dim] (fp32 inside)."""
    half = x.shape[-1] // 2
    freq = 500000.0 ** (-torch.arange(half, device=x.device) / half)
    a = positions[:, None, None].float() * freq
    lo, hi = x[..., :half].float(), x[..., half:].float()
    return torch.cat((lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()), -1).to(x.dtype)


class DecoderLayer:
    def __init__(self, seed=0):
        rng = np.random.default_rng(seed)
        w = lambda k, n: (rng.standard_normal((k, n)) / np.sqrt(k)).astype(np.float32)   # noqa: E731
        n_qkv = (HEADS + 2 * KV_HEADS) * DIM
        self.qkv, self.o = Linear(w(HIDDEN, n_qkv)), Linear(w(HEADS * DIM, HIDDEN))
        self.gate_up, self.down = Linear(w(HIDDEN, 2 * FFN)), Linear(w(FFN, HIDDEN))
        norm = lambda: torch.from_numpy(1 + 0.1 * rng.standard_normal(HIDDEN)).to(torch.bfloat16).cuda()   # noqa: E731
        self.norm_attn, self.norm_ffn, self.norm_next = norm(), norm(), norm()

    def __call__(self, x, block, cache, batch, slots, positions, window=0, sinks=0):
        """x: residual stream [tokens][HIDDEN]; block: output of the block before, still to be
        added.  Returns the residual stream, this layer's output still to be added, and the
        next layer's normed input."""
        T = x.shape[0]
        x, h = fq.fq_gated_residual_norm(block, x, self.norm_attn, eps=EPS)
        qkv = self.qkv(h).view(T, HEADS + 2 * KV_HEADS, DIM)
        q, k, v = qkv.split((HEADS, KV_HEADS, KV_HEADS), 1)
        fq.fq_kv_cache_write(cache, rotate(k, positions), v, slots)     # v: columns of the product
        a = fq.fq_paged_attention(rotate(q, positions), cache, batch, window=window, sinks=sinks)
        x, h = fq.fq_gated_residual_norm(self.o(a.view(T, -1)), x, self.norm_ffn, eps=EPS)
        gate, up = self.gate_up(h).chunk(2, 1)
        y = self.down(torch.nn.functional.silu(gate) * up)
        x, h = fq.fq_gated_residual_norm(y, x, self.norm_next, eps=EPS)
        return x, h

    def plain(self, x, window=0, sinks=0):
        """The same for one whole sequence, in 32-bit torch and without a cache."""
        def norm(t, w):
            return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w.float()

        x = x.float()
        T = x.shape[0]
        p = torch.arange(T, device=x.device)
        qkv = (norm(x, self.norm_attn) @ self.qkv.dense).view(T, HEADS + 2 * KV_HEADS, DIM)
        q, k, v = qkv.split((HEADS, KV_HEADS, KV_HEADS), 1)
        q, k = rotate(q, p), rotate(k, p)
        k, v = (t.repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1) for t in (k, v))
        s = q.transpose(0, 1) @ k.transpose(1, 2).contiguous() / DIM ** 0.5
        see = p[None, :] <= p[:, None]
        if window:
            see &= (p[None, :] > p[:, None] - window) | (p[None, :] < sinks)
        a = (s.masked_fill(~see, float("-inf")).softmax(-1) @ v).transpose(0, 1).reshape(T, -1)
        x = x + a @ self.o.dense
        gate, up = (norm(x, self.norm_ffn) @ self.gate_up.dense).chunk(2, 1)
        x = x + (torch.nn.functional.silu(gate) * up) @ self.down.dense
        return x, norm(x, self.norm_next)


def run(lengths=(150, 37, 90), steps=5, chunk=64, kind="int8", page=16, window=0, sinks=0, seed=0):
    """Prompts of the given lengths in chunks, then `steps` tokens of each together; returns
    (x, h) of every token by sequence, and the same of the plain layer."""
    layer = DecoderLayer(seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    n = len(lengths)
    xs = [torch.randn((t + steps, HIDDEN), generator=g, device="cuda").to(torch.bfloat16) for t in lengths]
    need = [-(-x.shape[0] // page) for x in xs]
    cache = fq.KVCache.empty(sum(need), page, KV_HEADS, DIM, kind)
    order = torch.randperm(sum(need), generator=g, device="cuda").to(torch.int32).split(need)
    table = torch.zeros((n, max(need)), dtype=torch.int32, device="cuda")
    for b, pages in enumerate(order):
        table[b, :len(pages)] = pages
    out = [[] for _ in lengths]

    def step(seqs, firsts, counts):
        """`counts[i]` tokens from `firsts[i]` on of each of the sequences."""
        cu = np.concatenate([[0], np.cumsum(counts)])
        ends = [a + c for a, c in zip(firsts, counts)]
        batch = fq.PagedBatch(torch.tensor(cu, dtype=torch.int32).cuda(), torch.tensor(ends, dtype=torch.int32).cuda(),
                              table[seqs], max(counts), max(ends))
        positions = torch.cat([torch.arange(a, e, device="cuda") for a, e in zip(firsts, ends)])
        owner = torch.repeat_interleave(torch.tensor(seqs).cuda(), torch.tensor(counts).cuda())
        slots = table[owner, positions // page].long() * page + positions % page
        x = torch.cat([xs[b][a:e] for b, a, e in zip(seqs, firsts, ends)])
        x, h = layer(x, torch.zeros_like(x), cache, batch, slots, positions, window, sinks)
        for i, b in enumerate(seqs):
            out[b].append((x[cu[i]:cu[i + 1]], h[cu[i]:cu[i + 1]]))

    for b, t in enumerate(lengths):
        for a in range(0, t, chunk):
            step([b], [a], [min(chunk, t - a)])
    for s in range(steps):
        step(list(range(n)), [t + s for t in lengths], [1] * n)
    got = [tuple(torch.cat(p) for p in zip(*o)) for o in out]
    return got, [layer.plain(x, window, sinks) for x in xs]


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--kind", default="int8", choices=("bf16", "int8", "int4"))
    p.add_argument("--window", type=int, default=0)
    p.add_argument("--sinks", type=int, default=0)
    a = p.parse_args()
    got, want = run(kind=a.kind, window=a.window, sinks=a.sinks)
    for b, (g, w) in enumerate(zip(got, want)):
        off = [((u.float() - v).norm() / v.norm()).item() for u, v in zip(g, w)]
        print(f"sequence {b}: {g[0].shape[0]} tokens, residual stream {off[0]:.2e} and normed output "
              f"{off[1]:.2e} off the 32-bit layer")


if __name__ == "__main__":
    main()
