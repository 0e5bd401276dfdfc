"""Decoder layers from the library's two halves: attention over an 8-bit
key/value cache and the sparse mixed-precision FFN over its neuron cache.

    python -m paper_2410_14740_amd.decoder [--layers 2] [--prompt 700,90,333] [--tokens 64]

runs ragged prompts in chunks and then decodes tokens on random LLaMA-shaped
weights, evicting blocks beyond a budget, and prints what it did.

One layer, rows x [tokens][d_model] (the residual stream, fp32):

    q, k, v = norm(x) Wq, norm(x) Wk, norm(x) Wv, q and k rotated by position
    x += attention(q, k, v) Wo
    x += FFN(norm(x))                       (m2c_predict_rank .. m2c_sparse_ffn)

A prompt goes in chunks: a chunk's queries see the tokens before it as the
cache holds them (`KVCache.attend_chunk`, or where `reads_back` has it faster
`KVCache.read` and `prompt_attention`) and their own, unrounded, and the chunk
is then appended. A token is rotated on its way into the cache
(`KVCache.append_rotated`) and attended over it. Keys are rotated before they are
cached, so evicting blocks leaves the others' positions as they are. The sum into
the stream after the attention is one with the norm for the FFN
(`norms.residual_norm`). Projections are torch's.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import m2c
from . import workloads as W
from .attention import KVCache, Rotary, prompt_attention
from .norms import residual_norm


def norm(x):
    """Root-mean-square norm of fp32 rows, as fp16 rows, in torch's operations."""
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).half()


def rotate(x, pos):
    """Rotary position embedding of x [tokens][heads][dim] at positions pos [tokens],
    in torch's operations (any width; angles in fp32)."""
    half = x.shape[-1] // 2
    freq = 10000.0 ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    a = pos.float()[:, None, None] * freq
    lo, hi = x[..., :half].float(), x[..., half:].float()
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1).to(x.dtype)


def rotary(dim, device="cuda"):
    """The rotation of a head of `dim` elements whose pairs turn once in 2 pi 10000^(2 i / dim) positions."""
    half = dim // 2
    return Rotary(10000.0 ** (-torch.arange(half, device=device, dtype=torch.float32) / half))


def reads_back(lens, before, n_heads, n_kv_heads, dim):
    """Whether chunks of lens[b] tokens on before[b] cached ones go faster over a
    copy of the cache in 16 bits than over its codes.

    Over codes a tile of 128 rows (tokens x heads of a group) and 64 keys takes
    0.43 ns more, as it converts them anew; the copy takes 50 us of calls and, per
    tile of keys and key/value head, 10 ns at 128 elements. Measured, in us over
    codes and over a copy: 64 / 8 heads of 128, 2048 and 700 tokens on 30000 and
    16385 2693, 2499; 4096 on 4000 863, 848; 2048 on 4000 369, 388; 1024 on 16000
    594, 591; 512 on 16000 340, 356. 40 / 40 heads, 4096 on 16000 1596, 1679. 32 / 8
    heads of 64, 1024 on 60000 904, 753; 512 on 60000 358, 428; 1024 on 16000 255, 258."""
    pairs = keys = 0
    for n, m in zip(lens, before):
        keys += (m + n) // 64 * n_kv_heads
        pairs += (m + n // 2) // 64 * n_kv_heads * -(-n * (n_heads // n_kv_heads) // 128)
    return pairs > 120000 + 24 * keys * dim // 128


class DecoderLayer:
    """One layer of `n_seqs` sequences of up to max_tokens tokens each.

    ffn: an m2c.Layer (its max_batch rows are what a call of its FFN takes);
    k, n16, n8: its active neurons and tier counts. budget: blocks that
    `evict` leaves per sequence and head beside the last one (0: no limit)."""

    def __init__(self, ffn, k, n16, n8, n_seqs, n_heads, n_kv_heads, max_tokens, weights,
                 block_tokens=64, budget=0):
        if budget < 0:
            raise ValueError(f"budget {budget}: need a number of blocks, or 0 for no limit")
        d = ffn.desc.d_model
        self.ffn, self.k, self.n16, self.n8, self.step = ffn, k, n16, n8, 0
        self.n_heads, self.n_kv_heads, self.dim = n_heads, n_kv_heads, d // n_heads
        self.wqkv, self.wo = weights  # [d][(n_heads + 2 n_kv_heads) dim], [d][d]
        self.budget = budget
        self.rotary = rotary(self.dim)
        self.cache = KVCache(n_seqs, n_kv_heads, self.dim, -(-max_tokens // block_tokens), block_tokens)
        self.tiers = torch.empty((ffn.desc.max_batch, ffn.desc.d_ff), dtype=torch.uint8, device="cuda")

    def project(self, x, pos=None):
        """Queries, keys and values of rows of the stream; queries and keys rotated
        by positions pos [rows] if given."""
        h, g = self.n_heads, self.n_kv_heads
        rows = (residual_norm(x)[1] @ self.wqkv).view(x.shape[0], h + 2 * g, self.dim)
        q, k, v = rows[:, :h], rows[:, h:h + g], rows[:, h + g:]
        if pos is not None:
            self.rotary.rotate(q, _places(pos), k=k, q_out=q, k_out=k)
        return q, k, v

    def feed_forward(self, x, attended=None):
        """x += attended Wo if given, x += FFN(norm(x)), max_batch rows at a time."""
        if attended is None:
            _, rows = residual_norm(x)
        else:
            _, rows = residual_norm(x, attended.reshape(x.shape[0], -1) @ self.wo, x_out=x)
        for a in range(0, x.shape[0], self.ffn.desc.max_batch):
            part = rows[a:a + self.ffn.desc.max_batch]
            n, L = part.shape[0], self.ffn
            L.predict_rank(part, n, self.k, self.n16, self.n8, None, self.tiers)
            L.cache_plan(self.tiers, n, self.step)
            L.cache_fill()
            L.sparse_ffn(part, n, x[a:a + n])
            self.step += 1

    def prefill(self, x, lens, before):
        """A chunk of every sequence: rows x are lens[b] tokens of sequence b,
        whose cache holds before[b]. Host lists; x is updated in place."""
        pos = torch.cat([torch.arange(p, p + n, dtype=torch.int32, device="cuda") for n, p in zip(lens, before)])
        cu = _starts(lens)
        if not any(before):
            q, k, v = self.project(x)
            q, k = self.cache.append_rotated(self.rotary, k, v, pos, q=q, cu=cu, k_out=True)
            out = prompt_attention(q, k, v, cu, max_q=max(lens))
        else:
            q, k, v = self.project(x, pos)
            out = self.attend(q, k, v, cu, lens, before)
            self.cache.append(k, v, cu=cu)
        self.feed_forward(x, out)

    def attend(self, q, k, v, cu, lens, before):
        """Chunks of rotated rows over the cache and themselves."""
        # after evictions the cache holds fewer tokens than their positions say
        if self.budget or not reads_back(lens, before, self.n_heads, self.n_kv_heads, self.dim):
            return self.cache.attend_chunk(q, cu, k, v, max_q=max(lens), max_len=max(before))
        both = [n + m for n, m in zip(lens, before)]
        cu_k = _starts(both)
        keys, values = self.cache.read(cu_k, sum(both))
        at = torch.cat([torch.arange(e - n, e, device="cuda") for n, e in zip(lens, np.cumsum(both).tolist())])
        keys[at], values[at] = k, v
        return prompt_attention(q, keys, values, cu, cu_k, max_q=max(lens))

    def decode(self, x, pos, max_len):
        """One token per sequence at positions pos (integer tensor); max_len: the
        longest sequence afterwards. x is updated in place."""
        q, k, v = self.project(x)
        q, _ = self.cache.append_rotated(self.rotary, k, v, _places(pos), q=q)
        out = self.cache.attend(q, max_len=max_len, track=self.budget > 0)
        self.feed_forward(x, out)

    def evict(self, first=1, recent=2):
        """Blocks beyond the budget leave, not the first `first` and the last
        `recent` of those that may (as many as the budget holds)."""
        first = min(first, self.budget)
        self.cache.evict(self.budget, first, min(recent, self.budget - first))


def _places(pos):
    """Positions as the library takes them."""
    return pos.to(torch.int32).contiguous()


def _starts(lens):
    return torch.tensor(np.cumsum([0, *lens]), dtype=torch.int32, device="cuda")


def random_layer(seed, index, d, d_ff, rank, k, n16, n8, slots, n_seqs, n_heads, n_kv_heads,
                 max_tokens, max_batch=32, block_tokens=64, budget=0):
    """A layer of seeded random weights (the FFN's as workloads.py draws them)."""
    data = W.make_layer(seed, index, d, d_ff, rank, 1)
    ffn = m2c.Layer(m2c.make_desc(d, d_ff, rank, k, slots, max_batch=max_batch), data)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 131 + index)
    dim = d // n_heads
    weights = tuple(torch.empty(s, dtype=torch.float16, device="cuda").normal_(0.0, d ** -0.5, generator=g)
                    for s in ((d, (n_heads + 2 * n_kv_heads) * dim), (d, n_heads * dim)))
    return DecoderLayer(ffn, k, n16, n8, n_seqs, n_heads, n_kv_heads, max_tokens, weights,
                        block_tokens, budget)


def run(layers, prompts, tokens, chunk=256):
    """Prefill prompts [list of fp32 tensors [len][d]] in chunks and decode
    `tokens` steps, the last output row of a sequence its next input. Returns
    the decoded rows [tokens][sequences][d] and the sequences' lengths in the
    cache."""
    n = len(prompts)
    if any(p.shape[0] == 0 for p in prompts):
        raise ValueError("a prompt without tokens: decoding starts from a prompt's last row")
    done, last = [0] * n, [None] * n
    while any(done[b] < prompts[b].shape[0] for b in range(n)):
        lens = [min(chunk, prompts[b].shape[0] - done[b]) for b in range(n)]
        x = torch.cat([prompts[b][done[b]:done[b] + lens[b]] for b in range(n)])
        for layer in layers:
            layer.prefill(x, lens, done)
        at = 0
        for b, m in enumerate(lens):
            last[b] = x[at + m - 1] if m else last[b]
            at += m
            done[b] += m
    x, held, rows = torch.stack(last), list(done), []  # held: tokens in the cache
    pos = torch.tensor(done, dtype=torch.int32, device="cuda")
    block, budget = layers[0].cache.block_tokens, layers[0].budget
    for _ in range(tokens):
        x = x.clone()
        held = [m + 1 for m in held]
        for layer in layers:
            layer.decode(x, pos, max(held))
        pos += 1
        rows.append(x)
        if budget and max(held) > (budget + 1) * block:
            for layer in layers:
                layer.evict()
            held = [min(m, budget * block + (m - 1) % block + 1) for m in held]
    for layer in layers:
        layer.cache.check()
    return torch.stack(rows) if rows else x[None][:0], layers[0].cache.len.cpu().tolist()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--prompt", default="700,90,333", help="prompt lengths")
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--budget", type=int, default=6, help="blocks kept per sequence and head (0: all)")
    a = ap.parse_args(argv)
    if a.tokens < 0:
        ap.error(f"--tokens {a.tokens}: need 0 or more")
    wl = W.WORKLOADS["tiny"]
    k, n16, n8 = wl.counts()
    lens = [int(x) for x in a.prompt.split(",")]
    layers = [random_layer(wl.seed, i, wl.d_model, wl.d_ff, wl.pred_rank, k, n16, n8, wl.cache_slots(),
                           len(lens), 16, 4, max(lens) + a.tokens, budget=a.budget)
              for i in range(a.layers)]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    prompts = [torch.randn((n, wl.d_model), generator=g, device="cuda") for n in lens]
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    run(layers, prompts, min(a.tokens, 2))  # warm
    for layer in layers:
        layer.cache.reset()
    start.record()
    rows, held = run(layers, prompts, a.tokens)
    end.record()
    end.synchronize()
    c = layers[0].cache
    used = sum(-(-n // c.block_tokens) for n in held) * c.n_kv_heads * (2 * c.block_tokens * c.head_dim + 8)
    rms = f", last row's rms {float(rows[-1].square().mean().sqrt()):.3f}" if a.tokens else ""
    print(f"{a.layers} layers of d_model {wl.d_model}: prompts of {lens} tokens, {a.tokens} decoded in "
          f"{start.elapsed_time(end):.1f} ms; the cache holds {held} tokens per sequence "
          f"({used / 1e6:.2f} MB per layer){rms}")


if __name__ == "__main__":
    main()
