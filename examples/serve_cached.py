"""Serving attention blocks of a merged model with a paged 8-bit key/value cache.

Each block is the attention half of a decoder layer whose four projections are merged QA-LoRA layers (the adapters folded
into the zero points, so that deployment runs plain quantized layers):

    x -> normalise -> q, k, v (qalora_forward_group) -> rotate by position -> qalora_kv_append
      -> qalora_kv_attention -> output projection (qalora_forward) -> + x

A batch of prompts is read in one step, then every sequence grows by a token per step; when a sequence has more than
`limit` tokens in the cache, qalora_kv_evict keeps the `recent` last ones and those that gathered the most attention,
`budget` in all, and its old blocks go back to the pool.

    python examples/serve_cached.py
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2309_14717_b200 import binding as Q  # noqa: E402


@dataclass(frozen=True)
class Config:
    hidden: int = 4096
    heads: int = 32
    kv_heads: int = 32
    head_dim: int = 128
    blocks: int = 2              # decoder blocks
    group_size: int = 32
    bits: int = 4
    rank: int = 64
    adapter_scale: float = 1.0
    block_tokens: int = 64       # tokens of a cache block
    pool_blocks: int = 512
    max_tokens: int = 4096       # of one sequence in the cache
    limit: int = 1024            # a sequence longer than this is cut ...
    budget: int = 512            # ... to this many tokens,
    recent: int = 128            # the last of which stay whatever they gathered
    seed: int = 0


def make_weights(cfg: Config) -> list:
    """Per decoder block {name: (W fp32 [K, N], A, B bf16)} on the CPU: random weights and adapters."""
    g = torch.Generator().manual_seed(cfg.seed)
    wide, narrow = cfg.heads * cfg.head_dim, cfg.kv_heads * cfg.head_dim
    shapes = {"q": (cfg.hidden, wide), "k": (cfg.hidden, narrow), "v": (cfg.hidden, narrow), "o": (wide, cfg.hidden)}
    out = []
    for _ in range(cfg.blocks):
        out.append({name: (torch.randn(k, n, generator=g) * k ** -0.5,
                           (torch.randn(k // cfg.group_size, cfg.rank, generator=g) * 0.02).bfloat16(),
                           (torch.randn(cfg.rank, n, generator=g) * 0.02).bfloat16())
                    for name, (k, n) in shapes.items()})
    return out


def normalise(x: torch.Tensor) -> torch.Tensor:
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def rotate(x: torch.Tensor, position: torch.Tensor) -> torch.Tensor:
    """Rotates the pairs (c, c + dim / 2) of rows [m, heads, dim] by position * 10000^(-2 c / dim)."""
    half = x.shape[-1] // 2
    angle = position.float()[:, None] * 10000.0 ** (-torch.arange(half, device=x.device) / half)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(x.dtype)


class Layer:
    """A quantized layer with its adapter merged into the zero points."""

    def __init__(self, cfg: Config, W, A, B):
        k, n = W.shape
        trained = Q.desc(k, n, cfg.group_size, cfg.bits, cfg.rank, cfg.adapter_scale)
        self.desc = Q.desc(k, n, cfg.group_size, cfg.bits, 0, 0.0)
        self.codes, qparams = Q.alloc_packed(trained)
        self.qparams = torch.empty_like(qparams)
        Q.qalora_quantize(trained, W.cuda(), self.codes, qparams)
        Q.qalora_merge(trained, qparams, A.cuda(), B.cuda(), self.qparams)
        self.width = n

    def entry(self, x, y):
        return (self.desc, x, self.codes, self.qparams, None, None, y)


class Block:
    """The attention half of a decoder layer and its cache."""

    def __init__(self, cfg: Config, weights: dict):
        self.cfg = cfg
        self.layers = {name: Layer(cfg, *w) for name, w in weights.items()}
        self.kv = Q.kv_desc(cfg.heads, cfg.kv_heads, cfg.head_dim, cfg.block_tokens, cfg.pool_blocks)
        self.codes, self.scales, self.score = Q.alloc_kv_cache(self.kv)

    def forward(self, x, position, max_new, max_len, starts, lens, table, work):
        cfg, m = self.cfg, x.shape[0]
        h = normalise(x)
        y = {name: torch.empty(m, self.layers[name].width, dtype=torch.bfloat16, device=x.device) for name in "qkv"}
        group = Q.group_layers([self.layers[name].entry(h, y[name]) for name in "qkv"])
        scratch = torch.empty(max(Q.qalora_forward_group_workspace_bytes(group, m), 16), dtype=torch.uint8, device=x.device)
        Q.qalora_forward_group(group, m, scratch)
        q = rotate(y["q"].view(m, cfg.heads, cfg.head_dim), position)
        k = rotate(y["k"].view(m, cfg.kv_heads, cfg.head_dim), position)
        Q.qalora_kv_append(self.kv, max_new, starts, lens, table, k, y["v"].view(m, cfg.kv_heads, cfg.head_dim), self.codes,
                           self.scales, self.score)
        attended = torch.empty(m, cfg.heads, cfg.head_dim, dtype=torch.bfloat16, device=x.device)
        Q.qalora_kv_attention(self.kv, max_new, max_len, starts, lens, table, q, self.codes, self.scales, cfg.head_dim ** -0.5,
                              attended, score_in=self.score, score_out=self.score, workspace=work)
        out, o = torch.empty_like(x), self.layers["o"]
        Q.qalora_forward(o.desc, m, attended.view(m, -1), o.codes, o.qparams, None, None, out,
                         Q.alloc_workspace(o.desc, m, Q.OP_FORWARD))
        return x + out


class Server:
    """A batch of sequences; which blocks of the pool each holds is kept on the host and is the same for every decoder block."""

    def __init__(self, cfg: Config, batch: int, weights=None):
        self.cfg = cfg
        self.blocks = [Block(cfg, w) for w in (weights or make_weights(cfg))]
        self.free = list(range(cfg.pool_blocks))[::-1]
        self.held = [[] for _ in range(batch)]        # blocks of each sequence
        self.lens = [0] * batch                       # its tokens in the cache
        self.seen = [0] * batch                       # its tokens so far: positions
        self.max_blocks = -(-cfg.max_tokens // cfg.block_tokens)

    def _table(self, held):
        rows = [h + [-1] * (self.max_blocks - len(h)) for h in held]
        return torch.tensor(rows, dtype=torch.int32, device="cuda")

    def _take(self, tokens):
        return [self.free.pop() for _ in range(-(-tokens // self.cfg.block_tokens))]

    def step(self, x: torch.Tensor, new: list) -> torch.Tensor:
        """x bf16 [sum(new), hidden]: the next new[b] tokens of each sequence; returns the blocks' output."""
        position, starts = [], [0]
        for b, n in enumerate(new):
            position += range(self.seen[b], self.seen[b] + n)
            starts.append(starts[-1] + n)
            self.seen[b] += n
            self.lens[b] += n
            self.held[b] += self._take(self.lens[b] - len(self.held[b]) * self.cfg.block_tokens)
        as_int = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        # (one scratch for the step: the blocks' attention calls follow each other)
        work = Q.alloc_kv_workspace(self.blocks[0].kv, len(new), x.shape[0], max(new), max(self.lens), True)
        args = (max(new), max(self.lens), as_int(starts), as_int(self.lens), self._table(self.held), work)
        for block in self.blocks:
            x = block.forward(x, as_int(position), *args)
        return x

    def shorten(self) -> list | None:
        """Cuts the sequences that are longer than the limit; returns, per decoder block, which tokens were kept."""
        cfg = self.cfg
        long = [b for b, n in enumerate(self.lens) if n > cfg.limit]
        if not long:
            return None
        fresh = [self._take(cfg.budget) for _ in long]
        lens = torch.tensor([self.lens[b] for b in long], dtype=torch.int32, device="cuda")
        table, dst_table = self._table([self.held[b] for b in long]), self._table(fresh)
        dst_lens, all_kept = torch.empty_like(lens), []
        for block in self.blocks:
            kept = torch.empty(len(long), cfg.kv_heads, cfg.budget, dtype=torch.int32, device="cuda")
            Q.qalora_kv_evict(block.kv, max(self.lens), cfg.budget, cfg.recent, lens, table, block.codes, block.scales, block.score,
                              dst_table, dst_lens, kept)
            all_kept.append(kept)
        for b, blocks, n in zip(long, fresh, dst_lens.tolist()):
            self.free += self.held[b]
            self.held[b], self.lens[b] = blocks, n
        return all_kept


def main():
    cfg = Config()
    g = torch.Generator().manual_seed(1)
    new = [900, 500, 1020, 37]
    server = Server(cfg, len(new))
    hidden = lambda n: torch.randn(n, cfg.hidden, generator=g).bfloat16().cuda()  # noqa: E731
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    y = server.step(hidden(sum(new)), new)
    torch.cuda.synchronize()
    print(f"prompts of {new} tokens: output {tuple(y.shape)}, {sum(map(len, server.held))} blocks of {cfg.block_tokens} tokens held")
    start.record()
    steps, cut = 40, 0
    for _ in range(steps):
        y = server.step(hidden(len(new)), [1] * len(new))
        cut += server.shorten() is not None
    stop.record()
    torch.cuda.synchronize()
    assert torch.isfinite(y.float()).all()
    print(f"{steps} steps of one token each, {start.elapsed_time(stop) / steps:.2f} ms a step, {cut} evictions: lengths {server.lens}, "
          f"{sum(map(len, server.held))} blocks held")


if __name__ == "__main__":
    main()
