"""The serving example end to end on a small model: prompts, single-token steps and an eviction, against the whole path in
float64 (quantized layers, rotation, 8-bit cache, attention)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from conftest import ROOT, record_margin
from oracle import kv_oracle as KV
from oracle import qalora_oracle as O
from paper_2309_14717_b200 import binding as Q
from paper_2309_14717_b200.synthetic import to_f64

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("serve_cached", os.path.join(ROOT, "examples", "serve_cached.py"))
example = importlib.util.module_from_spec(spec)
# (a dataclass looks its module up by name)
import sys  # noqa: E402
sys.modules["serve_cached"] = example
spec.loader.exec_module(example)

CFG = example.Config(hidden=512, heads=4, kv_heads=2, head_dim=64, blocks=2, rank=16, block_tokens=16, pool_blocks=64, max_tokens=256,
                     limit=80, budget=48, recent=16, seed=3)
# Of a block's output, relative to its largest: bf16 roundings of the normalised input, of q, k, v, of the rotated q and
# k, of the attention's and the projection's outputs (2^-9 each, some of them twice in a score) and a code that a rounding
# of k or v moves by one (2^-8 of the largest); 2^-6 covers their sum.  The block's input is rounded once (2^-9) and
# dominates the output; the blocks' errors add up.
TOL = CFG.blocks * (2.0 ** -6 + 2.0 ** -9)


class Reference:
    def __init__(self, cfg, weights):
        self.cfg, self.blocks = cfg, []
        for w in weights:
            layers = {}
            for name, (W, A, B) in w.items():
                codes, alpha, beta = O.quantize(W.numpy(), cfg.group_size, cfg.bits)
                layers[name] = (codes, alpha, O.merge(beta, to_f64(A), to_f64(B), cfg.adapter_scale))
            shape = (cfg.pool_blocks, 2, cfg.kv_heads, cfg.block_tokens, cfg.head_dim)
            self.blocks.append({"layers": layers, "codes": np.zeros(shape, np.int8), "scales": np.zeros(shape[:3], np.float32),
                                "score": np.zeros((shape[0], shape[2], shape[3]))})

    def project(self, block, name, x):
        codes, alpha, beta = block["layers"][name]
        return O.forward(x, codes, alpha, beta, self.cfg.group_size)

    def rotate(self, x, position):
        half = x.shape[-1] // 2
        angle = np.asarray(position, dtype=np.float64)[:, None] * 10000.0 ** (-np.arange(half) / half)
        cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = x[..., :half], x[..., half:]
        return np.concatenate([a * cos - b * sin, a * sin + b * cos], -1)

    def step(self, x, position, starts, lens, table):
        cfg, m = self.cfg, len(x)
        for block in self.blocks:
            h = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + 1e-6)
            q, k, v = (self.project(block, n, h).reshape(m, -1, cfg.head_dim) for n in "qkv")
            q, k = self.rotate(q, position), self.rotate(k, position)
            KV.append(block["codes"], block["scales"], block["score"], starts, lens, table, k.astype(np.float32), v.astype(np.float32))
            r = KV.attention(block["codes"], block["scales"], starts, lens, table, q, cfg.head_dim ** -0.5, block["score"], True)
            block["score"] = r["score"]
            x = x + self.project(block, "o", r["out"].reshape(m, -1))
        return x


def test_prompts_steps_and_eviction():
    cfg, new = CFG, [70, 33, 1]
    weights = example.make_weights(cfg)
    server, ref = example.Server(cfg, len(new), weights), Reference(cfg, weights)
    g = torch.Generator().manual_seed(5)
    launches, cut = Q.qalora_kernel_launches(), 0
    for t in range(14):
        x = torch.randn(sum(new), cfg.hidden, generator=g).bfloat16()
        position = [p for b, n in enumerate(new) for p in range(server.seen[b], server.seen[b] + n)]
        y = server.step(x.cuda(), new)
        starts, table = np.cumsum([0] + new), server._table(server.held).cpu().numpy()
        want = ref.step(to_f64(x), position, starts, np.array(server.lens), table)
        got = y.float().cpu().numpy()
        record_margin("serve_example", "y", float(np.abs(got - want).max() / np.abs(want).max()), TOL)
        lens_before = list(server.lens)
        kept = server.shorten()
        if kept is not None:
            cut += 1
            b = [i for i, n in enumerate(lens_before) if n > cfg.limit]
            new_table = server._table(server.held).cpu().numpy()
            for block, picked in zip(ref.blocks, kept):
                picked = picked.cpu().numpy()
                # what the device kept is what gathered most, up to the error of the weights; its choice is then taken over
                for i, seq in enumerate(b):
                    slots = np.arange(lens_before[seq])
                    blk = table[seq][slots // cfg.block_tokens]
                    for h in range(cfg.kv_heads):
                        s = block["score"][blk, h, slots % cfg.block_tokens].copy()
                        inside = np.zeros(len(s), bool)
                        inside[picked[i, h]] = True
                        assert inside.sum() == cfg.budget and inside[-cfg.recent:].all()
                        assert s[inside][:-cfg.recent].min() >= s[~inside].max() - 0.1 * s.max()
                        block["score"][blk, h, slots % cfg.block_tokens] = np.where(inside, 1.0 + s, 0.0)
                KV.evict(block["codes"], block["scales"], block["score"], np.array(lens_before)[b], table[b], cfg.budget, cfg.recent,
                         new_table[b])
                for i, seq in enumerate(b):
                    slots = np.arange(cfg.budget)
                    blk = new_table[seq][slots // cfg.block_tokens]
                    block["score"][blk, :, slots % cfg.block_tokens] -= 1.0
            assert [server.lens[i] for i in b] == [cfg.budget] * len(b)
        new = [1, 1, 1]
    assert cut >= 1, "no sequence was cut"
    held = [x for h in server.held for x in h]
    assert len(set(held) | set(server.free)) == cfg.pool_blocks == len(held) + len(server.free), "blocks lost or held twice"
    assert Q.qalora_kernel_launches() > launches
