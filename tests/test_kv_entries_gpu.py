"""Device-side entries that break a call's bounds: no access outside the buffers, and the other sequences' results stay."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from paper_2309_14717_b200 import binding as Q
from test_kv_cache_gpu import Cache, bf16, check, dev, starts_of

pytestmark = pytest.mark.gpu

LARGEST, LEAST = 2 ** 31 - 1, -2 ** 31


@pytest.mark.parametrize("first", [LARGEST, LARGEST - 40, LEAST, -200, -7, 40, 64, 100000])
@pytest.mark.parametrize("block", [16, 128])
def test_read_from_any_position(first, block):
    rng, n, kv_heads, dim = np.random.default_rng(1), 70, 2, 64
    c = Cache(rng, [64, 64], kv_heads, kv_heads, dim, block)
    room = c.table.shape[1] * block
    codes, scales, _ = c.up()
    out = [torch.full((2 * n, kv_heads, dim), 7.0, device="cuda") for _ in range(2)]
    Q.qalora_kv_read(c.d, n, dev(starts_of([n, n])), dev(np.array([first, 0], np.int32)), dev(c.table), codes, scales, *out)
    torch.cuda.synchronize()
    for which, t in enumerate(out):
        for b, start in enumerate([first, 0]):
            there = [i for i in range(n) if 0 <= start + i < room]
            want = np.full((n, kv_heads, dim), 7.0, np.float32)
            for h in range(kv_heads):
                if there:
                    want[there, h] = K.read(c.codes, c.scales, c.table, b, h, which, [start + i for i in there])
            assert np.array_equal(t[b * n:(b + 1) * n].cpu().numpy(), want)


@pytest.mark.parametrize("length", [LARGEST, LEAST, -1])
def test_append_of_any_length(length):
    rng, n, dim, block = np.random.default_rng(2), 20, 128, 16
    c = Cache(rng, [n, 32, n], 1, 1, dim, block)
    codes, scales, score = c.up()
    k = bf16(rng.standard_normal((3 * n, 1, dim))).astype(np.float32)
    lens = c.lens.copy()
    lens[1] = length
    Q.qalora_kv_append(c.d, n, dev(starts_of([n] * 3)), dev(lens), dev(c.table), dev(k).bfloat16(), dev(k).bfloat16(), codes, scales, score)
    torch.cuda.synchronize()
    own = set(int(x) for x in c.table[1])                          # (this sequence's blocks are unspecified, all others are not)
    keep = [i for i in range(c.blocks) if i not in own]
    rows = np.concatenate([k[:n], k[2 * n:]])
    K.append(c.codes, c.scales, c.score, starts_of([n, n]), c.lens[[0, 2]], c.table[[0, 2]], rows, rows)
    assert np.array_equal(codes.cpu().numpy()[keep], c.codes[keep])
    assert np.array_equal(scales.cpu().numpy()[keep], c.scales[keep])


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("length", [LARGEST, LEAST, -1])
@pytest.mark.parametrize("n", [1, 70])                             # few rows, and tiles of 128
def test_attention_of_any_length(n, length, scores):
    rng, heads, kv_heads, dim = np.random.default_rng(3), 4, 2, 128
    c = Cache(rng, [n + 30, n + 60, n], heads, kv_heads, dim, 32)
    q, new = bf16(rng.standard_normal((3 * n, heads, dim))), [n] * 3
    lens = c.lens.copy()
    lens[1] = length
    codes, scales, score = c.up()
    out = torch.zeros((3 * n, heads, dim), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((3 * n, heads), device="cuda")
    got = torch.full_like(score, -7.0) if scores else None
    longest = int(c.lens.max())
    ws = Q.alloc_kv_workspace(c.d, 3, 3 * n, n, longest, scores)
    Q.qalora_kv_attention(c.d, n, longest, dev(starts_of(new)), dev(lens), dev(c.table), dev(q).bfloat16(), codes, scales, dim ** -0.5,
                          out, lse, score if scores else None, got, ws)
    torch.cuda.synchronize()
    assert Q.workspace_status(ws) == 0
    if length < 0:                                                 # (no tokens: rows that attend to nothing)
        assert not out[n:2 * n].any() and torch.isneginf(lse[n:2 * n]).all()
    rows = np.r_[0:n, 2 * n:3 * n]
    at = torch.as_tensor(rows, device="cuda")
    if scores:
        got[dev(c.table[1], dtype=torch.long)] = -7.0              # (its own blocks are unspecified)
    c.lens, c.table = c.lens[[0, 2]], c.table[[0, 2]]
    check(c, q[rows], [n, n], dim ** -0.5, out[at], lse[at], got, c.score)


@pytest.mark.parametrize("length", [LARGEST, LEAST])
def test_evict_of_any_length(length):
    rng, kv_heads, dim, block, budget, recent = np.random.default_rng(4), 2, 64, 16, 24, 8
    c = Cache(rng, [50, 50, 50], kv_heads, kv_heads, dim, block, spare=6)
    dst = c.free[:6].reshape(3, 2).astype(np.int32)
    codes, scales, score = c.up()
    dst_lens, kept = torch.full((3,), -9, dtype=torch.int32, device="cuda"), torch.full((3, kv_heads, budget), -9, dtype=torch.int32, device="cuda")
    lens = c.lens.copy()
    lens[1] = length
    Q.qalora_kv_evict(c.d, 50, budget, recent, dev(lens), dev(c.table), codes, scales, score, dev(dst), dst_lens, kept)
    torch.cuda.synchronize()
    want = 50 if length > 0 else 0                                 # (a length above max_len counts as max_len)
    n = [24, min(want, 24), 24]
    assert dst_lens.cpu().tolist() == n
    kept = kept.cpu().numpy()
    for b in range(3):
        for h in range(kv_heads):
            assert (kept[b, h, n[b]:] == -1).all()
            if n[b]:
                s = np.array([c.score[c.table[b, t // block], h, t % block] for t in range(50)])
                best = sorted(np.argsort(-s[:42], kind="stable")[:16].tolist()) + list(range(42, 50))
                assert kept[b, h].tolist() == best
