"""Sizes at which the cache operators change their division of the work: evictions of many blocks (more pieces than the GPU
holds at once) for every block size, selections by few threads of many pairs, prompts that fill every block size, and
attention of sequences on both sides of the rule that gives each thread block a whole one.  Bounds as in
test_kv_cache_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from paper_2309_14717_b200 import binding as Q
from test_kv_cache_gpu import Cache, attend, bf16, check, dev, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,budget,recent,kv_heads,dim,block", [
    ([1300, 1200, 1100, 1290], 1000, 100, 8, 128, block) for block in (16, 32, 64, 128)] + [
    ([2300, 2200, 2100, 2290], 2000, 7, 8, 64, block) for block in (16, 32, 64, 128)] + [
    ([3000, 2900, 2800, 2700], 400, 33, 40, 64, 16), ([3000, 500, 401, 400], 400, 0, 40, 128, 32)])
def test_evict_of_many_blocks_is_bit_exact(lens, budget, recent, kv_heads, dim, block):
    rng = np.random.default_rng(dim + block)
    width = -(-budget // block)
    c = Cache(rng, lens, kv_heads, kv_heads, dim, block, spare=len(lens) * width)
    dst = c.free[:len(lens) * width].reshape(len(lens), width)
    codes, scales, score = c.up()
    dst_lens = torch.full((len(lens),), -5, dtype=torch.int32, device="cuda")
    kept = torch.full((len(lens), kv_heads, budget), -5, dtype=torch.int32, device="cuda")
    Q.qalora_kv_evict(c.d, max(lens), budget, recent, dev(c.lens), dev(c.table), codes, scales, score, dev(dst), dst_lens, kept)
    torch.cuda.synchronize()
    want_lens, want_kept = K.evict(c.codes, c.scales, c.score, c.lens, c.table, budget, recent, dst)
    assert np.array_equal(dst_lens.cpu().numpy(), want_lens)
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(scales.cpu().numpy(), c.scales)
    assert np.array_equal(codes.cpu().numpy(), c.codes)
    assert np.array_equal(score.cpu().numpy(), c.score)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_append_and_read_of_prompts(block, dim):
    rng, new, kv_heads = np.random.default_rng(block + dim), [300, 1, 129, 0], 3
    c = Cache(rng, [305, 1, 129, 40], kv_heads, kv_heads, dim, block)
    k, v = (bf16(rng.standard_normal((sum(new), kv_heads, dim))).astype(np.float32) for _ in range(2))
    codes, scales, score = c.up()
    starts = dev(starts_of(new))
    Q.qalora_kv_append(c.d, max(new), starts, dev(c.lens), dev(c.table), dev(k).bfloat16(), dev(v).bfloat16(), codes, scales, score)
    got = [torch.full((sum(new), kv_heads, dim), float("nan"), device="cuda") for _ in range(2)]
    first = np.array([5, 0, 0, 40], np.int32)
    Q.qalora_kv_read(c.d, max(new), starts, dev(first), dev(c.table), codes, scales, *got)
    torch.cuda.synchronize()
    K.append(c.codes, c.scales, c.score, starts_of(new), c.lens, c.table, k, v)
    assert np.array_equal(scales.cpu().numpy(), c.scales)
    assert np.array_equal(codes.cpu().numpy(), c.codes)
    assert np.array_equal(score.cpu().numpy(), c.score)
    for which, t in enumerate(got):
        for b, n in enumerate(new):
            for h in range(kv_heads):
                want = K.read(c.codes, c.scales, c.table, b, h, which, range(first[b], first[b] + n)) if n else np.zeros((0, dim))
                rows = t[starts_of(new)[b]:starts_of(new)[b] + n, h].double().cpu().numpy()
                assert np.array_equal(rows, want.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,block", [
    ([512], [1], 4, 4, 128, 64), ([513], [1], 4, 4, 128, 64), ([1024, 900], [1, 1], 4, 4, 128, 32), ([2049, 30], [1, 1], 8, 2, 64, 128),
    ([1025, 0, 70], [3, 2, 3], 20, 5, 128, 16), ([600] * 9 + [1], [1] * 10, 32, 32, 64, 64), ([900, 33, 1000, 1024] * 3, [1] * 12, 32, 32, 128, 64),
    ([300, 320, 7], [4, 4, 4], 16, 4, 64, 16), ([321, 5], [2, 2], 12, 2, 128, 128),
])
@pytest.mark.parametrize("scores", [False, True])
def test_few_rows_whole_or_in_even_shares(lens, new, heads, kv_heads, dim, block, scores):
    rng = np.random.default_rng(sum(lens) + heads)
    c = Cache(rng, lens, heads, kv_heads, dim, block)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    out, lse, got, _ = attend(c, q, new, dim ** -0.5, scores)
    check(c, q, new, dim ** -0.5, out, lse, got, c.score)


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,block", [
    ([1500], [700], 8, 1, 64, 128), ([1300, 300, 9], [600, 20, 9], 8, 1, 128, 32), ([700], [700], 16, 2, 128, 64),
    ([515, 0, 130], [515, 3, 130], 12, 3, 64, 16), ([2100], [260], 5, 1, 128, 16),
])
def test_gathered_weights_of_prompts_with_few_heads(lens, new, heads, kv_heads, dim, block):
    """(clusters of 8, 4 and 2 thread blocks share the rows of a token tile, some of them without a row tile)"""
    rng = np.random.default_rng(sum(lens) + heads)
    c = Cache(rng, lens, heads, kv_heads, dim, block)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    out, lse, got, _ = attend(c, q, new, dim ** -0.5, True)
    check(c, q, new, dim ** -0.5, out, lse, got, c.score)
    assert torch.equal(attend(c, q, new, dim ** -0.5, True)[2], got)
