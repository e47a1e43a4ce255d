"""Attention over the 8-bit cache where a call's rows, tokens or numbers lie at an edge.  Bounds as in
test_kv_cache_gpu.py unless a test states its own."""
import numpy as np
import pytest
import torch

from test_kv_cache_gpu import Cache, attend, bf16, check

pytestmark = pytest.mark.gpu

NAN = float("nan")


# ------------------------------------------------------------------- row tiles without a product
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scores", [False, True])
def test_row_tiles_of_absent_rows(dim, scores):
    """Rows before a sequence's first token: zeros and -infinity, whatever their queries and their neighbours' hold."""
    rng = np.random.default_rng(dim)
    lens, new = [0, 90, 5, 300], [700, 600, 130, 300]
    c = Cache(rng, lens, 4, 2, dim, 32)
    q = bf16(rng.standard_normal((sum(new), 4, dim)))
    want, want_lse, want_score, _ = attend(c, q, new, 0.1, scores)
    check(c, q, new, 0.1, want, want_lse, want_score, c.score)
    starts, bad = np.concatenate([[0], np.cumsum(new)]), q.copy()
    for b in range(4):
        for i in range(new[b] - lens[b]):                     # (absent rows only)
            if i % 3 == 0:
                bad[starts[b] + i] = NAN
    for _ in range(5):
        out, lse, score, _ = attend(c, bad, new, 0.1, scores)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert not scores or torch.equal(score, want_score)


@pytest.mark.parametrize("heads,kv_heads,dim,n", [(8, 8, 128, 1000), (4, 2, 128, 900), (8, 8, 64, 1000)])
def test_parts_of_a_prompt_that_a_row_tile_does_not_see(heads, kv_heads, dim, n):
    """Few row tiles and many tokens: the tokens are cut into parts, and the first row tiles see none of the later ones.
    Queries of NaN spoil their own rows alone."""
    rng = np.random.default_rng(n + dim)
    c = Cache(rng, [n], heads, kv_heads, dim, 64)
    q = bf16(rng.standard_normal((n, heads, dim)))
    want, want_lse, _, _ = attend(c, q, [n], 0.1)
    check(c, q, [n], 0.1, want, want_lse)
    spoilt = np.arange(5, n, 16)                              # in every quarter of every row tile
    bad = q.copy()
    bad[spoilt] = NAN
    at = torch.as_tensor(spoilt, device="cuda")
    for _ in range(5):
        out, lse, _, _ = attend(c, bad, [n], 0.1)
        assert torch.isnan(out[at].float()).all()
        # (a row of NaN changes when the other rows of its warp move to a new maximum: their last bits, within the bounds)
        out[at], lse[at] = want[at], want_lse[at]
        check(c, q, [n], 0.1, out, lse)


@pytest.mark.parametrize("heads,kv_heads,dim,n,cached", [(2, 2, 128, 400, 3000), (4, 2, 64, 300, 4000)])
def test_long_prompts_repeat_their_bits(heads, kv_heads, dim, n, cached):
    """Many steps of scores that follow weights in the same place of tensor memory."""
    rng = np.random.default_rng(cached)
    c = Cache(rng, [cached + n, cached], heads, kv_heads, dim, 64)
    q = bf16(rng.standard_normal((2 * n, heads, dim)))
    want, want_lse, _, _ = attend(c, q, [n, n], 0.1)
    check(c, q, [n, n], 0.1, want, want_lse)
    for _ in range(10):
        out, lse, _, _ = attend(c, q, [n, n], 0.1)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
