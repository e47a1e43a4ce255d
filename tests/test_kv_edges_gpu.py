"""Attention over the 8-bit cache where a call's rows, tokens or numbers lie at an edge.  Bounds as in
test_kv_cache_gpu.py unless a test states its own."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from paper_2309_14717_b200 import binding as Q
from test_kv_cache_gpu import Cache, attend, bf16, check, dev, starts_of

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


# --------------------------------------------------------------------- m as a bound of the rows
def attend_bounded(c, q, new, m, max_new, max_len, scale, scores, starts=None):
    """As attend(), with `m` rows of q, out and lse of which the sequences have the first sum(new); the others hold NaN
    queries and must stay as they are."""
    used = sum(new)
    rows = torch.full((m, c.d.heads, c.d.head_dim), NAN, dtype=torch.bfloat16, device="cuda")
    rows[:used] = dev(q).bfloat16()
    codes, scales, score = c.up()
    out = torch.full((m, c.d.heads, c.d.head_dim), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((m, c.d.heads), 9.0, device="cuda")
    got = torch.full_like(score, -7.0) if scores else None
    ws = Q.alloc_kv_workspace(c.d, len(new), m, max_new, max_len, scores)
    ws.fill_(0xFF)
    Q.qalora_kv_attention(c.d, max_new, max_len, dev(starts_of(new) if starts is None else starts), dev(c.lens), dev(c.table), rows, codes,
                          scales, scale, out, lse, score if scores else None, got, ws)
    torch.cuda.synchronize()
    assert Q.workspace_status(ws) == 0
    assert (out[used:] == 9).all() and (lse[used:] == 9).all()
    return out[:used], lse[:used], got


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,m,max_new", [
    ([70, 3, 200, 129] * 6, [1] * 24, 4, 4, 128, 32, 1), ([70, 3, 200, 129] * 6, [1] * 24, 4, 4, 128, 25, 1),       # a padded batch of tokens
    ([90], [1], 8, 2, 64, 2, 1), ([90], [3], 8, 2, 64, 100, 100), ([90], [3], 8, 2, 128, 4, 4),                     # one sequence
    ([50, 60, 70, 80], [1, 2, 3, 4], 4, 1, 128, 256, 64), ([50, 60, 70, 80], [1, 0, 3, 0], 4, 4, 64, 256, 64),      # far below the bounds
    ([150, 90], [100, 5], 4, 4, 128, 200, 100), ([150, 90, 33], [5, 90, 1], 4, 2, 64, 300, 100),                    # prompts and tokens
    ([40, 77, 9], [4, 4, 4], 2, 2, 128, 64, 4), ([40, 77, 9], [17, 2, 1], 2, 2, 128, 64, 17), ([0, 5], [2, 1], 2, 1, 64, 40, 20),
])
def test_rows_below_their_bounds(lens, new, heads, kv_heads, dim, m, max_new, scores):
    rng = np.random.default_rng(m + max_new)
    c = Cache(rng, lens, heads, kv_heads, dim, 32)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    out, lse, got = attend_bounded(c, q, new, m, max_new, max(lens), 0.1, scores)
    check(c, q, new, 0.1, out, lse, got, c.score)


@pytest.mark.parametrize("scores", [False, True])
def test_a_sequence_that_breaks_its_bounds_leaves_its_neighbours(scores):
    """starts that fall make one sequence's rows unspecified; short and long neighbours are answered all the same."""
    rng = np.random.default_rng(5)
    heads, kv_heads, dim, new = 4, 2, 128, [3, 0, 40]
    c = Cache(rng, [60, 50, 90], heads, kv_heads, dim, 32)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    out, lse, got = attend_bounded(c, q, new, 43, 40, 90, 0.1, scores, np.array([0, 3, 3, 43], np.int32))
    check(c, q, new, 0.1, out, lse, got, c.score)
    c.lens = np.array([60, 50, 90, 70], np.int32)              # the third has rows 50 .. 3: none
    c.table = np.concatenate([c.table, c.table[1:2]])
    new = [3, 47, 0, 0]
    q = bf16(rng.standard_normal((50, heads, dim)))
    starts = np.array([0, 3, 50, 3, 3], np.int32)
    out, lse, got = attend_bounded(c, q, new, 100, 60, 90, 0.1, scores, starts)
    c.lens, c.table = c.lens[:2], c.table[:2]
    check(c, q, new[:2], 0.1, out, lse, got, c.score)


def test_captured_attention_replays_with_other_rows():
    """One graph for any rows within its bounds: starts and lens change between replays."""
    rng = np.random.default_rng(6)
    heads, kv_heads, dim, m, max_new, max_len = 4, 2, 128, 96, 64, 300
    c = Cache(rng, [300, 300, 300, 300], heads, kv_heads, dim, 32)
    (codes, scales, score), table = c.up(), dev(c.table)
    q = torch.zeros((m, heads, dim), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros((m, heads, dim), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, heads), device="cuda")
    starts, lens = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    got = torch.zeros_like(score)
    ws = Q.alloc_kv_workspace(c.d, 4, m, max_new, max_len, True)

    def step():
        Q.qalora_kv_attention(c.d, max_new, max_len, starts, lens, table, q, codes, scales, 0.1, out, lse, score, got, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for new, length in ([[1, 1, 1, 1], [300, 20, 1, 77]], [[64, 1, 9, 0], [64, 300, 150, 3]], [[0, 0, 30, 2], [10, 0, 30, 5]], [[17, 16, 33, 8], [200] * 4]):
        c.lens = np.array(length, np.int32)
        rows = bf16(rng.standard_normal((sum(new), heads, dim)))
        q.fill_(NAN), out.fill_(9), lse.fill_(9), got.fill_(-7)
        q[:sum(new)] = dev(rows).bfloat16()
        starts.copy_(dev(starts_of(new))), lens.copy_(dev(c.lens))
        graph.replay()
        torch.cuda.synchronize()
        assert (out[sum(new):] == 9).all()
        check(c, rows, new, 0.1, out[:sum(new)], lse[:sum(new)], got, c.score)


# ------------------------------------------------------------------ value scales anywhere in float32
def check_values(c, q, new, scale, out, lse):
    """Bounds that follow the values a row weights: 2^-8 |out| (bf16), 2^-10 + 2^-16 + 2 d of sum weight |value| (weights in fp16;
    an exponent of up to 150 added to a score in float32; d as in test_kv_cache_gpu.py), 2^-26 of the largest weight * value scale for
    each token (a weighted scale is at least 2^8 for the largest, and fp16 numbers are 2^-24 apart at the least; codes go to 127),
    127 * 2^-80 of the largest value scale (with many rows, smaller ones count as zeros) and 2^-133 (the least bf16 number)."""
    T, group, row = c.codes.shape[3], c.d.heads // c.d.kv_heads, 0
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, n in enumerate(new):
        for i in range(n):
            t = np.arange(int(c.lens[b]) - n + i + 1)
            blk = c.table[b][t // T]
            if not len(t):                                      # (a row before the first token)
                assert (o[row] == 0).all() and np.isneginf(l[row]).all()
                row += 1
                continue
            for h in range(c.d.heads):
                kv = h // group
                key, val = (c.codes[blk, w, kv, t % T].astype(np.float64) * c.scales[blk, w, kv].astype(np.float64)[:, None] for w in (0, 1))
                s = scale * (key @ q[row, h])
                d = 2.0 ** -18 * (1 + scale * (np.abs(key) @ np.abs(q[row, h])).max())
                w = np.exp(s - s.max())
                total = w.sum()
                w /= total
                want, spread = w @ val, w @ np.abs(val)
                tol = (2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 ** -16 + 2 * d) * spread
                       + len(t) * 2.0 ** -26 * (w * c.scales[blk, 1, kv]).max() + 2.0 ** -133)
                if n * group > 16:
                    tol = tol + 127 * 2.0 ** -80 * np.float64(c.scales[:, 1].max())
                assert np.isfinite(o[row, h]).all()
                assert (np.abs(o[row, h] - want) <= tol).all(), (b, i, h, (np.abs(o[row, h] - want) / tol).max())
                norm = s.max() + np.log(total)
                assert abs(l[row, h] - norm) <= d + 2.0 ** -22 * abs(norm)
            row += 1


# lens, new, heads, kv_heads: few rows; tiles of 128; tiles whose tokens are cut into parts
ROWS_OF = {"few": ([150, 40, 97], [1, 4, 3], 4, 2), "prompt": ([400, 150], [140, 20], 4, 2), "parts": ([900], [70], 2, 2)}


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("form", ["few", "prompt", "parts"])
@pytest.mark.parametrize("values", ["subnormal", "subnormal and zero", "tiny, then ordinary", "ordinary, then tiny", "largest", "both ends", "zero"])
def test_value_scales_at_the_ends_of_float32(values, form, dim):
    lens, new, heads, kv_heads = ROWS_OF[form]
    rng = np.random.default_rng(dim + len(values))
    c = Cache(rng, lens, heads, kv_heads, dim, 16)
    v = c.scales[:, 1]                                          # [blocks][kv_heads], by place in the sequence below
    place = np.zeros(c.blocks, int)
    for row in c.table:
        place[row] = np.arange(len(row))
    even = (place % 2 == 0)[:, None]
    v[:] = {"subnormal": 1e-41 * v, "subnormal and zero": np.where(even, 3e-39 * v, 0), "tiny, then ordinary": np.where(place[:, None] < 2, 1e-40, v),
            "ordinary, then tiny": np.where(place[:, None] < 2, v, 1e-37), "largest": 2.6e36 / v.max() * v,
            "both ends": np.where(even, 2.6e36, 1e-44), "zero": 0 * v}[values].astype(np.float32)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    out, lse, _, _ = attend(c, q, new, 0.05)
    check_values(c, q, new, 0.05, out, lse)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("form", ["few", "prompt", "parts"])
@pytest.mark.parametrize("run", [1, 8])
@pytest.mark.parametrize("power", [-20, -25, -30, -38])
def test_weight_on_values_far_below_the_largest(power, run, form, dim):
    """Rows that attend sharply to blocks whose value scale is 2^power of the others': runs of them before, between and behind
    the others (a run of 8 is a tile of 128 tokens)."""
    lens, new, heads, kv_heads = ROWS_OF[form]
    rng = np.random.default_rng(dim - power)
    c = Cache(rng, lens, heads, kv_heads, dim, 16)
    for row in c.table:
        small = np.arange(len(row)) // run % 2 == 0
        c.scales[row[small], 1] *= np.float32(2.0 ** power)
        c.scales[row[~small], 0] *= np.float32(0.01)            # their keys are short ...
        c.codes[row[small], 0, :, :, 0] = 100                   # ... and the others' agree with the queries
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    q[..., 0] = 64.0
    out, lse, _, _ = attend(c, q, new, 1.0)
    check_values(c, q, new, 1.0, out, lse)


@pytest.mark.parametrize("n", [1, 3, 40])
def test_attention_over_what_append_stores_at_the_extremes(n):
    """Zeros, subnormals and the largest numbers as values, stored by append and read by attention in one sequence."""
    rng = np.random.default_rng(9)
    heads, kv_heads, dim, length = 4, 2, 64, 90
    c = Cache(rng, [length], heads, kv_heads, dim, 16)
    codes, scales, score = c.up()
    v = torch.randn((length, kv_heads, dim), generator=torch.Generator().manual_seed(3))
    v[:16], v[16:32], v[32:48], v[48:64] = v[:16] * 1e-39, 0, v[32:48].sign() * 3.3e38, v[48:64] * 1e-36
    k = torch.randn((length, kv_heads, dim), generator=torch.Generator().manual_seed(4))
    Q.qalora_kv_append(c.d, length, dev(starts_of([length])), dev(c.lens), dev(c.table), k.bfloat16().cuda(), v.bfloat16().cuda(), codes, scales)
    torch.cuda.synchronize()
    c.codes, c.scales = codes.cpu().numpy(), scales.cpu().numpy()
    for length in (10, 30, 45, 60, 90):
        c.lens = np.array([length], np.int32)
        q = bf16(rng.standard_normal((n, heads, dim)))
        out, lse, _, _ = attend(c, q, [n], 0.125)
        check_values(c, q, [n], 0.125, out, lse)


# ------------------------------------------------------------------------ NaN, and weights of zero
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,bad", [
    ([200], [200], 4, 2, 128, range(0, 200, 29)), ([200], [200], 4, 2, 128, [7]), ([200], [200], 2, 2, 64, [6]), ([200], [200], 2, 2, 64, [5]),
    ([500, 300], [90, 120], 2, 1, 128, [13, 150]), ([90], [20], 4, 1, 64, [3]),                                     # tiles of rows
    ([1100], [100], 2, 2, 128, [31, 70]),                                                                            # cut into parts
    ([200, 64, 30], [3, 2, 4], 4, 2, 128, [1, 3, 7]), ([900], [8], 2, 2, 64, [4]), ([40] * 3, [5] * 3, 3, 3, 128, [0, 9, 14]),   # few rows
])
def test_a_query_of_nan_spoils_the_weights_of_what_it_sees(lens, new, heads, kv_heads, dim, bad):
    rng = np.random.default_rng(sum(lens) + dim)
    c = Cache(rng, lens, heads, kv_heads, dim, 32)
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    for i in bad:
        q[i, i % heads, i % dim] = NAN
    with np.errstate(invalid="ignore"):
        r = K.attention(c.codes, c.scales, starts_of(new), c.lens, c.table, q, 0.1, c.score, True)
    assert np.isnan(r["score"]).any() and np.isfinite(r["score"]).any()
    out, lse, got, _ = attend(c, q, new, 0.1, True)
    got, mine = got.double().cpu().numpy(), np.zeros(c.score.shape, bool)
    for b, n in enumerate(c.lens):
        t = np.arange(int(n))
        mine[c.table[b][t // 32], :, t % 32] = True
    assert (np.isnan(got) == (np.isnan(r["score"]) & mine)).all()
    fine = mine & ~np.isnan(got)
    d = 2.0 ** -18 * (1 + np.nanmax(r["reach"]))
    assert (np.abs(got - r["score"])[fine] <= (d * (r["score"] - c.score) + 2.0 ** -22 * r["score"] + 1e-30)[fine]).all()
    assert (np.isnan(lse.cpu().numpy()) == np.isnan(r["lse"])).all()
    assert (np.isnan(out.float().cpu().numpy()) == np.isnan(r["out"])).all()


@pytest.mark.parametrize("lens,new,dim", [([260], [260], 128), ([500], [70], 64), ([1100], [40], 128), ([300, 90], [4, 9], 64)])
def test_tokens_without_weight_gather_nothing(lens, new, dim):
    """Sharp scores: a token whose weights are all below 2^-150 keeps its score, and with none before it has exactly 0."""
    rng = np.random.default_rng(dim)
    c = Cache(rng, lens, 2, 2, dim, 16)
    for row in c.table:
        c.codes[row[::3], 0, :, :, 0] = -127
    q = bf16(rng.standard_normal((sum(new), 2, dim)))
    q[..., 0] = 400.0
    r = K.attention(c.codes, c.scales, starts_of(new), c.lens, c.table, q, 1.0, None, True)
    none = (r["score"] > 0) & (r["score"] < 2.0 ** -150)
    assert none.sum() > 50
    for score_in in (False, True):
        _, _, got, before = attend(c, q, new, 1.0, True, score_in=score_in)
        assert torch.equal(got[dev(none)], before[dev(none)] if score_in else torch.zeros_like(got[dev(none)]))


@pytest.mark.parametrize("places", [(6, 7), (0, 1, 2, 3, 4, 5)])
def test_exponentials_of_gathered_weights(places):
    """Rows at `places` of eight weight the tokens mildly, the others only token 0: a token gathers the exponentials of the former,
    which with many rows are polynomials on the FMA pipe for places 6 and 7 and the exponential unit's for the others.  How the
    weights of the tokens relate to each other knows nothing of the rows' sums.  Its bound, twice (a token and the mean):
    ln 2 * (4 * 2^-24 for a score within +-1 after four roundings + 2^-21 for score minus logarithm, within 8 .. 16) + 2^-22
    (either exponential) + 2^-24 for each row that is added."""
    dim, n, cached = 64, 24, 256
    c = Cache(np.random.default_rng(1), [n + cached], 1, 1, dim, 16)
    c.codes[:, 0] = 0
    rng = np.random.default_rng(2)
    for t in range(n + cached):
        c.codes[c.table[0, t // 16], 0, 0, t % 16, 0] = rng.integers(-127, 128)
    c.codes[c.table[0, 0], 0, 0, 0, 1] = 127
    c.scales[:, 0] = np.float32(1 / 127)
    mild = [i for i in range(n) if i % 8 in places]
    q = np.zeros((n, 1, dim))
    q[:, 0, 1], q[mild, 0, 1], q[mild, 0, 0] = 200.0, 0.0, 0.6875
    r = K.attention(c.codes, c.scales, starts_of([n]), c.lens, c.table, q, 1.0, None, True)
    _, _, got, _ = attend(c, q, [n], 1.0, True, score_in=False)
    t = np.arange(1, cached)
    ratio = got.double().cpu().numpy()[c.table[0][t // 16], 0, t % 16] / r["score"][c.table[0][t // 16], 0, t % 16]
    assert np.abs(ratio / ratio.mean() - 1).max() <= 2 * (np.log(2) * (2.0 ** -22 + 2.0 ** -21) + 2.0 ** -22 + len(mild) * 2.0 ** -24)


# ------------------------------------------------------------------------- scores of any magnitude
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("heads,dim,new,power", [(1, 64, 1, 110), (2, 128, 3, 110), (1, 64, 50, 12), (2, 128, 50, 12), (1, 64, 50, 110),
                                                 (2, 128, 50, 110), (1, 128, 50, 24)])
def test_scores_far_beyond_any_weight(heads, dim, new, power, sign):
    """Scores of +-2^power * 64 .. 123: every row weights one token alone (no two have the same score), the first row its only
    one.  What a row gives its token is 1; with many rows but for its score's rounding, 2^-22 of it after four operations, and 0
    with scores beyond 2^24."""
    rng = np.random.default_rng(dim + new)
    for length in (new, 55):
        c = Cache(rng, [length], heads, heads, dim, 16)
        key = rng.permutation(60)[:length] + 64
        c.codes[:, 0] = 0
        for t in range(length):
            c.codes[c.table[0, t // 16], 0, :, t % 16, 0] = key[t]
        c.scales[:, 0] = np.float32(2.0 ** (power // 2))
        q = np.zeros((new, heads, dim))
        q[..., 0] = sign * 2.0 ** (power - power // 2)
        out, lse, got, _ = attend(c, q, [new], 1.0, True, score_in=False)
        gathered = np.zeros((length, heads))
        for i in range(new):
            t = int(np.argmax(sign * key[:length - new + i + 1]))
            blk = c.table[0, t // 16]
            want = torch.as_tensor(c.codes[blk, 1, :, t % 16].astype(np.float64) * c.scales[blk, 1].astype(np.float64)[:, None])
            assert (out[i].double().cpu() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
            norm = sign * 2.0 ** power * float(key[t])
            assert (np.abs(lse[i].double().cpu().numpy() - norm) <= 2.0 ** -22 * abs(norm)).all()
            gathered[t] += 1
        t = np.arange(length)
        if new * heads > 16 and power > 17:
            gathered[:] = 0
        off = 0 if new * heads <= 16 else np.expm1(2.0 ** -22 * 2.0 ** power * 127) if power < 17 else 0
        assert (np.abs(got.cpu().numpy()[c.table[0][t // 16], :, t % 16] - gathered) <= off * gathered).all()


# ------------------------------------------------------------------------------ shared beginnings
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 0, 2], [60, 40, 33], [60, 1, 2]])
def test_sequences_that_share_their_beginning(new):
    """Blocks of a common beginning, named by every sequence's table: the same numbers as with copies of them; with gathered
    weights one call for each sequence, whose sums add up in the shared blocks."""
    rng = np.random.default_rng(sum(new))
    lens, heads, kv_heads, dim, block, common = [150, 200, 131], 4, 2, 128, 32, 3
    c = Cache(rng, lens, heads, kv_heads, dim, block)
    for row in c.table[1:]:
        for j in range(common):
            c.codes[row[j]], c.scales[row[j]], c.score[row[j]] = (x[c.table[0, j]] for x in (c.codes, c.scales, c.score))
    q = bf16(rng.standard_normal((sum(new), heads, dim)))
    want, want_lse, _, _ = attend(c, q, new, 0.1)
    c.table[1:, :common] = c.table[0, :common]
    out, lse, _, _ = attend(c, q, new, 0.1)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    check(c, q, new, 0.1, out, lse)
    codes, scales, score = c.up()
    starts = starts_of(new)
    for b in range(3):
        if new[b]:
            rows = dev(q[starts[b]:starts[b + 1]]).bfloat16()
            ws = Q.alloc_kv_workspace(c.d, 1, new[b], new[b], lens[b], True)
            Q.qalora_kv_attention(c.d, new[b], lens[b], dev(starts_of([new[b]])), dev(c.lens[b:b + 1]), dev(c.table[b:b + 1]), rows, codes,
                                  scales, 0.1, torch.empty_like(rows), None, score, score, ws)
    torch.cuda.synchronize()
    r = K.attention(c.codes, c.scales, starts, c.lens, c.table, q, 0.1, c.score, True)
    d = 2.0 ** -18 * (1 + r["reach"].max())
    assert (np.abs(score.double().cpu().numpy() - r["score"]) <= d * (r["score"] - c.score) + 3 * 2.0 ** -22 * r["score"] + 1e-30).all()


# ------------------------------------------------------------------------------ bounds-check build
def test_edges_entries_and_sizes_pass_the_bounds_check_build():
    """The tests here, those of entries that lead outside and those of the division of work, once more in a child process that
    loads the build with index checks and workspace guards."""
    import os
    import subprocess
    import sys
    if os.environ.get("QALORA_LIBRARY") == "debug":
        pytest.skip("already inside the bounds-check run")
    from paper_2309_14717_b200 import build as B
    B.build(debug=True)
    env = dict(os.environ, QALORA_LIBRARY="debug")
    env.pop("QALORA_PARITY_MARGINS", None)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", "tests/test_kv_edges_gpu.py",
                        "tests/test_kv_entries_gpu.py", "tests/test_kv_sizes_gpu.py"], cwd=root, env=env, capture_output=True, text=True,
                       timeout=1500)
    tail = "\n".join((p.stdout + p.stderr).splitlines()[-40:])
    assert p.returncode == 0, tail
    assert " passed" in p.stdout and "bounds-check build" in p.stdout, tail
