"""The key/value cache operators against the float64 oracle (oracle/kv_oracle.py).

Codes and scales are decided by a fixed float32 sequence: bit-exact.  Bounds of the floating
outputs, per element, from the operators' own roundings:
  weights  relative error d = 2^-18 * (1 + reach): a score is a sum of exact products rounded in
           float32 (a few units of 2^-24 of sum |q||k| = reach), scaled twice and raised by an
           exponential of relative error 2^-22;
  out      2^-8 |out| (one rounding to bf16 is 2^-9) + (2^-10 + 2 d) * sum weight |value| (weights are rounded
           to fp16: 2^-11) + 2^-24 * the largest |value| (weights far below a row's largest are fp16
           subnormals);
  lse      d + 2^-22 |lse|;   score  d * gathered + 2^-22 |score|.
"""
import os

import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from paper_2309_14717_b200 import binding as Q

pytestmark = pytest.mark.gpu


def dev(x, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype).cuda()


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


class Cache:
    """A pool with random codes everywhere (also behind the sequences' ends) and a scattered table."""

    def __init__(self, rng, lens, heads, kv_heads, dim, block, spare=0, spread=1.0, room=0):
        self.lens = np.asarray(lens, np.int32)
        width = max(1, -(-(int(self.lens.max(initial=0)) + room) // block))
        self.blocks = len(lens) * width + spare + 2
        self.d = Q.kv_desc(heads, kv_heads, dim, block, self.blocks)
        order = rng.permutation(self.blocks)
        self.table = order[:len(lens) * width].reshape(len(lens), width).astype(np.int32)
        self.free = order[len(lens) * width:].astype(np.int32)
        self.codes = rng.integers(-127, 128, (self.blocks, 2, kv_heads, block, dim)).astype(np.int8)
        self.scales = (np.exp2(rng.uniform(-spread, spread, (self.blocks, 2, kv_heads))) / 100).astype(np.float32)
        self.score = rng.uniform(0, 1, (self.blocks, kv_heads, block)).astype(np.float32)

    def poison(self):
        """What lies outside the sequences must not matter: NaN scales and scores, absurd codes, entries outside the pool."""
        T = self.codes.shape[3]
        for b, n in enumerate(self.lens):
            for j in range(self.table.shape[1]):
                blk = self.table[b, j]
                keep = min(max(int(n) - j * T, 0), T)
                self.codes[blk, :, :, keep:] = -128
                self.score[blk, :, keep:] = np.nan
                if keep == 0:
                    self.scales[blk] = np.nan
        for b, n in enumerate(self.lens):
            self.table[b, -(-int(n) // T):] = [-1, 2 ** 31 - 1][b % 2]
        for blk in self.free:
            self.scales[blk] = np.nan
            self.score[blk] = np.nan
        return self

    def up(self):
        return dev(self.codes), dev(self.scales), dev(self.score)


def attend(c, q, new, scale, scores=False, max_new=None, max_len=None, score_in=True, stream=None, q_dev=None, lse=True):
    starts = starts_of(new)
    m = int(starts[-1])
    codes, scales, score = c.up()
    out = torch.full((m, c.d.heads, c.d.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    l = torch.full((m, c.d.heads), float("nan"), dtype=torch.float32, device="cuda") if lse else None
    max_new = max(new) if max_new is None else max_new
    max_len = int(c.lens.max()) if max_len is None else max_len
    ws = Q.alloc_kv_workspace(c.d, len(new), m, max_new, max_len, scores)
    ws.fill_(0xFF)
    got = torch.full_like(score, -7.0) if scores else None
    Q.qalora_kv_attention(c.d, max_new, max_len, dev(starts), dev(c.lens), dev(c.table), q_dev if q_dev is not None else dev(q).bfloat16(),
                          codes, scales, scale, out, l, score if scores and score_in else None, got, ws, stream=stream)
    torch.cuda.synchronize()
    assert Q.workspace_status(ws) == 0
    return out, l, got, score


def bf16(x):
    return torch.as_tensor(x, dtype=torch.float32).bfloat16().double().numpy()


def check(c, q, new, scale, out, lse, got=None, score_in=None):
    starts = starts_of(new)
    r = K.attention(c.codes, c.scales, starts, c.lens, c.table, q, scale, score_in, got is not None)
    d = 2.0 ** -18 * (1 + r["reach"])
    big = 127 * np.nanmax(c.scales[:, 1])
    o = out.double().cpu().numpy()
    tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -10 + 2 * d[..., None]) * r["spread"] + 2.0 ** -24 * big
    there = np.isfinite(r["lse"])
    assert (o[~there] == 0).all()
    worst = float((np.abs(o - r["out"]) / tol).max(initial=0.0))
    assert worst <= 1, f"out: {worst} of the bound"
    l = lse.double().cpu().numpy()
    assert np.isneginf(l[~there]).all()
    assert (np.abs(l[there] - r["lse"][there]) <= d[there] + 2.0 ** -22 * np.abs(r["lse"][there])).all()
    if got is not None:
        s = got.double().cpu().numpy()
        T, most = c.codes.shape[3], float(d.max(initial=0.0))
        mine = np.zeros(s.shape, bool)
        for b, n in enumerate(c.lens):
            if new[b] > 0:
                t = np.arange(int(n))
                mine[c.table[b][t // T], :, t % T] = True
        base = np.zeros(s.shape) if score_in is None else score_in
        want = np.where(mine, r["score"], 0)
        gathered = np.where(mine, r["score"] - np.where(mine, base, 0), 0)
        assert (s[~mine] == -7).all()
        assert (np.abs(s - want)[mine] <= (most * gathered + 2.0 ** -22 * np.abs(want) + 1e-30)[mine]).all()


# ---------------------------------------------------------------------------------- append, read
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("kv_heads,dim", [(1, 64), (3, 128), (2, 64)])
def test_append_step_by_step_is_bit_exact(kv_heads, dim, block):
    rng = np.random.default_rng(block + dim)
    c = Cache(rng, [0, 0, 0, 0], kv_heads, kv_heads, dim, block, room=330)
    codes, scales, score = c.up()
    table = dev(c.table)
    want = [c.codes.copy(), c.scales.copy(), c.score.copy()]
    lens = np.zeros(4, np.int32)
    for new in ([1, 0, 17, block], [1, block + 1, 0, 0], [1, 1, 1, 1], [0, 2, 130, 3], [15, 1, 1, block - 1]):
        lens = (lens + new).astype(np.int32)
        starts, m = starts_of(new), int(sum(new))
        fused = torch.randn((m, 2 * kv_heads + 1, dim), device="cuda", generator=torch.Generator("cuda").manual_seed(int(lens.sum())))
        fused = (fused * torch.exp2(torch.randint(-3, 4, (m, 1, 1), device="cuda").float())).bfloat16()
        k, v = fused[:, :kv_heads], fused[:, kv_heads:2 * kv_heads]                  # rows of a fused projection
        Q.qalora_kv_append(c.d, max(new), dev(starts), dev(lens), table, k, v, codes, scales, score)
        K.append(*want, starts, lens, c.table, k.float().cpu().numpy(), v.float().cpu().numpy())
        torch.cuda.synchronize()
        assert np.array_equal(scales.cpu().numpy(), want[1])
        assert np.array_equal(codes.cpu().numpy(), want[0])
        assert np.array_equal(score.cpu().numpy(), want[2])
    # and read back, whole and in part, in both types
    first, count = np.array([0, 3, 1, 0], np.int32), np.array([int(lens[0]), 1, int(lens[2]) - 1, 0])
    starts, m = starts_of(count), int(count.sum())
    for dtype in (torch.float32, torch.bfloat16):
        k, v = (torch.full((m, kv_heads, dim), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        Q.qalora_kv_read(c.d, int(count.max()), dev(starts), dev(first), table, codes, scales, k, v)
        only = torch.full_like(v, float("nan"))
        Q.qalora_kv_read(c.d, int(count.max()), dev(starts), dev(first), table, codes, scales, None, only)
        torch.cuda.synchronize()
        assert torch.equal(only, v)
        for b in range(4):
            for h in range(kv_heads):
                for which, got in enumerate((k, v)):
                    ref = K.read(want[0], want[1], c.table, b, h, which, range(first[b], first[b] + count[b]))
                    ref = torch.as_tensor(ref).float().to(dtype)                     # a product of 8 and 24 bits, rounded once or twice
                    assert torch.equal(got[starts[b]:starts[b + 1], h].cpu(), ref)


def test_append_extremes():
    """Infinities, NaNs, zeros, subnormals, the largest bf16 numbers, exact ties, and rows that are not there."""
    rng = np.random.default_rng(3)
    c = Cache(rng, [0] * 7, 2, 2, 64, 16, room=40)
    new = [5, 20, 3, 2, 4, 6, 33]
    lens = np.array([5, 20, 3, 2, 4, 2, 33], np.int32)                               # sequence 5: six rows, two tokens
    starts, m = starts_of(new), sum(new)
    k = torch.randn((m, 2, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
    v = torch.randn((m, 2, 64), generator=torch.Generator().manual_seed(2)).bfloat16()
    k[0, 0, 3], k[1, 1, 5], k[2, 0, 0] = float("inf"), float("nan"), float("-inf")
    k[5:25] = 0
    k[25:28] *= 1e-39                                                                # subnormal scales
    v[25:28] = torch.where(v[25:28] > 0, 1e-40, 0.0).bfloat16()
    k[28:30] = torch.where(k[28:30] > 0, 3.3e38, -3.3e38).bfloat16()
    k[30:34] = torch.arange(4 * 2 * 64).reshape(4, 2, 64).bfloat16() % 128 - 63.5    # halves under scale 1 and 0.5
    k[30, :, 0], v[30:34] = 127.0, k[30:34] / 2
    codes, scales, score = c.up()
    want = [c.codes.copy(), c.scales.copy(), c.score.copy()]
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    Q.qalora_kv_append(c.d, max(new), dev(starts), dev(lens), dev(c.table), k.cuda(), v.cuda(), codes, scales, score, flag)
    assert K.append(*want, starts, lens, c.table, k.float().numpy(), v.float().numpy())
    torch.cuda.synchronize()
    assert int(flag) == 1
    assert np.array_equal(scales.cpu().numpy(), want[1])
    assert np.array_equal(codes.cpu().numpy(), want[0])
    assert np.array_equal(score.cpu().numpy(), want[2])
    Q.qalora_kv_append(c.d, max(new), dev(starts), dev(lens), dev(c.table), k.cuda().nan_to_num(0, 1, -1), v.cuda(), codes, scales,
                       None, flag.zero_())
    torch.cuda.synchronize()
    assert int(flag) == 0


def test_append_skips_what_breaks_the_bounds():
    rng = np.random.default_rng(4)
    c = Cache(rng, [0] * 3, 1, 1, 64, 16, room=32)
    c.table[1] = [-1, c.blocks]                                                      # no such blocks
    codes, scales, score = c.up()
    k = torch.randn((9, 1, 64), device="cuda").bfloat16()
    # the third sequence claims more tokens than its table holds: only its own blocks may change
    Q.qalora_kv_append(c.d, 3, dev(starts_of([3, 3, 3])), dev(np.array([3, 3, 34], np.int32)), dev(c.table), k, k, codes, scales, score)
    torch.cuda.synchronize()
    touched = {int(c.table[0, 0]), int(c.table[2, 1])}
    for blk in set(range(c.blocks)) - touched:
        assert np.array_equal(codes[blk].cpu().numpy(), c.codes[blk])
    # starts that leave the rows: nothing of that sequence is stored
    before = codes.clone()
    Q.qalora_kv_append(c.d, 3, dev(np.array([0, 20, 3, 2], np.int32)), dev(np.array([3, 3, 3], np.int32)), dev(c.table), k, k, codes,
                       scales, score)
    torch.cuda.synchronize()
    assert torch.equal(codes, before)


# ---------------------------------------------------------------------------------- attention
FEW = [  # lens, new, heads, kv_heads, dim, block
    ([1], [1], 1, 1, 64, 16), ([1], [1], 8, 1, 128, 128), ([15, 16, 17], [1, 1, 1], 4, 4, 128, 16),
    ([63, 64, 65, 129], [1, 1, 1, 1], 8, 2, 128, 64), ([127, 128, 129, 1], [1, 1, 1, 1], 4, 4, 64, 32),
    ([300, 0, 5, 77], [1, 1, 1, 1], 6, 2, 64, 128), ([200, 31], [5, 3], 5, 5, 128, 16), ([90, 400], [2, 0], 14, 2, 128, 32),
    ([50, 3, 0], [4, 6, 2], 8, 8, 64, 16), ([1000], [1], 32, 2, 128, 64), ([257, 96], [3, 2], 16, 2, 128, 128),
    ([513], [1], 40, 1, 64, 64), ([40, 70, 33], [30, 17, 33], 4, 4, 128, 32), ([180], [31], 6, 1, 64, 16),
]
PROMPT = [
    ([128], [128], 2, 2, 128, 64), ([129, 60], [129, 60], 2, 1, 128, 32), ([300, 257], [300, 40], 4, 2, 64, 128),
    ([400, 0, 130], [133, 70, 130], 3, 3, 64, 16), ([77, 500], [100, 1], 4, 4, 128, 16), ([260], [65], 16, 2, 128, 128),
]


def _attention_case(lens, new, heads, kv_heads, dim, block, scores, spread=1.0, gain=1.0):
    rng = np.random.default_rng(sum(lens) + 7 * heads + dim)
    c = Cache(rng, lens, heads, kv_heads, dim, block, spread=spread)
    clean = Cache.__new__(Cache)
    clean.__dict__.update(c.__dict__)
    clean.codes, clean.scales, clean.score, clean.table = c.codes.copy(), c.scales.copy(), c.score.copy(), c.table.copy()
    c.poison()
    q = bf16(rng.standard_normal((sum(new), heads, dim)) * gain)
    return c, clean, q


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,block", FEW + PROMPT)
def test_attention_matches_the_oracle(lens, new, heads, kv_heads, dim, block, scores):
    c, clean, q = _attention_case(lens, new, heads, kv_heads, dim, block, scores)
    scale = dim ** -0.5
    out, lse, got, _ = attend(c, q, new, scale, scores)
    check(clean, q, new, scale, out, lse, got, clean.score)


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,block", [FEW[3], FEW[10], PROMPT[2]])
def test_attention_value_scales_far_apart_and_sharp_scores(lens, new, heads, kv_heads, dim, block):
    c, clean, q = _attention_case(lens, new, heads, kv_heads, dim, block, True, spread=5.0, gain=3.0)
    c.scales[c.table[0, 0], 1] = clean.scales[c.table[0, 0], 1] = 0               # a block of zeros, whatever its codes say
    out, lse, got, _ = attend(c, q, new, 0.3, True, score_in=False)
    check(clean, q, new, 0.3, out, lse, got, None)


@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,block", [FEW[3], FEW[9], PROMPT[1]])
def test_attention_repeats_its_bits_on_any_stream_and_with_larger_bounds(lens, new, heads, kv_heads, dim, block):
    c, clean, q = _attention_case(lens, new, heads, kv_heads, dim, block, True)
    side = torch.cuda.Stream()
    a = attend(c, q, new, 0.1, True)
    for _ in range(3):
        with torch.cuda.stream(side):
            b = attend(c, q, new, 0.1, True, stream=side)
        assert all(torch.equal(x.cpu().view(torch.uint8), y.cpu().view(torch.uint8)) for x, y in zip(a[:2], b[:2]))
        assert torch.equal(a[2].nan_to_num(-3), b[2].nan_to_num(-3))
    out, lse, got, _ = attend(c, q, new, 0.1, True, max_new=sum(new), max_len=int(c.lens.max()) + 1000)
    check(clean, q, new, 0.1, out, lse, got, clean.score)
    out, _, _, _ = attend(c, q, new, 0.1, False, lse=False)
    check(clean, q, new, 0.1, out, a[1])


@pytest.mark.parametrize("case", [FEW[6], PROMPT[2]])
def test_attention_strided_queries_scores_in_place_and_a_row_of_nan(case):
    lens, new, heads, kv_heads, dim, block = case
    c, clean, q = _attention_case(lens, new, heads, kv_heads, dim, block, True)
    m = sum(new)
    fused = torch.full((m, heads + 3, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, :heads] = dev(q).bfloat16()
    out, lse, got, _ = attend(c, q, new, 0.2, True, q_dev=fused[:, :heads])
    check(clean, q, new, 0.2, out, lse, got, clean.score)
    # in place: score_out is score_in
    codes, scales, score = c.up()
    ws = Q.alloc_kv_workspace(c.d, len(new), m, max(new), max(lens), True)
    Q.qalora_kv_attention(c.d, max(new), max(lens), dev(starts_of(new)), dev(c.lens), dev(c.table), fused[:, :heads], codes, scales, 0.2,
                          torch.empty_like(out), None, score, score, ws)
    torch.cuda.synchronize()
    mine = got != -7
    assert torch.equal(score[mine], got[mine])
    # a NaN in one query spoils that row and head alone
    bad = fused[:, :heads].clone()
    bad[1, 0, 5] = float("nan")
    spoilt, _, _, _ = attend(c, q, new, 0.2, False, q_dev=bad)
    assert torch.isnan(spoilt[1, 0]).all()
    spoilt[1, 0], out[1, 0] = 0, 0
    assert torch.equal(spoilt, out)


@pytest.mark.parametrize("power", [-100, -60, 60, 100])
def test_attention_queries_of_any_magnitude(power):
    """The query's power of two moves into the scale: outputs do not change with it."""
    c, clean, q = _attention_case(*FEW[4], False)
    ref = attend(c, q, FEW[4][1], 0.125)[0]
    big = q * 2.0 ** power
    out = attend(c, big, FEW[4][1], float(np.float32(0.125 * 2.0 ** -power)) if power < 0 else 0.125 * 2.0 ** -power)[0]
    assert torch.equal(out, ref)


def test_attention_of_generated_tokens_equals_attention_of_the_prompt():
    """The same rows in one call, one by one, and as drafts: the same numbers within the bounds of both."""
    lens, new, heads, kv_heads, dim, block = [150], [150], 4, 2, 128, 32
    c, clean, q = _attention_case(lens, new, heads, kv_heads, dim, block, True)
    out, lse, _, _ = attend(c, q, new, 0.1)
    for i in list(range(0, 150, 37)) + [149]:
        one = Cache.__new__(Cache)
        one.__dict__.update(c.__dict__)
        one.lens = np.array([i + 1], np.int32)
        o, l, _, _ = attend(one, q[i:i + 1], [1], 0.1)
        assert (o[0].float() - out[i].float()).abs().max() <= 2.0 ** -6 * out[i].float().abs().max()
        assert (l[0] - lse[i]).abs().max() <= 1e-4


@pytest.mark.parametrize("scores", [False, True])
def test_attention_many_sequences(scores):
    """More sequences than one launch plans for, most of them short; a few without new rows."""
    rng = np.random.default_rng(11)
    lens = rng.integers(0, 40, 1500).tolist()
    new = [int(x) for x in (rng.random(1500) < 0.9)]
    c = Cache(rng, lens, 2, 1, 64, 16)
    q = bf16(rng.standard_normal((sum(new), 2, 64)))
    out, lse, got, _ = attend(c, q, new, 0.125, scores)
    check(c, q, new, 0.125, out, lse, got, c.score)


def test_cache_beyond_2_to_the_31_bytes():
    """Blocks whose offsets pass 2^31 elements (codes) hold the same numbers as blocks near the start."""
    kv_heads, dim, block = 32, 128, 128
    blocks = 2 ** 31 // (2 * kv_heads * dim * block) + 40
    d = Q.kv_desc(32, kv_heads, dim, block, blocks)
    codes = torch.empty((blocks, 2, kv_heads, block, dim), dtype=torch.int8, device="cuda")
    scales = torch.full((blocks, 2, kv_heads), float("nan"), device="cuda")
    score = torch.zeros((blocks, kv_heads, block), device="cuda")
    assert codes.numel() > 2 ** 31
    n = 300
    g = torch.Generator("cuda").manual_seed(0)
    k, v = (torch.randn((n, kv_heads, dim), device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn((n + 1, 32, dim), device="cuda", generator=g).bfloat16()
    found = []
    for base in (0, blocks - 12):
        table = torch.arange(base, base + 3, dtype=torch.int32, device="cuda")[None]
        far = torch.arange(base + 6, base + 9, dtype=torch.int32, device="cuda")[None]
        lens, starts = dev(np.array([n], np.int32)), dev(np.array([0, n], np.int32))
        Q.qalora_kv_append(d, n, starts, lens, table, k, v, codes, scales, score)
        one = []
        for rows in (q[:n], q[n:]):
            m = rows.shape[0]
            out = torch.empty((m, 32, dim), dtype=torch.bfloat16, device="cuda")
            lse = torch.empty((m, 32), device="cuda")
            ws = Q.alloc_kv_workspace(d, 1, m, m, n, True)
            Q.qalora_kv_attention(d, m, n, dev(np.array([0, m], np.int32)), lens, table, rows, codes, scales, 0.1, out, lse, score, score, ws)
            one += [out, lse]
        dst_lens, kept = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, kv_heads, 200), dtype=torch.int32, device="cuda")
        Q.qalora_kv_evict(d, n, 200, 20, lens, table, codes, scales, score, far, dst_lens, kept)
        back = [torch.empty((200, kv_heads, dim), device="cuda") for _ in range(2)]
        Q.qalora_kv_read(d, 200, dev(np.array([0, 200], np.int32)), dev(np.array([0], np.int32)), far, codes, scales, *back)
        torch.cuda.synchronize()
        found.append(one + [kept, dst_lens] + back + [score[far[0].long()]])
    assert torch.isfinite(found[0][0].float()).all()
    for a, b in zip(*found):
        assert torch.equal(a, b)


def test_captured_step_replays_while_the_sequences_grow():
    """append + attention as one CUDA graph: lens is a device array, only its content moves on."""
    rng = np.random.default_rng(8)
    c = Cache(rng, [0, 0], 4, 2, 128, 16, room=64)
    d, (codes, scales, score) = c.d, c.up()
    table, starts, lens = dev(c.table), dev(np.array([0, 1, 2], np.int32)), dev(np.zeros(2, np.int32))
    k, v = (torch.zeros((2, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros((2, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((2, 4), device="cuda")
    ws = Q.alloc_kv_workspace(d, 2, 2, 1, 64, True)

    def step():
        lens.add_(1)
        Q.qalora_kv_append(d, 1, starts, lens, table, k, v, codes, scales, score)
        Q.qalora_kv_attention(d, 1, 64, starts, lens, table, q, codes, scales, 0.1, out, lse, score, score, ws)

    step()                                                     # (sets up the kernels outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens.zero_()
    codes.copy_(dev(c.codes)), scales.copy_(dev(c.scales)), score.copy_(dev(c.score))
    want, off = [c.codes.copy(), c.scales.copy(), c.score.copy()], 0.0
    for t in range(1, 40):
        x = [torch.randn((2, h, 128), generator=torch.Generator().manual_seed(t * 3 + i)).bfloat16() for i, h in enumerate((2, 2, 4))]
        k.copy_(x[0]), v.copy_(x[1]), q.copy_(x[2])
        graph.replay()
        torch.cuda.synchronize()
        now = np.array([t, t], np.int32)
        K.append(*want, [0, 1, 2], now, c.table, x[0].float().numpy(), x[1].float().numpy())
        assert np.array_equal(codes.cpu().numpy(), want[0])
        r = K.attention(want[0], want[1], [0, 1, 2], now, c.table, x[2].double().numpy(), 0.1, want[2], True)
        want[2] = r["score"].astype(np.float32)
        dd = 2.0 ** -18 * (1 + r["reach"])
        tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -10 + 2 * dd[..., None]) * r["spread"] + 2.0 ** -24
        assert (np.abs(out.double().cpu().numpy() - r["out"]) <= tol).all()
        off += float(dd.max())                                 # every step adds its own error
        assert np.allclose(score.cpu().numpy(), want[2], rtol=off + t * 2.0 ** -22, atol=1e-30)


# ---------------------------------------------------------------------------------- evict
@pytest.mark.parametrize("lens,budget,recent,kv_heads,dim,block", [
    ([40, 20, 64, 0], 20, 5, 2, 64, 16), ([300], 100, 0, 3, 128, 32), ([300, 299], 100, 100, 1, 128, 64), ([129, 128, 127, 1], 128, 1, 2, 64, 128),
    ([1000, 5], 1, 0, 1, 64, 16), ([1000, 900], 999, 500, 2, 128, 16), ([5000, 4097, 33], 1500, 100, 2, 64, 64), ([20000], 3001, 64, 1, 64, 128),
])
@pytest.mark.parametrize("ties", [False, True])
def test_evict_is_bit_exact(lens, budget, recent, kv_heads, dim, block, ties):
    rng = np.random.default_rng(budget + recent)
    width = -(-min(budget, max(lens)) // block)
    c = Cache(rng, lens, kv_heads, kv_heads, dim, block, spare=len(lens) * width)
    if ties:                                                   # few distinct scores, both zeros, infinities and a NaN
        c.score = rng.choice(np.array([0.0, -0.0, 1.5, 1.5, 2.0, np.inf, -1.0], np.float32), c.score.shape)
        c.score.flat[rng.integers(0, c.score.size, 3)] = np.nan
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
    assert np.array_equal(score.cpu().numpy(), c.score, equal_nan=True)


@pytest.mark.parametrize("length", [50001, 210001, 400003])
def test_evict_of_very_long_sequences(length):
    """Clusters of several blocks, and (beyond 393 216 tokens) keys that do not fit shared memory."""
    block, budget, recent = 128, 5001, 77
    width, kept_width = -(-length // block), -(-budget // block)
    d = Q.kv_desc(1, 1, 64, block, width + kept_width)
    codes, scales, score = Q.alloc_kv_cache(d)
    g = torch.Generator("cuda").manual_seed(length)
    codes.random_(-127, 128, generator=g)
    scales.uniform_(0.5, 1, generator=g)
    score.copy_(torch.randint(0, 1 << 14, score.shape, generator=g, device="cuda"))          # with ties
    order = torch.randperm(d.num_blocks, generator=g, device="cuda").int()
    table, dst = order[None, :width].contiguous(), order[None, width:].contiguous()
    lens, dst_lens = dev(np.array([length], np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = torch.zeros((1, 1, budget), dtype=torch.int32, device="cuda")
    flat = score[table[0].long(), 0].flatten()[:length]
    old = torch.sort(flat[:length - recent], descending=True, stable=True)[1][:budget - recent]
    want = torch.cat([old.sort()[0], torch.arange(length - recent, length, device="cuda")])
    Q.qalora_kv_evict(d, length, budget, recent, lens, table, codes, scales, score, dst, dst_lens, kept)
    torch.cuda.synchronize()
    assert int(dst_lens) == budget and torch.equal(kept[0, 0].long(), want)
    assert torch.equal(score[dst[0].long(), 0].flatten()[:budget], flat[want])


def test_evict_then_go_on_generating():
    """The shortened sequence is a sequence like any other: append to it and attend over it."""
    rng = np.random.default_rng(21)
    c = Cache(rng, [90, 40], 4, 2, 64, 16, spare=8)
    dst = c.free[:8].reshape(2, 4)
    codes, scales, score = c.up()
    dst_lens, kept = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 2, 50), dtype=torch.int32, device="cuda")
    Q.qalora_kv_evict(c.d, 90, 50, 10, dev(c.lens), dev(c.table), codes, scales, score, dev(dst), dst_lens, kept)
    k, v, q = (torch.randn((2, h, 64), generator=torch.Generator().manual_seed(h)).bfloat16() for h in (2, 2, 4))
    dst_lens.add_(1)
    starts = dev(np.array([0, 1, 2], np.int32))
    out, lse = torch.empty((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4), device="cuda")
    ws = Q.alloc_kv_workspace(c.d, 2, 2, 1, 51)
    Q.qalora_kv_append(c.d, 1, starts, dst_lens, dev(dst), k.cuda(), v.cuda(), codes, scales, score)
    Q.qalora_kv_attention(c.d, 1, 51, starts, dst_lens, dev(dst), q.cuda(), codes, scales, 0.125, out, lse, None, None, ws)
    torch.cuda.synchronize()
    K.evict(c.codes, c.scales, c.score, c.lens, c.table, 50, 10, dst)
    c.lens, c.table = np.array([51, 41], np.int32), dst
    K.append(c.codes, c.scales, c.score, [0, 1, 2], c.lens, dst, k.float().numpy(), v.float().numpy())
    check(c, q.double().numpy(), [1, 1], 0.125, out, lse)


# ---------------------------------------------------------------------------------- bounds-check build
def test_small_cases_pass_the_bounds_check_build():
    """These tests once more in a child process that loads the build with index checks and workspace guards."""
    import subprocess
    import sys
    if os.environ.get("QALORA_LIBRARY") == "debug":
        pytest.skip("already inside the bounds-check run")
    from paper_2309_14717_b200 import build as B
    B.build(debug=True)
    env = dict(os.environ, QALORA_LIBRARY="debug")
    env.pop("QALORA_PARITY_MARGINS", None)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", "tests/test_kv_cache_gpu.py",
                        "-k", "not beyond and not very_long"], cwd=root, env=env, capture_output=True, text=True, timeout=1500)
    tail = "\n".join((p.stdout + p.stderr).splitlines()[-40:])
    assert p.returncode == 0, tail
    assert " passed" in p.stdout and "bounds-check build" in p.stdout, tail
