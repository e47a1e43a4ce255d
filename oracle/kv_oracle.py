"""Plain definitions of the key/value cache operators (numpy, float64; loops over tokens and heads).

The one place where float32 is normative is the cached code: scale and code are integers or
float32 values decided by a fixed sequence of IEEE float32 operations, which `append` and
`evict` repeat; everything computed FROM codes is float64.

Layout: codes int8 [blocks][2][kv_heads][block][dim], scales float32 [blocks][2][kv_heads],
score float32 [blocks][kv_heads][block]; table [batch][max_blocks], lens [batch], starts [batch + 1].
"""
import numpy as np

F = np.float32


def _rint_div(x, scale):
    """clamp(rint(x / scale)) in float32; infinities saturate, NaN gives 0, and so does a scale of 0."""
    if not scale > 0:
        return np.zeros(x.shape, np.int8)
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.rint(x.astype(F) / F(scale))
    t = np.where(np.isnan(t), F(0), np.clip(t, -127, 127))
    return t.astype(np.int8)


def _need(x):
    fin = np.abs(x[np.isfinite(x)])
    return F(fin.max()) / F(127) if fin.size else F(0)


def append(codes, scales, score, starts, lens, table, k, v):
    """k, v float32 [m][kv_heads][dim].  Changes codes, scales and (unless None) score in place; returns
    whether something was not finite."""
    blocks, _, heads, T, _ = codes.shape
    odd = False
    for b in range(len(lens)):
        n, length = int(starts[b + 1] - starts[b]), int(lens[b])
        first = length - n
        lo = max(first, 0)
        for j in range(lo // T, -(-length // T) if length > lo else 0):
            blk = int(table[b][j])
            s0, s1 = max(lo, j * T), min(length, (j + 1) * T)
            for h in range(heads):
                for which, src in enumerate((k, v)):
                    x = src[starts[b] + s0 - first:starts[b] + s1 - first, h]
                    odd |= not np.isfinite(x).all()
                    need, before = _need(x), scales[blk, which, h]
                    scale = np.maximum(before, need) if s0 > j * T else need
                    if s0 > j * T and scale > before:
                        old = codes[blk, which, h, :s0 - j * T]
                        old[:] = np.rint(old.astype(F) * (before / scale)).astype(np.int8)
                    scales[blk, which, h] = scale
                    codes[blk, which, h, s0 - j * T:s1 - j * T] = _rint_div(x, scale)
                if score is not None:
                    score[blk, h, s0 - j * T:s1 - j * T] = 0
    return odd


def read(codes, scales, table, b, h, which, tokens):
    """float64 [len(tokens)][dim] of one sequence, head and plane."""
    T = codes.shape[3]
    blk = np.array([table[b][t // T] for t in tokens], dtype=np.int64)
    slot = np.array([t % T for t in tokens], dtype=np.int64)
    return codes[blk, which, h, slot].astype(np.float64) * scales[blk, which, h].astype(np.float64)[:, None]


def attention(codes, scales, starts, lens, table, q, softmax_scale, score_in=None, want_score=False):
    """q float64 [m][heads][dim].  Returns a dict: out [m][heads][dim], lse [m][heads], `spread` = sum of weight *
    |value| (what a relative error of the weights can move an output by), `reach` [m][heads] = the largest
    softmax_scale * sum |q||k| of the row (what rounding in a score can scale with), and score (float64, a copy
    of score_in or zeros, with the weights added)."""
    m, heads, dim = q.shape
    kv_heads, T = codes.shape[2], codes.shape[3]
    group = heads // kv_heads
    r = {"out": np.zeros((m, heads, dim)), "spread": np.zeros((m, heads, dim)), "lse": np.full((m, heads), -np.inf),
         "reach": np.zeros((m, heads))}
    if want_score:
        r["score"] = np.zeros((codes.shape[0], kv_heads, T)) if score_in is None else score_in.astype(np.float64).copy()
    for b in range(len(lens)):
        n, length = int(starts[b + 1] - starts[b]), int(lens[b])
        if n == 0 or length == 0:
            continue
        t = np.arange(length)
        for h in range(kv_heads):
            key, val = read(codes, scales, table, b, h, 0, t), read(codes, scales, table, b, h, 1, t)
            for i in range(n):
                pos, row = length - n + i, int(starts[b]) + i
                if pos < 0:
                    continue
                for g in range(h * group, (h + 1) * group):
                    s = softmax_scale * (key[:pos + 1] @ q[row, g])
                    top = s.max()
                    e = np.exp(s - top)
                    w = e / e.sum()
                    r["lse"][row, g] = top + np.log(e.sum())
                    r["out"][row, g] = w @ val[:pos + 1]
                    r["spread"][row, g] = w @ np.abs(val[:pos + 1])
                    r["reach"][row, g] = softmax_scale * (np.abs(key[:pos + 1]) @ np.abs(q[row, g])).max()
                    if want_score:
                        for u in range(pos + 1):
                            r["score"][int(table[b][u // T]), h, u % T] += w[u]
    return r


def select(score, length, budget, recent):
    """Places to keep of one sequence and head: the last `recent`, and the largest of the others (ties to the earlier)."""
    if length <= budget:
        return np.arange(length)
    old = np.asarray(score[:length - recent], dtype=np.float64)
    order = sorted(range(len(old)), key=lambda t: (not np.isnan(old[t]), 0.0 if np.isnan(old[t]) else -old[t], t))
    return np.array(sorted(order[:budget - recent]) + list(range(length - recent, length)), dtype=np.int64)


def evict(codes, scales, score, lens, table, budget, recent, dst_table):
    """Changes the destination blocks in place; returns (dst_lens, kept)."""
    kv_heads, T, dim = codes.shape[2], codes.shape[3], codes.shape[4]
    kept = np.full((len(lens), kv_heads, budget), -1, np.int32)
    dst_lens = np.minimum(np.asarray(lens), budget).astype(np.int32)
    for b, length in enumerate(lens):
        for h in range(kv_heads):
            t = np.arange(int(length))
            src = np.array([table[b][u // T] for u in t], dtype=np.int64)
            keep = select(score[src, h, t % T], int(length), budget, recent)
            kept[b, h, :len(keep)] = keep
            moved = score[src[keep], h, keep % T]
            values = [codes[src[keep], w, h, keep % T].astype(F) * scales[src[keep], w, h][:, None] for w in (0, 1)]
            for j in range(-(-len(keep) // T)):
                blk, part = int(dst_table[b][j]), slice(j * T, min((j + 1) * T, len(keep)))
                n = part.stop - part.start
                for w in (0, 1):
                    scale = _need(values[w][part])
                    scales[blk, w, h] = scale
                    codes[blk, w, h, :n] = _rint_div(values[w][part], scale)
                score[blk, h, :n] = moved[part]
    return dst_lens, kept
