"""Pins of the key/value cache oracle (CPU): hand-worked blocks, bounds of the rounding, attention against
closed forms, the meaning of the gathered weights, the selection against a brute force."""
import itertools

import numpy as np
import pytest

from oracle import kv_oracle as K

F = np.float32


def _empty(blocks, heads, T, dim):
    return (np.zeros((blocks, 2, heads, T, dim), np.int8), np.zeros((blocks, 2, heads), F), np.zeros((blocks, heads, T), F))


def test_append_hand_worked_block_with_a_growing_scale():
    codes, scales, score = _empty(1, 1, 16, 2)
    k = np.array([[[127.0, -63.5]]], F)                 # scale 1: codes 127, -64 (ties to even: -63.5 -> -64)
    K.append(codes, scales, score, [0, 1], [1], [[0]], k, k * 0)
    assert scales[0, 0, 0] == 1 and list(codes[0, 0, 0, 0]) == [127, -64]
    assert scales[0, 1, 0] == 0 and not codes[0, 1].any()                          # a block of zeros
    k2 = np.array([[[254.0, 3.0]]], F)                  # scale 2: the earlier codes become rint(63.5) = 64 and -32
    K.append(codes, scales, score, [0, 1], [2], [[0]], k2, k2 * 0)
    assert scales[0, 0, 0] == 2 and list(codes[0, 0, 0, 0]) == [64, -32] and list(codes[0, 0, 0, 1]) == [127, 2]
    k3 = np.array([[[1.0, -1.0]]], F)                   # a smaller token leaves the scale: 0.5 -> 0, -0.5 -> -0
    K.append(codes, scales, score, [0, 1], [3], [[0]], k3, k3 * 0)
    assert scales[0, 0, 0] == 2 and list(codes[0, 0, 0, 2]) == [0, 0]


def test_append_error_is_at_most_half_a_step_and_the_scale_is_used_up():
    rng = np.random.default_rng(0)
    codes, scales, score = _empty(4, 2, 16, 8)
    k, v = (rng.standard_normal((40, 2, 8)).astype(F) for _ in range(2))
    K.append(codes, scales, score, [0, 40], [40], [[2, 0, 3]], k, v)
    for which, x in enumerate((k, v)):
        for h in range(2):
            got = K.read(codes, scales, [[2, 0, 3]], 0, h, which, range(40))
            step = scales[[2, 0, 3], which, h].repeat(16)[:40, None]
            assert (np.abs(got - x[:, h]) <= 0.5 * step * (1 + 1e-6)).all()
            for j, blk in enumerate((2, 0, 3)):
                n = min(16, 40 - 16 * j)
                assert np.abs(codes[blk, which, h, :n]).max() == 127


def test_append_not_finite_and_rows_that_are_not_there():
    codes, scales, score = _empty(1, 1, 16, 2)
    score += 9
    k = np.array([[[1.0, 2.0]], [[np.inf, np.nan]], [[-np.inf, 4.0]]], F)
    assert K.append(codes, scales, score, [0, 3], [2], [[0]], k, k)                # 2 tokens, 3 rows: the first is not there
    assert scales[0, 0, 0] == F(4) / F(127)
    assert codes[0, 0, 0, :3].tolist() == [[127, 0], [-127, 127], [0, 0]]
    assert score[0, 0, :3].tolist() == [0, 0, 9]


def _random_cache(rng, lens, T, heads, dim):
    width = max(-(-n // T) for n in lens) if max(lens) else 1
    blocks = len(lens) * width + 1
    codes = rng.integers(-127, 128, (blocks, 2, heads, T, dim)).astype(np.int8)
    scales = (rng.uniform(0.5, 2, (blocks, 2, heads)) / 100).astype(F)
    return codes, scales, rng.permutation(blocks)[:len(lens) * width].reshape(len(lens), width)


def test_attention_of_one_token_and_of_equal_keys():
    rng = np.random.default_rng(1)
    codes, scales, table = _random_cache(rng, [1, 37], 16, 1, 4)
    q = rng.standard_normal((2, 2, 4))
    r = K.attention(codes, scales, [0, 1, 2], [1, 37], table, q, 0.5)
    v0 = K.read(codes, scales, table, 0, 0, 1, [0])[0]
    k0 = K.read(codes, scales, table, 0, 0, 0, [0])[0]
    assert np.allclose(r["out"][0], v0) and np.allclose(r["lse"][0], 0.5 * q[0] @ k0)
    codes[table[1], 0] = 0                                                          # equal keys: the mean of the values
    r = K.attention(codes, scales, [0, 1, 2], [1, 37], table, q, 0.5)
    assert np.allclose(r["out"][1], K.read(codes, scales, table, 1, 0, 1, range(37)).mean(0)) and np.allclose(r["lse"][1], np.log(37))


def test_attention_new_tokens_see_what_they_would_have_seen_one_by_one():
    rng = np.random.default_rng(2)
    codes, scales, table = _random_cache(rng, [21], 16, 2, 4)
    q = rng.standard_normal((5, 4, 4))
    whole = K.attention(codes, scales, [0, 5], [21], table, q, 0.7, want_score=True)
    total = np.zeros_like(whole["score"])
    for i in range(5):
        one = K.attention(codes, scales, [0, 1], [17 + i], table, q[i:i + 1], 0.7, want_score=True)
        assert np.allclose(one["out"][0], whole["out"][i]) and np.allclose(one["lse"][0], whole["lse"][i])
        total += one["score"]
    assert np.allclose(total, whole["score"])
    assert whole["score"].sum() == pytest.approx(5 * 4)                             # every row's weights add up to one


def test_rows_without_tokens_are_zero():
    rng = np.random.default_rng(3)
    codes, scales, table = _random_cache(rng, [2, 0], 16, 1, 4)
    r = K.attention(codes, scales, [0, 3, 4], [2, 0], table, rng.standard_normal((4, 1, 4)), 1.0, want_score=True)
    for row in (0, 3):
        assert not r["out"][row].any() and np.isneginf(r["lse"][row]).all()
    assert r["score"].sum() == pytest.approx(2)


@pytest.mark.parametrize("length,budget,recent", [(7, 7, 3), (7, 9, 2), (7, 4, 0), (7, 4, 4), (8, 5, 2), (1, 1, 0)])
def test_selection_is_the_best_subset(length, budget, recent):
    rng = np.random.default_rng(length * 10 + budget)
    for _ in range(20):
        score = rng.integers(0, 4, length).astype(F)
        keep = K.select(score, length, budget, recent)
        assert (np.diff(keep) > 0).all() and len(keep) == min(length, budget)
        if length > budget:
            assert set(range(length - recent, length)) <= set(keep.tolist())
            free = [c for c in itertools.combinations(range(length - recent), budget - recent)]
            best = max(free, key=lambda c: (sum(score[list(c)]), [-x for x in c]))
            assert tuple(keep[:budget - recent]) == best


def test_evict_of_whole_sequences_keeps_values_within_half_a_step():
    rng = np.random.default_rng(5)
    codes, scales, table = _random_cache(rng, [30, 12], 16, 2, 4)
    blocks = codes.shape[0]
    codes = np.concatenate([codes, np.zeros((4,) + codes.shape[1:], np.int8)])
    scales = np.concatenate([scales, np.zeros((4, 2, 2), F)])
    score = rng.uniform(0, 1, (blocks + 4, 2, 16)).astype(F)
    dst = np.arange(blocks, blocks + 4).reshape(2, 2)
    dst_lens, kept = K.evict(codes, scales, score, [30, 12], table, 20, 5, dst)
    assert dst_lens.tolist() == [20, 12] and (kept[1, :, 12:] == -1).all()
    for b, n in enumerate((20, 12)):
        for h in range(2):
            for w in range(2):
                got = K.read(codes, scales, dst, b, h, w, range(n))
                was = K.read(codes, scales, table, b, h, w, kept[b, h, :n])
                step = scales[dst[b], w, h].repeat(16)[:n, None]
                assert (np.abs(got - was) <= 0.5 * step * (1 + 1e-6)).all()
