"""Pins of the oracle of cached keys and values in 4 bits (CPU): hand-worked
values, brute force over the format's values, closed forms and PyTorch."""
import math

import numpy as np
import pytest
import torch

import oracle

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _group(*x):
    g = np.zeros(32)
    g[:len(x)] = x
    return g


def test_quantise_by_hand():
    # the largest magnitude is 7: scale 2^0; every border between two levels
    x = _group(7, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.75, -7, -0.1, 0.74)
    code, scale = oracle.kv4_quantise(x)
    assert scale.tolist() == [127]
    assert code[:14].tolist() == [7, 0, 1, 2, 2, 4, 4, 6, 6, 7, 10, 15, 8, 1]
    # just above 7 the scale doubles
    code, scale = oracle.kv4_quantise(_group(7.0625, 1))
    assert scale.tolist() == [128] and code[:2].tolist() == [6, 1]
    assert oracle.kv4_quantise(_group(3.5))[1].tolist() == [126]
    assert oracle.kv4_quantise(np.zeros(64))[1].tolist() == [2, 2]  # the least exponent, -125
    big = float(torch.finfo(torch.bfloat16).max)
    code, scale = oracle.kv4_quantise(_group(big, -big))
    assert scale.tolist() == [252] and code[:2].tolist() == [7, 15]
    assert oracle.kv4_values(code, scale)[0] == 6 * 2.0 ** 125 == 1.5 * 2.0 ** 127


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_group_with_a_value_that_is_not_finite_reads_back_as_nan(bad):
    x = np.ones(64)
    x[40] = bad
    code, scale = oracle.kv4_quantise(x)
    assert scale[1] == 255 and scale[0] != 255
    v = oracle.kv4_values(code, scale)
    assert np.isnan(v[32:]).all() and (v[:32] == 1).all()


def test_quantise_is_the_nearest_value_of_the_least_scale():
    rng = np.random.default_rng(0)
    for _ in range(50):
        x = rng.normal(size=32) * np.exp2(rng.uniform(-20, 20))
        code, scale = oracle.kv4_quantise(x)
        e = int(scale[0]) - 127
        assert np.abs(x).max() <= 7 * 2.0 ** e and np.abs(x).max() > 7 * 2.0 ** (e - 1)
        all_values = np.array([s * v * 2.0 ** e for v in LEVELS for s in (1, -1)])
        got = oracle.kv4_values(code, scale)
        np.testing.assert_array_equal(np.abs(got - x), np.abs(all_values[:, None] - x).min(0))
        # off by half a step of the neighbouring levels at most
        step = np.where(np.abs(x) < 2 * 2.0 ** e, 0.5, np.where(np.abs(x) < 4 * 2.0 ** e, 1.0, 2.0)) * 2.0 ** e
        assert (np.abs(got - x) <= step / 2).all()


@pytest.mark.parametrize("d,block", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_pages_hold_what_was_stored_and_nothing_else_changes(d, block):
    rng = np.random.default_rng(d + block)
    pool = rng.integers(0, 256, (3, 2, block * d * 17 // 16), dtype=np.uint8)
    before = pool.copy()
    k, v = rng.normal(size=(2, 5, 2, d))
    slots = [2 * block + 7, 0, -1, block - 1, 3 * block]  # the third and the last name no token
    oracle.kv4_store(pool, k, v, slots, block)
    for row in (0, 1, 3):
        page, t = divmod(slots[row], block)
        for h in range(2):
            got = oracle.kv4_token(pool, page, h, t, block, d)
            for g, x in zip(got, (k[row, h], v[row, h])):
                np.testing.assert_array_equal(g, oracle.kv4_values(*oracle.kv4_quantise(x)))
    # d / 2 + d / 32 bytes of K and of V for each head of three tokens (some may keep their value)
    assert (pool != before).sum() <= 3 * 2 * 2 * (d // 2 + d // 32)
    assert (pool[1] == before[1]).all()


def test_layout_by_hand():
    # d = 64, block = 64: K codes 2048 bytes, K scales 128, then V the same
    pool = np.zeros((1, 1, 64 * 64 * 17 // 16), dtype=np.uint8)
    k, v = np.zeros((1, 1, 64)), np.zeros((1, 1, 64))
    k[0, 0, 33], v[0, 0, 2] = 6.0, -3.0
    oracle.kv4_store(pool, k, v, [11], 64)
    p = pool[0, 0]
    assert p[11 * 32 + 16] == 0x70 and p[2048 + 11 * 2 + 1] == 127 and p[2048 + 11 * 2] == 2
    # octet 1, pair 1, token 3 of the octet; -3 under 2^-1 is code 7 with the sign
    assert p[2176 + (32 + 1) * 8 + 3] == 0x0F and p[2176 + 2048 + (2 + 0) * 8 + 3] == 126


def test_plan_by_hand():
    # block 64; request 0 holds 63 tokens in page 9, request 1 nothing, request 2 exactly a page
    table = np.array([[9, -1, -1], [-1, -1, -1], [4, -1, -1]])
    q, kv, slots, pos, counts, t = oracle.page_plan([63, 0, 64], [2, 0, 1], table, [20, 21, 22], 64, 5)
    assert q.tolist() == [0, 2, 2, 3] and kv.tolist() == [65, 0, 65]
    assert slots.tolist() == [9 * 64 + 63, 20 * 64, 21 * 64, -1, -1]
    assert pos.tolist() == [63, 64, 64, -1, -1] and counts.tolist() == [3, 2, 0]
    assert t.tolist() == [[9, 20, -1], [-1, -1, -1], [4, 21, -1]]
    # one free page: the last token is not placed; a table of one page: nor the second
    assert oracle.page_plan([63, 0, 64], [2, 0, 1], table, [20], 64, 3)[4].tolist() == [3, 1, 1]
    q, kv, slots, _, counts, _ = oracle.page_plan([63, 0, 64], [2, 0, 1], table[:, :1], [20, 21], 64, 3)
    assert slots.tolist() == [9 * 64 + 63, -1, -1] and kv.tolist() == [64, 0, 64] and counts.tolist() == [3, 0, 2]
    # two slots for four tokens
    q, kv, slots, _, counts, _ = oracle.page_plan([0, 0], [3, 1], [[-1], [-1]], [5, 6], 64, 2)
    assert q.tolist() == [0, 2, 2] and slots.tolist() == [320, 321] and counts.tolist() == [2, 1, 2]


@pytest.mark.parametrize("causal", [False, True])
def test_attention_is_softmax_attention_over_the_stored_values(causal):
    rng = np.random.default_rng(3)
    d, block, heads = 64, 64, 4
    pool = np.zeros((4, 2, block * d * 17 // 16), dtype=np.uint8)
    kv_len, table = [70, 5], np.array([[2, 0], [3, -1]])
    for b in range(2):
        slots = [table[b, t // block] * block + t % block for t in range(kv_len[b])]
        oracle.kv4_store(pool, *rng.normal(size=(2, kv_len[b], 2, d)), slots, block)
    q = rng.normal(size=(9, heads, d))
    o, lse, done = oracle.kv4_attention(q, pool, table, [1, 4, 8], kv_len, block, causal)
    assert done.tolist() == [False] + [True] * 7 + [False]
    for b, (a, e) in enumerate([(1, 4), (4, 8)]):
        k, v, there = oracle.kv4_cached(pool, table[b], kv_len[b], block, d)
        assert there.all()
        n, m = kv_len[b], e - a
        mask = torch.ones(m, n, dtype=torch.bool).tril(n - m) if causal else None
        up = lambda x: torch.tensor(x).repeat_interleave(2, 0)  # noqa: E731
        want = torch.nn.functional.scaled_dot_product_attention(
            torch.tensor(q[a:e]).transpose(0, 1), up(k), up(v), attn_mask=mask).transpose(0, 1)
        np.testing.assert_allclose(o[a:e], want.numpy(), atol=1e-12)
        s = (torch.tensor(q[a:e]).transpose(0, 1) @ up(k).transpose(1, 2)) / math.sqrt(d)
        s = s if mask is None else s.masked_fill(~mask, -math.inf)
        np.testing.assert_allclose(lse[a:e], torch.logsumexp(s, -1).T.numpy(), atol=1e-12)


def test_attention_rows_that_see_nothing():
    pool = np.zeros((1, 1, 64 * 64 * 17 // 16), dtype=np.uint8)
    q = np.ones((4, 1, 64))
    # no tokens; a page left out; two tokens for three causal queries
    for args in (([0, 4], [0]), ([0, 4], [30])):
        o, lse, done = oracle.kv4_attention(q, pool, [[-1]], *args, 64)
        assert done.all() and (o == 0).all() and np.isneginf(lse).all()
    o, lse, _ = oracle.kv4_attention(q, pool, [[0]], [0, 3], [2], 64, causal=True)
    assert np.isneginf(lse[0]).all() and np.isfinite(lse[1:3]).all()
