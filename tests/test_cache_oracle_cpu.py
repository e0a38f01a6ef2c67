"""Pins of the cache oracle: its e4m3 codes against torch's, its attention against
the prompt attention's oracle, its eviction against hand-made cases."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import cache_oracle as co


def test_codes_are_torchs():
    all_codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn)
    want = all_codes.float().numpy()
    assert np.array_equal(co.VALUES[~np.isnan(want)], want[~np.isnan(want)])
    assert np.isnan(co.VALUES[[0x7F, 0xFF]]).all()
    rng = np.random.default_rng(0)
    steps = co.VALUES[:127]
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000), steps,
                        (steps[1:] + steps[:-1]) / 2, [0.0, 448.0]])
    x = np.concatenate([x, -x]).clip(-448, 448).astype(np.float32)
    got = co.encode(x)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("amax,s", [(448.0, 1.0), (448.1, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8),
                                    (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7), (0.0, 2.0 ** -100),
                                    (1e-35, 2.0 ** -100), (3.38e38, 2.0 ** 120)])
def test_scale(amax, s):
    assert co.scale_for(amax) == s
    assert amax <= 448 * co.scale_for(amax)


def empty(pages, H, hd):
    return {"k": np.full((pages, H, 64, hd), 0x7F, np.uint8),
            "v": np.full((pages, H, 4, hd, 16), 0x7F, np.uint8),
            "kv_scale": np.ones((pages, H, 2)), "mass": np.zeros((pages, H, 64), np.float32)}


def test_chunks_give_the_prompt_attention():
    """A prompt appended in ragged chunks: with the cache's values rounded as they
    are, the rows' attention is the prompt attention's of those values."""
    rng = np.random.default_rng(1)
    H, nq, hd, S = 2, 2, 96, 150
    qkv = rng.normal(size=(H, S, nq + 2, hd))
    pool, table = empty(4, H, hd), np.array([[2, 0, 3]])
    qs, at = [], 0
    for n in (1, 62, 1, 70, 16):
        qs.append(co.append(pool, qkv[:, at:at + n], table, [at], [0, n], 500000.0, 16.0)[0])
        at += n
    # (after the last chunk: a scale that grew may have rounded small codes again)
    q = np.concatenate(qs, axis=1)
    o = np.concatenate([co.attend(pool, q[:, a:e], table, [a], [0, e - a])[0]
                        for a, e in ((0, 100), (100, S))])
    cos, sin = ao.rope_angles(S, hd, 500000.0, 16.0)
    for h in range(H):
        k, v, there = co.tokens(pool, table, 0, h, S)
        assert there.all()
        exact_k = ao.apply_rope(qkv[h, :, nq], cos, sin)
        assert np.abs(k - exact_k).max() <= 2.0 ** -4 * np.abs(exact_k).max()
        for j in range(nq):
            s = ao.apply_rope(qkv[h, :, j], cos, sin) @ k.T / np.sqrt(hd)
            s[np.triu_indices(S, 1)] = -np.inf
            p = np.exp(s - s.max(1, keepdims=True))
            ref = p / p.sum(1, keepdims=True) @ v
            assert np.abs(o[:, h, j] - ref).max() < 1e-12


def test_growing_scale_and_non_finite_rows():
    pool, table = empty(1, 1, 96), np.array([[0]])
    x = np.ones((1, 3, 3, 96))
    co.append(pool, x, table, [0], [0, 3], 1e4, 1.0)
    s0 = pool["kv_scale"][0, 0].copy()
    y = np.full((1, 2, 3, 96), 100.0)
    y[0, 1, 2, 5] = np.inf
    co.append(pool, y, table, [3], [0, 2], 1e4, 1.0)
    assert s0[1] == 2.0 ** -8 and pool["kv_scale"][0, 0, 1] == 2.0 ** -2
    k, v, _ = co.tokens(pool, table, 0, 0, 5)
    assert np.array_equal(v[:, 0], [1, 1, 1, 96, 0])  # 100 / 0.25 = 400, halfway 384 | 416
    assert np.isnan(k[4]).all() and not np.isnan(k[:4]).any()
    assert (pool["k"][0, 0, 5:] == 0x7F).all()


def test_evict_order():
    pool, table = empty(6, 1, 96), np.array([[0, 1]])
    co.append(pool, np.random.default_rng(2).normal(size=(1, 100, 3, 96)), table, [0], [0, 100],
              1e4, 1.0)
    pool["mass"][:2] = 0.0
    pool["mass"][0, 0, 7] = 2.0
    pool["mass"][1, 0, 3] = np.nan
    k0 = co.tokens(pool, table, 0, 0, 100)[0]
    kept, n = co.evict(pool, table, [100], 8, 3, np.array([[4]]))
    # the NaN, the 2.0 and, of the equal zeros, the first three; then the recent ones
    assert kept.tolist() == [[[0, 1, 2, 7, 67, 97, 98, 99]]] and n.tolist() == [8]
    k1 = co.tokens(pool, np.array([[4]]), 0, 0, 8)[0]
    assert np.array_equal(k1, k0[kept[0, 0]])
