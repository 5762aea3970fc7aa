"""Pins of the 8-bit cache's oracle: the installed PyTorch's 8-bit float, brute force, and cases worked out by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import cross_attn, kv8, tree_verify_attn


def test_code_values_are_the_8_bit_floats():
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.CODE_VALUES, want, equal_nan=True)
    assert np.array_equal(np.signbit(kv8.CODE_VALUES), np.arange(256) >= 128)


def test_encode_is_nearest_with_ties_to_even():
    rng = np.random.default_rng(0)
    v = kv8.CODE_VALUES[:0x7f]
    mid = (v[:-1] + v[1:]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), rng.standard_normal(2000) * 3,
                        np.exp(rng.uniform(-12, 6, 2000))])
    x = np.concatenate([x, -x])
    got = kv8.encode(x)
    assert np.array_equal(np.signbit(kv8.decode(got)), np.signbit(x))
    away = np.abs(np.abs(x)[:, None] - v[None])
    assert np.array_equal(np.abs(np.abs(kv8.decode(got)) - np.abs(x)), away.min(1))
    tie = (away == away.min(1)[:, None]).sum(1) > 1
    assert tie.sum() == 2 * len(mid) and np.all(got[tie] % 2 == 0)


def test_encode_beyond_the_range():
    assert kv8.encode(np.array([448.0, 449.0, 1e30, np.inf])).tolist() == [0x7e] * 4
    assert kv8.encode(np.array([-448.0, -np.inf])).tolist() == [0xfe] * 2
    assert np.all(np.isnan(kv8.decode(kv8.encode(np.array([np.nan, -np.nan])))))


@pytest.mark.parametrize("top,want", [
    (448.0, 0), (math.nextafter(448.0, 1e9), 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, kv8.EXP_MIN),
    (1e-40, kv8.EXP_MIN), (3.3e38, kv8.EXP_MAX)])
def test_exponent(top, want):
    assert kv8.exponent(np.array([0.0, -top, np.inf, np.nan])) == want


def test_append_by_hand():
    """One row of 1s in a block (exponent -8), then a row of 512s: exponent 1, and 1 is 0.5 * 2**1."""
    codes, exps = np.full((1, 1, 70, 2), 0x7f, np.uint8), np.full((1, 1, 2), 5, np.int8)
    codes, exps, L = kv8.kv8_append(codes, exps, np.ones((1, 1, 1, 2), np.float32), [0])
    assert L.tolist() == [1] and exps[0, 0].tolist() == [-8, 5] and kv8.decode(codes[0, 0, 0]).tolist() == [256.0] * 2
    codes, exps, L = kv8.kv8_append(codes, exps, np.full((1, 3, 1, 2), 512, np.float32), L, np.array([[0, 2, 1]]), [1])
    assert L.tolist() == [3] and exps[0, 0].tolist() == [1, 5]
    assert kv8.decode(codes[0, 0, :3, 0]).tolist() == [0.5, 256.0, 256.0]
    assert np.all(codes[0, 0, 3:] == 0x7f)  # past the end: as it was
    back = kv8.kv8_read(codes, exps, L, 4)
    assert back[0, 0, :, 0].tolist() == [1.0, 512.0, 512.0, 0.0]


def test_a_grown_exponent_keeps_what_it_can():
    """Codes that stay normal keep their values where the exponent grows."""
    rng = np.random.default_rng(1)
    x = rng.uniform(64, 400, (1, 40, 1, 64)).astype(np.float32)
    empty = np.zeros((1, 1, 64, 64), np.uint8), np.zeros((1, 1, 1), np.int8)
    codes, exps, L = kv8.kv8_append(*empty, x, [0])
    before = kv8.kv8_read(codes, exps, L, 40)
    codes, exps, L = kv8.kv8_append(codes, exps, np.full((1, 1, 1, 64), 8000, np.float32), L)
    assert np.array_equal(kv8.kv8_read(codes, exps, L, 41)[:, :, :40], before)


def test_attention_is_that_of_the_16_bit_calls_on_the_values():
    rng = np.random.default_rng(2)
    B, H, Hkv, D, cap, n, kv_len = 2, 4, 2, 64, 150, 5, [130, 0]
    codes, exps = [], []
    for _ in range(2):
        empty = np.zeros((B, Hkv, cap, D), np.uint8), np.zeros((B, Hkv, 3), np.int8)
        c, e, _ = kv8.kv8_append(*empty, rng.standard_normal((B, 130, Hkv, D)).astype(np.float32), [0, 0])
        codes.append(c)
        exps.append(e)
    K, V = (kv8.kv8_values(c, e).astype(np.float32) for c, e in zip(codes, exps))
    q1 = rng.standard_normal((B, 1, H, D)).astype(np.float32)
    got, size = kv8.kv8_attn(q1, *codes, *exps, kv_len)
    np.testing.assert_allclose(got, cross_attn(q1, K, V, kv_len), atol=1e-12)
    assert np.all(got[1] == 0) and np.all(size >= np.abs(got) - 1e-12)
    q, kt, vt = (rng.standard_normal((B, n, h, D)).astype(np.float32) for h in (H, Hkv, Hkv))
    parent = np.array([[-1, 0, 0, 1, 3], [-1, 0, 1, 2, 3]], np.int32)
    got, _ = kv8.kv8_attn(q, *codes, *exps, kv_len, parent, kt, vt)
    for b, L in enumerate(kv_len):  # there the tree's rows follow the cached ones
        K[b, :, L:L + n], V[b, :, L:L + n] = kt[b].transpose(1, 0, 2), vt[b].transpose(1, 0, 2)
    np.testing.assert_allclose(got, tree_verify_attn(q, parent, K, V, kv_len), atol=1e-12)
