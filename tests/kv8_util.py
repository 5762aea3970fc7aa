"""Inputs and comparisons of the 8-bit cache's tests."""
import numpy as np
import torch

from oracle import kv8
from paper_2402_02082_gb300 import binding as gb

F8 = torch.float8_e4m3fn


def bf16_bits(x):
    """Nearest bf16 of fp32 values, as bit patterns."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(
        np.uint16)


def dev(x):
    if x is None:
        return None
    if x.dtype == np.uint16:
        return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).view(torch.bfloat16).cuda()
    if x.dtype == np.uint8:
        return torch.from_numpy(np.ascontiguousarray(x)).cuda().view(F8)
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(t):
    """A result as fp64."""
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(rng, shape, dtype, spread=0.5):
    """Keys, values or queries: tokens of different magnitude."""
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[:-1] + (1,)))
    return bf16_bits(x) if dtype == "bf16" else x.astype(np.float32)


def cache(rng, B, H, cap, D, kv_len, spread=0.5, stale=0x7f):
    """Codes [B, H, cap, D] and exponents of a cache whose sequences hold kv_len rows; what lies past them is stale:
    codes that stand for NaN, and exponents that no block has."""
    codes = np.full((B, H, cap, D), stale, dtype=np.uint8)
    exps = np.full((B, H, -(-cap // kv8.BLOCK)), 127, dtype=np.int8)
    for b in range(B):
        L = int(kv_len[b])
        for h in range(H):
            x = rng.standard_normal((L, D)) * np.exp(spread * rng.standard_normal((L, 1)))
            for blk in range(-(-L // kv8.BLOCK)):
                part = x[blk * kv8.BLOCK:(blk + 1) * kv8.BLOCK]
                e = kv8.exponent(part)
                exps[b, h, blk] = e
                codes[b, h, blk * kv8.BLOCK:blk * kv8.BLOCK + len(part)] = kv8.encode(part * 2.0 ** -e)
    return codes, exps


def random_tree(rng, n):
    return np.array([-1] + [int(rng.integers(max(0, i - 6), i)) for i in range(1, n)], dtype=np.int32)


def workspace(B, H, H_kv, D, cap, dtype, n):
    desc = gb.make_desc(B, H, D, cap, gb.GLIDE_BF16 if dtype == "bf16" else gb.GLIDE_F32, H_kv=0 if H == H_kv else H_kv)
    size = gb.glide_kv8_workspace_bytes(desc, n)
    assert size > 0
    return torch.zeros(size, dtype=torch.uint8, device="cuda")


def check(got, want, size, dtype):
    """bf16: the result is rounded once (2^-9 of it), and each weight of the sum may be held with an error of 2^-9 of
    it; fp32: scores of magnitude up to 30 from sums of 128 products in fp32 give weights to about 2^-16.  Twice each."""
    assert got.shape == want.shape
    bad = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[bad & ~np.isnan(want)],
                                                                           want[bad & ~np.isnan(want)])
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -15
    err, most = np.abs(got - want)[~bad], (unit * (np.abs(want) + size) + 1e-30)[~bad]
    assert np.all(err <= most), f"{np.max(err / most):.2f} times what is allowed"
