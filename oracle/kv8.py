"""fp64 oracle for the 8-bit cache (test infrastructure only).

A code is a signed 8-bit float: 1 sign bit, 4 exponent bits (bias 7), 3
mantissa bits; 0x7f and 0xff are NaN, there is no infinity, the largest
magnitude is 448.  A block of 64 tokens of a cached head shares an int8
exponent: value = code * 2**exp.

Layouts are the library's: codes [.., B, H_kv, S_cap, D] uint8, exponents
[.., B, H_kv, ceil(S_cap/64)] int8, new rows [.., B, n, H_kv, D] (bf16 as uint16
bit patterns, or fp32).  Leading layer dimensions are optional.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np

from .attention import ancestors_or_self, kv_head, widen

BLOCK = 64
EXP_MIN, EXP_MAX = -117, 119


def _code_values() -> np.ndarray:
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        if (c & 0x7f) == 0x7f:
            v = math.nan
        elif e == 0:
            v = m * 2.0 ** -9
        else:
            v = (8 + m) * 2.0 ** (e - 10)
        out[c] = -v if c & 0x80 else v
    return out


CODE_VALUES = _code_values()
_POSITIVE = CODE_VALUES[:0x7f]


def decode(codes: np.ndarray) -> np.ndarray:
    return CODE_VALUES[codes]


def encode(y: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; the largest code beyond it; NaN for NaN (0x7f)."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 0x7e)       # first code with value >= a
    lo = hi - 1
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    c = np.where(a >= _POSITIVE[0x7e], 0x7e, c)
    c = np.where(np.isnan(y), 0x7f, c)
    return (c | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def exponent(x: np.ndarray) -> int:
    """The least e with max |x| <= 448 * 2**e over the finite elements, within the allowed range."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = EXP_MIN
    while e < EXP_MAX and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def _stack(x: np.ndarray, rank: int) -> np.ndarray:
    return x[None] if x.ndim == rank else x


def kv8_append(codes: np.ndarray, exps: np.ndarray, new: np.ndarray, kv_len: Sequence[int],
               path: Optional[np.ndarray] = None, length: Optional[Sequence[int]] = None):
    """(codes, exps, new_kv_len) after the new rows joined one tensor (K or V) of the cache."""
    shape_c, shape_e = codes.shape, exps.shape
    codes, exps, new = _stack(codes, 4).copy(), _stack(exps, 3).copy(), widen(_stack(new, 4))
    layers, B, H, cap, D = codes.shape
    n = new.shape[2]
    out_len = np.zeros(B, dtype=np.int32)
    for b in range(B):
        start = min(max(int(kv_len[b]), 0), cap)
        m = n if length is None else min(max(int(length[b]), -1), n - 1) + 1
        m = min(m, cap - start)
        out_len[b] = start + m
        nodes = [min(max(int(path[b][k]), 0), n - 1) if path is not None else k for k in range(m)]
        for layer in range(layers):
            for h in range(H):
                for blk in range(start // BLOCK, -(-(start + m) // BLOCK) if m else 0):
                    lo, hi = max(start, blk * BLOCK), min(start + m, (blk + 1) * BLOCK)
                    if lo >= hi:
                        continue
                    x = new[layer, b, [nodes[t - start] for t in range(lo, hi)], h]
                    e = exponent(x)
                    if blk * BLOCK < start:
                        old = min(max(int(exps[layer, b, h, blk]), EXP_MIN), EXP_MAX)
                        if old > e:
                            e = old
                        elif e > old:
                            kept = codes[layer, b, h, blk * BLOCK:start]
                            codes[layer, b, h, blk * BLOCK:start] = encode(decode(kept) * 2.0 ** (old - e))
                    codes[layer, b, h, lo:hi] = encode(x * 2.0 ** -e)
                    exps[layer, b, h, blk] = e
    return codes.reshape(shape_c), exps.reshape(shape_e), out_len


def kv8_values(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    rows = codes.shape[-2]
    e = np.repeat(np.clip(exps.astype(np.float64), EXP_MIN, EXP_MAX), BLOCK, axis=-1)[..., :rows]
    return decode(codes) * np.exp2(e)[..., None]


def kv8_read(codes: np.ndarray, exps: np.ndarray, kv_len: Sequence[int], rows: int) -> np.ndarray:
    v = kv8_values(codes, exps)[..., :rows, :].copy()
    v = np.moveaxis(v, -4, 0)
    for b, L in enumerate(kv_len):
        v[b, ..., max(int(L), 0):, :] = 0.0
    return np.moveaxis(v, 0, -4)


def kv8_attn(q: np.ndarray, K, V, K_exp, V_exp, kv_len: Sequence[int], parent: Optional[np.ndarray] = None,
             k_tree: Optional[np.ndarray] = None, v_tree: Optional[np.ndarray] = None, scale: float = 0.0):
    """(out, size): the attention of q [B, n, H, D] over the cached rows and, with a tree, over each
    query's ancestors and itself; size is the same weighting of the values' magnitudes (what a relative
    error of the weights can change)."""
    B, n, H, D = q.shape
    Hkv = K.shape[1]
    sc = scale if scale else 1.0 / np.sqrt(D)
    qd = widen(q)
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    kt = widen(k_tree) if k_tree is not None else None
    vt = widen(v_tree) if v_tree is not None else None
    for b in range(B):
        L = int(kv_len[b])
        anc = [sorted(ancestors_or_self(parent[b], i)) for i in range(n)] if parent is not None else [[]] * n
        for h in range(H):
            j = kv_head(h, H, Hkv)
            keys = kv8_values(K[b, j, :L], K_exp[b, j, :max(1, -(-L // BLOCK))])
            vals = kv8_values(V[b, j, :L], V_exp[b, j, :max(1, -(-L // BLOCK))])
            for i in range(n):
                k = np.concatenate([keys, kt[b, anc[i], j]]) if anc[i] else keys
                v = np.concatenate([vals, vt[b, anc[i], j]]) if anc[i] else vals
                if len(k) == 0:
                    continue
                s = (k @ qd[b, i, h]) * sc
                with np.errstate(invalid="ignore"):
                    p = np.exp(s - s.max())
                out[b, i, h] = (p @ v) / p.sum()
                size[b, i, h] = (p @ np.abs(v)) / p.sum()
    return out, size
