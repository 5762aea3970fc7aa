"""Inputs, expected results and tolerances of the paged cache's tests."""
import numpy as np
import torch

from oracle import paged
from paper_2402_02082_gb300 import binding as gb

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SENTINEL = 7.0


def i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int64), device="cuda").to(torch.int32)


def rounded(x, dtype):
    """fp64 values as the type holds them (on the host, fp64)."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TYPES[dtype]).double().numpy()


def dev(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(TYPES[dtype]).cuda()


def workspace(B, H, H_kv, D, dtype, T, max_q):
    d = gb.make_desc(B, H, D, 1, gb.GLIDE_BF16 if dtype == "bf16" else gb.GLIDE_F32, H_kv=H_kv)
    size = gb.glide_paged_workspace_bytes(d, T, max_q)
    assert size > 0
    return torch.zeros(size, dtype=torch.uint8, device="cuda")


def tolerance(want, mean, top, n, D, dtype):
    """Bound of |result - exact| by element: `mean` is the weighted mean of |v|, `top` the row's largest sum of |q k| scale.

    A score is a sum of D products in chains of at most D / 2 + 8 fp32 additions, each wrong by at most 2^-23 (a tensor
    core truncates) of that sum.  Its product with log2(e), the difference from the maximum and the exponential (2
    units) add 2^-22 of |score| + 1, and |score| <= top.  An error e of every score changes the softmax's mean by at most
    2 e mean.  The sums over n keys and the rescales add (n + 8) 2^-23 of mean.  bf16: each weight is rounded, 2^-8 of
    it, and so at most 2^-8 of mean, and the result is, 2^-8 of it.  fp32: one rounding of the result."""
    score = ((D / 2 + 8) * top * 2.0 ** -23 + (top + 1) * 2.0 ** -22)[:, None]
    tol = (2 * score + (n + 8) * 2.0 ** -23) * mean
    if dtype == "bf16":
        return tol + 2.0 ** -8 * mean + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7) + 1e-30
    return tol + 2.0 ** -24 * np.abs(want) + 1e-30


def check(got, want, tol, what=""):
    """Elements that are not finite have to be the same, the others within tol."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(np.where(np.isinf(want), got, 0), np.where(np.isinf(want), want, 0)), what
    err = np.abs(np.where(fin, got, 0) - np.where(fin, want, 0))
    tol = np.where(fin, tol, 0)
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), f"{what}: {err[worst]} > {tol[worst]} at {worst}"


def tokens(rng, *shape):
    """Rows of different magnitude."""
    return rng.standard_normal(shape) * np.exp(0.3 * rng.standard_normal(shape[:-1] + (1,)))


class Paged:
    """A step of requests with m[b] new tokens and kv[b] tokens over a pool whose other rows hold NaN."""

    def __init__(self, seed, m, kv, H, H_kv, D, P, dtype, pad=0, fused=False, spare=2, spread=1.0):
        rng = np.random.default_rng(seed)
        self.m, self.kv, self.H, self.H_kv, self.D, self.P, self.dtype = list(m), list(kv), H, H_kv, D, P, dtype
        B = len(m)
        width = max(1, max(-(-k // P) for k in kv)) + 1
        used = [-(-k // P) for k in kv]
        n_pages = sum(used) + spare
        ids = rng.permutation(n_pages)
        # entries behind a request's pages are never read: anything may stand there
        self.table = np.where(rng.random((B, width)) < 0.5, -5, 2 ** 31 - 1)
        self.K, self.V = (np.full((n_pages, H_kv, P, D), np.nan) for _ in range(2))
        at = 0
        for b in range(B):
            self.table[b, : used[b]] = ids[at: at + used[b]]
            at += used[b]
            for t in range(kv[b]):
                for X in (self.K, self.V):
                    X[self.table[b, t // P], :, t % P] = tokens(rng, H_kv, D)
        self.K, self.V = rounded(self.K, dtype), rounded(self.V, dtype)
        self.T = sum(m) + pad
        self.q = rounded(spread * tokens(rng, max(1, self.T), H, D)[: self.T], dtype)
        self.cu = np.concatenate([[0], np.cumsum(m)])
        self.fused = fused

    def upload(self):
        self.Kd, self.Vd = dev(self.K, self.dtype), dev(self.V, self.dtype)
        q = dev(self.q, self.dtype)
        if self.fused:  # rows of a wider tensor
            wide = torch.full((self.T, self.H + 3, self.D), float("nan"), dtype=q.dtype, device="cuda")
            wide[:, 1: self.H + 1] = q
            q = wide[:, 1: self.H + 1]
        self.qd, self.tabled, self.cud, self.kvd = q, i32(self.table), i32(self.cu), i32(self.kv)

    def run(self, max_q=None, max_kv=None, scale=0.0, flags=0, ws=None, stream=None):
        out = torch.full((self.T, self.H, self.D), SENTINEL, dtype=TYPES[self.dtype], device="cuda")
        mq, mk = max_q or max(1, max(self.m)), max(self.kv) if max_kv is None else max_kv
        ws = workspace(len(self.m), self.H, self.H_kv, self.D, self.dtype, self.T, mq) if ws is None else ws
        gb.glide_paged_attn(self.qd, self.Kd, self.Vd, self.tabled, self.cud, mq, self.kvd, mk, out, ws, scale, flags, stream)
        self.ws = ws
        return out

    def want(self, scale=0.0):
        scale = scale or self.D ** -0.5
        out = np.full((self.T, self.H, self.D), SENTINEL)
        tol = np.zeros_like(out)
        g = self.H // self.H_kv
        for b, (m, kv) in enumerate(zip(self.m, self.kv)):
            rows = slice(self.cu[b], self.cu[b] + m)
            sees = kv - m + 1 + np.arange(m)
            for h in range(self.H):
                k, v = (paged.gather(X, self.table[b], kv, h // g) for X in (self.K, self.V))
                o, mean, top = paged.attend(self.q[rows, h], k, v, sees, scale)
                out[rows, h] = o
                tol[rows, h] = tolerance(o, mean, top, max(kv, 1), self.D, self.dtype)
        return out, tol


class Prompt:
    """Packed prompts; padding rows hold NaN."""

    def __init__(self, seed, lens, H, H_kv, D, dtype, pad=0, fused=False, spread=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.H_kv, self.D, self.dtype, self.fused = list(lens), H, H_kv, D, dtype, fused
        n = sum(lens)
        self.T = n + pad
        x = rounded(tokens(rng, max(1, self.T), H + 2 * H_kv, D)[: self.T], dtype)
        x[n:] = np.nan
        self.q, self.k, self.v = x[:, :H] * spread, x[:, H: H + H_kv], x[:, H + H_kv:]
        self.q = rounded(self.q, dtype)
        self.cu = np.concatenate([[0], np.cumsum(lens)])

    def upload(self):
        parts = [dev(t, self.dtype) for t in (self.q, self.k, self.v)]
        if self.fused:
            wide = torch.cat(parts, 1)
            parts = wide.split([self.H, self.H_kv, self.H_kv], 1)
        self.qd, self.kd, self.vd = parts
        self.cud = i32(self.cu)

    def run(self, max_len=None, scale=0.0, flags=0, ws=None, stream=None):
        out = torch.full((self.T, self.H, self.D), SENTINEL, dtype=TYPES[self.dtype], device="cuda")
        ml = max_len or max(1, max(self.lens))
        ws = workspace(len(self.lens), self.H, self.H_kv, self.D, self.dtype, self.T, ml) if ws is None else ws
        gb.glide_prompt_attn(self.qd, self.kd, self.vd, self.cud, ml, out, ws, scale, flags, stream)
        self.ws = ws
        return out

    def want(self, scale=0.0):
        scale = scale or self.D ** -0.5
        out = np.full((self.T, self.H, self.D), SENTINEL)
        tol = np.zeros_like(out)
        g = self.H // self.H_kv
        for b, n in enumerate(self.lens):
            rows = slice(self.cu[b], self.cu[b] + n)
            for h in range(self.H):
                o, mean, top = paged.attend(self.q[rows, h], self.k[rows, h // g], self.v[rows, h // g], 1 + np.arange(n), scale)
                out[rows, h] = o
                tol[rows, h] = tolerance(o, mean, top, max(n, 1), self.D, self.dtype)
        return out, tol


def host(t):
    return t.detach().double().cpu().numpy()
