"""Waits of the tensor-core kernel of packed rows: work that takes longer than their limit of a second puts them off, and what
stands still is given up (no fault, no hang)."""
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import check, host, i32, tolerance, workspace

HERE = os.path.dirname(os.path.abspath(__file__))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def test_waits_that_are_put_off(tmp_path):
    exe = str(tmp_path / "wait_check")
    cmd = [build.nvcc(), *build.ARCH, "-std=c++17", "-O3", "--expt-relaxed-constexpr", "-I", build.CSRC,
           "-I", build.INCLUDE, os.path.join(HERE, "rows_wait_check.cu"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    waited, limit, released, done, status, *us = (int(x) for x in r.stdout.split())
    assert (waited, limit, released, done) == (1, 0, 0, 1)
    assert status == 4                           # kStatusTimeout: a wait that ran out
    assert 99000 <= us[0] <= 140000              # five times the limit
    assert 119000 <= us[1] <= 160000             # 20 ms behind the last time
    assert 119000 <= us[2] <= 160000


M, D, P = 17, 64, 256  # new tokens (too many for the kernel of few rows), and pages of 256 keys


def call(q, K, V, table, kv, H):
    out = torch.zeros((M, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, H, D, "bf16", M, M)
    gb.glide_paged_attn(q, K, V, table, i32([0, M]), M, i32([kv]), kv, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    return out


def heads():
    """Two items for every SM: their keys are not cut into chunks."""
    return 2 * torch.cuda.get_device_properties(0).multi_processor_count


def test_row_tiles_that_take_more_than_a_second():
    """2^28 keys of one page again and again, score 0 and values 1 (sums of whole numbers, which fp32 holds); the last key, that
    the last row alone sees, has score 60 and so all the weight but 2^28 e^-60 < 3e-18 of it."""
    H, kv = heads(), 2 ** 28
    K, V = torch.zeros((2, H, P, D), dtype=torch.bfloat16), torch.ones((2, H, P, D), dtype=torch.bfloat16)
    K[1, :, P - 1, 0] = 60.0
    V[1, :, P - 1] = torch.arange(D) - 20.0
    q = torch.zeros((M, H, D), dtype=torch.bfloat16)
    q[..., 0] = 8.0
    table = torch.zeros((1, kv // P), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    out = call(q.cuda(), K.cuda(), V.cuda(), table, kv, H).cpu().double()
    assert (out[: M - 1] == 1).all()
    assert ((out[M - 1] - V[1, 0, P - 1].double()).abs() < 3e-18 * 50).all()


@pytest.mark.parametrize("where", ["value", "key"])
def test_rows_that_are_computed_again_for_more_than_a_second(where):
    """Every row sees 2^20 keys, the first of them with an infinity in its value: each row is computed again, over all of them.
    With NaN in its key every row is NaN."""
    H, kv = heads(), 2 ** 20
    gen = torch.Generator().manual_seed(5)
    K = torch.randn((2, H, P, D), generator=gen).bfloat16()
    V = (torch.randn((2, H, P, D), generator=gen) + torch.arange(D)).bfloat16()
    q = torch.randn((M, H, D), generator=gen).bfloat16()
    (V if where == "value" else K)[0, :, 0, 3] = float("inf") if where == "value" else float("nan")
    table = torch.ones((1, kv // P), dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    got = host(call(q.cuda(), K.cuda(), V.cuda(), table, kv, H))
    if where == "key":
        assert np.isnan(got).all()
        return
    K, V, q = (x.double().numpy() for x in (K, V, q))
    times = np.full((2, P), 1.0)     # how often a row of a page is seen
    want, mean = np.zeros(got.shape), np.zeros(got.shape)
    top = np.zeros((M, H))
    for i in range(M):
        times[1] = kv // P - 2
        times[1, : P - M + 1 + i] += 1
        for h in range(H):
            s = np.einsum("prd,d->pr", K[:, h], q[i, h]) / 8
            w = np.exp(s - s.max()) * times
            w /= w.sum()
            with np.errstate(invalid="ignore"):
                want[i, h] = np.einsum("pr,prd->d", w, V[:, h])
            mean[i, h] = np.einsum("pr,prd->d", w, np.abs(np.where(np.isfinite(V[:, h]), V[:, h], 0)))
            top[i, h] = (np.abs(K[:, h]) @ np.abs(q[i, h])).max() / 8
    assert np.isposinf(want[..., 3]).all() and np.isfinite(np.delete(want, 3, -1)).all()
    tol = np.stack([tolerance(want[:, h], mean[:, h], top[:, h], kv, D, "bf16") for h in range(H)], 1)
    check(got, want, tol)
