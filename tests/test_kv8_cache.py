"""The 8-bit cache's rows on the GPU: quantised on write, read back, bit for bit as the oracle has them."""
import numpy as np
import pytest
import torch

from kv8_util import F8, cache, dev, host, rows
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def _append(case, stream=None):
    """Runs the call; K, V, K_exp, V_exp, new_kv_len as numpy."""
    K, V, Ke, Ve = (dev(case[w]) for w in ("K", "V", "Ke", "Ve"))
    B = case["kv_len"].shape[0]
    new_len = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    gb.glide_kv8_append(dev(case["k"]), dev(case["v"]), K, V, Ke, Ve, dev(case["kv_len"]), new_len, dev(case["path"]),
                        dev(case["length"]), stream=stream)
    torch.cuda.synchronize()
    return (K.view(torch.uint8).cpu().numpy(), V.view(torch.uint8).cpu().numpy(), Ke.cpu().numpy(), Ve.cpu().numpy(),
            new_len.cpu().numpy())


def _expect(case):
    k = kv8.kv8_append(case["K"], case["Ke"], case["k"], case["kv_len"], case["path"], case["length"])
    v = kv8.kv8_append(case["V"], case["Ve"], case["v"], case["kv_len"], case["path"], case["length"])
    return k[0], v[0], k[1], v[1], k[2]


def _same(got, want):
    for g, w, what in zip(got, want, ("K", "V", "K_exp", "V_exp", "new_kv_len")):
        if what in "KV":  # both NaN codes are NaN
            g, w = np.where(g % 128 == 127, 127, g), np.where(w % 128 == 127, 127, w)
        assert np.array_equal(g, w), f"{what}: {np.argwhere(g != w)[:5].tolist()}"


def _case(seed, B, H, D, cap, kv_len, n, dtype, length=None, path=None, layers=None, scale=1.0):
    rng = np.random.default_rng(seed)
    kv_len = np.array(kv_len, dtype=np.int32)
    lead = () if layers is None else (layers,)
    got = [cache(rng, B * (layers or 1), H, cap, D, np.tile(np.clip(kv_len, 0, cap), layers or 1)) for _ in range(2)]
    shape = lead + (B, n, H, D)
    c = dict(kv_len=kv_len, path=path, length=None if length is None else np.array(length, dtype=np.int32))
    for w, (codes, exps) in zip("KV", got):
        c[w], c[w + "e"] = codes.reshape(lead + (B, H, cap, D)), exps.reshape(lead + (B, H, -1))
        x = rows(rng, shape, "f32") * scale
        c[w.lower()] = x.astype(np.float32) if dtype == "f32" else rows(rng, shape, "bf16")
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,cap,kv_len", [
    (1, 64, [0, 63]), (1, 65, [64, 1]), (5, 200, [62, 63]), (64, 130, [0, 66]), (65, 200, [63, 64]),
    (200, 333, [0, 133]), (130, 130, [0, 0])])
def test_prompt(dtype, D, n, cap, kv_len):
    c = _case(n + D, 2, 3, D, cap, kv_len, n, dtype)
    _same(_append(c), _expect(c))


@pytest.mark.parametrize("layers", [None, 1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accepted_path(layers, dtype):
    n, B = 33, 4
    rng = np.random.default_rng(5)
    length = [0, 5, 3, 32]
    path = np.full((B, n), -1, dtype=np.int32)
    for b, m in enumerate(length):
        path[b, :m + 1] = [0] + sorted(rng.choice(np.arange(1, n), m, replace=False).tolist())
    c = _case(9, B, 2, 128, 190, [60, 61, 0, 100], n, dtype, length, path, layers)
    _same(_append(c), _expect(c))


@pytest.mark.parametrize("scale", [1e-38, 1e-6, 16.0, 3e4, 1e30])
def test_exponent_grows_or_stays(scale):
    """Rows that a block holds already are rounded again only where the new ones are larger."""
    c = _case(3, 2, 2, 64, 128, [7, 70], 20, "f32", scale=scale)
    _same(_append(c), _expect(c))


def test_ragged_lengths_and_ranges():
    """No new rows, all of them, and values out of range, which count as the nearest in it."""
    c = _case(4, 5, 2, 64, 100, [10, 64, -5, 1000, 40], 30, "bf16", [-1, 29, 500, 3, -9])
    _same(_append(c), _expect(c))
    path = np.array([[-3, 40, 2] + [0] * 27] * 5, dtype=np.int32)
    c = _case(4, 5, 2, 64, 100, [10, 64, 0, 70, 40], 30, "bf16", [2, 2, 2, 2, 2], path)
    _same(_append(c), _expect(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_non_finite_and_zero(dtype):
    c = _case(6, 1, 2, 64, 192, [3], 150, dtype)
    special = [np.inf, -np.inf, np.nan, 0.0, -0.0]
    for w in "kv":
        x = c[w] if dtype == "f32" else None
        for i, s in enumerate(special):
            value = np.float32(s)
            if dtype == "f32":
                x[0, 10 + i, 0, i] = value
            else:
                c[w][0, 10 + i, 0, i] = value.view(np.uint32) >> np.uint32(16)
        c[w][0, 61:125, 1] = 0  # a whole block of zeros
        c[w][0, 125:, 0] = np.float32(np.inf) if dtype == "f32" else 0x7f80  # a block with nothing finite
    got = _append(c)
    _same(got, _expect(c))
    assert got[2][0, 1, 1] == kv8.EXP_MIN


def test_every_step_of_a_decode():
    """One row at a time gives what the oracle gives, over a block's end."""
    rng = np.random.default_rng(8)
    c = _case(8, 1, 2, 64, 140, [50], 1, "bf16")
    for step in range(40):
        c["k"], c["v"] = rows(rng, (1, 1, 2, 64), "bf16", 1.0), rows(rng, (1, 1, 2, 64), "bf16", 1.0)
        got = _append(c)
        _same(got, _expect(c))
        c["K"], c["V"], c["Ke"], c["Ve"], c["kv_len"] = got


def test_append_on_a_stream():
    c = _case(11, 2, 3, 128, 300, [30, 100], 150, "bf16")
    st = torch.cuda.Stream()
    _same(_append(c, stream=st), _expect(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layers,cap,out,kv_len", [
    (None, 64, 1, [1, 0]), (None, 130, 130, [130, 129]), (None, 200, 65, [64, 200]), (3, 100, 99, [50, -4])])
def test_read(dtype, D, layers, cap, out, kv_len):
    rng = np.random.default_rng(cap)
    lead, B, H = (() if layers is None else (layers,)), 2, 3
    full = np.array(kv_len).clip(0, cap)
    sides = []
    for _ in range(2):
        codes, exps = cache(rng, B * (layers or 1), H, cap, D, np.tile(full, layers or 1))
        sides.append((codes.reshape(lead + (B, H, cap, D)), exps.reshape(lead + (B, H, -1))))
    (K, Ke), (V, Ve) = sides
    torch_type = torch.bfloat16 if dtype == "bf16" else torch.float32
    K_out, V_out = (torch.full(lead + (B, H, out, D), float("nan"), dtype=torch_type, device="cuda") for _ in range(2))
    gb.glide_kv8_read(dev(K), dev(V), dev(Ke), dev(Ve), dev(np.array(kv_len, dtype=np.int32)), K_out, V_out)
    torch.cuda.synchronize()
    for got, codes, exps in ((K_out, K, Ke), (V_out, V, Ve)):
        assert np.array_equal(host(got), kv8.kv8_read(codes, exps, full, out))


def test_read_every_code():
    codes = np.arange(256, dtype=np.uint8).repeat(64).reshape(1, 1, 128, 128)[:, :, :, :]
    exps = np.array([[[kv8.EXP_MIN, kv8.EXP_MAX]]], dtype=np.int8)
    for t in (torch.bfloat16, torch.float32):
        out = torch.empty((1, 1, 128, 128), dtype=t, device="cuda")
        out2 = torch.empty_like(out)
        gb.glide_kv8_read(dev(codes), dev(codes), dev(exps), dev(exps), dev(np.array([128], dtype=np.int32)), out, out2)
        want = kv8.kv8_read(codes, exps, [128], 128)
        for got in (host(out), host(out2)):
            assert np.array_equal(np.isnan(got), np.isnan(want))
            assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


def test_large_offsets():
    """A cache whose offsets pass 32 bits: 2.2e9 codes in a tensor."""
    B, H, cap, D, n = 1, 64, 270000, 128, 3
    K, V = (torch.zeros((B, H, cap, D), dtype=torch.uint8, device="cuda").view(F8) for _ in range(2))
    Ke, Ve = (torch.zeros((B, H, -(-cap // 64)), dtype=torch.int8, device="cuda") for _ in range(2))
    rng = np.random.default_rng(1)
    k, v = (rows(rng, (B, n, H, D), "bf16") for _ in range(2))
    kv_len, new_len = torch.tensor([cap - 6], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    gb.glide_kv8_append(dev(k), dev(v), K, V, Ke, Ve, kv_len, new_len)
    torch.cuda.synchronize()
    lo = (cap - 6) // 64 * 64
    for codes, exps, new in ((K, Ke, k), (V, Ve, v)):
        got = codes.view(torch.uint8)[:, :, lo:].cpu().numpy()
        zero = np.zeros((B, H, cap - lo, D), dtype=np.uint8)
        want, e, _ = kv8.kv8_append(zero, np.zeros((B, H, -(-(cap - lo) // 64)), dtype=np.int8), new, [cap - 6 - lo])
        assert np.array_equal(got, want) and np.array_equal(exps[:, :, lo // 64:].cpu().numpy(), e)
        assert not codes.view(torch.uint8)[:, -1, :lo].any()
    del K, V
    torch.cuda.empty_cache()
