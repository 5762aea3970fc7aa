"""Attention over the 8-bit cache against the fp64 oracle: cross-attention of a draft query, and verification of a
tree whose own keys and values are not quantised."""
import numpy as np
import pytest
import torch

from kv8_util import F8, cache, check, dev, host, random_tree, rows, workspace
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def make(seed, B, H, H_kv, D, kv_len, n, dtype, tree, cap=None, spread=0.5):
    rng = np.random.default_rng(seed)
    kv_len = np.array(kv_len, dtype=np.int32)
    cap = cap or int(kv_len.max()) + 7
    c = dict(B=B, H=H, H_kv=H_kv, D=D, n=n, dtype=dtype, cap=cap, kv_len=kv_len, scale=0.0)
    c["K"], c["Ke"] = cache(rng, B, H_kv, cap, D, kv_len, spread)
    c["V"], c["Ve"] = cache(rng, B, H_kv, cap, D, kv_len, spread)
    c["q"] = rows(rng, (B, n, H, D), dtype, 0.2)
    c["parent"] = np.stack([random_tree(rng, n) for _ in range(B)]) if tree else None
    c["k"], c["v"] = (rows(rng, (B, n, H_kv, D), dtype) if tree else None for _ in range(2))
    return c


def call(c, max_kv=None, max_ctas=0, stream=None, ws=None):
    t = {w: dev(c[w]) for w in ("q", "K", "V", "Ke", "Ve", "kv_len", "parent", "k", "v")}
    out = torch.full(c["q"].shape, float("nan"), dtype=DTYPES[c["dtype"]], device="cuda")
    ws = ws if ws is not None else workspace(c["B"], c["H"], c["H_kv"], c["D"], c["cap"], c["dtype"], c["n"])
    most = int(c["kv_len"].max()) if max_kv is None else max_kv
    torch.cuda.synchronize()
    side = (t["K"], t["V"], t["Ke"], t["Ve"], t["kv_len"], most, out, ws, c["scale"], max_ctas, stream)
    if c["parent"] is None:
        gb.glide_kv8_cross_attn(t["q"], *side)
    else:
        gb.glide_kv8_verify_attn(t["q"], t["parent"], t["k"], t["v"], *side)
    torch.cuda.synchronize()
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    return host(out)


def expect(c):
    return kv8.kv8_attn(c["q"], c["K"], c["V"], c["Ke"], c["Ve"], c["kv_len"], c["parent"], c["k"], c["v"], c["scale"])


def compare(c, **how):
    check(call(c, **how), *expect(c), c["dtype"])


HEADS = [(2, 2), (8, 2), (3, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
@pytest.mark.parametrize("kv_len", [[1], [64, 65], [31, 128, 129], [700, 0, 3, 257]])
def test_cross(dtype, D, H, H_kv, kv_len):
    compare(make(sum(kv_len) + D, len(kv_len), H, H_kv, D, kv_len, 1, dtype, False))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
@pytest.mark.parametrize("n,kv_len", [(1, [0]), (1, [1, 63]), (5, [0, 128]), (6, [127, 130]), (17, [500, 1]),
                                      (33, [64, 300]), (64, [0, 129])])
def test_verify(dtype, D, H, H_kv, n, kv_len):
    compare(make(n + sum(kv_len), len(kv_len), H, H_kv, D, kv_len, n, dtype, True))


@pytest.mark.parametrize("H,H_kv,n", [(256, 1, 1), (64, 1, 4), (16, 2, 32), (20, 4, 50), (65, 1, 2)])
def test_many_query_rows(H, H_kv, n):
    """Slabs of up to 256 query rows, groups that do not divide a tile among them."""
    compare(make(H + n, 2, H, H_kv, 128, [200, 75], n, "bf16", n > 1))


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("max_ctas", [1, 3, 7, 0])
def test_splits(tree, max_ctas):
    """Any division of the keys among CTAs gives the same result to rounding."""
    compare(make(21, 3, 4, 4, 128, [1000, 130, 2049], 9 if tree else 1, "bf16", tree), max_ctas=max_ctas)


@pytest.mark.parametrize("tree", [False, True])
def test_long(tree):
    compare(make(22, 1, 2, 1, 128, [9001], 12 if tree else 1, "bf16", tree))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_out_of_range(dtype):
    """Lengths beyond the bound count as the bound, negative ones as 0."""
    c = make(31, 3, 2, 2, 64, [100, 100, 100], 4, dtype, True)
    want = dict(c, kv_len=np.array([90, 0, 33], dtype=np.int32))
    got = call(dict(c, kv_len=np.array([5000, -3, 33], dtype=np.int32)), max_kv=90)
    check(got, *expect(want), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parents_out_of_range(dtype):
    """A parent that is not an earlier node makes a root."""
    c = make(32, 1, 2, 2, 64, [70], 6, dtype, True)
    c["parent"] = np.array([[-1, 0, 1, 2, 3, 4]], dtype=np.int32)
    bad = dict(c, parent=np.array([[9, 0, 2, -7, 3, 1 << 30]], dtype=np.int32))
    want = dict(c, parent=np.array([[-1, 0, -1, -1, 3, -1]], dtype=np.int32))
    check(call(bad), *expect(want), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.5, 1e-4])
def test_scale(dtype, scale):
    c = make(33, 2, 4, 2, 128, [333, 12], 7, dtype, True)
    c["scale"] = scale
    compare(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
def test_blocks_of_very_different_scale(dtype, tree):
    """Blocks whose keys or values are larger or smaller by powers of two up to 2^30, a block of zero values, and one
    that draws all the attention."""
    c = make(34, 1, 2, 2, 128, [640], 5 if tree else 1, dtype, tree)
    c["Ve"] = (c["Ve"] + np.array([0, -30, 12, -60, 30, -5, 0, 3, -20, 10, 0])[None, None]).astype(np.int8)
    c["V"][:, :, 256:320] = 0
    c["Ve"][:, :, 4] = kv8.EXP_MIN
    c["Ke"] = (c["Ke"] + np.array([0, 1, -8, 2, -3, 0, -60, 1, 0, -1, 0])[None, None]).astype(np.int8)
    compare(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_on_small_values(dtype):
    """All the weight on a block whose values are 2^-40 of the others': the result is that block's."""
    c = make(35, 1, 2, 2, 128, [320], 3, dtype, True)
    q = kv8.widen(c["q"])[:, 0]                                # [1, 2, D], the same query for every node
    c["q"][:] = c["q"][:, :1]
    x = q * 40.0 / np.sqrt((q ** 2).sum(-1, keepdims=True))
    for h in range(2):
        e = kv8.exponent(x[0, h])
        c["K"][0, h, 130], c["Ke"][0, h, 2] = kv8.encode(x[0, h] * 2.0 ** -e), e
    c["Ve"][:, :, 2] -= 40
    got, (want, size) = call(c), expect(c)
    check(got, want, size, dtype)


def test_rising_scores():
    """Scores that rise along the sequence by far more than a type's range: the running maximum moves in every tile."""
    for dtype in ("bf16", "f32"):
        c = make(36, 1, 1, 1, 64, [1500], 3, dtype, True)
        c["Ke"] = (c["Ke"].astype(np.int32) + np.arange(c["Ke"].shape[-1]) // 3).clip(-100, 8).astype(np.int8)
        got, (want, size) = call(c), expect(c)
        unit = 2.0 ** -6 if dtype == "bf16" else 2.0 ** -9    # scores up to 2000: their rounding shows in the weights
        assert np.all(np.abs(got - want) <= unit * (np.abs(want) + size))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_stays_where_it_is(dtype):
    """A NaN query row spoils its own output only; a NaN key or tree value those that see it."""
    c = make(37, 2, 4, 2, 64, [100, 200], 6, dtype, True)
    nan = 0x7fc0 if dtype == "bf16" else np.nan
    c["parent"] = np.array([[-1, 0, 0, 1, 1, 2]] * 2, dtype=np.int32)
    c["q"][0, 3, 1, 5] = nan        # one row of one head
    c["v"][1, 4, 0, 7] = nan        # node 4's value: seen by node 4 only
    c["k"][1, 2, 1, 0] = nan        # node 2's key: seen by nodes 2 and 5
    c["v"][0, 5, 1, 2] = 0x7f80 if dtype == "bf16" else np.inf  # node 5's value: seen by node 5 only
    got = call(c)
    want, size = expect(c)
    spoiled = np.isnan(want)
    assert spoiled[0, 3, 1].all() and spoiled[1, 4, 0, 7] and spoiled[1, 2, 2:].all() and spoiled[1, 5, 3].all()
    assert np.array_equal(np.isnan(got), spoiled)
    ok = np.isfinite(want)
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -15
    assert np.all(np.abs(got - want)[ok] <= (unit * (np.abs(want) + size))[ok])
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])


def test_on_another_stream_and_reused_workspace():
    ws = workspace(3, 8, 2, 128, 4000, "bf16", 64)
    st = torch.cuda.Stream()
    for i, (n, kv) in enumerate([(33, [800, 20, 300]), (1, [5, 5, 5]), (64, [0, 2000, 64]), (2, [129, 1, 77])]):
        c = make(40 + i, 3, 8, 2, 128, kv, n, "bf16", True)
        check(call(c, stream=st, ws=ws), *expect(c), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeats_are_identical(dtype):
    c = make(50, 4, 8, 8, 128, [2000, 333, 1500, 64], 26, dtype, True)
    first = call(c)
    for _ in range(5):
        assert np.array_equal(call(c), first)


def test_bytes_for_codes():
    """uint8 tensors for the codes are as good as float8 ones."""
    c = make(51, 1, 2, 2, 64, [100], 1, "bf16", False)
    t = {w: dev(c[w]) for w in ("q", "K", "V", "Ke", "Ve", "kv_len")}
    out = torch.empty_like(t["q"])
    ws = workspace(1, 2, 2, 64, c["cap"], "bf16", 1)
    gb.glide_kv8_cross_attn(t["q"], t["K"].view(torch.uint8), t["V"].view(torch.uint8), t["Ke"], t["Ve"], t["kv_len"],
                            100, out, ws)
    assert np.array_equal(host(out), call(c)) and t["K"].dtype == F8
