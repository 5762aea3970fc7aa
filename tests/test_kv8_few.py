"""Few query rows over the 8-bit cache (the kernel without tensor memory), and the same calls on the streaming kernel,
which a bound on the CTAs selects."""
import numpy as np
import pytest
import torch

from kv8_util import F8, check, dev, host, workspace
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


# clusters of 1, 2, 4 and 8 CTAs; keys that end on, before and after a tile; more warps than tiles and more tiles than warps
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv_len", [[31], [32, 33], [255, 256, 257], [511, 40], [1030, 2, 700], [2500]])
@pytest.mark.parametrize("H,H_kv,n", [(1, 1, 1), (5, 1, 1), (16, 2, 1), (32, 2, 1), (3, 3, 7), (8, 2, 2), (2, 2, 16), (15, 3, 3)])
def test_rows_and_keys(D, kv_len, H, H_kv, n):
    c = make(H + n + sum(kv_len), len(kv_len), H, H_kv, D, kv_len, n, "bf16", n > 1)
    want = expect(c)
    check(call(c), *want, "bf16")
    check(call(c, max_ctas=1), *want, "bf16")


def test_chains_and_stars():
    """Trees as deep as their nodes and as flat as can be."""
    for n, parent in ((16, list(range(-1, 15))), (16, [-1] + [0] * 15), (16, [-1] * 16)):
        c = make(n, 2, 2, 2, 128, [300, 0], n, "bf16", True)
        c["parent"] = np.array([parent] * 2, dtype=np.int32)
        check(call(c), *expect(c), "bf16")


def test_bound_far_above_the_lengths():
    """What lies between a length and its bound (stale NaN codes, exponents that no block has) is not used."""
    c = make(77, 3, 4, 4, 128, [33, 0, 200], 5, "bf16", True, cap=3000)
    check(call(c, max_kv=2900), *expect(c), "bf16")
    c = make(78, 3, 4, 4, 64, [33, 0, 200], 1, "bf16", False, cap=3000)
    check(call(c, max_kv=2900), *expect(c), "bf16")


def test_repeats_are_identical():
    c = make(79, 2, 8, 8, 128, [2000, 333], 6, "bf16", True)
    first = call(c)
    for _ in range(5):
        assert np.array_equal(call(c), first)


def test_in_a_graph():
    c = make(80, 2, 4, 2, 128, [700, 65], 3, "bf16", True)
    t = {w: dev(c[w]) for w in ("q", "K", "V", "Ke", "Ve", "kv_len", "parent", "k", "v")}
    out = torch.zeros_like(t["q"])
    ws = workspace(2, 4, 2, 128, c["cap"], "bf16", 3)
    st = torch.cuda.Stream()

    def run():
        gb.glide_kv8_verify_attn(t["q"], t["parent"], t["k"], t["v"], t["K"], t["V"], t["Ke"], t["Ve"], t["kv_len"], 700, out,
                                 ws)
    with torch.cuda.stream(st):
        run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            run()
            run()
    out.zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    check(host(out), *expect(c), "bf16")


@pytest.mark.parametrize("rows", [1, 20])
def test_large_offsets(rows):
    """A cache whose offsets pass 32 bits: the last head's keys lie beyond 2^31 codes."""
    H, cap, D = 64, 270000, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.zeros((1, H, cap, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    for t in (K, V):  # codes of magnitude up to 15, either sign
        t[0, H - 1] = torch.randint(0, 0x58, (cap, D), generator=gen, device="cuda", dtype=torch.uint8)
        t[0, H - 1] |= torch.randint(0, 2, (cap, D), generator=gen, device="cuda", dtype=torch.uint8) << 7
    Ke, Ve = (torch.full((1, H, -(-cap // 64)), -3, dtype=torch.int8, device="cuda") for _ in range(2))
    q = torch.randn((1, 1, H * rows, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    kv_len = torch.tensor([cap], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    desc = gb.make_desc(1, H * rows, D, cap, gb.GLIDE_BF16, H_kv=H if rows > 1 else 0)
    ws = torch.zeros(gb.glide_kv8_workspace_bytes(desc, 1), dtype=torch.uint8, device="cuda")
    gb.glide_kv8_cross_attn(q, K.view(F8), V.view(F8), Ke, Ve, kv_len, cap, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    k, v = (t[0, H - 1].view(F8).double() * 0.125 for t in (K, V))
    w = torch.softmax(q[0, 0, -rows:].double() @ k.T / D ** 0.5, -1)
    check(host(out[0, 0, -rows:]), (w @ v).cpu().numpy(), (w @ v.abs()).cpu().numpy(), "bf16")
    assert not out[0, 0, :-rows].any()  # zero keys weigh alike, zero values
    del K, V, k, v, w
    torch.cuda.empty_cache()
