"""Causal attention of packed prompts against the oracle."""
import numpy as np
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import SENTINEL, Prompt, check, host, tolerance, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


CASES = [
    # lens, H, H_kv, D, dtype, pad, fused
    ([1], 1, 1, 64, "bf16", 0, False),
    ([2, 0, 1], 4, 4, 128, "bf16", 0, True),
    ([31, 64, 1, 0, 65], 4, 2, 64, "bf16", 7, True),
    ([127, 128, 129], 2, 2, 128, "bf16", 0, False),
    ([255, 256, 257], 2, 1, 128, "bf16", 3, True),
    ([512, 3, 600], 3, 1, 128, "bf16", 0, True),
    ([300, 700], 8, 1, 64, "bf16", 1, True),
    ([1300], 4, 4, 128, "bf16", 0, True),
    ([2300], 2, 1, 64, "bf16", 0, False),
    ([1800, 5, 1601], 1, 1, 128, "bf16", 4, True),
    ([1, 1, 1, 1, 1, 1, 1, 200], 5, 5, 128, "bf16", 0, False),
    ([90], 34, 2, 64, "bf16", 0, True),
    ([9, 1, 30], 64, 1, 128, "bf16", 0, False),
    ([5, 2], 130, 1, 64, "bf16", 0, True),
    ([70], 40, 1, 64, "bf16", 1, True),
    ([60, 128], 4, 4, 64, "f32", 3, False),
    ([33, 1, 100], 6, 2, 128, "f32", 0, True),
]


@pytest.mark.parametrize("flags", [0, gb.GLIDE_FLAG_FORCE_FMA])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows(case, flags):
    lens, H, H_kv, D, dtype, pad, fused = CASES[case]
    s = Prompt(100 + case, lens, H, H_kv, D, dtype, pad=pad, fused=fused)
    s.upload()
    out = s.run(flags=flags)
    want, tol = s.want()
    check(host(out), want, tol)
    assert torch.equal(s.run(flags=flags, ws=s.ws, max_len=max(lens)), out)
    assert gb.glide_read_device_status(s.ws) == gb.GLIDE_OK


@pytest.mark.parametrize("max_len", [12, 33])
def test_many_sequences(max_len):
    rng = np.random.default_rng(0)
    s = Prompt(1, rng.integers(0, 12, 1024).tolist(), 2, 1, 64, "bf16", pad=2)
    s.upload()
    want, tol = s.want()
    check(host(s.run(max_len=max_len)), want, tol)


@pytest.mark.parametrize("n", [1, 31, 32, 33])
@pytest.mark.parametrize("B", [1, 9, 40])
def test_short_sequences(B, n):
    """On both sides of the lengths and of the numbers of rows that decide the kernel."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, n + 1, B)
    lens[B // 2] = n
    s = Prompt(10 + n, lens.tolist(), 8, 2, 64, "bf16", pad=1, fused=True)
    s.upload()
    check(host(s.run()), *s.want())


def test_more_row_tiles_than_are_listed():
    """4096 row tiles of four tokens: 1024 sequences of 13 tokens, 32 query heads over one cached head."""
    B, n, H, D = 1024, 13, 32, 64
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((B * n, H + 2, D), generator=gen, device="cuda").bfloat16()
    q, k, v = x.split([H, 1, 1], 1)
    cu = torch.arange(B + 1, device="cuda", dtype=torch.int32) * n
    out = torch.full((B * n, H, D), SENTINEL, dtype=torch.bfloat16, device="cuda")
    gb.glide_prompt_attn(q, k, v, cu, n, out, workspace(B, H, 1, D, "bf16", B * n, n))
    Q, K, V = (t.double().view(B, n, -1, D).transpose(1, 2) for t in (q, k, v))
    hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    p = torch.softmax((Q @ K.transpose(-1, -2) * D ** -0.5).masked_fill(hidden, -float("inf")), -1)
    want, mean = p @ V, p @ V.abs()
    top = (Q.abs() @ K.abs().transpose(-1, -2)).amax(-1).reshape(-1) * D ** -0.5
    want, mean = (t.reshape(-1, D).cpu().numpy() for t in (want, mean))
    check(host(out.view(B, n, H, D).transpose(1, 2)).reshape(-1, D), want, tolerance(want, mean, top.cpu().numpy(), n, D, "bf16"))


def test_rows_past_max_len():
    s = Prompt(2, [300, 20, 150], 2, 2, 64, "bf16")
    s.upload()
    want, tol = s.want()
    for b, n in enumerate(s.lens):
        want[s.cu[b] + 140: s.cu[b + 1]] = SENTINEL
        tol[s.cu[b] + 140: s.cu[b + 1]] = 0
    check(host(s.run(max_len=140)), want, tol)


@pytest.mark.parametrize("flags", [0, gb.GLIDE_FLAG_FORCE_FMA])
def test_what_is_not_finite(flags):
    """An infinity or NaN of one token reaches the tokens that see it, and no other sequence's."""
    s = Prompt(3, [200, 300, 40], 4, 2, 128, "bf16")
    c = s.cu
    s.v[c[0] + 150, 0, 4] = np.inf
    s.v[c[0] + 180, 0, 4] = -np.inf
    s.v[c[1] + 299, 1, 9] = np.nan
    s.k[c[1] + 130, 0, 3] = np.nan
    s.k[c[2], 1, 3] = -np.inf
    s.q[c[2], 2] = np.abs(s.q[c[2], 2])
    s.q[c[1] + 10, 3, 0] = np.inf
    s.upload()
    want, tol = s.want()
    check(host(s.run(flags=flags)), want, tol)


def test_large_scores():
    """Scores far apart: almost all the weight on one key."""
    s = Prompt(4, [260, 131], 2, 2, 64, "bf16", spread=20.0)
    s.upload()
    want, tol = s.want()
    check(host(s.run()), want, tol)


def test_two_graphs_of_one_workspace():
    a, b = Prompt(5, [200, 90], 4, 2, 128, "bf16"), Prompt(6, [33, 500], 4, 2, 128, "bf16")
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for s in (a, b):
        s.upload()
        outs.append(s.run(ws=ws))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            gb.glide_prompt_attn(s.qd, s.kd, s.vd, s.cud, max(s.lens), outs[-1], ws)
        graphs.append(g)
    for _ in range(2):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for s, o in zip((a, b), outs):
        check(host(o), *s.want())


def test_two_streams_at_once():
    """Calls that run beside one another, on workspaces of their own, give what they give alone."""
    cases = [Prompt(7, [200, 90, 400], 4, 2, 128, "bf16"), Prompt(8, [2300], 2, 1, 64, "bf16"), Prompt(9, [5, 1, 3], 4, 4, 64, "bf16")]
    alone, streams = [], [torch.cuda.Stream() for _ in cases]
    for s in cases:
        s.upload()
        alone.append(s.run())
    torch.cuda.synchronize()
    outs = [[] for _ in cases]
    for _ in range(10):
        for i, (s, stream) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(stream):
                outs[i].append(s.run(ws=s.ws))
    torch.cuda.synchronize()
    for want, got in zip(alone, outs):
        assert all(torch.equal(want, g) for g in got)
