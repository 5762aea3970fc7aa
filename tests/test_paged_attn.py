"""Attention of new tokens over pages against the oracle, with NaN in every row of the pool that no token sees."""
import numpy as np
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import SENTINEL, Paged, check, host, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


CASES = [
    # m, kv, H, H_kv, D, P, dtype, pad, fused
    ([1], [1], 1, 1, 64, 16, "bf16", 0, False),
    ([1], [33], 4, 4, 128, 16, "bf16", 0, False),
    ([1], [700], 8, 2, 128, 16, "bf16", 0, True),
    ([1, 1, 1, 1], [1, 17, 250, 129], 8, 8, 64, 32, "bf16", 3, False),
    ([1, 0, 1], [300, 50, 0], 12, 4, 128, 64, "bf16", 1, True),
    ([6, 6, 2], [900, 6, 131], 4, 4, 128, 64, "bf16", 0, False),
    ([5, 1, 3], [64, 65, 63], 8, 1, 64, 16, "bf16", 2, True),
    ([4, 16], [128, 257], 8, 2, 128, 16, "bf16", 0, False),
    ([17, 1, 33], [400, 513, 33], 6, 2, 128, 16, "bf16", 0, True),
    ([40, 7], [300, 7], 3, 3, 64, 128, "bf16", 5, False),
    ([129, 300, 1], [129, 555, 800], 2, 2, 128, 256, "bf16", 0, True),
    ([200, 0, 77, 1], [700, 0, 100, 1], 8, 2, 128, 32, "bf16", 9, True),
    ([130], [1500], 4, 1, 64, 16, "bf16", 0, False),
    ([40], [2600], 4, 1, 128, 16, "bf16", 0, True),          # few rows, long contexts: the keys are cut into chunks
    ([33, 1, 20], [1700, 2500, 300], 2, 2, 64, 32, "bf16", 2, False),
    ([260, 70], [2100, 1900], 3, 1, 128, 64, "bf16", 1, False),
    ([300], [290], 1, 1, 128, 16, "bf16", 0, False),
    ([150, 40], [1650, 20], 2, 1, 64, 128, "bf16", 0, True),
    ([3, 9], [1, 4], 4, 2, 128, 16, "bf16", 0, False),       # rows before any key: zeros
    ([150, 20], [90, 19], 4, 2, 128, 16, "bf16", 0, False),
    ([1, 5, 20], [77, 5, 300], 4, 2, 64, 16, "f32", 2, True),
    ([2, 30], [1, 30], 3, 1, 128, 32, "f32", 0, False),
    # many row tiles, few of them, with long contexts: chunks of entries that are listed
    ([40, 33, 1, 0, 20, 7], [2600, 1700, 2000, 30, 900, 2400], 32, 1, 64, 16, "bf16", 0, True),
    # more requests than a warp's lanes, and than are sorted, one of them long
    ([3, 0, 1, 9] * 10, [40, 7, 300, 20] * 8 + [2500, 0, 130, 9, 3, 3, 1, 1990], 32, 1, 64, 16, "bf16", 3, False),
    # many short requests
    ([1, 1, 2, 0] * 45, [1, 30, 2, 0] * 45, 2, 2, 64, 16, "bf16", 1, False),
    ([1, 1, 0, 1] * 50, [70, 129, 5, 300] * 49 + [0, 2300, 8, 1], 32, 1, 64, 16, "bf16", 0, False),
]


@pytest.mark.parametrize("flags", [0, gb.GLIDE_FLAG_FORCE_FMA])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows(case, flags):
    m, kv, H, H_kv, D, P, dtype, pad, fused = CASES[case]
    s = Paged(case, m, kv, H, H_kv, D, P, dtype, pad=pad, fused=fused)
    s.upload()
    out = s.run(flags=flags)
    want, tol = s.want()
    check(host(out), want, tol)
    # again on the same workspace, with looser bounds: the same bits
    again = s.run(max_q=max(m) + 3, max_kv=(s.table.shape[1]) * P, flags=flags,
                  ws=torch.zeros(256 << 20, dtype=torch.uint8, device="cuda"))
    check(host(again), want, tol)
    assert torch.equal(s.run(flags=flags, ws=s.ws), s.run(flags=flags, ws=s.ws))
    assert gb.glide_read_device_status(s.ws) == gb.GLIDE_OK


def test_scale():
    s = Paged(77, [1, 20, 200], [300, 150, 260], 4, 2, 128, 16, "bf16")
    s.upload()
    for scale in (0.31, 0.01):
        want, tol = s.want(scale)
        check(host(s.run(scale=scale)), want, tol)


@pytest.mark.parametrize("m", [[3, 2], [12, 40], [200, 150]])
def test_bounds_below_the_lengths(m):
    """Rows past max_q stay as they were; keys past max_kv_len are not there."""
    kv = [m[0] + 100, m[1] + 30]
    s = Paged(5, m, kv, 4, 2, 64, 16, "bf16")
    s.upload()
    most = 90
    out = host(s.run(max_q=2, max_kv=most))
    kept = Paged(5, m, kv, 4, 2, 64, 16, "bf16")
    kept.kv = [min(x, most) for x in kv]
    want, tol = kept.want()
    for b in range(2):
        want[s.cu[b] + 2: s.cu[b + 1]] = SENTINEL
        tol[s.cu[b] + 2: s.cu[b + 1]] = 0
    check(out, want, tol)


@pytest.mark.parametrize("flags", [0, gb.GLIDE_FLAG_FORCE_FMA])
@pytest.mark.parametrize("m, kv", [([1, 1], [200, 300]), ([4, 5], [140, 300]), ([150, 140], [300, 140]), ([40, 70], [2400, 1800])])
def test_what_is_not_finite(m, kv, flags):
    """In rows that some tokens see and others do not, and in the queries."""
    H, H_kv, D, P = 4, 2, 128, 16
    s = Paged(9, m, kv, H, H_kv, D, P, "bf16")
    rng = np.random.default_rng(2)

    def put(X, b, t, h, d, x):
        X[s.table[b, t // P], h, t % P, d] = x
    for b in range(2):
        put(s.V, b, kv[b] - 1, 0, 3, np.inf)           # the last token's value
        put(s.V, b, kv[b] - m[b] // 2 - 1, 0, 7, -np.inf)
        put(s.V, b, kv[b] - m[b] // 2 - 1, 0, 3, np.nan)
        put(s.V, b, 5, 1, 100, np.inf)
    put(s.K, 1, kv[1] - 1, 1, 9, np.nan)                # a key that the last token alone sees
    put(s.K, 0, kv[0] - 1, 1, 9, np.inf)                # a score of +inf or -inf
    s.q[0, 1] = np.nan
    s.q[s.cu[1], 2, 5] = np.inf
    s.q[s.cu[1], 2, rng.integers(6, D)] = 0
    s.upload()
    want, tol = s.want()
    check(host(s.run(flags=flags)), want, tol)


def test_scores_of_minus_infinity_everywhere():
    s = Paged(21, [1, 2], [40, 50], 2, 2, 64, 16, "bf16")
    s.K[s.table[0, 0], :, : , 0] = -np.inf
    s.K[s.table[0, 1], :, :, 0] = -np.inf
    s.K[s.table[0, 2], :, :, 0] = -np.inf
    s.q[:, :, 0] = 1.0
    s.upload()
    want, tol = s.want()
    assert np.isnan(want[0]).all() and np.isfinite(want[1:]).all()
    check(host(s.run()), want, tol)


def test_another_stream_and_a_graph():
    s = Paged(31, [1, 9, 70], [300, 200, 170], 8, 2, 128, 16, "bf16")
    s.upload()
    want, tol = s.want()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out = s.run(ws=ws)
    side.synchronize()
    check(host(out), want, tol)
    g = torch.cuda.CUDAGraph()
    out = torch.empty_like(out)
    with torch.cuda.graph(g):
        gb.glide_paged_attn(s.qd, s.Kd, s.Vd, s.tabled, s.cud, 70, s.kvd, 300, out, ws)
    for _ in range(3):
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        check(host(out), want, tol)
    # other lengths under the same bounds
    s.kvd.copy_(i32([250, 10, 170]))
    s.kv = [250, 10, 170]
    g.replay()
    torch.cuda.synchronize()
    check(host(out), *s.want())


def test_a_pool_beyond_32_bits():
    """Pages far behind in a pool of more than 2^32 bytes and 2^31 elements."""
    n, H, P, D = 530000, 2, 16, 128
    K, V = (torch.zeros((n, H, P, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for m, kv in (([1, 1], [100, 90]), ([40, 130], [100, 200])):
        s = Paged(3, m, kv, 2, 2, D, P, "bf16")
        s.upload()
        far = len(s.Kd)
        K[-far:], V[-far:] = s.Kd, s.Vd
        want, tol = s.want()
        s.Kd, s.Vd = K, V
        s.tabled = torch.where((s.tabled >= 0) & (s.tabled < far), s.tabled + (n - far), s.tabled)
        check(host(s.run()), want, tol)


def test_a_workspace_shared_with_tree_verification():
    """A step whose keys are cut into chunks leaves at zero what other calls on its workspace take their counters from."""
    s = Paged(70, [40], [2600], 4, 1, 128, 16, "bf16")
    s.upload()
    out = s.run()
    assert not s.ws[: 256 + 4 * 1024 * s.H].any()
    n, B, H, D, S = 5, 3, 4, 128, 700
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, K, V = (torch.randn(shape, generator=gen, device="cuda").bfloat16() for shape in ((B, n, H, D), (B, H, S, D), (B, H, S, D)))
    kv, parent = i32([600, 1, 333]), i32([[-1, 0, 1, 1, 0]] * B)
    results = []
    for ws in (s.ws, torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")):
        for flags in (0, gb.GLIDE_FLAG_FORCE_FMA):
            results.append(gb.tree_verify_attn(q, parent, K, V, kv, 600, torch.empty((B, n, H, D), device="cuda"), ws, flags=flags))
        results.append(s.run(ws=ws))
    assert all(torch.equal(a, b) for a, b in zip(results[:3], results[3:]))
    assert torch.equal(results[2], out)
