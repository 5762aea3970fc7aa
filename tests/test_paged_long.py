"""Contexts as long as a 32-bit length can say.  Page numbers may repeat, so a few pages hold them all."""
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import check, host, i32, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def test_a_token_over_the_longest_context():
    """2^31 - 1 keys of one page again and again, with score 0 and values 1; the last of them, in a page of its own, has score
    60 and so all the weight: the others together have 2^31 e^-60 < 2e-17 of it, which moves a column by less than
    2e-17 (1 + 43) < 1e-15, the whole numbers in V alone are held without rounding.  The row behind it holds NaN."""
    D, P, H, kv = 64, 256, 4, 2 ** 31 - 1
    width = -(-kv // P)
    K, V = torch.zeros((2, 1, P, D), dtype=torch.bfloat16), torch.zeros((2, 1, P, D), dtype=torch.bfloat16)
    q = torch.zeros((1, H, D), dtype=torch.bfloat16)
    q[:, :, 0], q[:, :, 1] = 8.0, torch.arange(H)
    last = (kv - 1) % P
    assert last == P - 2
    K[1, 0, last, 0] = 60.0                                   # 8 * 60 / sqrt(64)
    V[0, 0] = 1.0
    V[1, 0, last] = torch.arange(D) - 20.0
    K[1, 0, P - 1], V[1, 0, P - 1] = float("nan"), float("nan")
    table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    out = torch.zeros((1, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, 1, D, "bf16", 1, 1)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), table, i32([0, 1]), 1, i32([kv]), kv, out, ws)
    assert ((out.cpu().double() - V[1, 0, last].double()).abs() < 1e-15).all()
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK


def expected(q, K, V, table, kv, i, m):
    """(want, tolerance) [H, D] of row i of m new tokens: a softmax over the pool's rows, each as often as it is seen.

    A score is off by no more than in paged_util.tolerance.  Sums: a tensor core may lose 2^-25 of the sum so far at every key (it
    takes in at most 2^17 keys: 2^-8 of the mean of |v|) and 2^-23 at every 16 (2^-10); sums beyond that are in fp32, in few
    steps.  Each weight is rounded to bf16, 2^-8 of it, and the result."""
    H, D = q.shape[1:]
    H_kv, P = K.shape[1:3]
    n = kv - m + 1 + i
    times = torch.bincount(table[: n // P], minlength=len(K)).double()[:, None].expand(len(K), P).clone()
    if n % P:
        times[table[n // P], : n % P] += 1
    K, V, q = (x.double().cuda() for x in (K, V, q))
    K, V = (x.transpose(0, 1).reshape(H_kv, -1, D).repeat_interleave(H // H_kv, 0) for x in (K, V))
    s = torch.einsum("hkd,hd->hk", K, q[i]) * D ** -0.5
    top = (torch.einsum("hkd,hd->hk", K.abs(), q[i].abs()).amax(1) * D ** -0.5)[:, None]
    w = torch.exp(s - s.amax(1, keepdim=True)) * times.reshape(1, -1).cuda()
    w /= w.sum(1, keepdim=True)
    want, mean = torch.einsum("hk,hkd->hd", w, V), torch.einsum("hk,hkd->hd", w, V.abs())
    score = (D / 2 + 8) * top * 2.0 ** -23 + (top + 1) * 2.0 ** -22
    tol = (2 * score + 2.0 ** -8 + 2.0 ** -10 + 2.0 ** -8) * mean + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7)
    return host(want), host(tol)


SMS = 152
CASES = [
    # new tokens, keys, H, H_kv, D: few rows, a warp's keys in two spans and three; rows of a group
    (1, 2 ** 20 + 300, 2 * SMS + 2, 2 * SMS + 2, 64),
    (2, 2 ** 21 + 2 ** 19, 4 * SMS, 2 * SMS, 128),
    (5, 2 ** 21 + 777, 2 * SMS, SMS, 128),
    (3, 2 ** 24 + 2 ** 22 + 5, 2, 1, 64),
    # row tiles: an item in three segments, in eight; a call with its keys in chunks of more than one segment
    (17, 2 ** 18 + 5000, 2 * SMS, 2 * SMS, 64),
    (20, 2 ** 20, 2 * SMS, 2 * SMS, 128),
    (17, 2 ** 20 + 130, 8, 8, 128),
    (33, 2 ** 22 + 70, 2, 1, 64),
    (200, 2 ** 19 + 2 ** 18, 3 * SMS, SMS, 64),
    (40, 2 ** 19 + 1, SMS - 2, SMS - 2, 64),
]


@pytest.mark.parametrize("like", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_sums_of_very_many_keys(case, like):
    """Weights that are all alike, of values that are not 0 in the mean; and stretches of keys whose scores and values differ."""
    m, kv, H, H_kv, D = CASES[case]
    P, gen = 256, torch.Generator().manual_seed(case)
    stretches, each = 5, 3
    K = torch.zeros((stretches * each, H_kv, P, D)) if like else torch.randn((stretches * each, H_kv, P, D), generator=gen)
    V = 1 + torch.rand((stretches * each, H_kv, P, D), generator=gen)
    q = torch.randn((m, H, D), generator=gen)
    width = -(-kv // P)
    table = torch.randint(each, (width,), generator=gen) + torch.arange(width) * stretches // width * each
    if not like:  # a maximum that rises and falls from stretch to stretch
        q[..., 0] = 4.0
        for x, shift in enumerate((0.0, 2.0, -3.0, 2.5, 1.0)):
            K[x * each: (x + 1) * each, ..., 0] = shift * D ** 0.5 / 4
            V[x * each: (x + 1) * each] += x
    q, K, V = (x.bfloat16() for x in (q, K, V))
    out = torch.zeros((m, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, H_kv, D, "bf16", m, m)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), i32(table.numpy())[None], i32([0, m]), m, i32([kv]), kv, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    got = host(out)
    for i in sorted({0, m // 2, m - 1}):
        want, tol = expected(q, K, V, table, kv, i, m)
        check(got[i], want, tol, f"row {i}")
    again = torch.zeros_like(out)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), i32(table.numpy())[None], i32([0, m]), m, i32([kv]), kv, again, ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("m, H, D", [(1, SMS, 64), (3, SMS, 128), (17, SMS, 64), (40, SMS, 128)])
def test_requests_of_very_different_lengths(m, H, D):
    """In one call: one of many sums, one of few tokens, one of none but the new ones."""
    P, gen, lens = 256, torch.Generator().manual_seed(m), [m, 2 ** 20 + 300, 700, 2 ** 17 + 1280]
    K = torch.randn((8, H, P, D), generator=gen).bfloat16()
    V = (1 + torch.rand((8, H, P, D), generator=gen)).bfloat16()
    q = torch.randn((m * len(lens), H, D), generator=gen).bfloat16()
    table = torch.randint(8, (len(lens), -(-max(lens) // P)), generator=gen)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device="cuda")
    ws = workspace(len(lens), H, H, D, "bf16", len(q), m)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), i32(table.numpy()), i32([m * b for b in range(len(lens) + 1)]), m, i32(lens),
                        max(lens), out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    got = host(out)
    for b, kv in enumerate(lens):
        for i in {0, m - 1}:
            want, tol = expected(q[b * m: (b + 1) * m], K, V, table[b], kv, i, m)
            check(got[b * m + i], want, tol, f"request {b}, row {i}")


@pytest.mark.parametrize("m, H, D, kv", [(1, 2 * SMS + 2, 64, 2 ** 20 + 300), (17, 2 * SMS, 64, 2 ** 17 + 5000), (40, 8, 128, 2 ** 20 + 1)])
def test_infinite_values_in_long_contexts(m, H, D, kv):
    """One in the first keys, that every row sees, one in the last key, that the last row alone sees, and NaN in a key and a value
    behind it that no row sees.  (A warp's spans, an item's segments, segments of chunks.)"""
    P, gen = 256, torch.Generator().manual_seed(m)
    K = torch.randn((6, H, P, D), generator=gen).bfloat16()
    V = (1 + torch.rand((6, H, P, D), generator=gen)).bfloat16()
    q = torch.randn((m, H, D), generator=gen).bfloat16()
    width, last = -(-kv // P), (kv - 1) % P
    table = torch.randint(1, 4, (width,), generator=gen)
    table[0], table[-1] = 4, 5
    V[4, :, 2, 3] = float("inf")
    V[5, :, last, 7] = -float("inf")
    if last + 1 < P:
        K[5, :, last + 1], V[5, :, last + 1] = float("nan"), float("nan")
    out = torch.zeros((m, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, H, D, "bf16", m, m)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), i32(table.numpy())[None], i32([0, m]), m, i32([kv]), kv, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    got = host(out)
    finite_K, finite_V = (torch.where(X.isfinite(), X, 0) for X in (K, V))
    for i in sorted({0, m - 1}):
        want, tol = expected(q, finite_K, finite_V, table, kv, i, m)
        assert (got[i, :, 3] == float("inf")).all()
        assert (got[i, :, 7] == -float("inf")).all() if i == m - 1 else True
        odd = [3, 7] if i == m - 1 else [3]
        got[i][:, odd], want[:, odd] = 0, 0
        check(got[i], want, tol, f"row {i}")


def test_a_prompt_of_more_keys_than_one_sum_takes():
    n, H, H_kv, D = 2 ** 17 + 2 ** 14 + 77, 2, 1, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n, H + 2 * H_kv, D), generator=gen, device="cuda")
    x[:, H + H_kv:] = 1 + x[:, H + H_kv:].abs()
    q, k, v = x.bfloat16().split([H, H_kv, H_kv], 1)
    out = torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, H_kv, D, "bf16", n, n)
    gb.glide_prompt_attn(q, k, v, i32([0, n]), n, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    pool = [t.transpose(0, 1)[:, None].reshape(1, 1, n, D) for t in (k, v)]  # one page of all keys
    for i in (5, 2 ** 17 - 1, 2 ** 17, 2 ** 17 + 129, n - 1):
        want, tol = expected(q[i: i + 1], *(t[:, :, : i + 1] for t in pool), torch.tensor([0]), i + 1, 0, 1)
        check(host(out[i]), want, tol, f"row {i}")
