"""Finite values near the largest that a type holds: a weight that is 0 counts as 0 for them, and a sum of weights times
values that passes the type's range has a mean that does not."""
import numpy as np
import pytest

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import Paged, Prompt, check, host, rounded

pytestmark = pytest.mark.gpu
FMA = gb.GLIDE_FLAG_FORCE_FMA


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


# one warp a row, a block a row, few new tokens, row tiles, keys in chunks
PAGES = [
    ([1, 3], [20, 30], 4, 2, 64, "f32", 0),
    ([1, 6], [200, 70], 4, 2, 64, "f32", 0),
    ([2], [150], 2, 1, 128, "f32", 0),
    ([1, 5], [25, 31], 4, 2, 128, "bf16", FMA),
    ([2, 40], [130, 220], 4, 2, 128, "bf16", FMA),
    ([1, 2], [200, 333], 4, 2, 128, "bf16", 0),
    ([4, 4], [140, 900], 8, 2, 64, "bf16", 0),
    ([150, 40], [300, 140], 4, 2, 128, "bf16", 0),
    ([30, 140], [290, 170], 4, 2, 64, "bf16", 0),
    ([40], [2600], 4, 1, 128, "bf16", 0),
]


def far_below(s, K, V, at):
    """Rows of K and V whose scores lie 200 below the others' and whose values are large; an infinity in another column, which
    makes the tensor-core kernels compute the row again."""
    scale = s.D ** -0.5
    for n, x in enumerate(at):
        K[x][..., 0] = -200.0 / (8.0 * scale)
        V[x][..., 1 + n % 5] = (-1) ** n * 1e38
    V[at[0]][..., 40] = np.inf


@pytest.mark.parametrize("infinite", [False, True])
@pytest.mark.parametrize("case", range(len(PAGES)))
def test_a_weight_of_zero(case, infinite):
    """exp(-200) 1e38 < 1e-48: the columns are what the other keys make of them."""
    m, kv, H, H_kv, D, dtype, flags = PAGES[case]
    s = Paged(100 + case, m, kv, H, H_kv, D, 16, dtype)
    s.q[..., 0], s.K[..., 0] = 8.0, 0.0
    for b in range(len(m)):
        at = [(s.table[b, t // 16], slice(None), t % 16) for t in (0, 3, kv[b] // 2, kv[b] - m[b])]
        far_below(s, s.K, s.V, at)
    if not infinite:
        s.V[np.isinf(s.V)] = 1.0
    s.q, s.K, s.V = (rounded(x, dtype) for x in (s.q, s.K, s.V))
    s.upload()
    want, tol = s.want()
    assert np.isinf(want).any() == infinite
    check(host(s.run(flags=flags)), want, tol)


@pytest.mark.parametrize("case", range(len(PAGES)))
def test_a_sum_beyond_the_range(case):
    """Many values of 3e38 with like weights, all of one sign in one column, of both in others; and of fp32's largest."""
    m, kv, H, H_kv, D, dtype, flags = PAGES[case]
    s = Paged(200 + case, m, kv, H, H_kv, D, 16, dtype, spread=0.3)
    rng = np.random.default_rng(case)
    for b in range(len(m)):
        for t in range(kv[b]):
            v = s.V[s.table[b, t // 16], :, t % 16]
            v[:, 5] = 3e38
            v[:, 6] = rng.choice([-3e38, 3e38])
            v[:, D - 1] = 3e38 * rng.random()
            if t % 7 == 0:
                v[:, 17] = -3e38
            v[:, 9] = np.finfo(np.float32).max if dtype == "f32" else 3.3e38
    s.V = rounded(s.V, dtype)
    assert np.isinf(s.V).sum() == 0
    s.upload()
    want, tol = s.want()
    got = host(s.run(flags=flags))
    # the mean of fp32's largest values is that value, which no rounding passes
    assert np.isfinite(want).all() and np.isfinite(got).all()
    check(got, want, tol)


PROMPTS = [([20, 1, 31], 4, 2, 64, "f32", 0), ([60, 128], 4, 4, 64, "f32", 0), ([17, 32, 5], 8, 8, 128, "bf16", 0),
           ([130, 40], 4, 2, 128, "bf16", FMA), ([300, 1, 140], 4, 2, 128, "bf16", 0), ([33, 260], 6, 2, 64, "bf16", 0)]


@pytest.mark.parametrize("infinite", [False, True])
@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(case, infinite):
    lens, H, H_kv, D, dtype, flags = PROMPTS[case]
    s = Prompt(300 + case, lens, H, H_kv, D, dtype, spread=0.5)
    s.k, s.v = s.k.copy(), s.v.copy()
    for b, n in enumerate(lens):
        if n < 10:
            continue
        at = [(s.cu[b] + t,) for t in (1, 3, n // 2)]
        s.q[..., 0], s.k[s.cu[b]: s.cu[b + 1], :, 0] = 8.0, 0.0
        for x in at:
            s.k[x][..., 0] = -200.0 * D ** 0.5 / 8.0
            s.v[x][..., 3] = -1e38
        s.v[s.cu[b] + 4: s.cu[b + 1], :, 11] = 2.9e38
        if infinite:
            s.v[at[0]][..., 40] = np.inf
    s.q, s.k, s.v = (rounded(x, dtype) for x in (s.q, s.k, s.v))
    s.upload()
    want, tol = s.want()
    assert np.isinf(want).any() == infinite
    check(host(s.run(flags=flags)), want, tol)
