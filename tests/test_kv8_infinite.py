"""Infinities in what an attention call over the 8-bit cache meets, against the definition in 64 bits, in every kernel:
an infinite query makes its row NaN; an infinite key of the tree makes a row that sees it NaN where the score is +inf and
has no weight where it is -inf."""
import numpy as np
import pytest

from kv8_util import check
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

pytestmark = pytest.mark.gpu

INF = {"bf16": {1: 0x7f80, -1: 0xff80}, "f32": {1: np.inf, -1: -np.inf}}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def _expect(c):
    with np.errstate(invalid="ignore"):
        return expect(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("max_ctas", [0, 1])
@pytest.mark.parametrize("H,H_kv", [(4, 4), (12, 1), (40, 2)])
def test_query(dtype, sign, max_ctas, H, H_kv):
    c = make(3, 4, H, H_kv, 128, [1, 0, 40, 1], 1, dtype, False)
    c["q"][:, 0, ::2, 5] = INF[dtype][sign]
    want, size = _expect(c)
    assert np.isnan(want[0, 0, ::2]).all() and not want[1].any() and np.isfinite(want[:, 0, 1::2]).all()
    check(call(c, max_ctas=max_ctas), want, size, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("max_ctas", [0, 1, 3])
@pytest.mark.parametrize("kv_len", [0, 1, 700])
@pytest.mark.parametrize("H,n", [(2, 3), (8, 3), (2, 20), (2, 40), (2, 64)])
def test_tree_key(dtype, sign, max_ctas, kv_len, H, n):
    c = make(n + kv_len, 2, H, 2, 128, [kv_len, 300], n, dtype, True)
    c["parent"][:] = [-1, 0, 0] + [1] * (n - 3)
    c["k"][:, 0, 0, 9] = INF[dtype][sign]    # the root's, which every row sees
    c["k"][:, 2, 1, 3] = INF[dtype][-sign]   # a leaf's
    want, size = _expect(c)
    spoiled = np.isnan(want).all(-1)
    assert spoiled[1, :, :H // 2].any() and not spoiled[1, :, :H // 2].all()
    assert spoiled[0, 0, :H // 2].all() or kv_len
    check(call(c, max_ctas=max_ctas), want, size, dtype)
