"""An infinity among the values of the tree is the infinity of its column in every row that sees it, however small the
row's weight for it, in every kernel and however many CTAs share the keys."""
import numpy as np
import pytest

from kv8_util import check
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

pytestmark = pytest.mark.gpu

INF = {"bf16": {1: 0x7f80, -1: 0xff80}, "f32": {1: np.inf, -1: -np.inf}}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_ctas", [0, 1, 3])
@pytest.mark.parametrize("kv_len", [40, 700, 2100])
@pytest.mark.parametrize("n", [3, 12, 20, 40, 64])
def test_value_of_vanishing_weight(dtype, max_ctas, kv_len, n):
    c = make(n + kv_len, 1, 2, 2, 64, [kv_len], n, dtype, True)
    c["parent"][:] = [-1, 0, 0] + [1] * (n - 3)
    c["q"][:] = c["q"][:, :1]
    q = kv8.widen(c["q"])[:, 0]                        # [1, 2, 64], every node's
    k = -1600.0 * q / (q ** 2).sum(-1, keepdims=True)  # scores of -200
    k = k.astype(np.float32)
    c["k"][:] = ((k.view(np.uint32) >> np.uint32(16)).astype(np.uint16) if dtype == "bf16" else k)[:, None]
    c["v"][:, 1, 0, 7], c["v"][:, 2, 1, 63] = INF[dtype][1], INF[dtype][-1]
    want, size = expect(c)
    assert np.isposinf(want[0, 1, 0, 7]) and np.isneginf(want[0, 2, 1, 63]) and np.isinf(want).sum() == n - 1
    check(call(c, max_ctas=max_ctas), want, size, dtype)
