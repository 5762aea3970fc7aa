"""What a row does not see has no say in its result, whatever its size: values and keys of a type's largest magnitude
in nodes that are neither the row nor its ancestors."""
import numpy as np
import pytest

from kv8_util import bf16_bits, check
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

pytestmark = pytest.mark.gpu

LARGEST = {"bf16": 3.3895313892515355e38, "f32": 3.4028234663852886e38}
# query rows of every kernel: few rows, and tiles of 8, 16, 32, 48 and 64 rows (H / H_kv of them a node)
ROWS = [(2, 2, 3), (2, 2, 8), (2, 2, 16), (2, 2, 20), (2, 2, 40), (2, 2, 64), (8, 2, 33)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def _check_nodes(got, want, size, dtype, nodes):
    check(got[:, nodes], want[:, nodes], size[:, nodes], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["v", "k"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv,n", ROWS)
def test_unseen_node(dtype, what, D, H, H_kv, n):
    """The last node is a leaf: its own row alone sees it."""
    c = make(n + D, 2, H, H_kv, D, [300, 40], n, dtype, True)
    big = np.where(np.arange(D) % 2, LARGEST[dtype], -LARGEST[dtype]).astype(np.float32)
    c[what][:, n - 1] = bf16_bits(big) if dtype == "bf16" else big
    want, size = expect(c)
    for max_ctas in (0, 1):
        _check_nodes(call(c, max_ctas=max_ctas), want, size, dtype, slice(0, n - 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv,n", ROWS)
def test_seen_by_some(dtype, H, H_kv, n):
    """Values of 2^100 in one branch: the rows of the other do not lose their own."""
    c = make(n, 1, H, H_kv, 128, [500], n, dtype, True)
    c["parent"][:] = [-1] + [max(0, i - 2) for i in range(1, n)]    # odd nodes below 1, even ones below 2 (and 0)
    c["parent"][:, 2] = 0
    x = kv8.widen(c["v"])
    x[:, 1] *= 2.0 ** 100
    c["v"] = bf16_bits(x) if dtype == "bf16" else x.astype(np.float32)
    want, size = expect(c)
    for max_ctas in (0, 1):
        check(call(c, max_ctas=max_ctas), want, size, dtype)
