"""Query rows that share a cached head and are of very different size: none has a say in another's result."""
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv,n", ROWS)
def test_largest_query(dtype, D, H, H_kv, n):
    """The last node's queries are of the type's largest magnitude."""
    c = make(n + D, 2, H, H_kv, D, [300, 40], n, dtype, True)
    big = np.where(np.arange(D) % 2, LARGEST[dtype], -LARGEST[dtype]).astype(np.float32)
    c["q"][:, n - 1] = bf16_bits(big) if dtype == "bf16" else big
    want, size = expect(c)
    for max_ctas in (0, 1):
        check(call(c, max_ctas=max_ctas)[:, :n - 1], want[:, :n - 1], size[:, :n - 1], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [10, 16, 24])
@pytest.mark.parametrize("H,H_kv,n", ROWS + [(16, 1, 1), (40, 1, 1)])
def test_small_query_beside_a_large_one(dtype, power, H, H_kv, n):
    """Keys so large that queries of 2^-power of one neighbour's have scores of ordinary size."""
    c = make(n + H, 2, H, H_kv, 128, [300, 77], n, dtype, n > 1)
    c["Ke"] = (c["Ke"] + 8).astype(np.int8)
    q = kv8.widen(c["q"]) * 2.0 ** -8
    q[:, 0, 0] *= 2.0 ** power
    c["q"] = bf16_bits(q) if dtype == "bf16" else q.astype(np.float32)
    want, size = expect(c)
    rest = np.ones((n, H), dtype=bool)
    rest[0, 0] = False
    for max_ctas in (0, 1):
        got = call(c, max_ctas=max_ctas)
        check(got[:, rest], want[:, rest], size[:, rest], dtype)
