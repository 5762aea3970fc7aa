"""Long runs of one CTA over a slab: the block scales that it holds last 16 tiles of 128 keys, and are read again in
time for the tile after, for each size of a row tile.  Blocks differ in scale, so that another block's shows."""
import numpy as np
import pytest

from kv8_util import check
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def _case(seed, H, H_kv, D, kv_len, n):
    """Keys of magnitude 1/4 .. 2 and values of 1/4 .. 8, by block."""
    c = make(seed, len(kv_len), H, H_kv, D, kv_len, n, "bf16", n > 1)
    rng = np.random.default_rng(seed + 1)
    for w, top in (("K", -4), ("V", -2)):
        c[w] = kv8.encode(64.0 * rng.standard_normal(c[w].shape))
        c[w + "e"] = rng.integers(-8, top, c[w + "e"].shape).astype(np.int8)
    return c


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv,n", [(2, 2, 7), (2, 2, 12), (2, 2, 29), (2, 2, 45), (2, 2, 64), (8, 2, 33), (6, 2, 1)])
@pytest.mark.parametrize("kv_len", [[2048, 1920], [2049, 4097], [4224, 100, 6273]])
def test_scales_last(D, H, H_kv, n, kv_len):
    c = _case(n + D, H, H_kv, D, kv_len, n)
    want, size = expect(c)
    for max_ctas in (1, 2):  # so few that the tcgen05 kernel serves every number of rows
        check(call(c, max_ctas=max_ctas), want, size, "bf16")
