"""Value blocks whose scale rises along a sequence by more than fp32's exponent range holds between two weights: the
softmax sum keeps the share of the rows before the rise."""
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


# the exponent before the rise (None: values of zero), and after it
STEPS = [(None, 37), (None, 100), (-60, 70), (-80, 110)]


def _step(c, blocks, low, high):
    """The first `blocks` blocks of the values at scale `low`, the others at `high`."""
    c["V"][:, :, :64 * blocks] = np.where(low is None, 0, c["V"][:, :, :64 * blocks])
    c["Ve"][:, :, :blocks] = kv8.EXP_MIN if low is None else low
    c["Ve"][:, :, blocks:] = high
    return c


# keys before the rise: a cluster of eight CTAs' first tiles; of one CTA's run, the blocks whose scales it holds at once
@pytest.mark.parametrize("low,high", STEPS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (12, 1), (30, 1), (40, 1), (64, 1)])
def test_cached_blocks(low, high, dtype, H, H_kv):
    c = _step(make(H, 1, H, H_kv, 128, [4096], 1, dtype, False), 32, low, high)
    want = expect(c)
    for max_ctas in (0, 1):
        check(call(c, max_ctas=max_ctas), *want, dtype)


@pytest.mark.parametrize("low,high", STEPS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 6, 13, 20, 40, 64])
def test_tree_before_the_cache(low, high, dtype, D, n):
    c = _step(make(n, 1, 2, 2, D, [40], n, dtype, True), 0, low, high)
    x = kv8.widen(c["v"]) * (0.0 if low is None else 2.0 ** (low + 7))
    c["v"] = x.astype(np.float32)
    if dtype == "bf16":
        c["v"] = (c["v"].view(np.uint32) >> np.uint32(16)).astype(np.uint16)  # exact: a power of two
    want = expect(c)
    for max_ctas in (0, 1):
        check(call(c, max_ctas=max_ctas), *want, dtype)
