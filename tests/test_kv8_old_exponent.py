"""An exponent outside the allowed range counts as the nearest in it when rows join its block, as it does in reading and
attention: the rows that are there keep their values as far as the grown exponent lets them."""
import numpy as np
import pytest

from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_cache import _append, _case, _expect, _same


def _with(old, n, scale, dtype="f32"):
    c = _case(13, 2, 2, 64, 200, [40, 100], n, dtype, scale=scale)
    for w in ("Ke", "Ve"):
        c[w][:, :, :2] = old
    return c


@pytest.mark.parametrize("old", [-128, 127])
def test_oracle(old):
    c = _with(old, 5, 1e-35)
    K, _, Ke, _, new_len = _expect(c)
    before, after = (kv8.kv8_read(k, e, [40, 100], 100) for k, e in ((c["K"], c["Ke"]), (K, Ke)))
    step = 2.0 ** (Ke[:, :, :2].max() - 10)  # half the least step of the codes
    assert np.all(np.abs(after - before) <= np.maximum(step, np.abs(before) / 16))


@pytest.mark.gpu
@pytest.mark.parametrize("old", [-128, -118, 120, 127])
@pytest.mark.parametrize("scale", [0.0, 1e-35, 1.0])
@pytest.mark.parametrize("n", [5, 100])
def test_append(old, scale, n):
    build.build()
    gb.lib()
    c = _with(old, n, scale)
    _same(_append(c), _expect(c))
