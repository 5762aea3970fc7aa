"""Appending to an 8-bit cache that is nearly or wholly full: the rows that join are written after those that are there,
as many as the cache has room for, and none of those that are there is overwritten."""
import numpy as np
import pytest

from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_cache import _append, _case, _expect, _same


def test_oracle_by_hand():
    """Two of the tree's five nodes join a cache of 70 rows that holds 67; then three where one has room; then none."""
    codes, exps = np.full((1, 1, 70, 2), 0x7f, np.uint8), np.full((1, 1, 2), -8, np.int8)
    codes[0, 0, :67] = kv8.encode(np.full((67, 2), 256.0))
    new = np.arange(1, 6, dtype=np.float32).repeat(2).reshape(1, 5, 1, 2)
    path = np.array([[0, 3, 4, -1, -1]])
    codes, exps, L = kv8.kv8_append(codes, exps, new, [67], path, [1])
    assert L.tolist() == [69]
    assert kv8.kv8_read(codes, exps, L, 70)[0, 0, :, 0].tolist() == [1.0] * 67 + [1.0, 4.0, 0.0]
    codes, exps, L = kv8.kv8_append(codes, exps, new, L, path, [2])
    assert L.tolist() == [70]
    assert kv8.kv8_read(codes, exps, L, 70)[0, 0, 66:, 0].tolist() == [1.0, 1.0, 4.0, 1.0]
    before = codes.copy()
    codes, exps, L = kv8.kv8_append(codes, exps, new, L, path, [2])
    assert L.tolist() == [70] and np.array_equal(codes, before)


# rows of the call (those of 64 and fewer, and of more, take different kernels), and of each sequence that join
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [33, 64, 100])
@pytest.mark.parametrize("with_path", [False, True])
def test_near_the_end(dtype, n, with_path):
    build.build()
    gb.lib()
    cap, B = 230, 6
    kv_len = [cap - 10, cap - 3, cap - 2, cap, 1000, cap - n]
    joins = [3, 3, 3, 2, 2, n]
    path = None
    if with_path:
        path = np.tile(np.arange(n - 1, -1, -1, dtype=np.int32), (B, 1))
    c = _case(n, B, 2, 64, cap, kv_len, n, dtype, [m - 1 for m in joins], path)
    K, V, Ke, Ve, new_len = got = _append(c)
    assert new_len.tolist() == [cap - 7, cap, cap, cap, cap, cap]
    for b, held in enumerate(min(x, cap) for x in kv_len):
        whole = held // 64  # blocks that no new row is in
        for now, was in ((K, c["K"]), (V, c["V"])):
            assert np.array_equal(now[b, :, :whole * 64], was[b, :, :whole * 64])
        for now, was in ((Ke, c["Ke"]), (Ve, c["Ve"])):
            assert np.array_equal(now[b, :, :whole], was[b, :, :whole])
        if held == cap:
            assert np.array_equal(K[b], c["K"][b]) and np.array_equal(V[b], c["V"][b])
    _same(got, _expect(c))
