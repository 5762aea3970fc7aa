"""The paged cache's oracle against worked examples, invariants and closed forms."""
import numpy as np
import pytest

from oracle import attention, paged


def test_plan_by_hand():
    """Two live requests and a finished one; pages of 4 tokens."""
    table = [[7, -1, -1], [3, 5, -1], [2, -1, -1]]
    r = paged.page_plan([3, -1, 1], [4, 6, 2], [1, 2, 1], table, [9, 8, -1, -1], 2, 4, 6)
    # the stack is 9, 8, then the finished request's 3, 5; request 0 needs a second page and gets 5
    assert r["free"].tolist() == [9, 8, 3, 5] and r["new_n_free"] == 3
    assert r["table"].tolist() == [[7, 5, -1], [3, 5, -1], [2, -1, -1]]
    assert r["cu_q"].tolist() == [0, 3, 3, 4]
    assert r["slots"].tolist() == [20, 21, 22, 10, -1, -1] and r["positions"].tolist() == [4, 5, 6, 2, 0, 0]
    assert r["new_kv_len"].tolist() == [7, 0, 3] and r["new_held"].tolist() == [2, 0, 1]


def test_plan_runs_short():
    """The first request that the stack has not enough for, and every later one that needs pages, is left out."""
    table = np.full((4, 4), -1)
    table[2, 0] = 6
    r = paged.page_plan([4, 9, 2, 1], [0, 0, 1, 0], [0, 0, 1, 0], table, [0, 1, 2], 3, 4, 20)
    assert r["new_held"].tolist() == [1, 0, 1, 0] and r["new_kv_len"].tolist() == [4, 0, 3, 0]
    assert r["slots"][:4].tolist() == [8, 9, 10, 11] and set(r["slots"][4:13]) == {-1}
    assert r["slots"][13:15].tolist() == [25, 26] and r["slots"][15] == -1 and r["new_n_free"] == 2


@pytest.mark.parametrize("seed", range(5))
def test_pages_are_neither_lost_nor_shared(seed):
    rng = np.random.default_rng(seed)
    B, P, width, n = 12, 16, 9, 70
    ids = rng.permutation(n)
    held = rng.integers(0, 5, B)
    kv = np.maximum(0, held * P - rng.integers(0, P, B))
    table = np.full((B, width), -1)
    at = 0
    for b in range(B):
        table[b, : held[b]] = ids[at: at + held[b]]
        at += held[b]
    free = np.full(n, -1)
    free[: n - at] = ids[at:]
    q = rng.integers(-2, 40, B)
    T = int(np.maximum(q, 0).sum())
    r = paged.page_plan(q, kv, held, table, free, n - at, P, T)
    kept = [r["table"][b, j] for b in range(B) for j in range(r["new_held"][b])] + list(r["free"][: r["new_n_free"]])
    assert sorted(kept) == list(range(n))
    slots = r["slots"][r["slots"] >= 0]
    assert len(set(slots)) == len(slots)


def test_attend_is_causal_attention():
    rng = np.random.default_rng(3)
    K, V, q = rng.standard_normal((9, 8)), rng.standard_normal((9, 8)), rng.standard_normal((1, 8))
    out, mean, top = paged.attend(q, K, V, [9], 8 ** -0.5)
    want = attention.cross_attn(q[None, :, None].astype(np.float64), K[None, None], V[None, None], [9])
    assert np.allclose(out, want[0, 0]) and (mean >= np.abs(out) - 1e-12).all() and top[0] > 0
    K[5:], V[5:] = np.nan, np.inf
    assert np.allclose(paged.attend(q, K, V, [5], 8 ** -0.5)[0], paged.attend(q, K[:5], V[:5], [5], 8 ** -0.5)[0])
    assert (paged.attend(q, K, V, [0], 1.0)[0] == 0).all()


def test_append():
    pool = np.zeros((3, 2, 4, 1))
    got = paged.append(pool, np.arange(1, 9).reshape(4, 2, 1), [5, -1, 11, 12])
    assert got[1, 0, 1, 0] == 1 and got[1, 1, 1, 0] == 2 and got[2, 0, 3, 0] == 5 and got.sum() == 1 + 2 + 5 + 6
