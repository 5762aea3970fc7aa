"""Page tables and slots of a step, built on the GPU, against the oracle: equal in every entry."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def run(q, kv, held, table, free, n_free, P, T, positions=True):
    B = len(q)
    d = dict(table=i32(table), free=i32(free), cu_q=i32([-9] * (B + 1)), slots=i32([-9] * T), new_kv_len=i32([-9] * B),
             new_held=i32([-9] * B), new_n_free=i32([-9]))
    if positions:
        d["positions"] = i32([-9] * T)
    gb.glide_page_plan(i32(q), i32(kv), i32(held), d["table"], d["free"], i32([n_free]), P, d["cu_q"], d["slots"],
                       d["new_kv_len"], d["new_held"], d["new_n_free"], d.get("positions"))
    torch.cuda.synchronize()
    return {k: t.cpu().numpy() for k, t in d.items()}


def check(q, kv, held, table, free, n_free, P, T, positions=True):
    got = run(q, kv, held, table, free, n_free, P, T, positions)
    want = paged.page_plan(q, kv, held, table, free, n_free, P, T)
    want["new_n_free"] = [want["new_n_free"]]
    for k, x in got.items():
        assert np.array_equal(x, want[k]), k


def requests(seed, B, P, kv_max, q_max, finished, spare):
    rng = np.random.default_rng(seed)
    q = np.where(rng.random(B) < finished, -rng.integers(1, 5, B), rng.integers(0, q_max + 1, B))
    kv = rng.integers(0, kv_max + 1, B)
    held = -(-kv // P) + rng.integers(0, 2, B)
    width = -(-(kv_max + q_max) // P) + 1
    need = np.maximum(0, -(-(kv + np.maximum(q, 0)) // P) - held)[q > 0].sum()
    n_free = int(need * spare)
    ids = rng.permutation(int(held.sum()) + n_free + 3)
    table = np.full((B, width), -1)
    at = 0
    for b in range(B):
        table[b, : held[b]] = ids[at: at + held[b]]
        at += held[b]
    free = np.full(len(ids), -1)
    free[:n_free] = ids[at: at + n_free]
    return q, kv, held, table, free, n_free, int(np.maximum(q, 0).sum())


@pytest.mark.parametrize("seed, B, P, kv_max, q_max, finished, spare, pad", [
    (0, 1, 16, 40, 1, 0.0, 1.0, 0), (1, 1, 256, 0, 700, 0.0, 1.0, 3), (2, 31, 16, 100, 1, 0.2, 1.0, 0),
    (3, 33, 32, 333, 50, 0.3, 0.5, 9), (4, 257, 64, 1000, 7, 0.1, 0.9, 1), (5, 1024, 16, 700, 60, 0.1, 0.7, 5),
    (6, 1024, 128, 4000, 400, 0.5, 1.0, 0), (7, 100, 16, 200, 30, 1.0, 1.0, 4), (8, 64, 16, 50, 0, 0.3, 1.0, 2)])
def test_steps(seed, B, P, kv_max, q_max, finished, spare, pad):
    q, kv, held, table, free, n_free, T = requests(seed, B, P, kv_max, q_max, finished, spare)
    check(q, kv, held, table, free, n_free, P, T + pad, positions=seed != 4)


def test_more_tokens_than_rows():
    """The step's rows end inside a request's tokens; later requests have none."""
    q, kv, held, table, free, n_free, T = requests(11, 40, 16, 90, 20, 0.1, 1.0)
    for rows in (T // 2, 1, 0):
        check(q, kv, held, table, free, n_free, 16, rows)


def test_a_table_too_short():
    q, kv, held, table, free, n_free, T = requests(12, 40, 16, 90, 40, 0.1, 1.0)
    table = table[:, :6]
    check(q, kv, np.minimum(held, 6), table, free, n_free, 16, T)


def test_values_out_of_range():
    """Lengths, counts and page numbers that no step has: clamped, and nothing outside the buffers is touched."""
    table = [[5, -3, 2 ** 31 - 1, 0], [1, 2, 3, 4], [6, 7, 8, 9]]
    big = 2 ** 31 - 1
    check([2, 3, 1], [-5, 40, 10], [-2, 9, 4], table, [11, 12, 13], big, 16, 6)
    check([big, big, big], [0, 0, 0], [0, 0, 0], table, [11, 12, 13], -4, 16, 6)
    check([1, 1, 1], [big, big - 1, 0], [4, 4, 0], table, [11, 12, 13], 3, 256, 6)
    check([1, -1, -1], [0, 64, 64], [0, 4, 4], table, [11, 12, 13], 2, 16, 6)  # a stack without room for what comes back


def test_steps_in_turn():
    """A serving loop: the outputs of one step are the next one's inputs."""
    rng = np.random.default_rng(5)
    B, P, width, n = 24, 16, 12, 150
    state = dict(kv=np.zeros(B, int), held=np.zeros(B, int), table=np.full((B, width), -1), free=rng.permutation(n), n=n)
    for _ in range(12):
        q = np.where(state["kv"] > 120, -1, rng.integers(0, 30, B))
        args = (q, state["kv"], state["held"], state["table"], state["free"], state["n"], P, 400)
        check(*args)
        r = paged.page_plan(*args)
        state = dict(kv=r["new_kv_len"], held=r["new_held"], table=r["table"], free=r["free"], n=r["new_n_free"])
        kept = [r["table"][b, j] for b in range(B) for j in range(r["new_held"][b])] + list(r["free"][: r["new_n_free"]])
        assert sorted(kept) == list(range(n))
