"""One workspace for calls of every kind and shape, in any order: what a call leaves there is never another call's counter."""
import random

import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import Paged, i32

pytestmark = pytest.mark.gpu
ZEROS = 64 << 10  # the bytes that are zero between calls


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def _rand(seed, *shape, t=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(t)


def cross(B, H, H_kv, D, S, dtype=torch.bfloat16):
    q, K, V = _rand(1, B, 1, H, D, t=dtype), _rand(2, B, H_kv, S, D, t=dtype), _rand(3, B, H_kv, S, D, t=dtype)
    kv = i32([max(1, S - 17 * b) for b in range(B)])
    return lambda ws: gb.glide_cross_attn(q, K, V, kv, S, torch.zeros((B, 1, H, D), device="cuda"), ws)


def tree(B, H, H_kv, D, S, n, dtype=torch.bfloat16, flags=0):
    q, K, V = _rand(4, B, n, H, D, t=dtype), _rand(5, B, H_kv, S + n, D, t=dtype), _rand(6, B, H_kv, S + n, D, t=dtype)
    kv, parent = i32([max(1, S - 5 * b) for b in range(B)]), i32([[-1] + [i // 2 for i in range(n - 1)]] * B)
    return lambda ws: gb.tree_verify_attn(q, parent, K, V, kv, S, torch.zeros((B, n, H, D), device="cuda"), ws, flags=flags)


def accept(B, n, V=300):
    parent = [-1] + [i // 2 for i in range(n - 1)]
    draft = torch.randint(V, (B, n), generator=torch.Generator().manual_seed(7)).int().cuda()
    logits = _rand(8, B, n, V, t=torch.float32)
    for i in range(1, n):
        logits[:, parent[i], :].scatter_(1, draft[:, i: i + 1].long(), 9.0)
    par = i32([parent] * B)

    def run(ws):
        o = [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((B, n), (B,), (B,))]
        gb.tree_accept(draft, par, logits, *o, ws)
        return torch.cat([x.reshape(-1) for x in o])
    return run


def expand(B, gamma, V=5000):
    probs, root = torch.softmax(_rand(9, B, gamma, V, t=torch.float32), -1), i32(list(range(B)))

    def run(ws):
        o = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B, 33), (B, 33), (B,))]
        gb.cape_expand(probs, root, 32, *o, ws)
        return torch.cat([x.reshape(-1) for x in o])
    return run


def paged(seed, m, kv, H, H_kv, D):
    s = Paged(seed, m, kv, H, H_kv, D, 16, "bf16")
    s.upload()
    return lambda ws: s.run(ws=ws)


def kv8(B, H, D, S, n):
    kv, blocks = i32([S] * B), -(-S // 64)
    K, V = (torch.randint(0, 0x70, (B, H, S, D), generator=torch.Generator().manual_seed(x), dtype=torch.uint8).cuda()
            .view(torch.float8_e4m3fn) for x in (1, 2))
    e = torch.zeros((B, H, blocks), dtype=torch.int8, device="cuda")
    q, kt, vt = _rand(11, B, n, H, D), _rand(12, B, n, H, D), _rand(13, B, n, H, D)
    parent = i32([[-1] + [i // 2 for i in range(n - 1)]] * B)
    return lambda ws: gb.glide_kv8_verify_attn(q, parent, kt, vt, K, V, e, e, kv, S, torch.zeros_like(q), ws)


F = torch.float32
CALLS = {
    # scratch of few heads or sequences ..
    "cross 1": lambda: cross(1, 4, 4, 128, 9000), "cross f32": lambda: cross(2, 3, 3, 64, 3000, F),
    "tree 1": lambda: tree(1, 2, 2, 128, 5000, 9), "paged 1": lambda: paged(1, [40], [2600], 4, 1, 128),
    "paged 2": lambda: paged(2, [33, 20], [1700, 2500], 2, 2, 64), "kv8": lambda: kv8(1, 2, 64, 3000, 24),
    "expand": lambda: expand(3, 5),
    # .. and counters of many
    "fma 32": lambda: tree(8, 32, 32, 64, 300, 5, F), "fma group": lambda: tree(3, 64, 8, 128, 400, 20, F),
    "fma 1280": lambda: tree(40, 32, 32, 64, 100, 3, torch.bfloat16, gb.GLIDE_FLAG_FORCE_FMA),
    "fma 20480": lambda: tree(40, 512, 512, 64, 40, 2, torch.bfloat16, gb.GLIDE_FLAG_FORCE_FMA),
    "accept": lambda: accept(4, 60), "accept 9600": lambda: accept(160, 60), "tree 40": lambda: tree(40, 8, 8, 64, 200, 6),
    "expand 900": lambda: expand(900, 2),
}


def test_calls_in_any_order():
    calls = {name: make() for name, make in CALLS.items()}
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    want = {}
    for name, run in calls.items():  # each on a workspace of its own
        ws.zero_()
        want[name] = run(ws).clone()
        assert not ws[: ZEROS].any(), name
    ws.zero_()
    names = list(calls) * 4
    random.Random(5).shuffle(names)
    before = "nothing"
    for name in names:
        got = calls[name](ws)
        assert torch.equal(got, want[name]), f"{name} behind {before}"
        assert not ws[: ZEROS].any(), name
        before = name
