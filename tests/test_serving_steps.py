"""The paged calls as a serving loop makes them: prompts in, then chunks, proposals and single tokens of a ragged batch in
one call, requests that finish and hand their pages on; each step's attention against the oracle over what the requests have
seen so far, and one layer's pool against every key and value that was put in."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import TYPES, check, dev, host, i32, rounded, tokens, tolerance, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


@pytest.mark.parametrize("H, H_kv, D, P, dtype", [(8, 2, 128, 16, "bf16"), (4, 4, 64, 32, "bf16"), (4, 2, 64, 16, "f32")])
def test_a_run_of_steps(H, H_kv, D, P, dtype):
    rng = np.random.default_rng(H * D)
    B, width, n_pages, rows = 6, 40, 150, 900
    K, V = (torch.full((n_pages, H_kv, P, D), float("nan"), dtype=TYPES[dtype], device="cuda") for _ in range(2))
    table, free, n_free = i32(np.full((B, width), -1)), i32(rng.permutation(n_pages)), i32([n_pages])
    kv, held = i32(np.zeros(B)), i32(np.zeros(B))
    cu, slots, positions = i32(np.zeros(B + 1)), i32(np.zeros(rows)), i32(np.zeros(rows))
    new_kv, new_held, new_free = torch.zeros_like(kv), torch.zeros_like(held), torch.zeros_like(n_free)
    ws = workspace(B, H, H_kv, D, dtype, rows, 400)
    seen = [[np.zeros((0, H_kv, D)), np.zeros((0, H_kv, D))] for _ in range(B)]
    g, scale = H // H_kv, D ** -0.5
    plan = [[130, 40, 1, 0, 257, 16], [1, 1, 5, 33, 1, 6], [1, 6, 64, 1, 1, 1], [-1, 1, 200, 1, -1, 1], [77, 1, 1, 1, 300, 0],
            [1, 1, 1, 1, 1, 1]]
    for step, q_len in enumerate(plan):
        T = sum(max(0, m) for m in q_len) + 3
        gb.glide_page_plan(i32(q_len), kv, held, table, free, n_free, P, cu, slots[:T], new_kv, new_held, new_free,
                           positions[:T])
        kv, new_kv, held, new_held, n_free, new_free = new_kv, kv, new_held, held, new_free, n_free
        x = rounded(tokens(rng, T, H + 2 * H_kv, D), dtype)
        xd = dev(x, dtype)
        q, k, v = xd.split([H, H_kv, H_kv], 1)
        gb.glide_paged_append(k, v, K, V, slots[:T])
        out = torch.full((T, H, D), 3.0, dtype=TYPES[dtype], device="cuda")
        most = max(1, max(q_len))
        gb.glide_paged_attn(q, K, V, table, cu, most, kv, width * P, out, ws)
        first = step == 0
        if first:  # the first step's requests are whole prompts: the packed call gives the same
            packed = torch.full_like(out, 3.0)
            gb.glide_prompt_attn(q, k, v, cu, most, packed, ws)
        at, want, tol = 0, np.full((T, H, D), 3.0), np.zeros((T, H, D))
        for b, m in enumerate(q_len):
            if m < 0:
                seen[b] = [y[:0] for y in seen[b]]
                continue
            new = x[at: at + m]
            seen[b] = [np.concatenate([seen[b][0], new[:, H: H + H_kv]]), np.concatenate([seen[b][1], new[:, H + H_kv:]])]
            L = len(seen[b][0])
            assert positions[at: at + m].tolist() == list(range(L - m, L))
            for h in range(H):
                o, mean, top = paged.attend(new[:, h], seen[b][0][:, h // g], seen[b][1][:, h // g],
                                            L - m + 1 + np.arange(m), scale)
                want[at: at + m, h], tol[at: at + m, h] = o, tolerance(o, mean, top, max(1, L), D, dtype)
            at += m
        check(host(out), want, tol, f"step {step}")
        if first:
            check(host(packed), want, tol, "packed")
        assert kv.tolist() == [len(y[0]) for y in seen]
        assert slots[at: T].tolist() == [-1] * (T - at)
    Kh, Vh, tb = host(K), host(V), table.cpu().numpy()
    for b in range(B):
        for h in range(H_kv):
            for X, y in ((Kh, seen[b][0]), (Vh, seen[b][1])):
                assert np.array_equal(paged.gather(X, tb[b], len(y), h), y[:, h])
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK


def test_a_decoding_step_in_a_graph():
    """Plan, append and attention of a decoding step captured once and replayed: the lengths live on the device, and the step
    leaves them where the next replay reads them."""
    B, H, H_kv, D, P, width, n_pages = 4, 8, 2, 128, 16, 12, 60
    rng = np.random.default_rng(1)
    K, V = (torch.full((n_pages, H_kv, P, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, free, n_free = i32(np.full((B, width), -1)), i32(rng.permutation(n_pages)), i32([n_pages])
    kv, held, cu, slots = (i32(np.zeros(n)) for n in (B, B, B + 1, B))
    new = [torch.zeros_like(t) for t in (kv, held, n_free)]
    ws = workspace(B, H, H_kv, D, "bf16", B, 1)
    x = torch.zeros((B, H + 2 * H_kv, D), dtype=torch.bfloat16, device="cuda")
    q, k, v = x.split([H, H_kv, H_kv], 1)
    one, out = i32(np.ones(B)), torch.zeros((B, H, D), dtype=torch.bfloat16, device="cuda")

    def step():
        gb.glide_page_plan(one, kv, held, table, free, n_free, P, cu, slots, *new)
        gb.glide_paged_append(k, v, K, V, slots)
        gb.glide_paged_attn(q, K, V, table, cu, 1, new[0], width * P, out, ws)
        for a, b in zip((kv, held, n_free), new):
            a.copy_(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t in (kv, held):
        t.zero_()
    n_free.fill_(n_pages)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    seen = []
    for i in range(40):
        xh = rounded(tokens(rng, B, H + 2 * H_kv, D), "bf16")
        x.copy_(dev(xh, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        seen.append(xh)
        if i % 13 == 0 or i == 39:
            past = np.stack(seen, 1)
            for b in range(B):
                for h in range(H):
                    o, mean, top = paged.attend(xh[b, h][None], past[b, :, H + h // 4], past[b, :, H + H_kv + h // 4], [i + 1],
                                                D ** -0.5)
                    check(host(out[b, h])[None], o, tolerance(o, mean, top, i + 1, D, "bf16"))
    assert kv.tolist() == [40] * B and held.tolist() == [3] * B and n_free.tolist() == [n_pages - 3 * B]
