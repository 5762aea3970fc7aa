"""Calls whose cached heads do not fit the L2 cache together: they are worked on in groups, the last one of fewer heads."""
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import i32, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def attend(q, k, v, sees, scale):
    """(out, its weighted mean of |v|, the largest sum of |q k| scale) [n, H, D], [n, H, D], [n, H, 1] in fp64, a cached head a
    time: row i of q [n, H, D] sees the first sees[i] of k, v [S, H_kv, D]."""
    g = q.shape[1] // k.shape[1]
    hidden = torch.arange(k.shape[0], device=q.device)[None, :] >= sees[:, None]
    out, mean, top = [], [], []
    for h in range(k.shape[1]):
        K, V = k[:, h].double(), v[:, h].double()
        x = q[:, h * g: (h + 1) * g].double().transpose(0, 1)
        w = torch.softmax((x @ K.T * scale).masked_fill(hidden, -float("inf")), -1).nan_to_num(0.0)
        out.append(w @ V)
        mean.append(w @ V.abs())
        top.append(((x.abs() @ K.abs().T) * scale).masked_fill(hidden, 0.0).amax(-1, keepdim=True))
    return tuple(torch.cat(x).transpose(0, 1) for x in (out, mean, top))


def check(got, want, mean, top, n, D):
    """paged_util.tolerance."""
    score = (D / 2 + 8) * top * 2.0 ** -23 + (top + 1) * 2.0 ** -22
    tol = (2 * score + (n + 8) * 2.0 ** -23 + 2.0 ** -8) * mean + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -7) + 1e-30
    assert ((got.double() - want).abs() <= tol).all()


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


# lengths, H, H_kv, D.  A group has 48 MB of keys and values: 98304 keys of one head of 128, 196608 of 64.
PROMPTS = [
    ([13200], 16, 8, 128),                       # seven heads and one
    ([9000, 11000, 40, 7000], 8, 8, 128),        # three, three and two
    ([30000, 2500, 0, 17], 7, 7, 64),            # six and one
    ([300] * 140 + [8000], 12, 3, 128),          # more sequences than are sorted: two and one, the entries found by their counts
    ([900, 1, 640] * 45, 5, 5, 64),              # as many, one head a group less
]


@pytest.mark.parametrize("case", range(len(PROMPTS)))
def test_prompts(case):
    lens, H, H_kv, D = PROMPTS[case]
    assert sum(lens) * H_kv * D * 4 > 48 << 20 and sum(lens) * D * 4 < 48 << 20
    T = sum(lens) + 3
    x = rand(case, T, H + 2 * H_kv, D)
    q, k, v = x.split([H, H_kv, H_kv], 1)
    cu = torch.tensor([0] + lens).cumsum(0)
    out = torch.full((T, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = workspace(len(lens), H, H_kv, D, "bf16", T, max(lens))
    gb.glide_prompt_attn(q, k, v, i32(cu.numpy()), max(lens), out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    assert (out[T - 3:] == 7).all()
    if max(lens) < 12000:  # every row, as the CUDA-core kernel has it (a longer prompt takes it 15 s)
        fma = torch.full_like(out, 7.0)
        gb.glide_prompt_attn(q, k, v, i32(cu.numpy()), max(lens), fma, ws, flags=gb.GLIDE_FLAG_FORCE_FMA)
        # both results are rounded, the first one's weights too, and both have sums of up to n terms; means are at most the largest |v|
        n = max(lens)
        assert ((out.float() - fma.float()).abs() <= (3 * 2.0 ** -8 + 2 * (n + 8 + 30 * D) * 2.0 ** -23) * v[:sum(lens)].abs().max()).all()
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):  # some rows of each sequence
        rows = torch.unique(torch.tensor([0, 1, 127, 128, b - a - 1] + list(range(0, b - a, 97))))
        rows = rows[(rows >= 0) & (rows < b - a)].cuda()
        if len(rows):
            want = attend(q[a:b][rows], k[a:b], v[a:b], rows + 1, D ** -0.5)
            check(out[a:b][rows], *want, b - a, D)


# new tokens, keys, H, H_kv, D, P
CHUNKS = [
    ([16, 16], [16384, 16384], 32, 8, 128, 64),             # the keys cut into chunks: three groups of heads for the merge
    ([40, 18], [30000, 9000], 10, 5, 128, 16),              # two, two and one
    ([17], [70000], 3, 3, 128, 128),                        # one head a group
    ([64] * 6, [20000] * 6, 16, 8, 64, 32),
    ([200, 30], [40000, 13000], 24, 8, 64, 256),
    ([20] + [1] * 149, [9000] + [700] * 149, 16, 8, 128, 16),  # more requests than are sorted
]


@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunks(case):
    m, kv, H, H_kv, D, P = CHUNKS[case]
    assert sum(kv) * H_kv * D * 4 > 48 << 20
    B, T, pages = len(m), sum(m), [-(-n // P) for n in kv]
    K, V = rand(20 + case, sum(pages) + 1, H_kv, P, D), rand(40 + case, sum(pages) + 1, H_kv, P, D)
    ids = torch.randperm(sum(pages) + 1, generator=torch.Generator().manual_seed(case))
    table, at = torch.full((B, max(pages)), -1), 0
    for b, n in enumerate(pages):
        table[b, :n] = ids[at: at + n]
        at += n
    q, cu = rand(60 + case, T, H, D), torch.tensor([0] + m).cumsum(0)
    out = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(B, H, H_kv, D, "bf16", T, max(m))
    args = (q, K, V, i32(table.numpy()), i32(cu.numpy()), max(m), i32(kv), max(kv))
    gb.glide_paged_attn(*args, out, ws)
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
    again = torch.zeros_like(out)
    gb.glide_paged_attn(*args, again, ws)
    assert torch.equal(out, again)
    for b in list(range(min(B, 8))) + [B - 1]:
        k, v = (X[table[b, : pages[b]].cuda()].transpose(1, 2).reshape(-1, H_kv, D)[: kv[b]] for X in (K, V))
        rows = torch.unique(torch.tensor([0, m[b] // 2, m[b] - 1])).cuda()
        want = attend(q[cu[b]: cu[b + 1]][rows], k, v, kv[b] - m[b] + 1 + rows, D ** -0.5)
        check(out[cu[b]: cu[b + 1]][rows], *want, kv[b], D)
