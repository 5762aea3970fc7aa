"""Contexts as long as a 32-bit length can say.  Page numbers may repeat, so a few pages hold them all."""
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


def test_a_token_over_the_longest_context():
    """2^31 - 1 keys of one page again and again, with score 0 and values 1; the last of them, in a page of its own, has score
    60 and so all the weight: the others together have 2^31 e^-60 < 2e-17 of it, which moves a column by less than
    2e-17 (1 + 43) < 1e-15, the whole numbers in V alone are held without rounding.  The row behind it holds NaN."""
    D, P, H, kv = 64, 256, 4, 2 ** 31 - 1
    width = -(-kv // P)
    K, V = torch.zeros((2, 1, P, D), dtype=torch.bfloat16), torch.zeros((2, 1, P, D), dtype=torch.bfloat16)
    q = torch.zeros((1, H, D), dtype=torch.bfloat16)
    q[:, :, 0], q[:, :, 1] = 8.0, torch.arange(H)
    last = (kv - 1) % P
    assert last == P - 2
    K[1, 0, last, 0] = 60.0                                   # 8 * 60 / sqrt(64)
    V[0, 0] = 1.0
    V[1, 0, last] = torch.arange(D) - 20.0
    K[1, 0, P - 1], V[1, 0, P - 1] = float("nan"), float("nan")
    table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    out = torch.zeros((1, H, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(1, H, 1, D, "bf16", 1, 1)
    gb.glide_paged_attn(q.cuda(), K.cuda(), V.cuda(), table, i32([0, 1]), 1, i32([kv]), kv, out, ws)
    assert ((out.cpu().double() - V[1, 0, last].double()).abs() < 1e-15).all()
    assert gb.glide_read_device_status(ws) == gb.GLIDE_OK
