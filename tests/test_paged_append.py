"""New rows into a paged pool by their slots: bit for bit, and nothing else changes."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import TYPES, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


@pytest.mark.parametrize("T, H, D, P, dtype, fused", [
    (1, 1, 64, 16, "bf16", False), (1, 8, 128, 16, "f32", True), (7, 3, 64, 32, "f32", False), (100, 5, 128, 64, "bf16", True),
    (333, 40, 128, 16, "bf16", True), (2049, 8, 64, 256, "bf16", False), (5000, 32, 128, 128, "bf16", True)])
def test_rows(T, H, D, P, dtype, fused):
    gen = torch.Generator(device="cuda").manual_seed(T)
    wide = torch.randn((T, 3 + 2 * H, D), generator=gen, device="cuda").to(TYPES[dtype])
    wide[0, 3:] = float("nan")  # any bits are carried
    wide[-1, 3] = float("inf")
    k, v = wide[:, 3: 3 + H], wide[:, 3 + H:]
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    n = -(-T // P) + 2
    K, V = (torch.randn((n, H, P, D), generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    slots = torch.randperm(n * P, generator=gen, device="cuda")[:T].to(torch.int32)
    slots[torch.rand(T, generator=gen, device="cuda") < 0.2] = -1
    slots[T // 2:][torch.rand(T - T // 2, generator=gen, device="cuda") < 0.05] = n * P
    slots[0] = n * P - 1
    slots[1:][slots[1:] == n * P - 1] = -7
    ints = {torch.bfloat16: torch.int16, torch.float32: torch.int32}[TYPES[dtype]]
    want = [paged.append(x.view(ints).cpu().numpy(), y.contiguous().view(ints).cpu().numpy(), slots.tolist())
            for x, y in ((K, k), (V, v))]
    gb.glide_paged_append(k, v, K, V, slots)
    torch.cuda.synchronize()
    assert np.array_equal(K.view(ints).cpu().numpy(), want[0]) and np.array_equal(V.view(ints).cpu().numpy(), want[1])


def test_no_rows():
    K, V = (torch.ones((2, 1, 16, 64), device="cuda") for _ in range(2))
    k = torch.zeros((0, 1, 64), device="cuda")
    gb.glide_paged_append(k, k, K, V, i32([]))
    torch.cuda.synchronize()
    assert bool((K == 1).all()) and bool((V == 1).all())


def test_a_pool_beyond_32_bits():
    """Offsets of pages far behind: a pool of more than 2^32 bytes, and of more than 2^31 elements."""
    K = torch.zeros((530000, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((3, 2, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    n = K.shape[0] * 16
    slots = [n - 1, 0, 270000 * 16 + 5]
    gb.glide_paged_append(k, v, K, V, i32(slots))
    torch.cuda.synchronize()
    for i, s in enumerate(slots):
        assert torch.equal(K[s // 16, :, s % 16], k[i]) and torch.equal(V[s // 16, :, s % 16], v[i])
        K[s // 16, :, s % 16] = 0
    assert not bool(K.any())
