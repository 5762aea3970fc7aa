"""Bounds that are looser than the lengths, as a captured graph has them: in a call that takes the same kernel they change no
bit, on the same workspace."""
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import Paged, Prompt, check, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


@pytest.mark.parametrize("flags", [0, gb.GLIDE_FLAG_FORCE_FMA])
@pytest.mark.parametrize("m, kv, H, H_kv, D", [([150, 40], [300, 140], 4, 2, 128), ([20, 0, 33], [900, 5, 1200], 6, 3, 64)])
def test_pages(m, kv, H, H_kv, D, flags):
    P = 16
    s = Paged(1, m, kv, H, H_kv, D, P, "bf16")
    s.upload()
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    out = s.run(ws=ws, flags=flags)
    check(host(out), *s.want())
    for bound in (2048, 1 << 18):  # some more tiles; more than one O takes in
        table = torch.full((len(m), bound // P), -7, dtype=torch.int32, device="cuda")
        table[:, : s.tabled.shape[1]] = s.tabled
        s.tabled = table
        for _ in range(2):
            assert torch.equal(s.run(max_q=max(m) + 5, max_kv=bound, ws=ws, flags=flags), out), bound


def test_prompts():
    s = Prompt(2, [300, 1, 77], 4, 2, 128, "bf16", pad=2)
    s.upload()
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    out = s.run(ws=ws)
    check(host(out), *s.want())
    for bound in (s.T, 5000, 1 << 20):
        assert torch.equal(s.run(max_len=bound, ws=ws), out), bound
    assert torch.equal(s.run(ws=ws), out)
