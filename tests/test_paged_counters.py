"""What a call of packed rows leaves in its workspace's header: zeros, whatever its CTAs' last claims were."""
import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from paged_util import Paged, Prompt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()
    gb.lib()


def cases():
    yield Prompt(1, [40], 2, 1, 64, "bf16")                          # fewer items than CTAs: most CTAs have none
    yield Prompt(2, [3, 200, 0, 77] * 5, 16, 16, 64, "bf16")         # more
    yield Paged(3, [40], [2600], 4, 1, 128, 16, "bf16")              # keys in chunks, and the merge
    yield Paged(4, [20, 60], [0, 10], 4, 2, 128, 16, "bf16")         # rows that see nothing


def test_the_header_is_zero_after_many_calls():
    steps = list(cases())
    for s in steps:
        s.upload()
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")
    first = [s.run(ws=ws) for s in steps]
    for s in steps:
        s.run(ws=ws)
        torch.cuda.synchronize()
        assert not ws[:256].any()
    for _ in range(300):  # one behind the other, each beginning while the one before ends
        again = [s.run(ws=ws) for s in steps]
    assert not ws[:256].any()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
