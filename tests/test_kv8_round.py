"""The example's rounds: every call of a speculative round on an 8-bit cache, each against the oracle on what it was
given."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from kv8_util import check, host
from oracle import kv8
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    build.build()
    spec = importlib.util.spec_from_file_location("kv8_round", os.path.join(ROOT, "examples", "kv8_round.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def bits(t):
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def state(layer):
    return {w: (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x).cpu().numpy()
            for w, x in zip(("K", "V", "Ke", "Ve"), layer.cache)} | dict(L=layer.lengths[0].cpu().numpy())


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2)])
def test_rounds(example, heads, kv_heads, monkeypatch):
    B, D, prompt, rounds = 2, 128, 100, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = example.Layer(B, heads, kv_heads, D, prompt + rounds * (1 + example.MAX_TOKENS))
    seen = []

    def after(name):
        real = getattr(example.Layer, name)

        def call(self, *args):
            # copies: the next round writes the path, its length and the tree into the same tensors
            before, given, parent = state(self), [x.clone() for x in args], self.parent.cpu().numpy()
            r = real(self, *args)
            torch.cuda.synchronize()
            seen.append((name, before, given, state(self), None if r is None else r.clone(), parent))
            return r
        return call
    for name in ("append", "draft", "verify"):
        monkeypatch.setattr(example.Layer, name, after(name))
    layer.append(*(torch.randn((B, prompt, kv_heads, D), generator=gen, device="cuda", dtype=torch.bfloat16)
                   for _ in range(2)))
    for _ in range(rounds):
        example.round_of(layer, gen)
    assert [s[0] for s in seen] == ["append"] + (["draft"] * example.GAMMA + ["verify", "append"]) * rounds
    grown = 0
    for name, was, args, now, result, parent in seen:
        if name == "append":
            path = args[2].cpu().numpy() if len(args) > 2 else None
            length = args[3].cpu().numpy() if len(args) > 2 else None
            for codes, exps, new in (("K", "Ke", args[0]), ("V", "Ve", args[1])):
                c, e, L = kv8.kv8_append(was[codes], was[exps], bits(new), was["L"], path, length)
                assert np.array_equal(now[codes], c) and np.array_equal(now[exps], e) and np.array_equal(now["L"], L)
            grown += int((now["L"] - was["L"]).max())
        else:
            tree = (parent, bits(args[1]), bits(args[2])) if name == "verify" else (None, None, None)
            want, size = kv8.kv8_attn(bits(args[0]), was["K"], was["V"], was["Ke"], was["Ve"], was["L"], *tree)
            check(host(result), want, size, "bf16")
    assert grown > prompt + rounds  # some proposals were accepted
    assert gb.glide_read_device_status(layer.ws) == gb.GLIDE_OK
    K, V = (torch.empty((B, kv_heads, layer.most, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gb.glide_kv8_read(*layer.cache, layer.lengths[0], K, V)
    last = state(layer)
    assert np.array_equal(host(K), kv8.kv8_read(last["K"], last["Ke"], last["L"], layer.most))
    assert np.array_equal(host(V), kv8.kv8_read(last["V"], last["Ve"], last["L"], layer.most))
