"""Speculative rounds of one target layer on an 8-bit cache, the calls in the order a decoding loop makes them.

    python examples/kv8_round.py [--rounds 4] [--batch 2] [--prompt 700] [--heads 32] [--kv-heads 8]

A prompt's keys and values are quantised into the cache (glide_kv8_append); then every round
drafts (glide_kv8_cross_attn, once per drafted token), expands the proposal into a tree
(cape_expand), verifies it over the cache and the tree's own keys and values
(glide_kv8_verify_attn), accepts a path (tree_accept) and appends that path's rows
(glide_kv8_append again).  The models around the calls are stood in for by random numbers:
projections, distributions and logits are drawn, so a round shows the data flow and the
shapes, not language.  At the end the cache is read back in 16 bits (glide_kv8_read).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2402_02082_gb300 import binding as g  # noqa: E402

GAMMA, MAX_TOKENS, VOCAB = 5, 32, 1000


class Layer:
    """One target layer's 8-bit cache and the buffers that a decoding loop keeps."""

    def __init__(self, B: int, H: int, H_kv: int, D: int, S_cap: int):
        self.B, self.H, self.H_kv, self.D, self.S_cap = B, H, H_kv, D, S_cap
        blocks = (S_cap + g.GLIDE_KV8_BLOCK - 1) // g.GLIDE_KV8_BLOCK
        self.K, self.V = (torch.zeros((B, H_kv, S_cap, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                          for _ in range(2))
        self.K_exp, self.V_exp = (torch.zeros((B, H_kv, blocks), dtype=torch.int8, device="cuda") for _ in range(2))
        self.lengths = [torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2)]  # now, and after an append
        self.most = 0                                                                        # bound of the lengths
        n = 1 + MAX_TOKENS
        desc = g.make_desc(B, H, D, S_cap, g.GLIDE_BF16, H_kv=H_kv if H_kv != H else 0)
        self.ws = torch.zeros(g.glide_kv8_workspace_bytes(desc, n), dtype=torch.uint8, device="cuda")
        self.ws_cape = torch.zeros(g.glide_cape_workspace_bytes(B, GAMMA, VOCAB), dtype=torch.uint8, device="cuda")
        self.ws_acc = torch.zeros(g.glide_accept_workspace_bytes(B, n), dtype=torch.uint8, device="cuda")
        self.out_draft = torch.empty((B, 1, H, D), dtype=torch.bfloat16, device="cuda")
        self.out_tree = torch.empty((B, n, H, D), dtype=torch.bfloat16, device="cuda")
        ints = dict(dtype=torch.int32, device="cuda")
        self.tokens, self.parent, self.path = (torch.zeros((B, n), **ints) for _ in range(3))
        self.nodes, self.accepted, self.bonus = (torch.zeros(B, **ints) for _ in range(3))

    @property
    def cache(self):
        return self.K, self.V, self.K_exp, self.V_exp

    def append(self, k, v, path=None, accepted=None):
        g.glide_kv8_append(k, v, *self.cache, self.lengths[0], self.lengths[1], path, accepted)
        self.lengths.reverse()
        self.most = min(self.most + k.shape[1], self.S_cap)

    def draft(self, q):
        return g.glide_kv8_cross_attn(q, *self.cache, self.lengths[0], self.most, self.out_draft, self.ws)

    def verify(self, q, k, v):
        return g.glide_kv8_verify_attn(q, self.parent, k, v, *self.cache, self.lengths[0], self.most, self.out_tree, self.ws)


def round_of(layer: Layer, gen: torch.Generator) -> None:
    """One speculative round; everything stays on the GPU."""
    B, H, H_kv, D, n = layer.B, layer.H, layer.H_kv, layer.D, 1 + MAX_TOKENS

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    for _ in range(GAMMA):
        layer.draft(normal(B, 1, H, D))
    probs = torch.softmax(3.0 * normal(B, GAMMA, VOCAB, dtype=torch.float32), -1)
    g.cape_expand(probs, layer.bonus, MAX_TOKENS, layer.tokens, layer.parent, layer.nodes, layer.ws_cape)
    k, v = normal(B, n, H_kv, D), normal(B, n, H_kv, D)
    layer.verify(normal(B, n, H, D), k, v)
    # the target's logits: it likes the token of each node's first child in three of four nodes
    logits = normal(B, n, VOCAB, dtype=torch.float32)
    likes = (torch.rand((B, n - 1), generator=gen, device="cuda") < 0.75).float() * 20.0
    at = layer.parent[:, 1:].long().clamp(min=0) * VOCAB + layer.tokens[:, 1:].long().clamp(min=0)
    logits.view(B, -1).scatter_add_(1, at, likes)
    g.tree_accept(layer.tokens, layer.parent, logits, layer.path, layer.accepted, layer.bonus, layer.ws_acc)
    layer.append(k, v, layer.path, layer.accepted)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--prompt", type=int, default=700)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    a = ap.parse_args()
    D, gen = 128, torch.Generator(device="cuda").manual_seed(0)
    layer = Layer(a.batch, a.heads, a.kv_heads, D, a.prompt + a.rounds * (1 + MAX_TOKENS))
    shape = (a.batch, a.prompt, a.kv_heads, D)
    layer.append(*(torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2)))
    for r in range(a.rounds):
        before = layer.lengths[0].tolist()
        round_of(layer, gen)
        print(f"round {r}: lengths {before} -> {layer.lengths[0].tolist()}, accepted {layer.accepted.tolist()}")
    if g.glide_read_device_status(layer.ws) != g.GLIDE_OK:
        raise SystemExit("a kernel gave up a wait")
    K, V = (torch.empty((a.batch, a.kv_heads, layer.most, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g.glide_kv8_read(*layer.cache, layer.lengths[0], K, V)
    print(f"read back: K {tuple(K.shape)}, mean magnitude {K.float().abs().mean().item():.3f}")


if __name__ == "__main__":
    main()
