"""What the paged cache's calls refuse, before any work: through the C ABI and through the Python binding."""
import ctypes

import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build

FAKE = 0x10000  # 16-byte aligned, never dereferenced: every call below fails validation first
INVALID, UNSUPPORTED = gb.GLIDE_ERR_INVALID, gb.GLIDE_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    build.build()
    return gb.lib()


def desc(**kw):
    d = dict(B=2, H=4, D=128, S_cap=1, dtype=gb.GLIDE_BF16)
    d.update(kw)
    return ctypes.byref(gb.make_desc(**d))


def pool(**kw):
    c = dict(K=FAKE, V=FAKE + (1 << 30), n_pages=10, page_size=16)
    c.update(kw)
    return ctypes.byref(gb.PagePool(**c))


BAD_POOLS = [dict(K=None), dict(V=None), dict(K=FAKE + 8), dict(V=FAKE + 4), dict(n_pages=0), dict(n_pages=1 << 28)]
BAD_SIZES = [0, 1, 8, 24, 48, 512, -16]
BAD_DESCS = [dict(D=80), dict(H=0), dict(dtype=5), dict(H=6, H_kv=4), dict(H_kv=8)]


def test_plan(L):
    at = {k: FAKE + 4096 * i for i, k in enumerate(
        ["q", "kv", "held", "table", "free", "n", "cu", "slots", "pos", "nkv", "nheld", "nn"])}

    def call(B=3, T=10, P=16, W=5, cap=20, **kw):
        p = dict(at, **kw)
        return L.glide_page_plan(B, T, P, W, p["q"], p["kv"], p["held"], p["table"], p["free"], cap, p["n"], p["cu"],
                                 p["slots"], p["pos"], p["nkv"], p["nheld"], p["nn"], None)
    for b in [dict(B=0), dict(B=1025), dict(T=-1), dict(W=0), dict(cap=0)] + [{k: None} for k in at if k != "pos"] + \
            [{k: at[k] + 2} for k in at]:
        assert call(**b) == INVALID, b
    for P in BAD_SIZES:
        assert call(P=P) == UNSUPPORTED, P
    assert call(B=1024, W=1 << 22) == UNSUPPORTED
    # nothing written overlaps anything else
    for out in ("table", "free", "cu", "slots", "pos", "nkv", "nheld", "nn"):
        for other in at:
            if other != out:
                assert call(**{out: at[other]}) == INVALID, (out, other)
    assert call(nkv=at["kv"] + 8) == INVALID and call(slots=at["table"] + 56) == INVALID


def test_append(L):
    def call(d=None, c=None, k=FAKE + (1 << 32), v=FAKE + (1 << 33), ks=512, vs=512, T=5, slots=FAKE + (1 << 34)):
        return L.glide_paged_append(d or desc(), c or pool(), k, v, ks, vs, T, slots, None)
    for b in [dict(k=None), dict(v=None), dict(slots=None), dict(T=-1), dict(ks=511), dict(vs=504), dict(ks=516), dict(vs=-512),
              dict(k=FAKE + (1 << 32) + 8), dict(v=FAKE + (1 << 33) + 2), dict(slots=FAKE + (1 << 34) + 1),
              dict(k=FAKE + 1024), dict(v=FAKE + (1 << 30)), dict(slots=FAKE + 64), dict(c=pool(V=FAKE + 32))]:
        assert call(**b) == INVALID, b
    for c in BAD_POOLS:
        assert call(c=pool(**c)) == INVALID, c
    for d in BAD_DESCS:
        assert call(d=desc(**d)) == INVALID, d
    for P in BAD_SIZES:
        assert call(c=pool(page_size=P)) == UNSUPPORTED, P
    assert L.glide_paged_append(None, pool(), FAKE, FAKE, 512, 512, 5, FAKE, None) == INVALID
    assert L.glide_paged_append(desc(), None, FAKE, FAKE, 512, 512, 5, FAKE, None) == INVALID
    assert call(T=0, k=None, v=None, slots=None) == gb.GLIDE_OK  # a step without tokens


def test_workspace(L):
    def size(T=100, m=10, **kw):
        return gb.glide_paged_workspace_bytes(desc(**kw)._obj, T, m)
    assert 0 < size() <= size(T=1000, m=1000) <= size(T=100000, m=100000)
    assert size(T=-1) == 0 and size(m=0) == 0 and size(D=96) == 0 and size(B=0) == 0
    assert size(S_cap=0) > 0  # not looked at
    for m in range(1, 300):
        assert size(T=300, m=m) <= size(T=300, m=m + 1)
    for T in range(0, 300):
        assert size(T=T, m=64) <= size(T=T + 1, m=64)


def test_attention(L):
    def paged(d=None, q=FAKE, s=512, T=9, cu=FAKE, mq=4, c=None, table=FAKE, W=7, kv=FAKE, most=100, out=FAKE, ws=FAKE,
              wsb=1 << 40):
        return L.glide_paged_attn(d or desc(), q, s, T, cu, mq, c or pool(), table, W, kv, most, out, ws, wsb, None)

    def prompt(d=None, q=FAKE, s=512, k=FAKE, ks=512, v=FAKE, vs=512, T=9, cu=FAKE, mq=4, out=FAKE, ws=FAKE, wsb=1 << 40):
        return L.glide_prompt_attn(d or desc(), q, s, k, ks, v, vs, T, cu, mq, out, ws, wsb, None)
    for call in (paged, prompt):
        for b in [dict(q=None), dict(out=None), dict(ws=None), dict(cu=None), dict(T=-1), dict(mq=0), dict(s=511), dict(s=508),
                  dict(s=516), dict(q=FAKE + 8), dict(out=FAKE + 4), dict(ws=FAKE + 8), dict(cu=FAKE + 2), dict(wsb=16)]:
            assert call(**b) == INVALID, b
        for d in BAD_DESCS + [dict(B=0), dict(B=1025), dict(scale=-1.0), dict(scale=float("nan"))]:
            assert call(d=desc(**d)) == INVALID, d
    for b in [dict(table=None), dict(kv=None), dict(table=FAKE + 2), dict(kv=FAKE + 1), dict(W=0), dict(most=-1), dict(most=113)]:
        assert paged(**b) == INVALID, b
    for c in BAD_POOLS:
        assert paged(c=pool(**c)) == INVALID, c
    for P in BAD_SIZES:
        assert paged(c=pool(page_size=P)) == UNSUPPORTED, P
    for b in [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(ks=500), dict(vs=511), dict(ks=516)]:
        assert prompt(**b) == INVALID, b
    assert paged(T=0, q=None, out=None) == gb.GLIDE_OK and prompt(T=0, q=None, k=None, v=None, out=None) == gb.GLIDE_OK


def test_attention_refuses_overlaps(L):
    """out and the workspace on every input, and out's last 16 bytes on an input's first."""
    at = {n: FAKE + (x << 33) for x, n in enumerate(("q", "K", "V", "cu", "table", "kv", "out", "ws"))}
    out_bytes = 9 * 4 * 128 * 2

    def paged(**kw):
        a = {**at, **kw}
        return L.glide_paged_attn(desc(), a["q"], 512, 9, a["cu"], 4, pool(K=a["K"], V=a["V"]), a["table"], 7, a["kv"], 100,
                                  a["out"], a["ws"], 1 << 28, None)

    def prompt(**kw):
        a = {**at, **kw}
        return L.glide_prompt_attn(desc(), a["q"], 512, a["K"], 512, a["V"], 512, 9, a["cu"], 4, a["out"], a["ws"], 1 << 28, None)
    for call, names in ((paged, ("q", "K", "V", "cu", "table", "kv")), (prompt, ("q", "K", "V", "cu"))):
        for n in names:
            assert call(out=at[n]) == INVALID and call(ws=at[n]) == INVALID, n
            assert call(out=at[n] - out_bytes + 16) == INVALID, n
        assert call(out=at["ws"]) == INVALID
        assert call(q=at["out"] + out_bytes - 16) == INVALID


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_binding_refuses(L, device):
    """Host tensors, which are refused themselves, and every unusual argument beside good ones on the GPU."""
    B, H, H_kv, D, P, T = 2, 4, 2, 64, 16, 5

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device=device)

    def i(*shape):
        return t(*shape, dtype=torch.int32)
    K, V, ws = t(6, H_kv, P, D), t(6, H_kv, P, D), t(1 << 28 if device == "cuda" else 1 << 10, dtype=torch.uint8)
    plan = dict(q_len=i(B), kv_len=i(B), held=i(B), block_table=i(B, 3), free_pages=i(9), n_free=i(1), page_size=P,
                cu_q=i(B + 1), slots=i(T), new_kv_len=i(B), new_held=i(B), new_n_free=i(1), positions=i(T))
    app = dict(k_new=t(T, H_kv, D), v_new=t(T, H_kv, D), K=K, V=V, slots=i(T) - 1)
    att = dict(q=t(T, H, D), K=K, V=V, block_table=i(B, 3), cu_q=i(B + 1), max_q=4, kv_len=i(B), max_kv_len=48,
               out=t(T, H, D), workspace=ws)
    pro = dict(q=t(T, H, D), k=t(T, H_kv, D), v=t(T, H_kv, D), cu=i(B + 1), max_len=T, out=t(T, H, D), workspace=ws)

    def ints(good, *names):
        for n in names:
            x = good[n]
            yield from ((n, x.long()), (n, x.float()), (n, torch.cat([x, x])))
            if x.numel() > 1:
                yield n, torch.stack([x, x], -1)[..., 0]
            if device == "cuda":
                yield n, x.cpu()

    def rows(good, *names):
        for n in names:
            x = good[n]
            yield from ((n, x.half()), (n, x.float()), (n, x[:-1]), (n, x[0]), (n, x.transpose(0, 1)),
                        (n, torch.cat([x, x], -1)[..., : D]), (n, torch.stack([x, x], -1)[..., 0]))
            if device == "cuda":
                yield n, x.cpu()
    bad_pool = [("K", K[:, :, :8]), ("V", V[:-1]), ("K", K.float()), ("V", V.transpose(1, 2)), ("K", K[0]),
                ("V", torch.cat([V, V], -1)[..., :D])]
    for fn, good, bad in [
            (gb.glide_page_plan, plan, list(ints(plan, *(n for n in plan if n != "page_size")))),
            (gb.glide_paged_append, app, bad_pool + list(ints(app, "slots")) + list(rows(app, "k_new", "v_new"))),
            (gb.glide_paged_attn, att, bad_pool + list(ints(att, "block_table", "cu_q", "kv_len")) + list(rows(att, "q", "out"))
             + [("out", torch.cat([att["out"]] * 2, 1)[:, :H])]),
            (gb.glide_prompt_attn, pro, list(rows(pro, "q", "k", "v", "out")))]:
        if device == "cuda":
            fn(**good)
        else:
            with pytest.raises(ValueError):
                fn(**good)
        for name, value in bad:
            if fn is gb.glide_page_plan and name == "free_pages" and value.dtype == torch.int32 and value.dim() == 1 and \
                    value.is_contiguous() and value.device.type == "cuda":
                continue  # any number of entries
            with pytest.raises((TypeError, ValueError, gb.GlideError)):
                fn(**dict(good, **{name: value}))
                print("taken:", fn.__name__, name, value.dtype, tuple(value.shape), value.stride())
    if device == "cuda":
        for fn, good, bad in [(gb.glide_paged_attn, att, dict(max_kv_len=49)), (gb.glide_paged_attn, att, dict(workspace=ws[:16])),
                              (gb.glide_prompt_attn, pro, dict(max_len=0)), (gb.glide_page_plan, plan, dict(page_size=24)),
                              (gb.glide_page_plan, plan, dict(new_kv_len=plan["kv_len"])),
                              (gb.glide_paged_append, app, dict(k_new=K.view(-1, H_kv, D)[:T]))]:
            with pytest.raises(gb.GlideError):
                fn(**dict(good, **bad))
        torch.cuda.synchronize()
