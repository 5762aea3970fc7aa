"""What the 8-bit cache's calls refuse, before any work: through the C ABI and through the Python binding."""
import ctypes

import pytest
import torch

from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build

FAKE = 0x10000  # 16-byte aligned, never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def L():
    build.build()
    return gb.lib()


def desc(**kw):
    d = dict(B=2, H=4, D=128, S_cap=300, dtype=gb.GLIDE_BF16)
    d.update(kw)
    return ctypes.byref(gb.make_desc(**d))


def fake_cache(**kw):
    c = dict(K=FAKE, V=FAKE, K_exp=FAKE + 1, V_exp=FAKE + 3)
    c.update(kw)
    return ctypes.byref(gb.Kv8Cache(**c))


BAD_CACHES = [dict(K=None), dict(V=None), dict(K_exp=None), dict(V_exp=None), dict(K=FAKE + 8), dict(V=FAKE + 4)]
BAD_DESCS = [dict(D=80), dict(B=0), dict(B=1025), dict(H=0), dict(S_cap=0), dict(dtype=5), dict(H=6, H_kv=4)]


def test_append(L):
    def call(d=None, layers=1, c=None, k=FAKE, v=FAKE, kv=FAKE, n=5, path=None, ln=None, new=FAKE + 256):
        return L.glide_kv8_append(d or desc(), layers, c or fake_cache(), k, v, kv, n, path, ln, new, None)
    for b in [dict(layers=0), dict(k=None), dict(v=None), dict(kv=None), dict(new=None), dict(new=FAKE), dict(n=0),
              dict(n=301), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(kv=FAKE + 1), dict(path=FAKE + 2), dict(ln=FAKE + 3),
              dict(new=FAKE + 258)]:
        assert call(**b) == gb.GLIDE_ERR_INVALID, b
    assert L.glide_kv8_append(None, 1, fake_cache(), FAKE, FAKE, FAKE, 5, None, None, FAKE + 256, None) == gb.GLIDE_ERR_INVALID
    assert L.glide_kv8_append(desc(), 1, None, FAKE, FAKE, FAKE, 5, None, None, FAKE + 256, None) == gb.GLIDE_ERR_INVALID
    for c in BAD_CACHES:
        assert call(c=fake_cache(**c)) == gb.GLIDE_ERR_INVALID, c
    for d in BAD_DESCS:
        assert call(d=desc(**d)) == gb.GLIDE_ERR_INVALID, d


def test_read(L):
    def call(d=None, layers=1, c=None, kv=FAKE, rows=100, K=FAKE, V=FAKE):
        return L.glide_kv8_read(d or desc(), layers, c or fake_cache(), kv, rows, K, V, None)
    for b in [dict(layers=0), dict(kv=None), dict(K=None), dict(V=None), dict(rows=0), dict(rows=301), dict(kv=FAKE + 2),
              dict(K=FAKE + 8), dict(V=FAKE + 4)]:
        assert call(**b) == gb.GLIDE_ERR_INVALID, b
    for c in BAD_CACHES:
        assert call(c=fake_cache(**c)) == gb.GLIDE_ERR_INVALID, c
    for d in BAD_DESCS:
        assert call(d=desc(**d)) == gb.GLIDE_ERR_INVALID, d


def test_workspace(L):
    def size(n, **kw):
        return gb.glide_kv8_workspace_bytes(desc(**kw)._obj, n)
    assert size(1) > 0 and size(64) > 0
    assert size(0) == 0 and size(65) == 0 and size(1, D=96) == 0
    assert size(32, H=64, H_kv=8) > 0 and size(33, H=64, H_kv=8) == 0


def test_attention(L):
    def cross(d=None, q=FAKE, c=None, kv=FAKE, most=100, out=FAKE, ws=FAKE, wsb=1 << 40):
        return L.glide_kv8_cross_attn(d or desc(), q, c or fake_cache(), kv, most, out, ws, wsb, None)

    def verify(d=None, q=FAKE, n=5, par=FAKE, k=FAKE, v=FAKE, c=None, kv=FAKE, most=100, out=FAKE, ws=FAKE, wsb=1 << 40):
        return L.glide_kv8_verify_attn(d or desc(), q, n, par, k, v, c or fake_cache(), kv, most, out, ws, wsb, None)
    for call in (cross, verify):
        for b in [dict(q=None), dict(kv=None), dict(out=None), dict(ws=None), dict(most=-1), dict(most=301), dict(wsb=16),
                  dict(q=FAKE + 8), dict(kv=FAKE + 2), dict(out=FAKE + 4), dict(ws=FAKE + 8)]:
            assert call(**b) == gb.GLIDE_ERR_INVALID, b
        for c in BAD_CACHES:
            assert call(c=fake_cache(**c)) == gb.GLIDE_ERR_INVALID, c
        for d in BAD_DESCS:
            assert call(d=desc(**d)) == gb.GLIDE_ERR_INVALID, d
    for b in [dict(n=0), dict(n=65), dict(par=None), dict(k=None), dict(v=None), dict(par=FAKE + 1), dict(k=FAKE + 8),
              dict(v=FAKE + 2)]:
        assert verify(**b) == gb.GLIDE_ERR_INVALID, b
    assert verify(d=desc(H=64, H_kv=8), n=33) == gb.GLIDE_ERR_UNSUPPORTED
    assert cross(d=desc(H=512, H_kv=1)) == gb.GLIDE_ERR_UNSUPPORTED


@pytest.mark.gpu
def test_binding_refuses(L):
    B, H, cap, D, n = 2, 3, 100, 64, 4

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    f8, i8, i32 = torch.float8_e4m3fn, torch.int8, torch.int32
    side = dict(K=t(B, H, cap, D, dtype=f8), V=t(B, H, cap, D, dtype=f8), K_exp=t(B, H, 2, dtype=i8),
                V_exp=t(B, H, 2, dtype=i8))
    app = dict(k_new=t(B, n, H, D), v_new=t(B, n, H, D), **side, kv_len=t(B, dtype=i32), new_kv_len=t(B, dtype=i32))
    read = dict(**side, kv_len=t(B, dtype=i32), K_out=t(B, H, 50, D), V_out=t(B, H, 50, D))
    ws = t(1 << 22, dtype=torch.uint8)
    cross = dict(q_draft=t(B, 1, H, D), **side, kv_len=t(B, dtype=i32), max_kv_len=10, out=t(B, 1, H, D), workspace=ws)
    ver = dict(q_tree=t(B, n, H, D), parent_idx=t(B, n, dtype=i32), k_tree=t(B, n, H, D), v_tree=t(B, n, H, D), **side,
               kv_len=t(B, dtype=i32), max_kv_len=10, out=t(B, n, H, D), workspace=ws)
    common = [("K", side["K"].view(i8)), ("V", t(B, H, cap + 1, D, dtype=f8)), ("K", side["K"].cpu()),
              ("K_exp", t(B, H, 3, dtype=i8)), ("V_exp", t(B, H, 2, dtype=torch.uint8)), ("kv_len", t(B + 1, dtype=i32)),
              ("kv_len", t(B, dtype=torch.int64)), ("K", t(B, H, D, cap, dtype=f8).transpose(2, 3))]
    for fn, good, bad in [
            (gb.glide_kv8_append, app, [("k_new", t(B, n, H, D, dtype=torch.float32)), ("v_new", t(B, n + 1, H, D)),
                                        ("k_new", t(B, n, H, 2 * D)[..., ::2]), ("new_kv_len", t(B + 1, dtype=i32)),
                                        ("path", t(B, n + 1, dtype=i32)), ("length", t(B + 1, dtype=i32)),
                                        ("path", t(B, n, dtype=torch.int64)), ("v_new", app["v_new"].cpu())]),
            (gb.glide_kv8_read, read, [("K_out", t(B, H, 50, D, dtype=torch.float32)), ("V_out", t(B, H, 50, D + 1)),
                                       ("K_out", t(B, H, 50, 2 * D)[..., :D]), ("V_out", read["V_out"].cpu())]),
            (gb.glide_kv8_cross_attn, cross, [("q_draft", t(B, 2, H, D)), ("q_draft", t(B, 1, H, D, dtype=torch.float16)),
                                              ("out", t(B, 1, H, D, dtype=torch.float32)), ("out", t(B, 1, H, D + 1)),
                                              ("workspace", ws.cpu()), ("q_draft", t(B, 1, H, 2 * D)[..., ::2])]),
            (gb.glide_kv8_verify_attn, ver, [("parent_idx", t(B, n + 1, dtype=i32)), ("k_tree", t(B, n, H + 1, D)),
                                             ("v_tree", t(B, n, H, D, dtype=torch.float32)),
                                             ("out", t(B, n, H, D, dtype=torch.float32)), ("k_tree", ver["k_tree"].cpu()),
                                             ("parent_idx", ver["parent_idx"].cpu())])]:
        fn(**good)
        for name, value in bad + common:
            with pytest.raises((TypeError, ValueError)):
                fn(**dict(good, **{name: value}))
    with pytest.raises(gb.GlideError):
        gb.glide_kv8_cross_attn(**dict(cross, max_kv_len=cap + 1))
    with pytest.raises(gb.GlideError):
        gb.glide_kv8_cross_attn(**dict(cross, workspace=ws[:16]))
    with pytest.raises(gb.GlideError):
        gb.glide_kv8_append(**dict(app, new_kv_len=app["kv_len"]))
    torch.cuda.synchronize()
