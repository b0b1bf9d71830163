"""The cache's and the attention's C entry points without a GPU: arguments are refused before the device is touched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2506_05413_b200 import build, binding
    build.build()
    return binding.load()


P = ctypes.c_void_p(0x1000)     # never dereferenced: each call fails validation first
ODD = ctypes.c_void_p(0x1008)


def _append(lib, **change):
    a = dict(Q=P, ldq=512, K=P, ldk=256, V=P, ldv=256, T=3, H=4, kv=2, D=128, pos=P, rot=P, rows=10, inter=0, walsh=0,
             Qo=P, ldqo=512, Ko=None, ldko=0, slots=P, bits=4, pages=2, page=16, kc=P, vc=P, kp=P, vp=P, clip=0.9, st=None)
    a.update(change)
    return lib.smoothrot_kv_append(*a.values())


def _gather(lib, **change):
    a = dict(slots=P, T=3, kv=2, D=128, bits=4, pages=2, page=16, kc=P, vc=P, kp=P, vp=P, Ko=P, ldk=256, Vo=P, ldv=256, st=None)
    a.update(change)
    return lib.smoothrot_kv_gather(*a.values())


def _decode(lib, **change):
    a = dict(Q=P, ldq=512, B=2, H=4, kv=2, D=128, bits=16, pages=2, page=16, kc=P, vc=P, kp=None, vp=None, table=P, mp=4,
             n=P, scale=0.1, Y=P, ldy=512, ws=P, wsb=1 << 30, st=None)
    a.update(change)
    return lib.smoothrot_attn_decode(*a.values())


def _prefill(lib, **change):
    a = dict(Q=P, ldq=512, tq=5, K=P, ldk=256, V=P, ldv=256, tk=5, H=4, kv=2, D=128, cq=P, ck=P, B=1, causal=1, scale=0.1,
             Y=P, ldy=512, st=None)
    a.update(change)
    return lib.smoothrot_attn_prefill(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(H=-1), -1), (dict(kv=0), -1), (dict(D=96), -2), (dict(bits=8), -1), (dict(kv=3, D=64, ldk=192, ldv=192), -2),
    (dict(page=12), -1), (dict(page=2048), -1), (dict(page=0), -1), (dict(pages=-1), -1), (dict(clip=0.0), -1), (dict(clip=1.1), -1),
    (dict(inter=2), -1), (dict(walsh=-1), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(pos=None), -1), (dict(rot=None), -1),
    (dict(slots=None), -1), (dict(Q=None), -1), (dict(Qo=None), -1), (dict(ldq=256), -1), (dict(ldk=128), -1), (dict(kc=None), -1),
    (dict(kp=None), -1), (dict(Ko=P, ldko=128), -1), (dict(K=ODD), -3), (dict(ldv=260), -3), (dict(kc=ODD), -3), (dict(vp=ODD), -3),
    (dict(Qo=ODD), -3), (dict(rot=ODD), -3), (dict(Ko=ODD, ldko=256), -3), (dict(T=0, K=None, slots=None), 0),
])
def test_append(lib, change, status):
    assert _append(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(D=32), -2), (dict(bits=3), -1), (dict(page=24), -1), (dict(T=1 << 30), -1), (dict(slots=None), -1),
    (dict(Ko=None), -1), (dict(ldk=128), -1), (dict(vc=None), -1), (dict(vp=None), -1), (dict(Vo=ODD), -3), (dict(ldv=257), -3),
    (dict(T=0, slots=None), 0),
])
def test_gather(lib, change, status):
    assert _gather(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(B=-1), -1), (dict(B=8193), -1), (dict(H=0), -1), (dict(H=5), -1), (dict(D=256), -2), (dict(page=3), -1), (dict(mp=-1), -1),
    (dict(mp=1 << 28), -1), (dict(scale=float("nan")), -1), (dict(Q=None), -1), (dict(Y=None), -1), (dict(n=None), -1),
    (dict(table=None), -1), (dict(ldq=511), -1), (dict(bits=4), -1), (dict(kc=None), -1), (dict(Q=ODD), -3), (dict(ldy=516), -3),
    (dict(kc=ODD), -3), (dict(B=0, Q=None), 0),
])
def test_decode(lib, change, status):
    assert _decode(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(tq=-1), -1), (dict(tk=1 << 31), -1), (dict(B=-1), -1), (dict(H=5), -1), (dict(kv=0), -1), (dict(D=80), -2),
    (dict(causal=2), -1), (dict(scale=float("nan")), -1), (dict(Q=None), -1), (dict(K=None), -1), (dict(cq=None), -1),
    (dict(ldv=128), -1), (dict(Y=ODD), -3), (dict(K=ODD), -3), (dict(ldq=516), -3), (dict(tq=0, Q=None), 0), (dict(B=0, K=None), 0),
])
def test_prefill(lib, change, status):
    assert _prefill(lib, **change) == status


def test_decode_workspace(lib):
    need = lib.smoothrot_attn_decode_workspace_bytes(4, 32, 8, 128)
    assert 0 <= need <= 16 << 20
    assert lib.smoothrot_attn_decode_workspace_bytes(-1, 32, 8, 128) == 0 and lib.smoothrot_attn_decode_workspace_bytes(4, 5, 2, 128) == 0
    if need:
        assert _decode(lib, B=4, H=32, kv=8, ldq=4096, ldy=4096, wsb=need - 1) == -4
