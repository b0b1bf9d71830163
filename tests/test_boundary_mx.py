"""The C entry points of the microscaled operators and the norms without a GPU: arguments are refused before the device is touched."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2506_05413_b200 import build, binding
    build.build()
    return binding.load()


P = ctypes.c_void_p(0x1000)     # never dereferenced: each call fails validation first
ODD = ctypes.c_void_p(0x1008)


def _quant(lib, **change):
    a = dict(X=P, M=3, K=256, ld=256, group=32, pre=None, walsh=0, q=P, s=P, step=None, st=None)
    a.update(change)
    return lib.smoothrot_mx_quant(*a.values())


def _dequant(lib, **change):
    a = dict(q=P, s=P, step=None, M=3, K=256, group=32, Y=P, ld=256, st=None)
    a.update(change)
    return lib.smoothrot_mx_dequant(*a.values())


def _linear(lib, **change):
    a = dict(x=P, xs=P, xstep=None, M=3, w=P, ws=P, wstep=None, N=16, K=256, group=32, Y=P, ld=16, st=None)
    a.update(change)
    return lib.smoothrot_mx_linear(*a.values())


def _glu(lib, **change):
    a = dict(x=P, xs=P, xstep=None, M=3, g=P, gs=P, gstep=None, u=P, us=P, ustep=None, F=128, K=256, group=32, walsh=0, H=P, ldh=128,
             q=None, s=None, hstep=None, st=None)
    a.update(change)
    return lib.smoothrot_mx_glu(*a.values())


def _norm(lib, **change):
    a = dict(Y=P, ldy=256, H=P, ldh=256, M=3, K=256, post=0, pw=None, gate=None, bs=1.0, rs=1.0, w=P, eps=1e-5, Ho=P, ldho=256,
             Xo=ctypes.c_void_p(0x2000), ldxo=256, codes=0, clip=0.9, q=None, s=None, step=None, st=None)
    a.update(change)
    return lib.smoothrot_add_norm(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), -1), (dict(K=0), -1), (dict(group=64), -1), (dict(group=0), -1), (dict(walsh=16), -1), (dict(walsh=256), -1), (dict(K=192, ld=192), -2),
    (dict(K=64, ld=64), -2), (dict(K=65536, ld=65536), -2), (dict(X=None), -1), (dict(q=None), -1), (dict(s=None), -1), (dict(ld=128), -1),
    (dict(group=16), -1), (dict(step=P), -1), (dict(M=1 << 31), -1), (dict(X=ODD), -3), (dict(ld=260), -3), (dict(q=ODD), -3), (dict(s=ODD), -3),
    (dict(pre=ODD), -3), (dict(M=0, X=None, q=None, s=None), 0),
])
def test_quant(lib, change, status):
    assert _quant(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), -1), (dict(group=8), -1), (dict(K=100), -2), (dict(q=None), -1), (dict(s=None), -1), (dict(Y=None), -1), (dict(ld=255), -1),
    (dict(Y=ODD), -3), (dict(ld=260), -3), (dict(M=0, q=None), 0),
])
def test_dequant(lib, change, status):
    assert _dequant(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), -1), (dict(N=-8), -1), (dict(N=12, ld=16), -1), (dict(K=64), -2), (dict(K=1 << 21), -2), (dict(group=128), -1), (dict(x=None), -1),
    (dict(xs=None), -1), (dict(w=None), -1), (dict(ws=None), -1), (dict(Y=None), -1), (dict(ld=8), -1), (dict(ld=20), -3), (dict(x=ODD), -3),
    (dict(ws=ODD), -3), (dict(Y=ODD), -3), (dict(wstep=ODD), -3), (dict(M=0, x=None), 0), (dict(N=0, w=None), 0),
])
def test_linear(lib, change, status):
    assert _linear(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), -1), (dict(F=12), -1), (dict(walsh=64), -1), (dict(walsh=1), -1), (dict(F=40, walsh=32), -2), (dict(F=64, H=None, q=P, s=P), -2),
    (dict(K=96), -2), (dict(H=None), -1), (dict(q=P, s=P), -1), (dict(H=None, q=P), -1), (dict(H=None, q=P, s=P, hstep=P), -1),
    (dict(H=None, q=P, s=P, group=16), -1), (dict(s=P), -1), (dict(hstep=P), -1), (dict(ldh=64), -1), (dict(u=None), -1), (dict(gs=None), -1),
    (dict(g=ODD), -3), (dict(us=ODD), -3), (dict(H=ODD), -3), (dict(ldh=132), -3), (dict(ustep=ODD), -3), (dict(H=None, q=ODD, s=P), -3),
    (dict(M=0, x=None), 0), (dict(F=0, g=None), 0),
])
def test_glu(lib, change, status):
    assert _glu(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), -1), (dict(K=0), -1), (dict(post=2), -1), (dict(codes=8), -1), (dict(eps=0.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(bs=float("inf")), -1), (dict(rs=float("nan")), -1), (dict(codes=4, q=P, step=P, clip=0.0), -1), (dict(codes=4, q=P, step=P, clip=1.5), -1),
    (dict(K=12, ldy=16, ldh=16, ldho=16, ldxo=16), -2), (dict(codes=32, q=P, s=P, K=192), -2), (dict(K=40960, ldy=40960, ldh=40960, ldho=40960, ldxo=40960), -2),
    (dict(Y=None, H=None), -1), (dict(Y=None, post=1), -1), (dict(Y=None, gate=P), -1), (dict(pw=P), -1), (dict(Ho=None, Xo=None), -1), (dict(Ho=P, Xo=P), -1),
    (dict(codes=32, s=P), -1), (dict(codes=32, q=P), -1), (dict(codes=32, q=P, s=P, step=P), -1), (dict(codes=16, q=P, s=P), -1), (dict(codes=4, q=P), -1),
    (dict(ldy=128), -1), (dict(ldxo=128), -1), (dict(Y=ODD), -3), (dict(ldh=260), -3), (dict(Xo=ODD), -3), (dict(w=ODD), -3), (dict(gate=ODD), -3),
    (dict(post=1, pw=ODD), -3), (dict(codes=32, q=ODD, s=P), -3), (dict(codes=32, q=P, s=ODD), -3), (dict(M=0, Y=None, H=None), 0),
])
def test_norm(lib, change, status):
    assert _norm(lib, **change) == status


def test_scale_bytes(lib):
    from paper_2506_05413_b200 import binding
    assert binding.mx_scale_bytes(1, 128, 32) == 512 and binding.mx_scale_bytes(128, 128, 16) == 1024
    assert binding.mx_scale_bytes(129, 4096, 32) == 2 * 128 * 128 and binding.mx_scale_bytes(0, 128, 32) == 0
    assert binding.mx_scale_bytes(4, 100, 32) == 0 and binding.mx_scale_bytes(4, 128, 8) == 0


def test_the_binding_asks_for_cuda_tensors():
    from paper_2506_05413_b200 import binding as sr
    x, q, s = torch.zeros(2, 128, dtype=torch.float16), torch.zeros(2, 64, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for call in (lambda: sr.mx_quant(x, q, s), lambda: sr.mx_dequant(q, s, None, x), lambda: sr.mx_linear(q, s, q, s, x),
                 lambda: sr.mx_glu(q, s, q, s, q, s, h_out=x), lambda: sr.add_norm(x, x, h_out=x), lambda: sr.mx_quant(None, q, s)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        sr.add_norm(x, x, codes="mx8")


@pytest.mark.parametrize("change,status", [
    (dict(q=P), -1), (dict(step=P), -1), (dict(s=P), -1), (dict(codes=4, q=P, step=P, s=P), -1), (dict(ldho=512), -1), (dict(Xo=P, Ho=None, ldxo=264), -1),
    (dict(M=0, ldho=512), 0),
])
def test_norm_arguments_that_do_not_go_together(lib, change, status):
    assert _norm(lib, **change) == status
