"""What the 8-bit operators refuse, through the C ABI before any launch (CPU: no pointer is read)."""
import ctypes

import pytest

from tests.test_abi import pace

P, ODD, OFF, ONE = (ctypes.c_void_p(a) for a in (0x1000, 0x1008, 0x1002, 0x1001))


def quantize(**kw):
    a = dict(x=P, stride=256, M=4, K=256, rows=1, q=P, scale=P, stream=None)
    a.update(kw)
    return pace.lib().pace_quantize_fp8(*a.values()), pace.lib().pace_last_error().decode()


def norm(**kw):
    a = dict(x=P, stride=256, r=P, rstride=256, gamma=P, eps=1e-6, M=4, K=256, sum=P, y=None, q=P, scale=P, stream=None)
    a.update(kw)
    return pace.lib().pace_rmsnorm(*a.values()), pace.lib().pace_last_error().decode()


def gemm(**kw):
    a = dict(x=P, xs=P, xss=4, w=P, ws=P, bias=None, residual=None, C=P, cs=None, M=4, N=64, K=256, epilogue=0, sums=0, wsp=None, wsb=0, stream=None)
    a.update(kw)
    return pace.lib().pace_gemm_fp8(*a.values()), pace.lib().pace_last_error().decode()


@pytest.mark.parametrize("bad,word", [
    (dict(x=None), "null"), (dict(q=None), "null"), (dict(scale=None), "null"), (dict(x=ODD), "aligned"), (dict(q=ODD), "aligned"), (dict(scale=OFF), "aligned"), (dict(M=-1), "M=-1"),
    (dict(K=0), "K=0"), (dict(K=8), "K=8"), (dict(K=200), "K=200"), (dict(K=(1 << 20) + 16, stride=1 << 21), "2^20"), (dict(stride=248), "stride"),
    (dict(stride=260), "stride"), (dict(stride=-256), "stride"), (dict(rows=2), "rows"), (dict(rows=0), "rows"),
    (dict(M=1 << 30, K=16384, stride=16384), "too many"), (dict(M=(1 << 31) - 1, K=4096, stride=4096, rows=128), "too many")])
def test_quantize(bad, word):
    st, msg = quantize(**bad)
    assert st == 1 and word in msg


@pytest.mark.parametrize("bad,word", [
    (dict(x=None), "null"), (dict(gamma=None), "null"), (dict(q=None), "either"), (dict(scale=None), "either"), (dict(y=P), "either"),
    (dict(q=None, scale=None), "either"), (dict(y=P, q=None), "either"), (dict(x=ODD), "aligned"), (dict(r=ODD), "aligned"), (dict(gamma=ODD), "aligned"),
    (dict(sum=ODD), "aligned"), (dict(scale=OFF), "aligned"), (dict(q=ODD), "aligned"), (dict(y=ODD, q=None, scale=None), "aligned"), (dict(M=-1), "M=-1"), (dict(K=0), "K=0"), (dict(K=264), "K=264"),
    (dict(K=65552, stride=65552, rstride=65552), "65,536"), (dict(stride=248), "stride"), (dict(stride=257), "stride"), (dict(rstride=248), "residual"),
    (dict(rstride=252), "residual"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(M=1 << 26), "too many"), (dict(M=1 << 24, K=8192, stride=8192, rstride=8192), "too many")])
def test_norm(bad, word):
    st, msg = norm(**bad)
    assert st == 1 and word in msg


@pytest.mark.parametrize("bad,word", [
    (dict(x=None), "null"), (dict(xs=None), "null"), (dict(w=None), "null"), (dict(ws=None), "null"), (dict(C=None), "null"), (dict(x=ODD), "aligned"),
    (dict(w=ODD), "aligned"), (dict(xs=OFF), "aligned"), (dict(ws=OFF), "aligned"), (dict(bias=OFF), "aligned"), (dict(residual=ONE, epilogue=1), "aligned"), (dict(C=ONE), "aligned"),
    (dict(cs=OFF, epilogue=2), "aligned"), (dict(epilogue=3), "epilogue"), (dict(epilogue=-1), "epilogue"), (dict(sums=3), "sums"), (dict(sums=-1), "sums"), (dict(epilogue=1), "residual"), (dict(epilogue=2, N=63), "even"),
    (dict(M=-1), "M=-1"), (dict(N=0), "N=0"), (dict(K=0), "K=0"), (dict(K=264), "K=264"), (dict(K=(1 << 20) + 16), "2^20"), (dict(xss=3), "stride"),
    (dict(cs=P), "SwiGLU"), (dict(cs=P, epilogue=1, residual=P), "SwiGLU"), (dict(cs=P, epilogue=2, N=48), "32"), (dict(cs=P, epilogue=2, C=ODD), "aligned"),
    (dict(N=(1 << 30) + 1), "too many"), (dict(M=1 << 22, xss=1 << 22, N=1 << 22), "too many")])
def test_gemm(bad, word):
    st, msg = gemm(**bad)
    assert st == 1 and word in msg


def test_no_rows_are_no_error():
    assert quantize(M=0, x=None, q=None, scale=None)[0] == 0
    assert norm(M=0, x=None, r=None, sum=None, q=None, scale=None)[0] == 0
    assert gemm(M=0, x=None, xs=None, xss=0, C=None)[0] == 0


@pytest.mark.parametrize("M,N,K,bits", [(8, 28672, 3584, 8), (48, 3584, 14336, 16), (300, 640, 1280, 8)])
def test_gemm_workspace(M, N, K, bits):
    need = pace.lib().pace_gemm_fp8_workspace_size(M, N, K, bits, 0)
    assert pace.lib().pace_gemm_fp8_workspace_size(0, N, K, bits, 0) == 0 and pace.lib().pace_gemm_fp8_workspace_size(M, -N, K, bits, 0) == 0
    if need:
        kw = dict(M=M, N=N, K=K, xss=M, epilogue=2 if bits == 8 else 0, cs=P if bits == 8 else None)
        for ws, wsb, st, word in ((None, 0, 3, "workspace"), (P, need - 1, 3, "workspace"), (ODD, need, 1, "aligned")):
            got, msg = gemm(wsp=ws, wsb=wsb, **kw)
            assert got == st and word in msg
