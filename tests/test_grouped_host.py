"""CPU-only checks of the grouped entry points: what they refuse, what they take as nothing to do, and that the native
binding agrees with ctypes."""
import os

import pytest

from paper_2511_13764_amd import binding as B

P = 0x1000          # never dereferenced: every call below is refused, or has nothing to launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2511_13764_amd import build
        build.build()
    return B.load()


GROUPED = dict(dt=B.DTYPE_BF16, tB=1, M=16, N=8, K=24, groups=2, off=P, A=P, lda=24, Bm=P, ldb=24, sB=8 * 24, beta=0.0, C=P,
               ldc=8, c32=0, bias=None, sbias=0, epi=0)
WGRAD = dict(dt=B.DTYPE_BF16, M=16, N=8, K=24, groups=2, off=P, dY=P, ldy=8, X=P, ldx=24, beta=0.0, dW=P, ldw=24, sW=8 * 24, c32=0)
ADAPTERS = dict(dt=B.DTYPE_BF16, tB=1, M=16, N=8, K=24, R=4, segments=2, off=P, ids=P, adapters=3, X=P, ldx=24, W=P, ldw=24,
                down=P, ld_down=24, s_down=4 * 24, up=P, ld_up=4, s_up=32, scale=P, beta=0.0, Y=P, ldy=8, c32=0, bias=None,
                epi=0, H=P, ldh=4)


def grouped(**kw):
    a = {**GROUPED, **kw}
    return B.gemm_grouped(a["dt"], a["tB"], a["M"], a["N"], a["K"], a["groups"], a["off"], a["A"], a["lda"], a["Bm"], a["ldb"],
                          a["sB"], a["beta"], a["C"], a["ldc"], a["c32"], a["bias"], a["sbias"], a["epi"], stream=0, check=False)


def wgrad(**kw):
    a = {**WGRAD, **kw}
    return B.gemm_grouped_wgrad(a["dt"], a["M"], a["N"], a["K"], a["groups"], a["off"], a["dY"], a["ldy"], a["X"], a["ldx"],
                                a["beta"], a["dW"], a["ldw"], a["sW"], a["c32"], stream=0, check=False)


def adapters(**kw):
    a = {**ADAPTERS, **kw}
    return B.gemm_adapters(a["dt"], a["tB"], a["M"], a["N"], a["K"], a["R"], a["segments"], a["off"], a["ids"], a["adapters"],
                           a["X"], a["ldx"], a["W"], a["ldw"], a["down"], a["ld_down"], a["s_down"], a["up"], a["ld_up"],
                           a["s_up"], a["scale"], a["beta"], a["Y"], a["ldy"], a["c32"], a["bias"], a["epi"], a["H"], a["ldh"],
                           stream=0, check=False)


@pytest.mark.parametrize("kw", [
    dict(dt=9), dict(dt=B.DTYPE_F32, c32=0), dict(tB=2), dict(M=-1), dict(N=-1), dict(K=-1), dict(groups=-1), dict(groups=1 << 31),
    dict(M=1 << 31), dict(off=None), dict(A=None), dict(Bm=None), dict(C=None), dict(lda=23), dict(ldb=23), dict(tB=0, ldb=7),
    dict(ldc=7), dict(sB=-1), dict(sbias=-1), dict(epi=8), dict(epi=B.EPI_BIAS)])
def test_grouped_refuses(lib, kw):
    assert grouped(**kw) == B.INVALID_ARG


def test_grouped_with_nothing_to_do(lib):
    for kw in (dict(M=0), dict(N=0), dict(groups=0), dict(groups=0, off=None, Bm=None)):
        assert grouped(**kw) == B.OK, kw


def test_more_rows_than_a_launch_holds(lib):
    assert grouped(M=(1 << 31) - 1, groups=2) == B.UNSUPPORTED
    assert adapters(M=(1 << 31) - 1) == B.UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(dt=9), dict(dt=B.DTYPE_F32, c32=0), dict(M=-1), dict(N=-1), dict(K=-1), dict(groups=-1), dict(off=None), dict(dY=None),
    dict(X=None), dict(dW=None), dict(ldy=7), dict(ldx=23), dict(ldw=23), dict(sW=-1), dict(sW=8 * 24 - 1)])
def test_wgrad_refuses(lib, kw):
    assert wgrad(**kw) == B.INVALID_ARG


def test_wgrad_with_nothing_to_do(lib):
    for kw in (dict(N=0), dict(K=0), dict(groups=0)):
        assert wgrad(**kw) == B.OK, kw


@pytest.mark.parametrize("kw", [
    dict(dt=9), dict(dt=B.DTYPE_F32, c32=0), dict(tB=2), dict(M=-1), dict(N=-1), dict(K=-1), dict(R=-1), dict(segments=-1),
    dict(adapters=-1), dict(off=None), dict(X=None), dict(W=None), dict(Y=None), dict(down=None), dict(up=None), dict(H=None),
    dict(ldx=23), dict(ldw=23), dict(ld_down=23), dict(ld_up=3), dict(ldy=7), dict(ldh=3), dict(s_down=-1), dict(s_up=-1),
    dict(epi=8), dict(epi=B.EPI_BIAS), dict(tB=0, ldw=7), dict(tB=0, ldw=8, ld_down=3), dict(tB=0, ldw=8, ld_down=4, ld_up=7),
    dict(N=0, X=None)])
def test_adapters_refuse(lib, kw):
    assert adapters(**kw) == B.INVALID_ARG


def test_adapters_with_nothing_to_do(lib):
    assert adapters(M=0) == B.OK
    assert adapters(M=0, segments=0, off=None, ids=None) == B.OK


def test_workspace_rules(lib):
    import ctypes
    a = [B.DTYPE_BF16, 1, 16, 8, 24, 2, P, P, 24, P, 24, 192, 0.0, P, 8, 0, None, 0, 0]
    assert lib.gemm_grouped(*a, None, 1024, None) == B.INVALID_ARG
    assert lib.gemm_grouped(*a, ctypes.c_void_p(0x1010), 1024, None) == B.MISALIGNED_WORKSPACE


def test_native_calls_agree_with_ctypes(lib):
    """csrc/fastcall.c: the same codes for plain arguments, NotImplemented for any other."""
    import numpy as np
    calls = {"gemm_grouped": lambda M: (1, 1, M, 8, 24, 2, P, P, 24, P, 24, 192, 0.0, P, 8, 0, None, 0, 0, None, 0),
             "gemm_grouped_wgrad": lambda M: (1, 16, M, 24, 2, P, P, 8, P, 24, 0, P, 24, 192, True, None, 0),
             "gemm_adapters": lambda M: (1, 1, M, 8, 24, 4, 2, P, P, 3, P, 24, P, 24, P, 24, 96, P, 4, 32, None, 0.0, P, 8, False,
                                         None, 0, P, 4, None, 0)}
    assert set(calls) == set(B.FAST_GROUPED)
    for name, args in calls.items():
        f = B._native(name)
        assert f(*args(0)) == B.OK and f(*args(-1)) == B.INVALID_ARG, name
        for odd in (np.int64(0), 0.0, "0", 1 << 70, None):
            assert f(*args(odd)) is NotImplemented, (name, odd)
        assert f(*args(0)[:-1]) is NotImplemented
        assert f(*args(0)[:-1], object()) is NotImplemented
    assert grouped(M=np.int64(0)) == B.OK and wgrad(N=np.int64(-1)) == B.INVALID_ARG and adapters(M=np.int64(0)) == B.OK
