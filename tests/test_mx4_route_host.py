"""CPU-only checks of the 4-bit images, their products and the router: what they refuse, what they take as nothing to do, and that the
references the GPU tests use agree with themselves."""
import ctypes
import os

import numpy as np
import pytest

import mx4_reference as mx
import route_reference as rr
from paper_2511_13764_amd import binding as B

P = 0x1000          # never dereferenced: every call below is refused, or has nothing to launch


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2511_13764_amd import build
        build.build()
    return B.load()


def pack(**kw):
    a = {**dict(dt=B.DTYPE_BF16, trans=0, rows=4, K=40, X=P, ldx=40, x_rows=4, source=None, image=P, nb=1 << 20), **kw}
    return B.gemm_pack_mx4(a["dt"], a["trans"], a["rows"], a["K"], a["X"], a["ldx"], a["x_rows"], a["source"], a["image"], a["nb"],
                           stream=0, check=False)


def unpack(**kw):
    a = {**dict(dt=B.DTYPE_BF16, rows=4, K=40, image=P, out=P, ldo=40), **kw}
    return B.gemm_unpack_mx4(a["dt"], a["rows"], a["K"], a["image"], a["out"], a["ldo"], stream=0, check=False)


def mx4(**kw):
    a = {**dict(dt=B.DTYPE_BF16, M=4, N=8, K=40, A=P, lda=40, W=P, beta=0.0, C=P, ldc=8, c32=0, bias=None, epi=0), **kw}
    return B.gemm_mx4(a["dt"], a["M"], a["N"], a["K"], a["A"], a["lda"], a["W"], a["beta"], a["C"], a["ldc"], a["c32"], a["bias"],
                      a["epi"], stream=0, check=False)


def grouped(**kw):
    a = {**dict(dt=B.DTYPE_BF16, M=4, N=8, K=40, groups=2, off=P, A=P, lda=40, W=P, sW=2048, beta=0.0, C=P, ldc=8, c32=0, bias=None,
                sb=0, epi=0), **kw}
    return B.gemm_grouped_mx4(a["dt"], a["M"], a["N"], a["K"], a["groups"], a["off"], a["A"], a["lda"], a["W"], a["sW"], a["beta"],
                              a["C"], a["ldc"], a["c32"], a["bias"], a["sb"], a["epi"], stream=0, check=False)


def route(**kw):
    a = {**dict(dt=B.DTYPE_BF16, M=4, E=8, top=2, x=P, ld=8, valid=None, level=0, ids=P, gates=P, off=P, rows=P, place=P, bal=P), **kw}
    return B.gemm_route(a["dt"], a["M"], a["E"], a["top"], a["x"], a["ld"], a["valid"], a["level"], a["ids"], a["gates"], a["off"],
                        a["rows"], a["place"], a["bal"], stream=0, check=False)


def route_grad(**kw):
    a = {**dict(dt=B.DTYPE_BF16, M=4, E=8, top=2, x=P, ld=8, level=0, ids=P, off=P, bal=P, dg=P, dl=P, dx=P, ldd=8), **kw}
    return B.gemm_route_grad(a["dt"], a["M"], a["E"], a["top"], a["x"], a["ld"], a["level"], a["ids"], a["off"], a["bal"], a["dg"],
                             a["dl"], a["dx"], a["ldd"], stream=0, check=False)


@pytest.mark.parametrize("kw", [
    dict(dt=B.DTYPE_MX4), dict(dt=9), dict(trans=2), dict(rows=-1), dict(K=-1), dict(rows=1 << 31), dict(K=1 << 31), dict(X=None),
    dict(ldx=39), dict(x_rows=3), dict(x_rows=-1), dict(image=None), dict(image=P + 8), dict(nb=4 * 136 - 1), dict(trans=1, ldx=3),
    dict(trans=1, source=P), dict(source=P, x_rows=-1), dict(source=P, X=None)])
def test_pack_refuses(lib, kw):
    assert pack(**kw) == B.INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dt=B.DTYPE_MX4), dict(rows=-1), dict(K=-1), dict(image=None), dict(image=P + 4), dict(out=None), dict(ldo=39)])
def test_unpack_refuses(lib, kw):
    assert unpack(**kw) == B.INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(dt=B.DTYPE_F32), dict(dt=9), dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 31), dict(A=None), dict(W=None), dict(C=None),
    dict(lda=39), dict(ldc=7), dict(epi=8), dict(epi=B.EPI_BIAS), dict(W=P + 8), dict(dt=B.DTYPE_MX4, A=P + 8)])
def test_products_refuse(lib, kw):
    assert mx4(**kw) == B.INVALID_ARG
    assert grouped(**kw) == B.INVALID_ARG


@pytest.mark.parametrize("kw", [dict(groups=-1), dict(groups=1 << 31), dict(off=None), dict(sW=-16), dict(sW=2056), dict(sb=-1)])
def test_grouped_refuses(lib, kw):
    assert grouped(**kw) == B.INVALID_ARG


def test_nothing_to_do(lib):
    for kw in (dict(M=0), dict(N=0)):
        assert mx4(**kw) == B.OK and grouped(**kw) == B.OK, kw
    assert grouped(groups=0, off=None, W=None) == B.OK
    for kw in (dict(rows=0, x_rows=0), dict(K=0)):
        assert pack(**kw) == B.OK, kw
    assert unpack(rows=0) == B.OK and unpack(K=0) == B.OK
    assert route_grad(M=0) == B.OK
    assert grouped(M=(1 << 31) - 1) == B.UNSUPPORTED


def test_bytes(lib):
    for rows, K in ((1, 1), (3, 256), (5, 257), (7, 1000)):
        assert B.gemm_mx4_bytes(rows, K) == mx.nbytes(rows, K)
    for rows, K in ((0, 5), (5, 0), (-1, 5), (5, 1 << 31)):
        assert B.gemm_mx4_bytes(rows, K) == 0


@pytest.mark.parametrize("kw", [
    dict(dt=B.DTYPE_MX4), dict(M=-1), dict(E=0), dict(E=-1), dict(top=0), dict(top=9), dict(x=None), dict(ld=7), dict(ids=None),
    dict(off=None), dict(bal=None)])
def test_router_refuses(lib, kw):
    assert route(**kw) == B.INVALID_ARG
    assert route_grad(**{**kw}) == B.INVALID_ARG


def test_router_refuses_more(lib):
    for kw in (dict(gates=None), dict(rows=None), dict(place=None)):
        assert route(**kw) == B.INVALID_ARG
    for kw in (dict(dx=None), dict(ldd=7)):
        assert route_grad(**kw) == B.INVALID_ARG
    for kw in (dict(E=1025, ld=1025, ldd=1025), dict(E=64, ld=64, ldd=64, top=17), dict(M=1 << 30, top=2)):
        assert route(**{k: v for k, v in kw.items() if k != "ldd"}) == B.UNSUPPORTED
        assert route_grad(**kw) == B.UNSUPPORTED
    a = [B.DTYPE_BF16, 4, 8, 2, P, 8, None, 0, P, P, P, P, P, P]
    assert lib.gemm_route(*a, None, 1024, None) == B.INVALID_ARG
    assert lib.gemm_route(*a, ctypes.c_void_p(0x1010), 1024, None) == B.MISALIGNED_WORKSPACE
    a = [B.DTYPE_BF16, 4, 8, 40, P, 40, P, 0.0, P, 8, 0, None, 0]
    assert lib.gemm_mx4(*a, None, 1024, None) == B.INVALID_ARG
    assert lib.gemm_mx4(*a, ctypes.c_void_p(0x1010), 1024, None) == B.MISALIGNED_WORKSPACE


def test_workspace_bytes(lib):
    assert B.gemm_route_workspace_bytes(16, 8) == 0
    assert B.gemm_route_workspace_bytes(0, 8) == 0 and B.gemm_route_workspace_bytes(5, 2000) == 0
    assert 0 < B.gemm_route_workspace_bytes(100000, 1024) <= 8 << 20


def test_native_calls_agree_with_ctypes(lib):
    """csrc/fastcall.c: the same codes for plain arguments, NotImplemented for any other."""
    calls = {"gemm_pack_mx4": (lambda r: (1, 0, r, 40, P, 40, 4, None, P, 1 << 20, 0), 2),
             "gemm_unpack_mx4": (lambda r: (1, r, 40, P, P, 40, 0), 1),
             "gemm_mx4": (lambda M: (1, M, 8, 40, P, 40, P, 0.0, P, 8, False, None, 0, None, 0), 1),
             "gemm_grouped_mx4": (lambda M: (1, M, 8, 40, 2, P, P, 40, P, 2048, 0.0, P, 8, 0, None, 0, 0, None, 0), 1),
             "gemm_route_grad": (lambda M: (1, M, 8, 2, P, 8, True, P, P, P, P, P, P, 8, 0), 1),
             "gemm_route": (lambda M: (1, M, 8, 2, P, 8, P, 0, P, P, P, P, P, None, None, 0), 1)}
    assert set(calls) == set(B.FAST_MX4)
    for name, (args, at) in calls.items():
        f = B._native(name)
        nothing = B.INVALID_ARG if name == "gemm_route" else B.OK       # (without a place for the balance)
        assert f(*args(0)) == nothing and f(*args(-1)) == B.INVALID_ARG, name
        for odd in (np.int64(0), 0.0, "0", 1 << 70, None):
            assert f(*args(odd)) is NotImplemented, (name, odd)
        assert f(*args(0)[:-1]) is NotImplemented
        assert f(*args(0)[:-1], object()) is NotImplemented
    f = B._native("gemm_pack_mx4")
    assert f(1, 0, 0, 40, P, 40, 4, None, P, None, 0) is NotImplemented          # an address does not say how many bytes
    assert pack(rows=np.int64(0)) == B.OK and mx4(M=np.int64(-1)) == B.INVALID_ARG and route_grad(M=np.int64(0)) == B.OK


def test_image_reference():
    """Values of the grid times a power are what they are; others are off by at most half a step of theirs."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, 300)) * np.exp2(rng.integers(-20, 20, (9, 300)))
    img = mx.image(x)
    assert img.nbytes == mx.nbytes(9, 300)
    v = mx.values(img, 9, 300)
    assert np.array_equal(mx.values(mx.image(v), 9, 300), v)
    codes, powers = mx.quantise(x)
    scale = np.repeat(np.ldexp(1.0, powers.astype(int) - 127), 32, 1)[:, :300]
    y = np.abs(x) / scale
    step = np.where(y < 2, 0.5, np.where(y < 4, 1.0, 2.0))
    assert (np.abs(v - x) / scale <= np.where(y > 6, 2.0, step / 2)).all() and (y < 8).all()
    assert (np.abs(y).reshape(9, 300).max() >= 4)


@pytest.mark.parametrize("level", [False, True])
def test_router_gradient_is_the_difference(level):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 7))
    x[2] = -np.inf
    x[3, :5] = -np.inf
    ids = rr.route(x, 3, None, level)["ids"]
    assert (ids[2] == -1).all() and (ids[3] >= 0).sum() == 2
    share = rng.random(7)
    dg, dl = rng.standard_normal((6, 3)), 0.7
    g = rr.gradient(x, ids, share, dg, dl, level)
    h = 1e-5
    for t in range(6):
        for e in range(7):
            if x[t, e] == -np.inf:
                assert g[t, e] == 0
                continue
            up, down = x.copy(), x.copy()
            up[t, e] += h
            down[t, e] -= h
            d = (rr.value(up, ids, share, dg, dl, level) - rr.value(down, ids, share, dg, dl, level)) / (2 * h)
            assert abs(d - g[t, e]) < 1e-8            # (h^2 and 1e-16 / h)
