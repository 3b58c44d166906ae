"""The router against its definition in 64 bits (route_reference.py)."""
import numpy as np
import pytest
import torch

import route_reference as rr
from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, B.DTYPE_F32), "bf16": (torch.bfloat16, B.DTYPE_BF16), "f16": (torch.float16, B.DTYPE_F16)}


def outputs(M, E, top):
    def full(shape, v, dt):
        return torch.full(shape, v, dtype=dt, device="cuda")
    return dict(ids=full((M, top), 99, torch.int64), gates=full((M, top), 9.0, torch.float32), offsets=full((E + 1,), 99, torch.int64),
                rows=full((M * top,), 99, torch.int64), place=full((M, top), 99, torch.int64), balance=full((2 + E,), 9.0, torch.float32))


def call(dtype, t, M, E, top, valid=None, level=0, ws=True, ld=None):
    o = outputs(M, E, top)
    workspace = torch.empty(B.gemm_route_workspace_bytes(M, E), dtype=torch.uint8, device="cuda") if ws else None
    B.gemm_route(DT[dtype][1], M, E, top, t, ld or E, valid, level, *o.values(), workspace=workspace if ws and workspace.numel() else None)
    return o


def check_forward(o, want, E):
    for n in ("ids", "offsets", "rows", "place"):
        assert np.array_equal(o[n].cpu().numpy(), want[n]), n
    # exp, its sum over E, a quotient and (level) another sum and quotient: each within a few roundings of 2^-24
    eps = 2.0 ** -24
    assert np.allclose(o["gates"].cpu().numpy(), want["gates"], rtol=(E + 40) * eps, atol=1e-37)
    # sums of p over the rows: at most 2^15 rows one after the other, in parts of at most 256
    assert np.allclose(o["balance"].cpu().numpy(), want["balance"], rtol=(2 * E + 600) * eps, atol=1e-37)


def logits_of(rng, M, E, dtype, coarse=False):
    x = rng.integers(-3, 4, (M, E)).astype(float) if coarse else rng.standard_normal((M, E)) * 2
    t = torch.from_numpy(x).to(DT[dtype][0])
    return t.double().numpy(), t


SIZES = [(1, 1, 1), (1, 8, 2), (16, 8, 8), (130, 16, 3), (300, 5, 2), (700, 33, 4), (1000, 64, 4), (777, 160, 6), (515, 300, 8),
         (200, 1000, 16), (33, 1024, 1), (4099, 96, 5), (257, 8, 2), (6000, 7, 7)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,E,top", SIZES)
def test_route_and_gradient(dtype, M, E, top):
    rng = np.random.default_rng([M, E, top])
    for level, coarse in ((0, True), (1, False)):
        x, t = logits_of(rng, M, E, dtype, coarse)
        valid = (rng.random(M) < 0.8) if level else None
        wide = torch.full((M, E + 3), float("nan"), dtype=t.dtype)
        wide[:, :E] = t
        dv = torch.from_numpy(valid.astype(np.uint8)).cuda() if level else None
        want = rr.route(x, top, valid, level)
        o = call(dtype, wide.cuda(), M, E, top, dv, level, ld=E + 3)
        check_forward(o, want, E)
        dg = rng.standard_normal((M, top)).astype(np.float32)
        dg[want["ids"] < 0] = np.nan                                # not read
        dl = np.float32(3.0 * M)
        d = torch.full((M, E + 1), -77.0, dtype=t.dtype, device="cuda")
        B.gemm_route_grad(DT[dtype][1], M, E, top, wide.cuda(), E + 3, level, o["ids"], o["offsets"], o["balance"],
                          torch.from_numpy(dg).cuda(), torch.tensor([dl], device="cuda"), d, E + 1)
        share = np.diff(want["offsets"]) / max(1, want["offsets"][-1])
        ref = rr.gradient(x, want["ids"], share, dg.astype(float), float(dl), level)
        got = d.double().cpu().numpy()
        assert (got[:, E] == -77.0).all()
        # terms of at most 1 * max|dgates| and dloss E / n: their roundings in 32 bits, then the result's own
        n = max(1.0, want["balance"][1])
        term = np.nanmax(np.abs(np.where(np.isnan(dg), 0, dg))) + float(dl) * E / n * want["p"].max(1, keepdims=True)
        eps = torch.finfo(t.dtype).eps / 2 if dtype != "f32" else 2.0 ** -24
        tiny = 2.0 ** -25 if dtype == "f16" else 1e-38
        off = (2 * E + 60) * 2.0 ** -24 * term
        assert (np.abs(got[:, :E] - ref) <= off + eps * (np.abs(ref) + off) + tiny).all()


@pytest.mark.parametrize("M", [9, 2000])
def test_rows_that_cannot_choose(M):
    """Rows of -inf, rows with fewer experts than choices, NaN, +inf, the type's lowest value, all of them padding."""
    E, top = 12, 4
    rng = np.random.default_rng(6)
    x = rng.standard_normal((M, E)).astype(np.float32)
    x[0] = -np.inf
    x[1, 3:] = -np.inf
    x[2, 5] = np.nan
    x[3, :] = np.nan
    x[4, 7] = np.inf
    x[5, :] = np.finfo(np.float32).min
    x[6, 1:] = -np.inf
    x[7, ::2] = -np.inf
    for level in (0, 1):
        want = rr.route(x.astype(float), top, None, level)
        o = call("f32", torch.from_numpy(x).cuda(), M, E, top, None, level)
        for n in ("ids", "offsets", "rows", "place"):
            assert np.array_equal(o[n].cpu().numpy(), want[n]), n
        good = np.ones(M, bool)
        good[[2, 4]] = False                                        # NaN, as the formula
        got = o["gates"].cpu().numpy()
        assert np.allclose(got[good], want["gates"][good], rtol=1e-5, atol=1e-37)
        assert np.isnan(got[[2, 4]]).all() and np.isnan(o["balance"].cpu().numpy()[0])
        assert float(o["balance"][1]) == want["balance"][1] == M - 2
        dg = torch.ones((M, top), device="cuda")
        dg[0] = dg[3] = float("nan")
        d = torch.full((M, E), 5.0, device="cuda")
        B.gemm_route_grad(B.DTYPE_F32, M, E, top, torch.from_numpy(x).cuda(), E, level, o["ids"], o["offsets"], o["balance"], dg, None, d, E)
        share = np.diff(want["offsets"]) / want["offsets"][-1]
        ref = rr.gradient(x.astype(float), want["ids"], share, np.ones((M, top)), 0.0, level)
        got = d.cpu().numpy()
        assert (got[0] == 0).all() and (got[3] == 0).all()
        assert np.allclose(got[good], ref[good], rtol=1e-4, atol=1e-6)
    o = call("f32", torch.from_numpy(x).cuda(), M, E, top, torch.zeros(M, dtype=torch.uint8, device="cuda"), 1)
    assert (o["ids"] == -1).all() and (o["rows"] == -1).all() and (o["place"] == -1).all()
    assert (o["gates"] == 0).all() and (o["offsets"] == 0).all() and (o["balance"] == 0).all()
    d = torch.full((M, E), 5.0, device="cuda")
    B.gemm_route_grad(B.DTYPE_F32, M, E, top, torch.from_numpy(x).cuda(), E, 1, o["ids"], o["offsets"], o["balance"], None,
                      torch.ones(1, device="cuda"), d, E)
    assert (d == 0).all()


def test_no_rows():
    o = call("f32", None, 0, 8, 2)
    assert (o["offsets"] == 0).all() and (o["balance"] == 0).all()


@pytest.mark.parametrize("M,E,top", [(3000, 64, 4), (1500, 512, 8)])
def test_the_same_bits_with_any_workspace_and_from_a_graph(M, E, top):
    rng = np.random.default_rng(11)
    xs = [logits_of(rng, M, E, "bf16")[1].cuda() for _ in range(3)]
    x = xs[0].clone()
    o, d = outputs(M, E, top), torch.empty((M, E), dtype=torch.bfloat16, device="cuda")
    need = B.gemm_route_workspace_bytes(M, E)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dg, dl = torch.ones((M, top), device="cuda"), torch.ones(1, device="cuda")

    def run(workspace):
        B.gemm_route(B.DTYPE_BF16, M, E, top, x, E, None, 1, *o.values(), workspace=workspace)
        B.gemm_route_grad(B.DTYPE_BF16, M, E, top, x, E, 1, o["ids"], o["offsets"], o["balance"], dg, dl, d, E)

    def kept():
        return {**{n: v.clone() for n, v in o.items()}, "d": d.clone()}
    eager = []
    for i in range(3):
        x.copy_(xs[i])
        run(ws)
        eager.append(kept())
        for workspace in (ws, None, ws[:need // 3 // 256 * 256]):
            run(workspace)
            got = kept()
            for n in got:
                if workspace is ws or n not in ("balance", "d"):
                    assert torch.equal(got[n], eager[-1][n]), n
                else:                                               # (fewer workgroups add the probabilities up in other parts)
                    assert torch.allclose(got[n].float(), eager[-1][n].float(), rtol=1e-2 if n == "d" else 1e-5, atol=1e-6), n
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(ws)
    for i in (1, 2, 0, 0, 1):
        x.copy_(xs[i])
        for v in o.values():
            v.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        got = kept()
        for n in got:
            assert torch.equal(got[n], eager[i][n]), n
