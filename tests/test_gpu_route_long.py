"""The router on so many rows a workgroup that sums of 32 bits would lose the last ones: mean probabilities and the balance loss do not
depend on how many workgroups there were."""
import numpy as np
import pytest
import torch

from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,E,top,dtype", [(1 << 22, 4, 1, torch.float32), (1 << 21, 16, 2, torch.bfloat16), (1 << 17, 1000, 1, torch.bfloat16),
                                           (300 * 64 + 5, 5, 2, torch.float32)])
@pytest.mark.parametrize("padding", [0, 3])
def test_many_rows_without_a_workspace(M, E, top, dtype, padding):
    """All rows alike, so that every rounding of a sum goes the same way; every fourth one is padding, or none is."""
    print(f"[gpu-case] {M} rows of {E}", flush=True)
    row = torch.log(torch.arange(1, E + 1, dtype=torch.float64)).to(dtype)
    logits = row.cuda()[None].expand(M, E).contiguous()
    valid = (torch.arange(M, device="cuda") % 4 != padding).to(torch.uint8) if padding else None
    n = int(valid.sum()) if padding else M
    i64 = dict(dtype=torch.int64, device="cuda")
    ids, place, rows, offsets = (torch.empty(s, **i64) for s in ((M, top), (M, top), (M * top,), (E + 1,)))
    gates, balance = torch.empty((M, top), device="cuda"), torch.empty(2 + E, device="cuda")
    code = B.DTYPE_F32 if dtype == torch.float32 else B.DTYPE_BF16
    p = torch.softmax(row.double(), 0).numpy()
    best = np.argsort(-row.double().numpy(), kind="stable")[:top]
    share = np.zeros(E)
    share[best] = 1.0 / top
    u = 2.0 ** -24
    ws = torch.empty(B.gemm_route_workspace_bytes(M, E), dtype=torch.uint8, device="cuda")
    for workspace in (None, ws):
        B.gemm_route(code, M, E, top, logits, E, valid, 0, ids, gates, offsets, rows, place, balance, workspace=workspace)
        got = balance.double().cpu().numpy()
        assert got[1] == n
        # p: exp, its sum over E and a quotient; a lane's sum of 256 of them in 32 bits, sums of those in 64; then of at most 64 lanes of a wave,
        # 8 waves, 16 and 32 workgroups, and the quotient by n
        off = (E + 40 + 256 + 6 + 8 + 48 + 2) * u
        assert np.allclose(got[2:], p, rtol=off, atol=0), np.abs(got[2:] / p - 1).max()
        assert np.isclose(got[0], E * (share * p).sum(), rtol=off + (E + 10) * u, atol=0)
        want = np.zeros(E + 1, np.int64)
        want[1:] = np.cumsum(np.isin(np.arange(E), best) * n)
        assert np.array_equal(offsets.cpu().numpy(), want)
