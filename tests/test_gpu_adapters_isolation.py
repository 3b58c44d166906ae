"""What one request's adapter or rows hold reaches no other request's: infinities and NaN in one adapter's weights and in one
row, with segments and rows without an adapter beside them in the same tiles.

Where the definition gives an infinity or NaN in 64 bits the call has to give the same, everywhere else a value under the bounds of
test_gpu_grouped.py.  The weights put beside an infinity are of one sign, so that no sum's sign hangs on a rounding."""
import pytest
import torch

from paper_2511_13764_amd import binding as B
from test_gpu_grouped import DT, PINGPONG, TUNED, U, bounds, check, force, half_step, matrix, on_device, say, stack

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
KERNELS = [PINGPONG, ("bf16_128x128x64", "")] + TUNED[1:]
SIZES = [0, 1, 63, 5, 257, 300, 64, 7, 130, 0]
IDS = [3, 1, 0, 1, 2, -1, 1, 3, 1, 0]


def same_values(got, ref, absolute, terms, dtype, what, more):
    got = got.double().cpu()
    odd = ~torch.isfinite(ref)
    assert torch.equal(got.isnan(), ref.isnan()), (what, (got.isnan() != ref.isnan()).nonzero()[:4].tolist())
    keep = odd & ~ref.isnan()
    assert torch.equal(got[keep], ref[keep]), what
    zero = torch.zeros_like(ref)
    check(torch.where(odd, zero, got), torch.where(odd, zero, ref), torch.where(odd, zero, absolute), terms, dtype, what,
          torch.where(odd, zero, more))


def run(dtype, tB, sizes, ids, R, N, K, *, variant=None, form="", workspace=None, per_row=False, lead=0, behind=0, beta=0.0,
        bad_row=None):
    say(f"isolation {dtype} tB={tB} sizes={sizes} ids={ids} R={R} {N}x{K} {variant} {form} ws={workspace is not None} {per_row} {bad_row}")
    t, code = DT[dtype]
    gen = torch.Generator().manual_seed(R + N)
    at, bank = bounds(sizes, lead), 4
    M = at[-1] + behind
    X, _ = matrix(gen, M, K, t)
    X.abs_()                                                    # (with the first weights: H[:, 0] > 0)
    W, ldw = matrix(gen, *((N, K) if tB else (K, N)), t, sigma=0.5)
    down, ldd, sd, _ = stack(gen, bank, *((R, K) if tB else (K, R)), t, sigma=0.5)
    up, ldu, su, _ = stack(gen, bank, *((N, R) if tB else (R, N)), t, sigma=0.5)
    d = [down[a].view(R, K) if tB else down[a].view(K, R).t() for a in range(bank)]        # R x K
    u = [up[a].view(N, R) if tB else up[a].view(R, N).t() for a in range(bank)]            # N x R
    for a in range(bank):
        d[a][0] = d[a][0].abs()
    # adapter 1: infinities and NaN, in different columns; adapter 3: a column of down that makes a rank's sums NaN
    u[1][0, 0], u[1][N // 2, 0], u[1][N - 1, R - 1], u[1][N // 3, R // 2] = INF, -INF, NAN, NAN
    d[3][R - 1, K - 1] = NAN
    if bad_row is not None:
        X[bad_row, K // 2] = NAN
    Y, _ = matrix(gen, M, N, t)
    Y0 = Y.double().cpu()
    H = torch.full((M, R), NAN, dtype=t, device="cuda")
    sc = torch.rand(bank, generator=gen) + 0.5
    force(variant, form)
    try:
        B.gemm_adapters(code, tB, M, N, K, R, len(sizes), None if per_row else on_device(at), on_device(ids), bank, X, K, W, ldw, down,
                        ldd, sd, up, ldu, su, sc.cuda(), beta, Y, N, dtype == "f32", None, 0, H, R, workspace=workspace)
        torch.cuda.synchronize()
    finally:
        force(None)
    x, w = X.double().cpu(), W.double().cpu()
    w = w.t() if tB else w
    ref, ab, more = x @ w, x.abs() @ w.abs(), torch.zeros((M, N), dtype=torch.float64)
    h, h_ab = torch.zeros((M, R), dtype=torch.float64), torch.zeros((M, R), dtype=torch.float64)
    rel, tiny = half_step(t)
    for s, a in enumerate(ids):
        r = slice(at[s], at[s + 1])
        if at[s] == at[s + 1] or not 0 <= a < bank:
            continue
        f, da, ua = sc[a].double(), d[a].double().cpu(), u[a].double().cpu()
        h[r], h_ab[r] = f * (x[r] @ da.t()), f * (x[r].abs() @ da.abs().t())
        ref[r] += h[r] @ ua.t()
        ab[r] += h[r].abs() @ ua.abs().t()
        off = (K + 6) * U * h_ab[r] + (rel * h[r].abs() * (1 + K * U) + tiny if dtype != "f32" else 0)
        more[r] += 1.01 * off @ ua.abs().t()
    if beta:
        ref, ab = ref + beta * Y0, ab + abs(beta) * Y0.abs()
    none = torch.zeros_like(h)
    same_values(H, h, h_ab, K + 2, t, "H", none)
    same_values(Y, ref, ab, K + R, t, "Y", more)


def workspace():
    return torch.empty(16 << 20, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: " ".join(k).strip())
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tB", [0, 1])
def test_as_blocks_of_a_tile(kernel, dtype, tB):
    for R, N, K in ((16, 264, 256), (8, 520, 328), (72, 136, 64), (40, 256, 72)):
        run(dtype, tB, SIZES, IDS, R, N, K, variant=kernel[0], form=kernel[1], lead=1, behind=2)
    run(dtype, tB, SIZES, IDS, 200, 264, 136, variant=kernel[0], form=kernel[1], beta=0.5, bad_row=70)
    run(dtype, tB, [i % 3 for i in range(140)], [i % 5 - 1 for i in range(140)], 16, 72, 256, variant=kernel[0], form=kernel[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tB", [0, 1])
def test_as_the_plan_has_it(dtype, tB):
    """Without a workspace and with one; short segments, long ones and a row each."""
    for ws in (None, workspace()):
        for R, N, K in ((16, 264, 256), (13, 203, 137), (64, 1032, 512)):
            run(dtype, tB, SIZES, IDS, R, N, K, workspace=ws, lead=3, behind=5)
            run(dtype, tB, [i % 4 for i in range(40)], [i % 5 - 1 for i in range(40)], R, N, K, workspace=ws, bad_row=11)
            run(dtype, tB, [1] * 16, [i % 5 - 1 for i in range(16)], R, N, K, workspace=ws, per_row=True, bad_row=3)
        run(dtype, tB, [1] * 64, [i % 5 - 1 for i in range(64)], 520, 1000, 1064, workspace=ws, per_row=True)


@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("M,bank,R", [(16, 1, 700), (64, 8, 512), (256, 40, 144), (33, 0, 520)])
def test_no_segment_has_no_id(M, bank, R, tB):
    """segments == 0 without offsets: no row has an adapter, and `ids`, which holds none, is not read, also at sizes whose rows
    would otherwise be taken by their adapter."""
    gen = torch.Generator().manual_seed(M)
    N, K = 1000, 1064
    t = torch.bfloat16
    X, W = matrix(gen, M, K, t)[0], matrix(gen, *((N, K) if tB else (K, N)), t)[0]
    down, up = (torch.full((max(bank, 1), R * n), NAN, dtype=t, device="cuda") for n in (K, N))
    for ws in (None, workspace()):
        Y, H = (torch.full((M, n), NAN, dtype=t, device="cuda") for n in (N, R))
        # (one id would be the first adapter; M more lie behind it)
        ids = torch.zeros(M + 1, dtype=torch.int64, device="cuda")
        B.gemm_adapters(B.DTYPE_BF16, tB, M, N, K, R, 0, None, ids, bank, X, K, W, K if tB else N, down, K if tB else R, R * K, up,
                        R if tB else N, R * N, None, 0.0, Y, N, 0, None, 0, H, R, workspace=ws)
        assert not H.any()
        x, w = X.double().cpu(), W.double().cpu()
        w = w.t() if tB else w
        check(Y, x @ w, x.abs() @ w.abs(), K, t, "Y")
