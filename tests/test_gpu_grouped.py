"""Grouped products, their weight gradient and adapters against plain products in 64 bits.

Every element is held to a bound that follows from the arithmetic: one rounding to the result's type, at most half a
step (`eps / 2` relative), and fp32 sums of n terms in any order, at most n 2^-24 of the sum of the terms' absolute values
(the matrix instruction rounds no product).  A second product's 16-bit operand adds half a step of its own, times what it is
multiplied with."""
import sys

import pytest
import torch

from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": (torch.bfloat16, B.DTYPE_BF16), "f16": (torch.float16, B.DTYPE_F16), "f32": (torch.float32, B.DTYPE_F32)}
U = 2.0 ** -24
SENTINEL = -77.0                       # exact in every type


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)
    sys.stdout.flush()


def half_step(dtype):
    """Largest relative error of one rounding, and the largest absolute one among the type's subnormals."""
    f = torch.finfo(dtype)
    return f.eps / 2, f.smallest_normal * f.eps / 2


def matrix(gen, rows, cols, dtype, pad=0, sigma=1.0, lead=0, fill=float("nan")):
    """rows x cols with `pad` more elements a row, `lead` elements into its allocation, all others `fill`."""
    ld = cols + pad
    buf = torch.full((lead + rows * ld + 16,), fill, dtype=dtype)
    view = buf[lead:lead + rows * ld].view(rows, ld)
    view[:, :cols] = (torch.randn((rows, cols), generator=gen) * sigma).to(dtype)
    dev = buf.cuda()
    return dev[lead:lead + rows * ld].view(rows, ld), ld


def stack(gen, n, rows, cols, dtype, pad=0, gap=0, sigma=1.0, fill=float("nan")):
    """n matrices, `gap` elements between them: (device tensor n x stride, ld, stride, the matrices on the host)."""
    ld = cols + pad
    stride = rows * ld + gap
    buf = torch.full((max(n, 1), stride), fill, dtype=dtype)
    for i in range(n):
        buf[i, :rows * ld].view(rows, ld)[:, :cols] = (torch.randn((rows, cols), generator=gen) * sigma).to(dtype)
    return buf.cuda(), ld, stride, [buf[i, :rows * ld].view(rows, ld)[:, :cols].double() for i in range(n)]


def bounds(sizes, lead=0):
    out = [lead]
    for m in sizes:
        out.append(out[-1] + m)
    return out


def on_device(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


def force(variant, form=""):
    """Force a kernel by its name and its form's; None: the plan's choice."""
    if variant is None:
        B.gemm_force_variant(-1, 0)
        return
    B.gemm_force_variant(B.variants().index(variant), 0)
    if form:
        B.gemm_force_form(next(f for f in range(8) if B.gemm_form_name(f) == form))


def check(got, ref, absolute, terms, dtype, what, more=None):
    """got (device) against ref and the sum of absolute values of its `terms` terms (64 bits)."""
    got = got.double().cpu()
    rel, tiny = half_step(dtype)
    err = (terms + 4) * U * absolute + (0 if more is None else more)
    bound = err + rel * (ref.abs() + err) + tiny
    over = (got - ref).abs() - bound
    bad = ~(over <= 0)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, the first at {bad.nonzero()[0].tolist()}: "
                           f"{got[bad][0]} for {ref[bad][0]}, bound {bound[bad][0]}")


def act(y, relu):
    return y.clamp_min(0.0) if relu else y


# ------------------------------------------------------------------ grouped products

def run_grouped(dtype, tB, sizes, N, K, *, lead=0, behind=0, beta=0.0, c32=False, bias=False, relu=False, pads=(0, 0, 0),
                gap=0, a_lead=0, seed=1, variant=None, form="", workspace=None):
    say(f"grouped {dtype} tB={tB} sizes={sizes} {N}x{K} beta={beta} c32={c32} bias={bias} relu={relu} pads={pads} "
        f"gap={gap} a_lead={a_lead} {variant} {form}")
    t, code = DT[dtype]
    out_t = torch.float32 if c32 or dtype == "f32" else t
    gen = torch.Generator().manual_seed(seed)
    at = bounds(sizes, lead)
    M, G = at[-1] + behind, len(sizes)
    A, lda = matrix(gen, M, K, t, pads[0], lead=a_lead)
    Bm, ldb, sB, Bs = stack(gen, G, *((N, K) if tB else (K, N)), t, pads[1], gap, sigma=0.5)
    C, ldc = matrix(gen, M, N, out_t, pads[2], fill=SENTINEL)
    if beta == 0.0:
        C[:, :N] = float("nan")                                 # never read
    before = C.clone()
    bs = torch.randn((G, N + 3), generator=gen)
    epi = (B.EPI_BIAS if bias else 0) | (B.EPI_RELU if relu else 0)
    force(variant, form)
    try:
        B.gemm_grouped(code, tB, M, N, K, G, on_device(at), A, lda, Bm, ldb, sB, beta, C, ldc, out_t == torch.float32,
                       bs.cuda() if bias else None, N + 3, epi, workspace=workspace)
        torch.cuda.synchronize()
        ran = B.variants()[B.gemm_last_variant()], B.gemm_form_name(B.gemm_last_form())
    finally:
        force(None)
    Ah, C0 = A[:, :K].double().cpu(), before[:, :N].double().cpu()
    for e in range(G):
        r = slice(at[e], at[e + 1])
        w = Bs[e].t() if tB else Bs[e]
        ref, ab = Ah[r] @ w, Ah[r].abs() @ w.abs()
        if beta:
            ref, ab = ref + beta * C0[r], ab + abs(beta) * C0[r].abs()
        if bias:
            ref, ab = ref + bs[e, :N].double(), ab + bs[e, :N].double().abs()
        check(C[r, :N], act(ref, relu), ab, K, out_t, f"group {e}")
    # rows of no group and the padding of the others are as they were
    for r in (slice(0, at[0]), slice(at[-1], M)):
        assert torch.equal(C[r].view(torch.uint8), before[r].view(torch.uint8))
    assert (C[:, N:] == SENTINEL).all()
    return ran


ODD_SIZES = [0, 1, 63, 0, 64, 65, 7, 130, 0]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tB", [0, 1])
def test_grouped_types_and_layouts(dtype, tB):
    run_grouped(dtype, tB, ODD_SIZES, 200, 136)
    run_grouped(dtype, tB, ODD_SIZES, 203, 137, bias=True, relu=True)
    run_grouped(dtype, tB, ODD_SIZES, 96, 64, beta=0.5, c32=True, lead=3, behind=5)
    run_grouped(dtype, tB, [5, 300, 2], 130, 70, pads=(3, 5, 2), gap=7, lead=2, behind=9, a_lead=1, bias=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 2), (1, 65), (5, 7), (64, 1), (33, 9), (8, 8), (2, 200)])
def test_grouped_runs_shorter_than_a_chunk(dtype, tB, N, K):
    run_grouped(dtype, tB, [2, 0, 1, 70], N, K, bias=True)


PINGPONG, STREAM128 = ("bf16_pingpong_256x256x64", ""), ("bf16_stream_128x128x64", "")
STREAM_MID, STREAM64 = ("bf16_stream_64x128x64", "128x64"), ("bf16_stream_32x128x64", "64x64")
GENERIC = "generic_64x64x16_f32mfma"
TUNED = [PINGPONG, STREAM128, STREAM_MID, STREAM64]
DIVIDED = [(GENERIC, "128x128"), (GENERIC, "128x64"), (GENERIC, "64x64")]


@pytest.mark.parametrize("kernel", TUNED + DIVIDED, ids=lambda k: " ".join(k).strip())
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tB", [0, 1])
def test_grouped_kernels(kernel, dtype, tB):
    """Every kernel a plan may take, at tiles that end inside a group, a row, a column and a block of the reduction."""
    sizes = [0, 1, 63, 0, 257, 300, 64, 7, 130, 0]
    for N, K in ((264, 256), (520, 328), (256, 264), (8, 320)):
        assert run_grouped(dtype, tB, sizes, N, K, variant=kernel[0], form=kernel[1], bias=N == 264, relu=K == 328, lead=1, behind=2) == kernel
    run_grouped(dtype, tB, sizes, 264, 456, variant=kernel[0], form=kernel[1], beta=0.5, c32=True, pads=(8, 8, 3), gap=8)
    run_grouped(dtype, tB, sizes, 264, 256, variant=kernel[0], form=kernel[1], beta=-1.0, pads=(8, 8, 4), gap=8, bias=True)
    run_grouped(dtype, tB, [512, 256], 512, 512, variant=kernel[0], form=kernel[1])
    run_grouped(dtype, tB, [i % 3 for i in range(140)], 72, 256, variant=kernel[0], form=kernel[1])
    if kernel in TUNED:
        for K in (8, 64, 72, 128):                              # one block, part of one, two
            run_grouped(dtype, tB, sizes, 136, K, variant=kernel[0], form=kernel[1])


@pytest.mark.parametrize("form", ["128x128", "128x64", "64x64"])
@pytest.mark.parametrize("tB", [0, 1])
def test_grouped_divided_tiles_at_any_alignment(form, tB):
    for dtype, K in (("bf16", 257), ("f16", 199), ("f32", 129), ("f32", 128)):
        run_grouped(dtype, tB, [0, 1, 63, 257, 130, 7], 203, K, variant=GENERIC, form=form, pads=(1, 3, 1), gap=1, a_lead=1, bias=True)


def test_forced_kernels_that_cannot_run_are_refused():
    off, x = on_device([0, 8, 16]), torch.zeros(1 << 16, device="cuda")

    def call(variant, form="", K=256, dt=B.DTYPE_BF16, lda=256):
        force(variant, form)
        try:
            return B.gemm_grouped(dt, 1, 16, 64, K, 2, off, x, lda, x, 256, 0, 0.0, x, 64, 1, check=False)
        finally:
            force(None)
    assert call(*PINGPONG, dt=B.DTYPE_F32) == call(*STREAM128, lda=257) == call("bf16_128x128x64") == B.INVALID_ARG
    assert call(*STREAM64, K=7) == call("bf16_stream_32x128x64") == call(GENERIC, "32x32") == call(GENERIC, "64x64", K=64) == B.INVALID_ARG


def test_grouped_single_rows_and_many_groups():
    run_grouped("bf16", 1, [1], 64, 64)
    run_grouped("bf16", 1, [0, 0, 1, 0], 40, 72)
    run_grouped("bf16", 1, [i % 3 for i in range(150)], 72, 64, lead=1)
    run_grouped("bf16", 0, [1] * 64, 72, 64)
    run_grouped("f16", 1, [2] * 65, 72, 64, behind=1)
    run_grouped("bf16", 1, [0] * 200 + [5] + [0] * 60, 72, 64)


def test_grouped_empty_reduction_and_no_rows():
    run_grouped("bf16", 1, [3, 0, 70], 40, 0, bias=True, relu=True)
    run_grouped("bf16", 1, [3, 0, 70], 40, 0, beta=0.5)
    run_grouped("bf16", 1, [0, 0], 40, 64, behind=4)


@pytest.mark.parametrize("bad", [[5, 3, 9, 12], [-4, 2, 2, 50], [0, 100, 4, 12], [1 << 40, -(1 << 40), 3, 4], [12, 9, 5, 0]])
def test_offsets_out_of_order_or_range_stay_inside(bad):
    """The kernels move bounds into 0 .. M and take a group that ends before it starts as empty: every row that is written
    then has the product with the weights of a group that holds it, and no other is touched."""
    M, N, K, G = 12, 40, 64, 3
    say(f"bad offsets {bad}")
    gen = torch.Generator().manual_seed(9)
    A, lda = matrix(gen, M, K, torch.bfloat16)
    Bm, ldb, sB, Bs = stack(gen, G, N, K, torch.bfloat16)
    C = torch.full((M, N), SENTINEL, device="cuda")
    B.gemm_grouped(B.DTYPE_BF16, 1, M, N, K, G, on_device(bad), A, lda, Bm, ldb, sB, 0.0, C, N, 1)
    torch.cuda.synchronize()
    Ah, got = A[:, :K].double().cpu(), C.double().cpu()
    for m in range(M):
        holds = [e for e in range(G) if max(0, bad[e]) <= m < min(M, bad[e + 1])]
        refs = [Ah[m] @ Bs[e].t() for e in holds]
        untouched = bool((got[m] == SENTINEL).all())
        assert untouched or any(torch.allclose(got[m], r, rtol=0, atol=K * U * 64) for r in refs), m
        assert untouched or holds


def test_grouped_shared_weights():
    """A stride of 0: all groups take the same weights."""
    gen = torch.Generator().manual_seed(3)
    A, lda = matrix(gen, 50, 64, torch.bfloat16)
    W, ldw = matrix(gen, 48, 64, torch.bfloat16)
    C = torch.empty((50, 48), device="cuda")
    B.gemm_grouped(B.DTYPE_BF16, 1, 50, 48, 64, 3, on_device([0, 10, 11, 50]), A, lda, W, ldw, 0, 0.0, C, 48, 1)
    a, w = A.double().cpu(), W.double().cpu()
    check(C, a @ w.t(), a.abs() @ w.abs().t(), 64, torch.float32, "shared weights")


def test_a_row_of_nan_stays_its_own():
    """NaN and infinities in a row reach that row's results alone, also where the row is its group's last of a tile."""
    gen = torch.Generator().manual_seed(4)
    A, lda = matrix(gen, 140, 64, torch.bfloat16)
    A[69] = float("nan")
    A[70] = float("inf")
    Bm, ldb, sB, _ = stack(gen, 2, 72, 64, torch.bfloat16)
    C = torch.empty((140, 72), device="cuda", dtype=torch.bfloat16)
    B.gemm_grouped(B.DTYPE_BF16, 1, 140, 72, 64, 2, on_device([0, 70, 140]), A, lda, Bm, ldb, sB, 0.0, C, 72, 0)
    finite = torch.isfinite(C.float()).all(1)
    assert not finite[69] and not finite[70] and finite.sum() == 138 and torch.isnan(C[69].float()).all()


# ------------------------------------------------------------------ weight gradients

def run_wgrad(dtype, sizes, N, K, *, lead=0, behind=0, beta=0.0, c32=False, pads=(0, 0, 0), gap=0, y_lead=0, seed=2,
              variant=None, form=""):
    say(f"wgrad {dtype} sizes={sizes} {N}x{K} beta={beta} c32={c32} pads={pads} gap={gap} y_lead={y_lead} {variant} {form}")
    t, code = DT[dtype]
    out_t = torch.float32 if c32 or dtype == "f32" else t
    gen = torch.Generator().manual_seed(seed)
    at = bounds(sizes, lead)
    M, G = at[-1] + behind, len(sizes)
    dY, ldy = matrix(gen, M, N, t, pads[0], lead=y_lead)
    X, ldx = matrix(gen, M, K, t, pads[1])
    dY[:at[0]], dY[at[-1]:] = float("nan"), float("nan")        # rows of no group are not read into any
    dW, ldw, sW, W0 = stack(gen, G, N, K, out_t, pads[2], gap, fill=SENTINEL)
    if beta == 0.0:
        for e in range(G):
            dW[e, :N * ldw].view(N, ldw)[:, :K] = float("nan")
    before = dW.clone()
    force(variant, form)
    try:
        B.gemm_grouped_wgrad(code, M, N, K, G, on_device(at), dY, ldy, X, ldx, beta, dW, ldw, sW, out_t == torch.float32)
        torch.cuda.synchronize()
        ran = B.variants()[B.gemm_last_variant()], B.gemm_form_name(B.gemm_last_form())
    finally:
        force(None)
    y, x = dY[:, :N].double().cpu(), X[:, :K].double().cpu()
    for e in range(G):
        r = slice(at[e], at[e + 1])
        ref, ab = y[r].t() @ x[r], y[r].abs().t() @ x[r].abs()
        if beta:
            ref, ab = ref + beta * W0[e], ab + abs(beta) * W0[e].abs()
        check(dW[e, :N * ldw].view(N, ldw)[:, :K], ref, ab, sizes[e], out_t, f"group {e}")
        assert (dW[e, :N * ldw].view(N, ldw)[:, K:] == SENTINEL).all() and torch.equal(dW[e, N * ldw:], before[e, N * ldw:])
    return ran


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_wgrad_types(dtype):
    run_wgrad(dtype, ODD_SIZES, 136, 200)
    run_wgrad(dtype, ODD_SIZES, 137, 203, lead=3, behind=2)
    run_wgrad(dtype, [1, 300, 0, 129], 96, 64, beta=0.5, c32=True)
    run_wgrad(dtype, [1, 300, 0, 129], 70, 130, pads=(3, 5, 2), gap=7, lead=2, behind=9, y_lead=1, c32=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 2), (1, 65), (65, 1), (5, 70), (16, 200), (200, 16), (8, 8)])
def test_wgrad_narrow(dtype, N, K):
    run_wgrad(dtype, [0, 1, 2, 70, 200], N, K, c32=True)


SHORT = ("bf16_128x128x64", "")


@pytest.mark.parametrize("kernel", TUNED + [SHORT, (GENERIC, "64x64")], ids=lambda k: " ".join(k).strip())
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_wgrad_kernels(kernel, dtype):
    sizes = [0, 1, 63, 64, 65, 128, 0, 200, 7, 321]
    for N, K in ((264, 328), (8, 520), (256, 8), (136, 72)):
        assert run_wgrad(dtype, sizes, N, K, variant=kernel[0], form=kernel[1], lead=1, behind=3) == kernel
    run_wgrad(dtype, sizes, 264, 136, variant=kernel[0], form=kernel[1], beta=0.5, c32=True, pads=(8, 8, 3), gap=4)
    run_wgrad(dtype, sizes, 264, 136, variant=kernel[0], form=kernel[1], beta=1.0, c32=True)
    run_wgrad(dtype, sizes, 136, 264, variant=kernel[0], form=kernel[1], beta=-1.0, pads=(8, 8, 4), gap=4)
    run_wgrad(dtype, [256, 512], 256, 512, variant=kernel[0], form=kernel[1])


def test_wgrad_divided_tiles_at_any_alignment():
    for dtype in ("bf16", "f16", "f32"):
        run_wgrad(dtype, [0, 1, 63, 64, 65, 200, 31, 33], 203, 137, variant=GENERIC, form="64x64", pads=(1, 3, 1), gap=1, y_lead=1, c32=True)


def test_wgrad_no_rows_and_many_groups():
    run_wgrad("bf16", [0, 0, 0], 40, 64)
    run_wgrad("bf16", [0, 0, 0], 40, 64, beta=0.5, c32=True)
    run_wgrad("bf16", [0, 0, 0], 40, 64, beta=1.0)
    run_wgrad("bf16", [i % 5 for i in range(150)], 24, 40)


def test_wgrad_is_the_gradient():
    """d/dW of sum(G * grouped(X, W)) is wgrad(G, X): against the change of that sum when W moves along a direction (the
    sum is linear in W, so the difference is exact but for rounding)."""
    gen = torch.Generator().manual_seed(12)
    sizes, N, K = [5, 0, 90, 33], 48, 72
    at, G = bounds(sizes), 4
    X, _ = matrix(gen, at[-1], K, torch.float32)
    dY, _ = matrix(gen, at[-1], N, torch.float32)
    W, _, sW, _ = stack(gen, G, N, K, torch.float32)
    D, _, _, _ = stack(gen, G, N, K, torch.float32)
    off, Y = on_device(at), [torch.empty((at[-1], N), device="cuda") for _ in range(2)]
    for y, w in zip(Y, (W + D, W - D)):
        B.gemm_grouped(B.DTYPE_F32, 1, at[-1], N, K, G, off, X, K, w, K, sW, 0.0, y, N, 1)
    dW = torch.empty_like(W)
    B.gemm_grouped_wgrad(B.DTYPE_F32, at[-1], N, K, G, off, dY, N, X, K, 0.0, dW, K, sW, 1)
    dX = torch.empty_like(X)
    B.gemm_grouped(B.DTYPE_F32, 0, at[-1], K, N, G, off, dY, N, W, K, sW, 0.0, dX, K, 1)
    diff = ((Y[0].double() - Y[1].double()) / 2 * dY.double()).sum()
    along = (dW.double() * D.double()).sum()
    # both sums have 128 * 48 * 72 products of three normal numbers; their fp32 errors stay below 1e-5 of the sum's size
    size = (dY.double().abs().sum() * K) ** 0.5 * 10
    assert abs(diff - along) <= 1e-4 * size, (diff, along)
    # and along a direction of X
    DX, _ = matrix(gen, at[-1], K, torch.float32)
    for y, x in zip(Y, (X + DX, X - DX)):
        B.gemm_grouped(B.DTYPE_F32, 1, at[-1], N, K, G, off, x, K, W, K, sW, 0.0, y, N, 1)
    diff = ((Y[0].double() - Y[1].double()) / 2 * dY.double()).sum()
    along = (dX.double() * DX.double()).sum()
    assert abs(diff - along) <= 1e-4 * size, (diff, along)


# ------------------------------------------------------------------ adapters

def run_adapters(dtype, tB, sizes, ids, bank, R, N, K, *, lead=0, behind=0, beta=0.0, c32=False, bias=False, relu=False,
                 scale=True, pads=(0,) * 6, gap=0, x_lead=0, h_lead=0, seed=3, per_row=False, workspace=None, variant=None, form=""):
    say(f"adapters {dtype} tB={tB} sizes={sizes} ids={ids} bank={bank} R={R} {N}x{K} beta={beta} c32={c32} bias={bias} relu={relu} "
        f"scale={scale} pads={pads} gap={gap} lead={lead} behind={behind} per_row={per_row} ws={workspace is not None} {variant} {form}")
    t, code = DT[dtype]
    out_t = torch.float32 if c32 or dtype == "f32" else t
    gen = torch.Generator().manual_seed(seed)
    at = bounds(sizes, lead)
    M, S = at[-1] + behind, len(sizes)
    X, ldx = matrix(gen, M, K, t, pads[0], lead=x_lead)
    W, ldw = matrix(gen, *((N, K) if tB else (K, N)), t, pads[1], sigma=0.5)
    down, ldd, sd, downs = stack(gen, bank, *((R, K) if tB else (K, R)), t, pads[2], gap, sigma=0.5)
    up, ldu, su, ups = stack(gen, bank, *((N, R) if tB else (R, N)), t, pads[3], gap, sigma=0.5)
    Y, ldy = matrix(gen, M, N, out_t, pads[4], fill=SENTINEL)
    if beta == 0.0:
        Y[:, :N] = float("nan")
    Y0 = Y[:, :N].double().cpu()
    H, ldh = matrix(gen, M, R, t, pads[5], lead=h_lead, fill=SENTINEL)
    H[:, :R] = float("nan")
    sc = torch.rand(max(bank, 1), generator=gen) + 0.5
    bs = torch.randn(N, generator=gen)
    epi = (B.EPI_BIAS if bias else 0) | (B.EPI_RELU if relu else 0)
    force(variant, form)
    try:
        B.gemm_adapters(code, tB, M, N, K, R, S, None if per_row else on_device(at), None if ids is None else on_device(ids), bank,
                        X, ldx, W, ldw, down if bank else None, ldd, sd, up if bank else None, ldu, su, sc.cuda() if scale else None,
                        beta, Y, ldy, out_t == torch.float32, bs.cuda() if bias else None, epi, H, ldh, workspace=workspace)
        torch.cuda.synchronize()
        ran = B.variants()[B.gemm_last_variant()], B.gemm_form_name(B.gemm_last_form())
    finally:
        force(None)
    x, w = X[:, :K].double().cpu(), W[:, :W.shape[1] - pads[1]].double().cpu()
    w = w.t() if tB else w
    h, h_ab = torch.zeros((M, R), dtype=torch.float64), torch.zeros((M, R), dtype=torch.float64)
    ref, ab, more = x @ w, x.abs() @ w.abs(), torch.zeros((M, N), dtype=torch.float64)
    rel, tiny = half_step(t)
    for s in range(S):
        a = s if ids is None else ids[s]
        r = slice(at[s], at[s + 1])
        if not 0 <= a < bank:
            continue
        d, u, f = (downs[a].t() if tB else downs[a]), (ups[a].t() if tB else ups[a]), (sc[a].double() if scale else 1.0)
        h[r], h_ab[r] = f * (x[r] @ d), f * (x[r].abs() @ d.abs())
        ref[r] += h[r] @ u
        ab[r] += h[r].abs() @ u.abs()
        h_off = (K + 6) * U * h_ab[r] + (rel * h[r].abs() * (1 + K * U) + tiny if t != torch.float32 else 0)
        more[r] += 1.01 * h_off @ u.abs()
    if beta:
        ref, ab = ref + beta * Y0, ab + abs(beta) * Y0.abs()
    if bias:
        ref, ab = ref + bs.double(), ab + bs.double().abs()
    check(H[:, :R], h, h_ab, K + 2, t, "H")
    check(Y[:, :N], act(ref, relu), ab, K + R, out_t, "Y", more)
    assert (Y[:, N:] == SENTINEL).all() and (H[:, R:] == SENTINEL).all()
    return ran


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tB", [0, 1])
def test_adapters_types_and_layouts(dtype, tB):
    ids = [2, 0, -1, 1, 2, 3, 0, 1, 7]
    run_adapters(dtype, tB, ODD_SIZES, ids, 4, 16, 200, 136)
    run_adapters(dtype, tB, ODD_SIZES, ids, 4, 13, 203, 137, bias=True, relu=True)
    run_adapters(dtype, tB, ODD_SIZES, ids, 4, 64, 96, 64, beta=0.5, c32=True, lead=3, behind=5, scale=False)
    run_adapters(dtype, tB, [5, 300, 2], [1, 0, -5], 2, 70, 130, 72, pads=(3, 5, 2, 1, 2, 3), gap=7, lead=2, behind=9, x_lead=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("R,N,K", [(1, 1, 1), (2, 5, 3), (1, 64, 64), (9, 8, 200), (4, 200, 65)])
def test_adapters_runs_shorter_than_a_chunk(dtype, tB, R, N, K):
    run_adapters(dtype, tB, [2, 0, 1, 70], [1, 0, 0, 1], 2, R, N, K)


@pytest.mark.parametrize("rows", [1, 2, 16, 33, 130])
def test_adapters_one_row_each(rows):
    """Decode: every row its own segment, without offsets."""
    ids = [(7 * i) % 5 - (1 if i % 4 == 3 else 0) for i in range(rows)]
    ids = [-1 if i % 4 == 3 else a for i, a in enumerate(ids)]
    for tB in (0, 1):
        run_adapters("bf16", tB, [1] * rows, ids, 5, 16, 264, 192, per_row=True)
    run_adapters("f16", 1, [1] * rows, ids, 5, 33, 72, 71, per_row=True, bias=True)


def workspace():
    return torch.empty(16 << 20, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("kernel", [PINGPONG, ("bf16_128x128x64", "")] + TUNED[1:], ids=lambda k: " ".join(k).strip())
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tB", [0, 1])
def test_adapters_as_blocks_of_a_tile(kernel, dtype, tB):
    """Every kernel a projection's plan may take, with segments that begin, end and lie inside its tiles, ranks of part of a
    block, one and more."""
    sizes, ids = [0, 1, 63, 0, 257, 300, 64, 7, 130, 0], [3, 1, 0, 2, 2, -1, 0, 3, 1, 0]
    for R, N, K in ((16, 264, 256), (8, 520, 328), (40, 256, 72), (64, 8, 320), (72, 136, 64), (200, 264, 136)):
        assert run_adapters(dtype, tB, sizes, ids, 4, R, N, K, variant=kernel[0], form=kernel[1], bias=N == 264, relu=K == 328,
                            lead=1, behind=2) == kernel
    run_adapters(dtype, tB, sizes, ids, 4, 13, 264, 456, variant=kernel[0], form=kernel[1], beta=0.5, c32=True,
                 pads=(8, 8, 3, 5, 3, 1), gap=5, h_lead=1, scale=False)
    run_adapters(dtype, tB, [i % 3 for i in range(140)], [i % 5 for i in range(140)], 4, 16, 72, 256, variant=kernel[0], form=kernel[1])
    run_adapters(dtype, tB, [1] * 70, [i % 5 for i in range(70)], 4, 16, 72, 256, per_row=True, variant=kernel[0], form=kernel[1])
    run_adapters(dtype, tB, [512, 256], None, 2, 64, 512, 512, variant=kernel[0], form=kernel[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tB", [0, 1])
def test_adapters_apart_from_the_projection(dtype, tB):
    """Short segments with a workspace: the projection's sums there, split or not, the adapters behind it."""
    ids = [(5 * i) % 6 - 1 for i in range(40)]
    for R, N, K in ((16, 264, 2048), (64, 72, 136), (13, 203, 137), (1, 7, 9), (100, 300, 8)):
        run_adapters(dtype, tB, [i % 4 for i in range(40)], ids, 5, R, N, K, workspace=workspace(), bias=R == 13, relu=R == 13, lead=2, behind=3)
    run_adapters(dtype, tB, [1, 40, 0, 17, 16], ids[:5], 5, 24, 260, 1024, workspace=workspace(), beta=0.5, c32=True, pads=(3, 5, 2, 1, 2, 3), gap=7)
    run_adapters(dtype, tB, [1] * 16, ids[:16], 5, 16, 4096, 2048, workspace=workspace(), per_row=True, beta=-1.0)
    run_adapters(dtype, tB, [1], [0], 5, 16, 1024, 4096, workspace=workspace(), per_row=True)


def test_adapters_none_at_all():
    run_adapters("bf16", 1, [], [], 3, 8, 40, 64, behind=20)                # no segment
    run_adapters("bf16", 1, [5, 5], [0, 1], 0, 8, 40, 64)                   # no adapter
    run_adapters("bf16", 1, [5, 0, 70], [-1, -1, 9], 3, 8, 40, 64, bias=True)
    run_adapters("bf16", 1, [5, 6], None, 2, 8, 40, 0, beta=0.5)            # nothing to add up
    run_adapters("bf16", 1, [5, 6, 1], None, 3, 16, 40, 64)                 # segment s takes adapter s


def test_adapters_of_rank_zero_is_the_projection():
    gen = torch.Generator().manual_seed(5)
    X, W = (matrix(gen, r, 64, torch.bfloat16)[0] for r in (20, 48))
    Y, Z = (torch.empty((20, 48), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    B.gemm_adapters(B.DTYPE_BF16, 1, 20, 48, 64, 0, 2, on_device([0, 4, 20]), None, 2, X, 64, W, 64, None, 0, 0, None, 0, 0, None,
                    0.0, Y, 48, 0, None, 0, None, 0)
    B.gemm_bf16(0, 1, 20, 48, 64, X, 64, W, 64, 0.0, Z, 48, 0)
    assert torch.equal(Y, Z)


def test_adapters_without_columns_still_give_h():
    gen = torch.Generator().manual_seed(6)
    X, down = matrix(gen, 9, 64, torch.bfloat16)[0], stack(gen, 2, 8, 64, torch.bfloat16)
    H = torch.empty((9, 8), device="cuda", dtype=torch.bfloat16)
    B.gemm_adapters(B.DTYPE_BF16, 1, 9, 0, 64, 8, 2, on_device([0, 4, 9]), None, 2, X, 64, X, 64, down[0], 64, 512, None, 8, 0, None,
                    0.0, H, 8, 0, None, 0, H, 8)
    x = X.double().cpu()
    ref = torch.cat([x[:4] @ down[3][0].t(), x[4:] @ down[3][1].t()])
    ab = torch.cat([x[:4].abs() @ down[3][0].abs().t(), x[4:].abs() @ down[3][1].abs().t()])
    check(H, ref, ab, 64, torch.bfloat16, "H")


def test_adapter_gradients_by_the_same_calls():
    """dX and G are the call turned over, the adapters' gradients grouped weight gradients: against autograd in 64 bits."""
    gen = torch.Generator().manual_seed(8)
    sizes, R, N, K = [30, 0, 65, 7], 8, 72, 104
    at, n = bounds(sizes), len(sizes)
    M = at[-1]
    X, dY = matrix(gen, M, K, torch.float32)[0], matrix(gen, M, N, torch.float32)[0]
    W = matrix(gen, N, K, torch.float32, sigma=0.3)[0]
    down, _, sd, _ = stack(gen, n, R, K, torch.float32, sigma=0.3)
    up, _, su, _ = stack(gen, n, N, R, torch.float32, sigma=0.3)
    sc = (torch.rand(n, generator=gen) + 0.5).cuda()
    off = on_device(at)
    Y, H = torch.empty((M, N), device="cuda"), torch.empty((M, R), device="cuda")
    B.gemm_adapters(B.DTYPE_F32, 1, M, N, K, R, n, off, None, n, X, K, W, K, down, K, sd, up, R, su, sc, 0.0, Y, N, 1, None, 0, H, R)
    dX, G = torch.empty_like(X), torch.empty_like(H)
    B.gemm_adapters(B.DTYPE_F32, 0, M, K, N, R, n, off, None, n, dY, N, W, K, up, R, su, down, K, sd, sc, 0.0, dX, K, 1, None, 0, G, R)
    d_down, d_up = torch.empty_like(down), torch.empty_like(up)
    B.gemm_grouped_wgrad(B.DTYPE_F32, M, R, K, n, off, G, R, X, K, 0.0, d_down, K, sd, 1)
    B.gemm_grouped_wgrad(B.DTYPE_F32, M, N, R, n, off, dY, N, H, R, 0.0, d_up, R, su, 1)
    x, w, a, b = (v.double().cpu().requires_grad_() for v in (X, W, down.view(n, R, K), up.view(n, N, R)))
    y = torch.cat([x[at[i]:at[i + 1]] @ w.t() + sc[i].double().cpu() * (x[at[i]:at[i + 1]] @ a[i].t()) @ b[i].t() for i in range(n)])
    (y * dY.double().cpu()).sum().backward()
    for got, want in ((Y, y.detach()), (dX, x.grad), (d_down.view(n, R, K), a.grad), (d_up.view(n, N, R), b.grad)):
        # sums of at most a few thousand products of size 1: fp32 errors below 1e-5 of the results' size
        assert (got.double().cpu() - want).abs().max() <= 2e-5 * want.abs().max()
