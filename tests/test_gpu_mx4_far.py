"""4-bit images, their products and the router where places pass 32 bits: rows far apart, and images of more than 2^32 bytes; and what
is no number in every tile."""
import numpy as np
import pytest
import torch

import mx4_reference as mx
import route_reference as rr
from paper_2511_13764_amd import binding as B
from test_gpu_mx4 import PINGPONG, TILES, check, force_tile, left_of, weights_of

pytestmark = pytest.mark.gpu
DT = {"f32": (torch.float32, B.DTYPE_F32), "bf16": (torch.bfloat16, B.DTYPE_BF16), "f16": (torch.float16, B.DTYPE_F16)}


def far(t, ld):
    """The same rows, `ld` elements apart; between them whatever the memory holds."""
    out = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda")
    view = out.as_strided(t.shape, (ld, 1))
    view.copy_(t)
    return out, view


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("ld,force", [((1 << 23) + 8, None), ((1 << 23) - 8, TILES[0]), ((1 << 23) - 8, PINGPONG), ((1 << 28) + 8, None)])
def test_rows_far_apart(kind, ld, force):
    M, N, K = 20, 70, 320
    print(f"[gpu-case] rows {ld} apart, {force}", flush=True)
    rng = np.random.default_rng(ld)
    a, A, _ = left_of(kind, rng, M, K)
    w, W = weights_of(rng, N, K)
    A, _ = far(A, ld)
    C, rows = far(torch.zeros((M, N), dtype=DT[kind][0]), (1 << 27) + 3)
    if force:
        force_tile(force)
    try:
        B.gemm_mx4(DT[kind][1], M, N, K, A, ld, W, 0.0, C, (1 << 27) + 3, 0)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    check(rows.double().cpu().numpy(), a @ w.T, mx.most_off(a, w, False), DT[kind][0])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_rows_far_apart_are_copied(kind):
    M, N, K, ld = 20, 70, 320, (1 << 23) + 8
    rng = np.random.default_rng(ld)
    a, A, _ = left_of(kind, rng, M, K)
    w, W = weights_of(rng, N, K)
    A, _ = far(A, ld)
    C = torch.zeros((M, N), dtype=DT[kind][0], device="cuda")
    B.gemm_mx4(DT[kind][1], M, N, K, A, ld, W, 0.0, C, N, 0, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert B.variants()[B.gemm_last_variant()] != B.variants()[0]
    check(C.double().cpu().numpy(), a @ w.T, mx.most_off(a, w, False), DT[kind][0])


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("M", [3, 300])
def test_weights_of_more_than_4_gib(kind, M):
    """Zeros but for the last 70 rows."""
    N, K, some = 1100000, 8000, 70
    print(f"[gpu-case] {M} x {N} x {K} {kind}", flush=True)
    rng = np.random.default_rng(M)
    a, A, lda = left_of(kind, rng, M, K)
    w, small = weights_of(rng, some, K)
    W = torch.zeros(B.gemm_mx4_bytes(N, K), dtype=torch.uint8, device="cuda")
    row, blocks = mx.padded(K) // 2, mx.padded(K) // 256
    assert N * row > 1 << 32
    W[(N - some) * row:N * row] = small[:some * row]
    W[N * row:].view(blocks, N, 8)[:, N - some:] = small[some * row:].view(blocks, some, 8)
    half = torch.float16 if kind == "f16" else torch.bfloat16
    C = torch.full((M, N), -1.0, dtype=half, device="cuda")
    B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, W, 0.0, C, N, 0)
    check(C[:, N - some:].double().cpu().numpy(), a @ w.T, mx.most_off(a, w, kind == "mx4"), half)
    assert not bool(C[:, :N - some].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack_and_unpack_far(dtype):
    rows, K, ld = 20, 300, (1 << 28) + 1
    print(f"[gpu-case] pack, rows {ld} apart", flush=True)
    t = torch.randn((rows, K), generator=torch.Generator().manual_seed(1)).to(DT[dtype][0])
    X, view = far(t, ld)
    image = torch.empty(mx.nbytes(rows, K), dtype=torch.uint8, device="cuda")
    B.gemm_pack_mx4(DT[dtype][1], 0, rows, K, X, ld, rows, None, image)
    assert np.array_equal(image.cpu().numpy(), mx.image(t.double().numpy()))
    view.fill_(9.0)
    B.gemm_unpack_mx4(DT[dtype][1], rows, K, image, X, ld)
    assert np.array_equal(view.double().cpu().numpy(), mx.values(image.cpu().numpy(), rows, K))
    # stored turned over: 20 rows of 300 columns are 300 rows of a 20-column image
    view.copy_(t)
    turned = torch.empty(mx.nbytes(K, rows), dtype=torch.uint8, device="cuda")
    B.gemm_pack_mx4(DT[dtype][1], 1, K, rows, X, ld, K, None, turned)
    assert np.array_equal(turned.cpu().numpy(), mx.image(t.double().numpy().T))


@pytest.mark.parametrize("M", [20, 300])
def test_logits_far_apart(M):
    E, top, ld = 10, 2, (1 << 27) + 1 if M == 20 else (1 << 25) + 1
    print(f"[gpu-case] logits {ld} apart", flush=True)
    t = torch.randn((M, E), generator=torch.Generator().manual_seed(M)).bfloat16()
    X, _ = far(t, ld)
    want = rr.route(t.double().numpy(), top, None, True)
    o = dict(ids=torch.empty((M, top), dtype=torch.int64, device="cuda"), gates=torch.empty((M, top), device="cuda"),
             offsets=torch.empty(E + 1, dtype=torch.int64, device="cuda"), rows=torch.empty(M * top, dtype=torch.int64, device="cuda"),
             place=torch.empty((M, top), dtype=torch.int64, device="cuda"), balance=torch.empty(2 + E, device="cuda"))
    ws = torch.empty(max(256, B.gemm_route_workspace_bytes(M, E)), dtype=torch.uint8, device="cuda")
    B.gemm_route(B.DTYPE_BF16, M, E, top, X, ld, None, 1, *o.values(), workspace=ws)
    for n in ("ids", "offsets", "rows", "place"):
        assert np.array_equal(o[n].cpu().numpy(), want[n]), n
    D, rows = far(torch.full((M, E), 7.0, dtype=torch.bfloat16), ld)
    dgates = torch.randn((M, top), generator=torch.Generator().manual_seed(3))
    B.gemm_route_grad(B.DTYPE_BF16, M, E, top, X, ld, 1, o["ids"], o["offsets"], o["balance"], dgates.cuda(), None, D, ld)
    ref = rr.gradient(t.double().numpy(), want["ids"], np.zeros(E), dgates.double().numpy(), 0.0, True)
    # as in test_gpu_route.py: terms of at most max |dgates|, in 32 bits, then the result's rounding
    off = (2 * E + 60) * 2.0 ** -24 * float(dgates.abs().max())
    assert (np.abs(rows.double().cpu().numpy() - ref) <= off + 2.0 ** -8 * (np.abs(ref) + off)).all()


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("force", [*TILES, PINGPONG])
def test_what_is_no_number_in_every_tile(kind, force):
    """A row and a weight are not numbers; everything else is as without them, in tiles that overhang, too."""
    M, N, K = 270, 280, 576
    rng = np.random.default_rng(4)
    a, A, lda = left_of(kind, rng, M, K)
    w, W = weights_of(rng, N, K)
    if kind == "mx4":
        img = A.cpu().numpy()
        img[M * mx.padded(K) // 2 + 8 * (M + 7) + 3] = 255          # row 7, columns 416 .. 447
        A = torch.from_numpy(img).cuda()
    else:
        A[7, 300] = float("nan")
    img = W.cpu().numpy()
    img[N * mx.padded(K) // 2 + 8 * 265 + 1] = 255                  # weight 265, columns 128 .. 159
    C = torch.zeros((M, N), device="cuda")
    force_tile(force)
    try:
        B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, torch.from_numpy(img).cuda(), 0.0, C, N, 1)
    except B.BrgemmError:
        assert kind == "mx4" and force == "bf16_stream_32x128x64"
        pytest.skip("not a tile of images")
    finally:
        B.gemm_force_variant(-1, 0)
    got = C.double().cpu().numpy()
    keep = np.ones((M, N), bool)
    keep[7] = keep[:, 265] = False
    assert np.isnan(got[7]).all() and np.isnan(got[:, 265]).all()
    check(got[keep], (a @ w.T)[keep], mx.most_off(a, w, kind == "mx4")[keep], None)


def repeated(t, times):
    return t[None].expand(times, *t.shape).reshape(times * t.shape[0], *t.shape[1:]).contiguous()


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
def test_more_tiles_than_a_launch_holds(kind):
    """Weights that repeat every 1000 rows, 3000 rows beside them; looked at where the parts meet, too."""
    M, N, K, some = 3000, 1100000, 200, 1000
    print(f"[gpu-case] {M} x {N} x {K} {kind}", flush=True)
    rng = np.random.default_rng(8)
    a, A, lda = left_of(kind, rng, M, K)
    w, small = weights_of(rng, some, K)
    row = mx.padded(K) // 2
    W = torch.cat([repeated(small[:some * row], N // some), repeated(small[some * row:], N // some)])
    assert W.numel() == mx.nbytes(N, K)
    bias = rng.standard_normal(N).astype(np.float32)
    C = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, W, 0.0, C, N, 0, torch.from_numpy(bias).cuda(), B.EPI_BIAS)
    rows = np.r_[0:40, M - 40:M]
    for n0 in (0, 549000, 550000, 551000, N - some):
        want = a[rows] @ w.T + bias[n0:n0 + some]
        off = mx.most_off(a[rows], w, kind == "mx4") + 2.0 ** -23 * (np.abs(want) + np.abs(bias[n0:n0 + some]))
        check(C[rows, n0:n0 + some].double().cpu().numpy(), want, off, torch.bfloat16)


@pytest.mark.parametrize("kind", ["mx4", "bf16"])
def test_more_rows_than_a_launch_holds(kind):
    """134.3 million rows that repeat every 1000, 16 weights."""
    some, K, N = 1000, 64, 16
    M = 134300 * some
    print(f"[gpu-case] {M} x {N} x {K} {kind}", flush=True)
    rng = np.random.default_rng(9)
    a, small, lda = left_of(kind, rng, some, K)
    w, W = weights_of(rng, N, K)
    if kind == "mx4":
        row = mx.padded(K) // 2
        A = torch.cat([repeated(small[:some * row], M // some), repeated(small[some * row:], M // some)])
        assert A.numel() == mx.nbytes(M, K)
    else:
        A = repeated(small, M // some)
    C = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, W, 0.0, C, N, 0)
    want, off = a @ w.T, mx.most_off(a, w, kind == "mx4")
    for m0 in (0, M // 2 - some, M // 2, M - some):                 # (M / 2 is a multiple of 1000)
        check(C[m0:m0 + some].double().cpu().numpy(), want, off, torch.bfloat16)
