"""4-bit images and the products that read them, against their definition in 64 bits (mx4_reference.py)."""
import numpy as np
import pytest
import torch

import mx4_reference as mx
from paper_2511_13764_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": (torch.float32, B.DTYPE_F32), "bf16": (torch.bfloat16, B.DTYPE_BF16), "f16": (torch.float16, B.DTYPE_F16)}



def numbers(rng, rows, K, dtype):
    """Rows of every magnitude, representable in `dtype`, as a float64 array and a CPU tensor."""
    x = rng.standard_normal((rows, K)) * np.exp2(rng.integers(-6, 6, (rows, 1)))
    t = torch.from_numpy(x).to(DT[dtype][0])
    return t.double().numpy(), t


def bytes_of(image):
    return image.cpu().numpy()


def pack(dtype, t, rows, K, trans=0, ldx=None, x_rows=None, source=None):
    img = torch.full((mx.nbytes(rows, K) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    B.gemm_pack_mx4(DT[dtype][1], trans, rows, K, t, ldx if ldx else (rows if trans else K), rows if x_rows is None else x_rows, source,
                    img, mx.nbytes(rows, K))
    out = bytes_of(img)
    assert (out[-64:] == 0xA5).all()
    return out[:-64]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 31), (2, 32), (16, 256), (5, 257), (70, 512), (33, 1000), (130, 770)])
def test_pack(dtype, rows, K):
    x, t = numbers(np.random.default_rng([rows, K]), rows, K, dtype)
    want = mx.image(x)
    assert np.array_equal(pack(dtype, t.cuda(), rows, K), want)
    assert np.array_equal(pack(dtype, t.t().contiguous().cuda(), rows, K, trans=1), want)
    # wider rows than K, at an address of the element's own alignment, NaN around them
    wide = torch.full((rows, K + 5), float("nan"), dtype=t.dtype)
    wide[:, 1:K + 1] = t
    assert np.array_equal(pack(dtype, wide.cuda().view(-1)[1:], rows, K, ldx=K + 5), want)
    tall = torch.full((K, rows + 3), float("nan"), dtype=t.dtype)
    tall[:, 1:rows + 1] = t.t()
    assert np.array_equal(pack(dtype, tall.cuda().view(-1)[1:], rows, K, trans=1, ldx=rows + 3), want)


def test_pack_of_rows_from_elsewhere():
    x, t = numbers(np.random.default_rng(5), 9, 300, "bf16")
    source = torch.tensor([3, 3, -1, 8, 0, 9, 1 << 40, 5, -(1 << 40), 2, 7], device="cuda")
    want = np.stack([x[i] if 0 <= i < 9 else np.zeros(300) for i in source.tolist()])
    assert np.array_equal(pack("bf16", t.cuda(), 11, 300, x_rows=9, source=source), mx.image(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("trans", [0, 1])
def test_pack_at_the_ends_of_the_range(dtype, trans):
    """Every code and half-way point under the least, an ordinary and the largest power, subnormals, zeros of both signs, infinities, NaN."""
    halves = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.9, .2499, .2501, .7499, .7501, 1.2499, 4.999, 5.001,
                       -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -7])
    least = {"f32": -149, "bf16": -133, "f16": -24}[dtype]
    most = {"f32": 125, "bf16": 125, "f16": 13}[dtype]
    x = np.zeros((8, 96))
    x[0, :32] = halves
    x[1, :32] = halves * 2.0 ** most
    x[2, :32] = 2.0 ** least * np.arange(32)
    x[3, 32:64] = -0.0
    x[4, :32] = np.inf
    x[4, 40] = -np.inf
    x[5, 70] = np.nan
    x[6, :32] = halves * 2.0 ** -126 if dtype != "f16" else halves * 2.0 ** -14
    x[7, :32] = 2.0 ** (least + 3)
    t = torch.from_numpy(x).to(DT[dtype][0])
    got = pack(dtype, (t.t().contiguous() if trans else t).cuda(), 8, 96, trans=trans)
    assert np.array_equal(got, mx.image(t.double().numpy()))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 31), (16, 256), (5, 257), (130, 770)])
def test_unpack(dtype, rows, K):
    rng = np.random.default_rng([7, rows, K])
    img = rng.integers(0, 256, mx.nbytes(rows, K), dtype=np.uint8)
    want = mx.values(img, rows, K)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(want).float().to(DT[dtype][0])
    out = torch.full((rows * (K + 3) + 1,), -777.0, dtype=DT[dtype][0], device="cuda")
    B.gemm_unpack_mx4(DT[dtype][1], rows, K, torch.from_numpy(img).cuda(), out[1:], K + 3)
    got = out.cpu()
    body = got[1:].view(rows, K + 3)
    assert (got[0] == -777.0) and (body[:, K:] == -777.0).all()
    assert torch.equal(torch.nan_to_num(body[:, :K].float(), nan=123.0), torch.nan_to_num(want.float(), nan=123.0))


def left_of(kind, rng, M, K, pad=0):
    """The left operand: values, device tensor, leading dimension."""
    if kind == "mx4":
        img = mx.image(rng.standard_normal((M, K)) * np.exp2(rng.integers(-3, 4, (M, 1))))
        return mx.values(img, M, K), torch.from_numpy(img).cuda(), 0
    x, t = numbers(rng, M, K, kind)
    if not pad:
        return x, t.cuda(), K
    wide = torch.full((M, K + pad), float("nan"), dtype=t.dtype)
    wide[:, :K] = t
    return x, wide.cuda(), K + pad


def weights_of(rng, N, K, sigma=0.05):
    img = mx.image(rng.standard_normal((N, K)) * sigma)
    return mx.values(img, N, K), torch.from_numpy(img).cuda()


def check(got, want, off, half):
    """`half`: the type a result is rounded to, or None."""
    eps = torch.finfo(half).eps / 2 if half else 0.0
    tiny = 2.0 ** -25 if half == torch.float16 else 0.0             # half a subnormal step
    err = np.abs(got - want)
    assert (err <= off + eps * (np.abs(want) + off) + tiny).all(), float((err - off).max())


def force_tile(name, split=0):
    """A variant's name, and behind a colon its form's."""
    variant, _, form = name.partition(":")
    B.gemm_force_variant(B.variants().index(variant), split)
    if form:
        B.gemm_force_form(next(f for f in range(8) if B.gemm_form_name(f) == form))


def product(kind, M, N, K, act=False, beta=0.0, c32=True, pad=0, ldc_pad=0, force=None, split=0, ws=0, sigma=0.05, seed=0):
    rng = np.random.default_rng([seed, M, N, K])
    a, A, lda = left_of(kind, rng, M, K, pad)
    w, W = weights_of(rng, N, K, sigma)
    half = None if c32 else torch.float16 if kind == "f16" else torch.bfloat16
    bias = rng.standard_normal(N).astype(np.float32)
    c0 = torch.from_numpy(rng.standard_normal((M, N + ldc_pad))).to(half or torch.float32)
    C = (c0 if beta else torch.full_like(c0, float("nan"))).cuda()
    if ldc_pad:
        C[:, N:] = -77.0
    workspace = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None
    if force:
        force_tile(force, split)
    try:
        B.gemm_mx4(DT[kind][1] if kind != "mx4" else B.DTYPE_MX4, M, N, K, A, lda, W, beta, C, N + ldc_pad, c32,
                   torch.from_numpy(bias).cuda() if act else None, B.EPI_BIAS | B.EPI_RELU if act else 0, workspace=workspace)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    want, off = a @ w.T, mx.most_off(a, w, kind == "mx4")
    if beta:
        want = want + beta * c0[:, :N].double().numpy()
        off = off + 2.0 ** -23 * (np.abs(want) + np.abs(beta * c0[:, :N].double().numpy()))
    if act:
        want = want + bias
        off = off + 2.0 ** -23 * (np.abs(want) + np.abs(bias))
        want = np.maximum(want, 0.0)
    got = C.double().cpu().numpy()
    check(got[:, :N], want, off, half)
    assert (got[:, N:] == -77.0).all()


SIZES = [(1, 1, 1), (1, 15, 31), (2, 16, 32), (16, 100, 255), (17, 257, 256), (33, 64, 257), (65, 130, 1000), (130, 33, 2048), (300, 259, 515)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(20, 70, 333), (140, 300, 1001), (600, 520, 70), (17, 64, 2050)])
def test_rows_that_are_copied(kind, M, N, K):
    """With a workspace: rows off 16 bytes, and a K that ends inside 64 columns."""
    product(kind, M, N, K, ws=8 << 20)
    product(kind, M, N, K, act=True, c32=False, pad=3, ldc_pad=5, ws=8 << 20)
    product(kind, M, N, K, pad=8 - K % 8, ws=8 << 20, beta=2.0)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("tile", ["generic_64x64x16_f32mfma", *["bf16_stream_128x128x64", "bf16_stream_64x128x64", "bf16_stream_32x128x64:64x64"]])
@pytest.mark.parametrize("split", [2, 3, 8])
def test_split(kind, tile, split):
    """Slices of unequal length and, of eight, two without a block."""
    for M, N, K, kw in ((20, 70, 1472, {}), (130, 132, 1536, dict(act=True, c32=False)), (5, 33, 1536, dict(beta=0.5))):
        if split <= -(-K // 256):
            product(kind, M, N, K, force=tile, split=split, ws=16 << 20, **kw)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_split_by_itself(kind):
    """Few tiles of a long reduction; weights that binary16 does not hold, too."""
    for sigma in (0.05, 2.0 ** -40):
        product(kind, 20, 70, 8000, ws=16 << 20, sigma=sigma)
    assert B.gemm_last_split() > 1


def test_forced_splits_are_checked():
    X, W, C = (torch.zeros(1 << 20, dtype=torch.uint8, device="cuda") for _ in range(3))
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    for variant, split, want in ((0, 2, B.WORKSPACE_TOO_SMALL), (2, 2, B.INVALID_ARG), (0, 5, B.INVALID_ARG), (3, 1, B.INVALID_ARG)):
        B.gemm_force_variant(variant, split)
        try:
            assert B.gemm_mx4(B.DTYPE_BF16, 20, 70, 1024, X, 1024, W, 0.0, C, 70, 0, workspace=ws, check=False) == want, (variant, split)
        finally:
            B.gemm_force_variant(-1, 0)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(kind, M, N, K):
    product(kind, M, N, K)
    product(kind, M, N, K, act=True, c32=False, pad=3, ldc_pad=5)
    product(kind, M, N, K, beta=-0.5, ldc_pad=1)


PINGPONG = "bf16_pingpong_256x256x64"


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (256, 256, 256), (256, 512, 512), (300, 259, 515), (257, 256, 770), (512, 300, 1030), (130, 256, 4000), (520, 520, 5500)])
def test_large_tiles(M, N, K):
    """One block of the reduction, an even and an odd number, more than the ring's period; tiles that overhang either way."""
    product("mx4", M, N, K, force=PINGPONG)
    product("mx4", M, N, K, act=True, c32=False, ldc_pad=8 - N % 8, force=PINGPONG)
    product("mx4", M, N, K, act=True, c32=False, ldc_pad=1, force=PINGPONG)
    product("mx4", M, N, K, beta=-0.5, ldc_pad=1, force=PINGPONG)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 64), (256, 256, 128), (256, 512, 192), (300, 259, 256), (257, 256, 320), (512, 300, 832), (130, 256, 4032), (520, 520, 1408)])
def test_large_tiles_of_rows(kind, M, N, K):
    """Every number of blocks modulo the four that the weights' take, more than the rings' periods."""
    product(kind, M, N, K, force=PINGPONG)
    product(kind, M, N, K, act=True, c32=False, pad=8, ldc_pad=8 - N % 8, force=PINGPONG)
    product(kind, M, N, K, beta=-0.5, ldc_pad=1, force=PINGPONG)


TILES = ["bf16_stream_128x128x64", "bf16_stream_64x128x64", "bf16_stream_32x128x64:64x64", "bf16_stream_32x128x64"]


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 64), (128, 128, 128), (64, 64, 192), (130, 259, 256), (257, 130, 320), (40, 300, 832), (14, 200, 1600), (65, 66, 4032), (200, 200, 1408)])
def test_tiles(tile, kind, M, N, K):
    if kind == "mx4" and tile == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")
    product(kind, M, N, K - (30 if kind == "mx4" else 0), force=tile)
    product(kind, M, N, K, act=True, c32=False, pad=8, ldc_pad=3, force=tile)
    product(kind, M, N, K, beta=-0.5, ldc_pad=1, force=tile)


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [0, 0, 3], [63, 1, 0, 130], [130, 7, 301], [5, 0, 17, 1, 2, 0, 9]])
def test_experts_in_tiles(tile, kind, sizes):
    if kind == "mx4" and tile == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")
    experts(kind, sizes, 300, 576, lead=3, tail=2, act=True, force=tile)
    experts(kind, sizes, 128, 1024, shared=True, c32=True, force=tile)


@pytest.mark.parametrize("sigma", [2.0 ** -40, 2.0 ** -17, 2.0 ** -13, 2.0 ** 12, 2.0 ** 20])
@pytest.mark.parametrize("force", [None, PINGPONG, *TILES])
def test_weights_at_the_ends_of_binary16(sigma, force):
    product("f16", 70, 330, 576, sigma=sigma, force=force)
    product("bf16", 70, 330, 576, sigma=sigma, force=force)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [0, 0, 3], [255, 1, 0, 300], [256, 512], [130, 7, 301]])
def test_experts_in_large_tiles(kind, sizes):
    experts(kind, sizes, 300, 576, lead=3, tail=2, act=True, force=PINGPONG)
    experts(kind, sizes, 256, 1024, shared=True, c32=True, force=PINGPONG)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
def test_product_without_a_reduction(kind):
    product(kind, 20, 40, 0, act=True, beta=1.0)
    product(kind, 20, 40, 0, act=True, c32=False)


@pytest.mark.parametrize("sigma", [2.0 ** -40, 2.0 ** 20])
def test_weights_beyond_binary16(sigma):
    """Powers that binary16 does not hold, beside rows that are."""
    product("f16", 20, 48, 600, sigma=sigma)
    product("bf16", 20, 48, 600, sigma=sigma)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
def test_what_is_no_number_stays_in_its_row_and_column(kind):
    M, N, K = 40, 70, 520
    rng = np.random.default_rng(3)
    a, A, lda = left_of(kind, rng, M, K)
    w, W = weights_of(rng, N, K)
    if kind == "mx4":
        img = A.cpu().numpy()
        img[M * mx.padded(K) // 2 + 8 * (M + 7)] = 255              # row 7, columns 256 .. 287
        A = torch.from_numpy(img).cuda()
    else:
        A[7, 300] = float("inf")
    img = W.cpu().numpy()
    img[N * mx.padded(K) // 2 + 8 * 9 + 1] = 255                    # weight 9, columns 128 .. 159
    C = torch.zeros((M, N), device="cuda")
    B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, torch.from_numpy(img).cuda(), 0.0, C, N, 1)
    got = C.double().cpu().numpy()
    keep = np.ones((M, N), bool)
    keep[7] = keep[:, 9] = False
    assert not np.isfinite(got[7]).any() and np.isnan(got[:, 9]).all()
    check(got[keep], (a @ w.T)[keep], mx.most_off(a, w, kind == "mx4")[keep], None)


def experts(kind, sizes, N, K, lead=0, tail=0, act=False, shared=False, force=None, c32=False, seed=0):
    """Groups of `sizes` rows behind `lead` rows and before `tail` that belong to none."""
    rng = np.random.default_rng([seed, len(sizes), N, K])
    G, M = len(sizes), lead + sum(sizes) + tail
    a, A, lda = left_of(kind, rng, M, K)
    each = [weights_of(rng, N, K) for _ in range(1 if shared else G)]
    W = torch.stack([w for _, w in each])
    half = None if c32 else torch.float16 if kind == "f16" else torch.bfloat16
    bias = rng.standard_normal((G, N)).astype(np.float32)
    bounds = np.concatenate([[lead], lead + np.cumsum(sizes)])
    C = torch.full((M, N), -77.0, dtype=half or torch.float32, device="cuda")
    if force:
        force_tile(force)
    try:
        B.gemm_grouped_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, G, torch.from_numpy(bounds).cuda(), A, lda, W,
                           0 if shared else W.stride(0), 0.0, C, N, c32, torch.from_numpy(bias).cuda() if act else None, N,
                           B.EPI_BIAS | B.EPI_RELU if act else 0)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    got = C.double().cpu().numpy()
    assert (got[:lead] == -77.0).all() and (got[M - tail:] == -77.0).all()
    for e in range(G):
        w = each[0 if shared else e][0]
        at = slice(bounds[e], bounds[e + 1])
        want, off = a[at] @ w.T, mx.most_off(a[at], w, kind == "mx4")
        if act:
            want = want + bias[e]
            off = off + 2.0 ** -23 * (np.abs(want) + np.abs(bias[e]))
            want = np.maximum(want, 0.0)
        check(got[at], want, off, half)


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [[1], [0, 0, 3], [5, 0, 17, 1], [16, 33, 2, 0, 64, 9], [1] * 40, [130, 7, 301]])
def test_experts(kind, sizes):
    experts(kind, sizes, 130, 600, lead=3, tail=2, act=True)
    experts(kind, sizes, 40, 256, shared=True, c32=True)


def test_bounds_that_make_no_sense():
    M, N, K = 24, 48, 300
    rng = np.random.default_rng(8)
    a, A, lda = left_of("mx4", rng, M, K)
    each = [weights_of(rng, N, K) for _ in range(3)]
    W = torch.stack([w for _, w in each])
    for bounds, rows in ([-5, 4, 1 << 40, 2], [(0, 0, 4), (1, 4, 24)]), ([30, 8, 12, 10], [(1, 8, 12)]):
        C = torch.full((M, N), -77.0, device="cuda")
        B.gemm_grouped_mx4(B.DTYPE_MX4, M, N, K, 3, torch.tensor(bounds, device="cuda"), A, lda, W, W.stride(0), 0.0, C, N, 1)
        got, left = C.double().cpu().numpy(), np.ones(M, bool)
        for e, first, end in rows:
            check(got[first:end], a[first:end] @ each[e][0].T, mx.most_off(a[first:end], each[e][0], True), None)
            left[first:end] = False
        assert (got[left] == -77.0).all()


@pytest.mark.parametrize("kind", ["mx4", "bf16", "f16"])
def test_the_same_bits_again_and_from_a_graph(kind):
    """Captured on its own stream; its replays read what the buffers hold then, between eager calls."""
    M, N, K = 48, 144, 1030
    rng = np.random.default_rng(4)
    x = [numbers(rng, M, K, "bf16" if kind == "mx4" else kind)[1].cuda() for _ in range(3)]
    w = [numbers(rng, N, K, "bf16")[1].cuda() for _ in range(3)]
    X, Wn = x[0].clone(), w[0].clone()
    A = torch.empty(mx.nbytes(M, K), dtype=torch.uint8, device="cuda") if kind == "mx4" else X
    W = torch.empty(mx.nbytes(N, K), dtype=torch.uint8, device="cuda")
    C = torch.empty((M, N), device="cuda")
    offsets = torch.tensor([0, 20, 48], device="cuda")
    ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")

    def call():
        B.gemm_pack_mx4(B.DTYPE_BF16, 0, N, K, Wn, K, N, None, W)
        if kind == "mx4":
            B.gemm_pack_mx4(B.DTYPE_BF16, 0, M, K, X, K, M, None, A)
        code = B.DTYPE_MX4 if kind == "mx4" else DT[kind][1]
        B.gemm_mx4(code, M, N, K, A, K, W, 0.0, C, N, 1, workspace=ws)
        B.gemm_grouped_mx4(code, M, N, K, 2, offsets, A, K, W, 0, 1.0, C, N, 1, workspace=ws)

    eager = []
    for i in range(3):
        X.copy_(x[i])
        Wn.copy_(w[i])
        call()
        eager.append(C.clone())
        call()
        assert torch.equal(C, eager[-1])
    g = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=stream):
        call()
    for i in (1, 2, 0, 0, 1):
        X.copy_(x[i])
        Wn.copy_(w[i])
        C.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, eager[i])
        assert bool(torch.isfinite(eager[i]).all())


def test_backward_of_a_layer_in_four_bits():
    """dX = dY W and dW = dY^T X on images packed along what each sums over."""
    M, N, K = 70, 130, 300
    rng = np.random.default_rng(9)
    (y, Y), (x, X), (w, W) = (numbers(rng, *s, "bf16") for s in ((M, N), (M, K), (N, K)))

    def img(t, rows, k, trans):
        out = torch.empty(mx.nbytes(rows, k), dtype=torch.uint8, device="cuda")
        B.gemm_pack_mx4(B.DTYPE_BF16, trans, rows, k, t.cuda(), rows if trans else k, rows, None, out)
        return out
    dX, dW = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda")
    B.gemm_mx4(B.DTYPE_MX4, M, K, N, img(Y, M, N, 0), 0, img(W, K, N, 1), 0.0, dX, K, 1)
    B.gemm_mx4(B.DTYPE_MX4, N, K, M, img(Y, N, M, 1), 0, img(X, K, M, 1), 0.0, dW, K, 1)

    def q(v):
        return mx.values(mx.image(v), *v.shape)
    check(dX.double().cpu().numpy(), q(y) @ q(w.T).T, mx.most_off(q(y), q(w.T), True), None)
    check(dW.double().cpu().numpy(), q(y.T) @ q(x.T).T, mx.most_off(q(y.T), q(x.T), True), None)
