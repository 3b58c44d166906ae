"""Products with 4-bit weights whose powers are the format's least and largest, as images that others quantised may have them: 2^-127 .. 2^-125,
which 16-bit floats hold as subnormals, and 2^125 .. 2^127, with which a weight can be beyond every 16- and 32-bit float."""
import numpy as np
import pytest
import torch

import mx4_reference as mx
from paper_2511_13764_amd import binding as B
from test_gpu_mx4 import DT, PINGPONG, TILES, check, force_tile

pytestmark = pytest.mark.gpu
KINDS = ["mx4", "bf16", "f16"]
FORCES = [None, "generic_64x64x16_f32mfma", *TILES, PINGPONG]
LEAST, MOST = [0, 1, 2], [252, 253, 254]


def image_of(rng, rows, K, powers):
    """Every code, under powers drawn from `powers`; a power of blocks of zeros is one of them, too."""
    Kp = mx.padded(K)
    codes = rng.integers(0, 16, (rows, Kp), dtype=np.uint8)
    codes[:, 64:96] &= 8                                            # a block of zeros of both signs
    codes[:, K:] = 0
    planes = rng.choice(np.array(powers, np.uint8), (rows, Kp // 256, 8)).transpose(1, 0, 2)
    img = np.concatenate([(codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1), planes.reshape(-1)])
    return mx.values(img, rows, K), torch.from_numpy(img).cuda()


def rows_of(kind, rng, M, K, scale):
    """Rows of the size of `scale`, some of them zero."""
    if kind == "mx4":
        img = mx.image(rng.standard_normal((M, K)) * scale)
        return mx.values(img, M, K), torch.from_numpy(img).cuda(), 0
    x = rng.standard_normal((M, K)) * scale
    x[:, ::5] = 0.0
    t = torch.from_numpy(x).to(DT[kind][0])
    return t.double().numpy(), t.cuda(), K


def multiply(kind, M, N, K, A, lda, W, force=None, split=0, ws=None):
    C = torch.full((M, N), -5.0, device="cuda")
    print(f"[gpu-case] {kind} {M} x {N} x {K} {force} split {split}", flush=True)
    if force:
        force_tile(force, split)
    try:
        B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, W, 0.0, C, N, 1, workspace=ws)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    return C.double().cpu().numpy()


def skip_where_there_is_none(kind, force):
    if kind == "mx4" and force == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")


# Rows are such that products and sums are normal 32-bit floats, far from the least and the largest: of that size a weight of the least power
# times a row is 2^-116 and more, and sums of 576 with the largest are below 2^127.
SCALE = {"mx4": (2.0 ** 40, 2.0 ** -20), "bf16": (2.0 ** 40, 2.0 ** -20), "f16": (2.0 ** 12, 2.0 ** -13)}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", FORCES)
@pytest.mark.parametrize("powers", [LEAST, MOST, [0, 100, 127, 150], [90, 127, 253]])
@pytest.mark.parametrize("M,N,K", [(14, 70, 320), (260, 300, 576)])
def test_powers(kind, force, powers, M, N, K):
    skip_where_there_is_none(kind, force)
    rng = np.random.default_rng([M, *powers])
    a, A, lda = rows_of(kind, rng, M, K, SCALE[kind][max(powers) > 200])
    w, W = image_of(rng, N, K, powers)
    check(multiply(kind, M, N, K, A, lda, W, force), a @ w.T, mx.most_off(a, w, kind == "mx4"), None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("powers", [LEAST, MOST])
def test_powers_of_both_images_and_of_odd_rows(kind, powers):
    """Rows that only registers take (K off 64), copied and not; both images with powers at an end, of which the product still is a 32-bit float."""
    M, N, K = 40, 130, 601
    rng = np.random.default_rng(powers)
    w, W = image_of(rng, N, K, powers)
    a, A, lda = rows_of(kind, rng, M, K, SCALE[kind][powers is MOST]) if kind != "mx4" else (*image_of(rng, M, K, MOST if powers is LEAST else [5, 60]), 0)
    off = mx.most_off(a, w, kind == "mx4")
    for ws in (None, torch.empty(1 << 20, dtype=torch.uint8, device="cuda")):
        check(multiply(kind, M, N, K, A, lda, W, ws=ws), a @ w.T, off, None)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("tile", ["generic_64x64x16_f32mfma", *TILES])
@pytest.mark.parametrize("powers", [LEAST, MOST])
def test_powers_in_slices(kind, tile, powers):
    M, N, K = 20, 70, 1472
    rng = np.random.default_rng(powers)
    a, A, lda = rows_of(kind, rng, M, K, SCALE[kind][powers is MOST])
    w, W = image_of(rng, N, K, powers)
    ws = torch.empty(4 << 20, dtype=torch.uint8, device="cuda")
    check(multiply(kind, M, N, K, A, lda, W, tile, 3, ws), a @ w.T, mx.most_off(a, w, False), None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", FORCES)
def test_powers_of_experts(kind, force):
    """One expert with the largest powers between others."""
    skip_where_there_is_none(kind, force)
    sizes, N, K = [5, 130, 0, 301, 17], 300, 576
    M, G = sum(sizes), len(sizes)
    rng = np.random.default_rng(3)
    a, A, lda = rows_of(kind, rng, M, K, SCALE[kind][1])
    each = [image_of(rng, N, K, p) for p in ([120, 127], MOST, MOST, [110, 127], MOST)]
    W = torch.stack([w for _, w in each])
    bounds = np.concatenate([[0], np.cumsum(sizes)])
    C = torch.full((M, N), -5.0, device="cuda")
    print(f"[gpu-case] experts {kind} {force}", flush=True)
    if force:
        force_tile(force)
    try:
        B.gemm_grouped_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, G, torch.from_numpy(bounds).cuda(), A, lda, W,
                           W.stride(0), 0.0, C, N, 1)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    got = C.double().cpu().numpy()
    for e in range(G):
        at = slice(bounds[e], bounds[e + 1])
        check(got[at], a[at] @ each[e][0].T, mx.most_off(a[at], each[e][0], kind == "mx4"), None)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("force", FORCES)
def test_rows_at_the_ends_beside_the_largest_powers(kind, force):
    """The type's largest values beside weights of 0 under a power of 2^127 add nothing; beside others the sum is an infinity of its own sign,
    and so it is for an infinity in a row; NaN stays in its row."""
    M, N, K = 260, 300, 576
    rng = np.random.default_rng(5)
    a, _, _ = rows_of(kind, rng, M, K, SCALE[kind][1])
    w, W = image_of(rng, N, K, [254])
    big = float(torch.finfo(DT[kind][0]).max)
    a[2, 64:96] = big                                               # (weights of 0)
    a[100, 3] = np.inf
    a[101, 4] = np.nan
    if kind == "bf16":
        a[102, 3], a[258, 3] = big, -big
    t = torch.from_numpy(a).to(DT[kind][0])
    a = t.double().numpy()
    got = multiply(kind, M, N, K, t.cuda(), K, W, force)
    keep = np.ones(M, bool)
    keep[[100, 101, 102, 258]] = False
    with np.errstate(invalid="ignore"):
        want = a @ w.T
    check(got[keep], want[keep], mx.most_off(a[keep], w, False), None)
    assert np.isnan(got[101]).all()
    sign = np.sign(w[:, 3])
    assert (sign == 0).any() and (sign != 0).any()
    assert np.isnan(got[100][sign == 0]).all() and np.array_equal(got[100][sign != 0], sign[sign != 0] * np.inf)
    if kind == "bf16":
        for m, s in ((102, 1), (258, -1)):
            assert np.array_equal(got[m][sign != 0], s * sign[sign != 0] * np.inf)
            assert np.isfinite(got[m][sign == 0]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", FORCES)
@pytest.mark.parametrize("others", [[127], MOST])
def test_a_block_of_zeros_that_is_not_a_number(kind, force, others):
    """What the packer makes of a block with a NaN: zeros under the power 255."""
    skip_where_there_is_none(kind, force)
    M, N, K = 260, 300, 576
    rng = np.random.default_rng(6)
    a, A, lda = rows_of(kind, rng, M, K, SCALE[kind][1])
    w, W = image_of(rng, N, K, others)
    row = mx.padded(K) // 2
    for n in (9, 290):
        W[n * row + 16:n * row + 32] = 0
        W[N * row + n * 8 + 2] = 255                                # block 1: columns 32 .. 63
    got = multiply(kind, M, N, K, A, lda, W, force)
    keep = np.ones(N, bool)
    keep[[9, 290]] = False
    assert np.isnan(got[:, ~keep]).all()
    check(got[:, keep], (a @ w.T)[:, keep], mx.most_off(a, w, kind == "mx4")[:, keep], None)
