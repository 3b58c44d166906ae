"""Images whose size is no multiple of 16 bytes, one behind the other: made, read back and multiplied where they stand."""
import numpy as np
import pytest
import torch

import mx4_reference as mx
from paper_2511_13764_amd import binding as B
from test_gpu_mx4 import DT, PINGPONG, TILES, check, experts, force_tile, left_of, numbers

pytestmark = pytest.mark.gpu
KINDS = ["mx4", "bf16", "f16"]
BANKS = [(257, 256), (307, 608), (1, 100), (129, 1280)]         # N and the blocks of 256 odd


def say(what):
    print(f"[gpu-case] {what}", flush=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("N,K", BANKS)
def test_images_of_a_bank(dtype, trans, N, K):
    """Three images, each made and read back where it stands; nothing beside them is touched."""
    size = B.gemm_mx4_bytes(N, K)
    assert size % 16 == 8
    say(f"bank of {N} x {K} {dtype} trans {trans}")
    rng = np.random.default_rng([N, K])
    bank = torch.full((3 * size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    each = [numbers(rng, N, K, dtype) for _ in range(3)]
    for e in (1, 0, 2):
        t = each[e][1].t().contiguous() if trans else each[e][1]
        B.gemm_pack_mx4(DT[dtype][1], trans, N, K, t.cuda(), N if trans else K, N, None, bank[e * size:(e + 1) * size])
    got = bank.cpu().numpy()
    assert (got[3 * size:] == 0xA5).all()
    for e in range(3):
        assert np.array_equal(got[e * size:(e + 1) * size], mx.image(each[e][0])), e
        out = torch.empty((N, K), dtype=torch.float32, device="cuda")
        B.gemm_unpack_mx4(B.DTYPE_F32, N, K, bank[e * size:], out, K)
        assert np.array_equal(out.double().cpu().numpy(), mx.values(got[e * size:(e + 1) * size], N, K))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", [None, "generic_64x64x16_f32mfma", *TILES, PINGPONG])
@pytest.mark.parametrize("sizes,N,K", [([5, 0, 17, 1], 257, 256), ([3, 140, 33], 307, 608), ([300, 1, 259], 257, 1280), ([1] * 9, 1, 100)])
def test_experts_of_a_bank(kind, force, sizes, N, K):
    if kind == "mx4" and force == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")
    if kind != "mx4" and force not in (None, "generic_64x64x16_f32mfma") and K % 64:
        pytest.skip("tiles read whole 64 columns of 16-bit rows")
    say(f"experts {kind} {sizes} {N} x {K} {force}")
    experts(kind, sizes, N, K, lead=3, tail=2, act=True, force=force)


@pytest.mark.parametrize("sigma", [2.0 ** -40, 2.0 ** 20])
@pytest.mark.parametrize("force", [None, *TILES, PINGPONG])
def test_an_image_of_a_bank_in_a_product(sigma, force):
    """The second image as weights, beside rows and, on the other side, an image that stands likewise; powers that binary16 does not hold, too."""
    M, N, K = 261, 257, 1280
    rng = np.random.default_rng(7)
    banks = [torch.zeros(2 * mx.nbytes(n, K), dtype=torch.uint8) for n in (M, N)]
    a4, w = (mx.image(rng.standard_normal((n, K)) * s) for n, s in ((M, 1.0), (N, sigma)))
    for bank, image in zip(banks, (a4, w)):
        bank[image.size:] = torch.from_numpy(image)
    A4, W = (bank.cuda()[bank.numel() // 2:] for bank in banks)
    assert A4.data_ptr() % 16 == 8 and W.data_ptr() % 16 == 8
    w = mx.values(w, N, K)
    for kind in KINDS:
        if kind == "mx4" and force == TILES[3]:
            continue
        a, A, lda = (mx.values(a4, M, K), A4, 0) if kind == "mx4" else left_of(kind, rng, M, K)
        C = torch.full((M, N), float("nan"), device="cuda")
        say(f"product {kind} {force}")
        if force:
            force_tile(force)
        try:
            B.gemm_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, A, lda, W, 0.0, C, N, 1)
        finally:
            if force:
                B.gemm_force_variant(-1, 0)
        check(C.double().cpu().numpy(), a @ w.T, mx.most_off(a, w, kind == "mx4"), None)
