"""Grouped products with 4-bit images as a program may call them: added to what C holds, into and out of rows of any pitch, with biases apart from
one another or shared, rows that are copied first, more groups than one wave looks at."""
import numpy as np
import pytest
import torch

import mx4_reference as mx
from paper_2511_13764_amd import binding as B
from test_gpu_mx4 import DT, PINGPONG, TILES, check, force_tile, left_of, weights_of

pytestmark = pytest.mark.gpu
KINDS = ["mx4", "bf16", "f16"]


def run(kind, sizes, N, K, lead=3, tail=2, beta=0.0, pad=0, ldc_pad=0, act=False, stride_bias=None, c32=False, force=None, ws=0, gap=0, seed=0):
    """`gap`: bytes between one expert's image and the next's."""
    print(f"[gpu-case] {kind} {sizes} {N} x {K} beta {beta} pads {pad} {ldc_pad} {force}", flush=True)
    rng = np.random.default_rng([seed, len(sizes), N, K])
    G, M = len(sizes), lead + sum(sizes) + tail
    a, A, lda = left_of(kind, rng, M, K, 0 if kind == "mx4" else pad)
    each = [weights_of(rng, N, K) for _ in range(G)]
    step = mx.nbytes(N, K) + gap
    W = torch.full((G * step,), 0xFF, dtype=torch.uint8, device="cuda")
    for e in range(G):
        W[e * step:e * step + mx.nbytes(N, K)] = each[e][1]
    half = None if c32 else torch.float16 if kind == "f16" else torch.bfloat16
    sb = N if stride_bias is None else stride_bias
    bias = rng.standard_normal((G - 1) * sb + N).astype(np.float32)
    bounds = np.concatenate([[lead], lead + np.cumsum(sizes)])
    c0 = torch.from_numpy(rng.standard_normal((M, N + ldc_pad))).to(half or torch.float32)
    C = c0.cuda()
    workspace = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None
    if force:
        force_tile(force)
    try:
        B.gemm_grouped_mx4(B.DTYPE_MX4 if kind == "mx4" else DT[kind][1], M, N, K, G, torch.from_numpy(bounds).cuda(), A, lda, W,
                           step, beta, C, N + ldc_pad, c32, torch.from_numpy(bias).cuda() if act else None, sb,
                           B.EPI_BIAS | B.EPI_RELU if act else 0, workspace=workspace)
    finally:
        if force:
            B.gemm_force_variant(-1, 0)
    got, was = C.double().cpu().numpy(), c0.double().numpy()
    left = np.ones((M, N + ldc_pad), bool)
    for e in range(G):
        at = slice(bounds[e], bounds[e + 1])
        left[at, :N] = False
        w = each[e][0]
        want, off = a[at] @ w.T, mx.most_off(a[at], w, kind == "mx4")
        for add in ([beta * was[at, :N]] if beta else []) + ([bias[e * sb:e * sb + N]] if act else []):
            want = want + add
            off = off + 2.0 ** -23 * (np.abs(want) + np.abs(add))
        check(got[at, :N], np.maximum(want, 0.0) if act else want, off, half)
    assert np.array_equal(got[left], was[left])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", [None, "generic_64x64x16_f32mfma", *TILES, PINGPONG])
@pytest.mark.parametrize("sizes", [[5, 0, 17, 1], [3, 140, 33], [300, 1, 259]])
def test_added_to_what_is_there(kind, force, sizes):
    if kind == "mx4" and force == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")
    run(kind, sizes, 300, 576, beta=-0.5, ldc_pad=1, pad=8, force=force)
    run(kind, sizes, 259, 512, beta=2.0, ldc_pad=5, act=True, stride_bias=400, c32=True, force=force)
    run(kind, sizes, 256, 320, beta=1.0, act=True, stride_bias=0, gap=48, force=force)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("force", [None, "generic_64x64x16_f32mfma", *TILES, PINGPONG])
@pytest.mark.parametrize("ldc_pad", [0, 8, 4])
def test_rows_of_any_pitch(kind, force, ldc_pad):
    """The large tiles store whole lines where a group's rows of C allow it."""
    if kind == "mx4" and force == TILES[3]:
        pytest.skip("tiles of 32 and 16 rows are for 16-bit rows")
    run(kind, [270, 5, 600], 512, 256, lead=1, ldc_pad=ldc_pad, pad=16, act=True, force=force)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("sizes,N,K,pad", [([40, 0, 70, 33], 130, 601, 0), ([300, 5], 264, 1003, 3), ([25] * 9, 72, 100, 1), ([64, 64], 520, 512, 4)])
def test_rows_that_are_copied(kind, sizes, N, K, pad):
    """Groups of more than 16 rows whose rows end inside 64 columns or start off 16 bytes; without room they are read where they are."""
    for ws in (0, 1 << 10, 8 << 20):
        run(kind, sizes, N, K, pad=pad, ws=ws, act=True)
    run(kind, sizes, N, K, pad=pad, ws=8 << 20, beta=-0.5, ldc_pad=3, c32=True)


@pytest.mark.parametrize("kind", KINDS)
def test_many_groups(kind):
    """More than the 256 that are looked at together, most of them empty."""
    rng = np.random.default_rng(2)
    sizes = rng.integers(0, 3, 300).tolist()
    sizes[37], sizes[270] = 150, 40
    run(kind, sizes, 72, 256, act=True)
    run(kind, sizes, 72, 256, act=True, force=PINGPONG)
    run(kind, sizes, 72, 256, beta=0.5, force=TILES[0])
