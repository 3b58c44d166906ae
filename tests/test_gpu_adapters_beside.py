"""Adapters whose first product runs beside the projection's tiles in one launch, and those of long segments whose sums stay
apart, at segments that begin and end anywhere."""
import pytest
import torch

from paper_2511_13764_amd import binding as B
from test_gpu_grouped import run_adapters

pytestmark = pytest.mark.gpu

STREAM128, STREAM_MID, STREAM64 = (("bf16_stream_128x128x64", ""), ("bf16_stream_64x128x64", "128x64"),
                                   ("bf16_stream_32x128x64", "64x64"))


def workspace():
    return torch.empty(32 << 20, dtype=torch.uint8, device="cuda")


def segments(rows, longest):
    sizes = []
    while sum(sizes) < rows:
        sizes.append(min([1, 0, 2, longest, 17, 1, 16][len(sizes) % 7], rows - sum(sizes)))
    return sizes, [(5 * i) % 6 - 1 for i in range(len(sizes))]


@pytest.mark.parametrize("M,N,K,kernel", [(600, 4096, 512, STREAM128), (600, 4096, 64, STREAM128), (597, 2056, 1280, STREAM_MID),
                                          (150, 2056, 512, STREAM64), (599, 1032, 2048, STREAM64)])
@pytest.mark.parametrize("tB", [0, 1])
def test_first_product_beside_the_projection(M, N, K, kernel, tB):
    sizes, ids = segments(M, 70)
    for dtype, R in (("bf16", 16), ("f16", 40), ("bf16", 72)):
        assert run_adapters(dtype, tB, sizes, ids, 4, R, N, K, workspace=workspace(), bias=R == 40, relu=R == 40) == kernel
    run_adapters("bf16", tB, sizes, ids, 4, 24, N, K, workspace=workspace(), beta=0.5, c32=True, lead=3, behind=5,
                 pads=(8, 8, 3, 5, 3, 1), gap=5, scale=False)
    run_adapters("bf16", tB, sizes, ids, 4, 13, N, K, workspace=workspace())             # (along the rank: a launch of its own)


def test_one_segment_a_row_beside_the_projection():
    run_adapters("bf16", 1, [1] * 200, [i % 5 for i in range(200)], 4, 16, 2056, 512, workspace=workspace(), per_row=True)


@pytest.mark.parametrize("tB", [0, 1])
def test_long_segments_with_a_split_reduction(tB):
    """The projection's plan splits its reduction: its sums, a set for each slice, and the adapters behind them."""
    for sizes, R, N, K in (([0, 200, 258], 32, 704, 4096), ([64, 64], 16, 2048, 4096), ([256, 300, 0, 300], 64, 1024, 4104), ([64], 16, 4096, 1024)):
        run_adapters("bf16", tB, sizes, [2, 0, 1, 5][:len(sizes)], 3, R, N, K, workspace=workspace(), bias=True)


def test_the_same_result_again():
    """No order of additions is left to chance: the same call gives the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    M, N, K, R, G = 600, 4096, 512, 16, 60
    X, W = (torch.randn(s, device="cuda", generator=gen).bfloat16() for s in ((M, K), (N, K)))
    down, up = (torch.randn(s, device="cuda", generator=gen).bfloat16() for s in ((G, R, K), (G, N, R)))
    off = torch.arange(0, M + 1, M // G, device="cuda")
    ws, got = workspace(), []
    for _ in range(3):
        ws.fill_(255)
        Y, H = torch.empty((M, N), device="cuda", dtype=torch.bfloat16), torch.empty((M, R), device="cuda", dtype=torch.bfloat16)
        B.gemm_adapters(B.DTYPE_BF16, 1, M, N, K, R, G, off, None, G, X, K, W, K, down, K, R * K, up, R, N * R, None, 0.0, Y, N, 0,
                        None, 0, H, R, workspace=ws)
        got.append((Y, H))
    for Y, H in got[1:]:
        assert torch.equal(Y, got[0][0]) and torch.equal(H, got[0][1])


@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("M,bank", [(4, 1), (16, 1), (17, 2), (32, 8), (64, 3), (65, 4), (129, 32), (255, 5), (256, 64), (257, 4)])
def test_rows_taken_by_their_adapter(M, bank, tB):
    """Decode with few adapters: an adapter's rows go together, wherever they lie; some have none, some adapters no row."""
    ids = [(i * i + i // 7) % (bank + 2) - 1 for i in range(M)]            # -1 and `bank` are none
    for dtype, R, N, K in (("bf16", 16, 520, 320), ("f16", 40, 264, 1000), ("bf16", 13, 75, 71)):
        run_adapters(dtype, tB, [1] * M, ids, bank, R, N, K, per_row=True, workspace=workspace(), bias=R == 40, relu=R == 40)
    run_adapters("bf16", tB, [1] * M, [0] * M, bank, 16, 264, 128, per_row=True, workspace=workspace(), beta=0.5, c32=True)
    run_adapters("bf16", tB, [1] * M, ids, bank, 70, 136, 64, per_row=True)              # (no workspace)


@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("M,bank,R", [(33, 2, 520), (64, 1, 200), (65, 4, 200), (129, 3, 130), (255, 5, 77), (256, 40, 144), (257, 4, 64)])
def test_rows_taken_by_their_adapter_in_earnest(M, bank, R, tB):
    """... at sizes where it saves enough reading (of 30 MB and 2 MB an adapter); 257 rows go one by one."""
    ids = [(i * i + i // 7) % (bank + 2) - 1 for i in range(M)]
    run_adapters("bf16", tB, [1] * M, ids, bank, R, 1000, 1064, per_row=True, workspace=workspace(), bias=True, relu=True)
    run_adapters("f16", tB, [1] * M, [bank - 1] * M, bank, R, 1003, 1061, per_row=True, workspace=workspace(), beta=0.5, c32=True)
    run_adapters("bf16", tB, [1] * M, ids, bank, R, 1000, 1064, per_row=True)             # (no workspace)
