"""gemm_last_variant and gemm_last_form after a call with adapters: the kernel that they name is the one that ran."""
import pytest
import torch

from paper_2511_13764_amd import binding as B
from test_gpu_adapters_isolation import KERNELS
from test_gpu_grouped import force, matrix, on_device, say, stack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tB", [0, 1])
@pytest.mark.parametrize("M,N,K", [(64, 1024, 1024), (16, 4096, 4096), (100, 264, 512), (64, 96, 64), (300, 520, 328), (130, 4096, 2048),
                                   (700, 1024, 4096), (1030, 2056, 1024), (2048, 4096, 512)])
def test_the_kernel_named_is_the_one_that_ran(M, N, K, tB):
    """Without a workspace the adapters are blocks of the projection's tiles.  Forced, the kernel named gives the same bits."""
    gen = torch.Generator().manual_seed(M)
    R, t = 16, torch.bfloat16
    X, W = matrix(gen, M, K, t)[0], matrix(gen, *((N, K) if tB else (K, N)), t)[0]
    down, up = stack(gen, 2, *((R, K) if tB else (K, R)), t)[0], stack(gen, 2, *((N, R) if tB else (R, N)), t)[0]
    off = on_device([0, M // 3, M])

    def run():
        Y, H = torch.empty((M, N), dtype=t, device="cuda"), torch.empty((M, R), dtype=t, device="cuda")
        B.gemm_adapters(B.DTYPE_BF16, tB, M, N, K, R, 2, off, None, 2, X, K, W, K if tB else N, down, K if tB else R, R * K, up,
                        R if tB else N, R * N, None, 0.0, Y, N, 0, None, 0, H, R)
        return Y, (B.variants()[B.gemm_last_variant()], B.gemm_form_name(B.gemm_last_form()))
    Y, named = run()
    say(f"{M} x {N} x {K} tB={tB}: {named}")
    assert named in KERNELS
    force(*named)
    try:
        Z, again = run()
    finally:
        force(None)
    assert again == named and torch.equal(Y, Z)
