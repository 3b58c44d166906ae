"""Grouped calls that one launch does not hold, against the formula on the card (64 bits, a part of the columns at a time)."""
import pytest
import torch

from paper_2511_13764_amd import binding as B
from test_gpu_grouped import U, half_step, on_device, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K", [(2, 600000003), (8, 540000000)])
def test_weight_gradient_of_a_few_very_long_rows(N, K):
    say(f"wgrad of 3 rows, {N} x {K}")
    gen = torch.Generator(device="cuda").manual_seed(9)
    t = torch.bfloat16
    dY = torch.randn((3, N), device="cuda", generator=gen).to(t)
    X = torch.empty((3, K), dtype=t, device="cuda").normal_(generator=gen)
    dW = torch.full((N, K), float("nan"), dtype=t, device="cuda")
    B.gemm_grouped_wgrad(B.DTYPE_BF16, 3, N, K, 1, on_device([0, 3]), dY, N, X, K, 0.0, dW, K, N * K, 0)
    rel, tiny = half_step(t)
    for k in range(0, K, 1 << 22):
        x, y = X[:, None, k:k + (1 << 22)].double(), dY[:, :, None].double()
        ref, absolute = (y * x).sum(0), (y * x).abs().sum(0)
        err = (3 + 4) * U * absolute
        bad = ~((dW[:, k:k + (1 << 22)].double() - ref).abs() <= err + rel * (ref.abs() + err) + tiny)
        assert not bad.any(), (k, int(bad.sum()))
