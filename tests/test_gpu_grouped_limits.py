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


def test_adapters_of_one_row_and_very_many_columns():
    """More columns than one launch has workgroups of 16 of them for."""
    M, N, K, R = 1, (1 << 27) + 1000, 64, 8
    say(f"adapters of {M} row, {N} x {K}, rank {R}")
    gen = torch.Generator(device="cuda").manual_seed(10)
    t = torch.bfloat16

    def normal(*shape):
        return torch.empty(shape, dtype=t, device="cuda").normal_(generator=gen)
    X, W, down, up = normal(M, K), normal(N, K), normal(2, R, K), normal(2, N, R)
    Y, H = torch.full((M, N), float("nan"), dtype=t, device="cuda"), torch.empty((M, R), dtype=t, device="cuda")
    ws = torch.empty(4 * M * N + 512, dtype=torch.uint8, device="cuda")
    B.gemm_adapters(B.DTYPE_BF16, 1, M, N, K, R, M, None, on_device([1]), 2, X, K, W, K, down, K, R * K, up, R, N * R, None, 0.0, Y, N,
                    0, None, 0, H, R, workspace=ws)
    rel, tiny = half_step(t)
    terms = down[1].double() * X.double()
    h, h_abs = terms.sum(1), terms.abs().sum(1)
    h_off = (K + 6) * U * h_abs + rel * h.abs() * (1 + K * U) + tiny
    assert ((H[0].double() - h).abs() <= h_off).all()
    for n in range(0, N, 1 << 20):
        w, u = W[n:n + (1 << 20)].double() * X.double(), up[1, n:n + (1 << 20)].double()
        ref, absolute = w.sum(1) + (u * h).sum(1), w.abs().sum(1) + (u * h).abs().sum(1)
        err = (K + R + 4) * U * absolute + 1.01 * (u.abs() * h_off).sum(1)
        bad = ~((Y[0, n:n + (1 << 20)].double() - ref).abs() <= err + rel * (ref.abs() + err) + tiny)
        assert not bad.any(), (n, int(bad.sum()))
