"""Up to 32 rows that are taken by their adapter, in the launch that also gives the projection's sums."""
import pytest

from test_gpu_adapters_beside import workspace
from test_gpu_grouped import run_adapters

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tB", [1, 0])
@pytest.mark.parametrize("M,bank,R", [(16, 1, 600), (17, 1, 600), (17, 2, 640), (31, 1, 320), (31, 2, 330), (32, 1, 320), (32, 2, 330), (32, 8, 520)])
def test_few_rows_taken_by_their_adapter(M, bank, R, tB):
    """Widths and ranks at which that saves 30 MB and 2 MB an adapter of reading: 2 (M - (M + 15 (bank + 1)) / 16) R (N + K) bytes."""
    N, K = 1000, 1064
    assert 2.0 * (M - (M + 15 * (bank + 1)) // 16) * R * (N + K - 3) > 30e6 + 2e6 * bank and M >= 4 * bank
    for ids in ([(i * i + i // 7) % (bank + 2) - 1 for i in range(M)], [bank - 1] * M, [-1] * (M - 1) + [0]):
        run_adapters("bf16", tB, [1] * M, ids, bank, R, N, K, per_row=True, workspace=workspace(), bias=True, relu=True)
    ids = [(5 * i) % (bank + 1) for i in range(M)]                          # (`bank` is none)
    run_adapters("f16", tB, [1] * M, ids, bank, R, 1003, 1061, per_row=True, workspace=workspace(), beta=0.5, c32=True)
