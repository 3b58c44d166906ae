"""fp32 experts of few rows: 32 x 32 tiles whose waves share the reduction."""
import pytest

from paper_2511_13764_amd import binding as B
from test_gpu_grouped import GENERIC, run_grouped, run_wgrad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tB", [0, 1])
def test_small_tiles(tB):
    sizes = [0, 1, 31, 0, 32, 33, 7, 130, 0]
    for N, K in ((264, 256), (520, 328), (203, 137), (31, 33), (1, 1), (8, 1000)):
        assert run_grouped("f32", tB, sizes, N, K, variant=GENERIC, form="32x32", bias=N == 264, relu=K == 328, lead=1, behind=2) == (GENERIC, "32x32")
    run_grouped("f32", tB, sizes, 264, 456, variant=GENERIC, form="32x32", beta=0.5, pads=(3, 5, 2), gap=7, a_lead=1)
    run_grouped("f32", tB, [3, 0, 70], 40, 0, variant=GENERIC, form="32x32", bias=True, relu=True)
    run_grouped("f32", tB, [i % 3 for i in range(140)], 72, 256, variant=GENERIC, form="32x32")


def test_the_plan_takes_them_where_larger_ones_leave_cus_idle():
    for rows in ([4, 4, 4, 4], [1, 0, 0, 0], [60, 40, 0, 3]):
        assert run_grouped("f32", 1, rows, 512, 1024) == (GENERIC, "32x32")
    assert run_grouped("f32", 1, [900, 300, 300, 100], 1024, 512)[1] != "32x32"


def test_not_for_gradients_and_16_bits():
    for call in (lambda: run_wgrad("f32", [3, 70], 64, 64, variant=GENERIC, form="32x32"),
                 lambda: run_grouped("bf16", 1, [3, 70], 64, 256, variant=GENERIC, form="32x32")):
        with pytest.raises(B.BrgemmError) as e:
            call()
        assert e.value.code == B.INVALID_ARG


@pytest.mark.parametrize("dtype,tB", [("bf16", 0), ("bf16", 1), ("f16", 1)])
def test_small_tiles_of_unaligned_rows(dtype, tB):
    """Rows of 16-bit values that the tuned kernels cannot read."""
    sizes = [0, 1, 31, 0, 32, 33, 7, 130, 0]
    for N, K in ((203, 137), (31, 65), (1, 1), (9, 1001)):
        assert run_grouped(dtype, tB, sizes, N, K, variant=GENERIC, form="32x32", bias=K == 137, relu=K == 137, lead=1, behind=2) == (GENERIC, "32x32")
    run_grouped(dtype, tB, sizes, 75, 300, variant=GENERIC, form="32x32", beta=0.5, c32=True, pads=(3, 5, 2), gap=7, a_lead=1)
    assert run_grouped(dtype, tB, [4, 0, 9, 3], 701, 1333) == (GENERIC, "32x32")
    assert run_grouped(dtype, tB, [300, 200, 9, 130], 701, 333)[1] != "32x32"
