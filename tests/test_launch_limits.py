"""CPU-only checks of csrc/launch_limits.hpp, compiled for the host: calls that one launch does not hold end in parts that
cover them once."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2511_13764_amd import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_13764_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("clang++")


def compiled(tmp_path, body):
    src = tmp_path / "limits.cpp"
    src.write_text('#include "launch_limits.hpp"\n#include <cstdio>\n#include <cstdlib>\nusing namespace brg;\n' + body)
    exe = tmp_path / "limits"
    subprocess.run([CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return lambda *args: subprocess.run([str(exe), *map(str, args)], check=True, capture_output=True, text=True, timeout=60).stdout


@pytest.mark.skipif(CXX is None, reason="no host C++ compiler")
def test_parts_of_a_weight_gradient(tmp_path):
    """As launch_grouped_wgrad goes through them: always less than the whole, each within a launch, together all of it."""
    run = compiled(tmp_path, """
static long parts = 0;
static double area = 0;
static void go(int64_t M, int64_t N, int64_t groups, int depth)
{
    if (depth > 80 || M < 1 || N < 1 || groups < 1)
        exit(2);
    const ReductionPart p = reduction_part(M, N, groups);
    const int cut = (p.m != M) + (p.n != N) + (p.groups != groups);
    if (p.m > M || p.n > N || p.groups > groups || cut > 1)
        exit(3);
    if (cut == 0) {
        if (reduction_grid(((M + 63) / 64) * ((N + 63) / 64), groups) * 512 > 0xffffffffLL)
            exit(4);
        ++parts;
        area += (double)M * N * groups;
        return;
    }
    if ((p.m != M && p.m % 256) || (p.n != N && p.n % 256))
        exit(5);
    go(p.m, p.n, p.groups, depth + 1);
    go(p.m != M ? M - p.m : M, p.n != N ? N - p.n : N, p.groups != groups ? groups - p.groups : groups, depth + 1);
}
int main(int, char **a)
{
    const int64_t M = atoll(a[1]), N = atoll(a[2]), G = atoll(a[3]);
    go(M, N, G, 0);
    printf("%ld %d", parts, area == (double)M * N * G);
}
""")
    most = (1 << 31) - 1
    # (64 x 600e6: 9.375e6 tiles of 64 x 64 where 8388607 workgroups are a launch; 256 x 200e6: 12.5e6; 300 x 200e6: 15.6e6; 185344: 2896^2)
    for M, N, groups, parts in ((64, 600000000, 1, 2), (256, 200000000, 1, 2), (300, 200000000, 1, 2), (2, 536870400, 1, 1),
                                (1, most, 1, None), (most, 1, 1, None), (most, 200, 1, None), (185344, 185344, 1, 1), (185345, 185345, 1, 2),
                                (1 << 20, 1 << 20, 3, None), (4096, 4096, 3000, None), (1, 1, 1 << 22, None), (64, 64, 8, 1)):
        got, whole = run(M, N, groups).split()
        assert whole == "1" and (parts is None or int(got) == parts), (M, N, groups, got, whole)


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="its operands are not there")
@pytest.mark.parametrize("N,K", [(64, 600000000), (256, 200000000), (300, 200000000), (2, 536870400)])
def test_a_weight_gradient_of_long_rows_returns(N, K):
    """... without a GPU with the launch's error: the parts come to an end."""
    code = ("from paper_2511_13764_amd import binding as B; P = 4096\n"
            f"print(B.gemm_grouped_wgrad(1, 64, {N}, {K}, 1, P, P, {N}, P, {K}, 0.0, P, {K}, {N * K}, 1, stream=0, check=False))")
    env = {**os.environ, "HIP_VISIBLE_DEVICES": "-1"}
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(CSRC)), env=env, capture_output=True, text=True,
                       timeout=110)
    assert r.returncode == 0 and int(r.stdout) == B.HIP_ERROR, (r.returncode, r.stdout, r.stderr[-500:])


@pytest.mark.skipif(CXX is None, reason="no host C++ compiler")
def test_first_products_that_a_launch_holds(tmp_path):
    """Tiles of H and the workgroups beside them, 512 threads each, within 2^32 threads."""
    run = compiled(tmp_path, """
int main(int, char **a) { printf("%d", (int)first_product_fits(atoll(a[1]), atoll(a[2]), atoll(a[3]))); }
""")
    most = (1 << 31) - 1
    # 16 rows with an adapter each beside a projection of 16 columns a workgroup: 2^27 columns are 2^23 workgroups, one launch 2^23 - 1
    for tiles, rank, beside, fits in ((16, 16, 4096 // 16, 1), (16, 16, (1 << 23) - 17, 1), (16, 16, (1 << 23) - 16, 0), (1, 16, 200000000 // 16, 0),
                                      (16, 33, (1 << 23) - 49, 1), (16, 33, (1 << 23) - 48, 0), ((1 << 23) - 1, 1, 0, 1), ((1 << 23) - 1, 16, 1, 0),
                                      (most, most, most, 0), (0, 16, 0, 1)):
        assert int(run(tiles, rank, beside)) == fits, (tiles, rank, beside)
    assert ((1 << 23) - 1) * 512 < 1 << 32 <= (1 << 23) * 512


def test_more_groups_than_the_kernels_count():
    """The search for a workgroup's tile counts groups in 32 bits, up to 256 past the last: it would never end."""
    P = 4096                # (M = 0: nothing is launched)
    for more, code in ((0, B.OK), (1, B.INVALID_ARG), (1024, B.INVALID_ARG)):
        G = B.MOST_GROUPS + more
        assert B.gemm_grouped(B.DTYPE_BF16, 1, 0, 8, 24, G, P, P, 24, P, 24, 192, 0.0, P, 8, 0, stream=0, check=False) == code
        assert B.gemm_grouped_wgrad(B.DTYPE_BF16, 8, 0, 24, G, P, P, 8, P, 24, 0.0, P, 24, 192, 0, stream=0, check=False) == code
        assert B.gemm_adapters(B.DTYPE_BF16, 1, 0, 8, 24, 4, G, P, P, 3, P, 24, P, 24, P, 24, 96, P, 4, 32, P, 0.0, P, 8, 0, None, 0, P, 4,
                               stream=0, check=False) == code
    assert B.MOST_GROUPS + 2 + 2 * 256 < 1 << 31
