"""CPU-only: images of every size may stand one behind the other, as gemm_mx4_bytes spaces them."""
import pytest

from paper_2511_13764_amd import binding as B
from test_mx4_route_host import P, grouped, lib, mx4, pack, unpack          # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("N,K", [(256, 256), (257, 256), (257, 257), (256, 257), (307, 608), (1, 1), (3, 512), (5, 513)])
def test_a_bank_of_images_one_behind_the_other(lib, N, K):      # noqa: F811
    """Without a row nothing is launched; the stride is looked at all the same."""
    size = B.gemm_mx4_bytes(N, K)
    assert grouped(M=0, N=N, K=K, lda=K, ldc=N, sW=size) == B.OK
    assert grouped(M=0, N=N, K=K, lda=K, ldc=N, sW=3 * size) == B.OK
    odd = size % 16 != 0
    for more, want in ((8, B.OK if odd else B.INVALID_ARG), (4, B.INVALID_ARG), (1, B.INVALID_ARG), (16, B.OK)):
        assert grouped(M=0, N=N, K=K, lda=K, ldc=N, sW=size + more) == want, more


def test_where_images_may_not_start(lib):       # noqa: F811
    """257 x 256 is 8 bytes beyond a multiple of 16: its neighbour starts there, and nothing starts in between."""
    for at in (P + 4, P + 12, P + 1):
        assert pack(rows=257, K=256, ldx=256, x_rows=257, image=at) == B.INVALID_ARG
        assert unpack(rows=257, K=256, ldo=256, image=at) == B.INVALID_ARG
        assert mx4(N=257, K=256, lda=256, ldc=257, W=at) == B.INVALID_ARG
        assert mx4(dt=B.DTYPE_MX4, M=257, K=256, A=at) == B.INVALID_ARG
        assert grouped(N=257, K=256, lda=256, ldc=257, W=at) == B.INVALID_ARG
    assert pack(rows=256, K=256, ldx=256, x_rows=256, image=P + 8) == B.INVALID_ARG
    assert mx4(N=256, K=256, lda=256, ldc=256, W=P + 8) == B.INVALID_ARG
