// H beside the projection's tiles in one launch.  Where segments of a few rows take adapters' second product out of the tiles
// (lowrank.hpp), the projection's sums and H need nothing of each other, and a projection of less than 256 tiles leaves CUs idle
// for longer than H takes in a launch of its own: 611 rows in 130 segments, 4096 x 4096, ranks of 64: 34.6 us on 160 of 256 CUs
// after 16.6 on all of them, the whole call 75.8 us and 59.3 so; 604 rows in 60 segments, 4584 x 2304, ranks of 16: 40.0 and 34.9.
// The projection's workgroups come first.
#include "grouped_tuned.hpp"
#include "lowrank_first.hpp"

namespace brg {

namespace {

template <int BM, int BN, bool KMAJ, int KIND, int RT>
__global__ void __launch_bounds__(512, BN == 64 ? 4 : 2)
adapters_beside_kernel(Bf16Args p, FirstArgs f, GroupArgs g)
{
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    static_assert(FIRST_WAVES == 8 && FIRST_WAVES * FirstLds<KIND, KMAJ, 1, RT>::kWave <= S128<BN, BM>::kLds, "one launch for both");
    const int tiles = p.tiles_m * p.tiles_n;
    if ((int)blockIdx.x >= tiles) {
        first_tile<KIND, KMAJ, RT, true>(f, g, (LDS_AS char *)smem_generic, (int)blockIdx.x - tiles);
        return;
    }
    int tile, slice, tm, tn;
    slice_major_coords(tiles, 1, p.walk, tile, slice);
    group_walk(tile, p.tiles_m, p.tiles_n, p.walk, tm, tn);
    stream128_body<true, KMAJ ? LAY_K : LAY_MN, KIND, BN, false, BM, false, NoOffsets>(p, tm, tn, 0);
}

template <int BM, int BN, bool KMAJ, int KIND, int RT>
hipError_t launch(const GroupedCall &first, const Problem &p)
{
    Bf16Args a;
    fill_common_args(a, p);
    a.tiles_m = (int)((p.M + BM - 1) / BM);
    a.tiles_n = (int)((p.N + BN - 1) / BN);
    a.walk = make_walk(a.tiles_m, a.tiles_n, 1, p.K / BK, 1, (int64_t)kWalkRows * a.tiles_n);
    FirstArgs f = first_args(first);
    GroupArgs g;
    const int more = first_grid(first, RT, f, g);
    constexpr size_t lds = S128<BN, BM>::kLds;
    static thread_local const void *configured[32] = {nullptr};
    auto kern = adapters_beside_kernel<BM, BN, KMAJ, KIND, RT>;
    const hipError_t e = raise_lds((const void *)kern, lds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.tiles_m * a.tiles_n + more)), dim3(512), lds, p.stream, a, f, g);
    return hipGetLastError();
}

template <int BM, int BN, int KIND>
hipError_t launch_rank(const GroupedCall &first, const Problem &p)
{
    if (p.transB == 0)
        return launch<BM, BN, false, KIND, 2>(first, p);
    return first.p.N > 16 ? launch<BM, BN, true, KIND, 2>(first, p) : launch<BM, BN, true, KIND, 1>(first, p);
}

template <int BM, int BN>
hipError_t launch_kind(const GroupedCall &first, const Problem &p)
{
    return p.in_f16 ? launch_rank<BM, BN, KIND_F16>(first, p) : launch_rank<BM, BN, KIND_BF16>(first, p);
}

}  // namespace

// base: the projection's plan.  Its tiles leave CUs or halves of them free, and its reduction has no incomplete block.
bool adapters_beside_fits(const GroupedCall &first, const Problem &p, const Plan &base)
{
    const int bm = base.variant == V_BF16_STREAM32 ? 64 : 128, bn = base.variant == V_BF16_STREAM128 ? 128 : 64;
    const bool is = base.variant == V_BF16_STREAM128 ? base.form < 0 : base.variant == V_BF16_STREAM64 ? base.form == GEN_MID
                    : base.variant == V_BF16_STREAM32 && base.form == GEN_64;
    const int64_t tiles = ((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn);
    return is && base.split == 1 && in_16bit(p) && p.K % BK == 0 && bf16_rows_eligible(p) && (p.transB || first.p.N % 8 == 0) && adapters_down_fits(first) &&
           tiles < (bn == 128 ? 256 : 512) && first_product_fits(most_row_tiles(first.p.M, first.g.groups + 2 * first.g.cover, 16), first.p.N, tiles);
}

hipError_t adapters_beside(const GroupedCall &first, const Problem &p, const Plan &base)
{
    return base.variant == V_BF16_STREAM128 ? launch_kind<128, 128>(first, p) : base.variant == V_BF16_STREAM64 ? launch_kind<128, 64>(first, p)
           : launch_kind<64, 64>(first, p);
}

}  // namespace brg
