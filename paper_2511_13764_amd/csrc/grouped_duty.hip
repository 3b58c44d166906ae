// Grouped products on the general kernel's tiles with the work divided by kind (general_duty.hpp): fp32, and 16-bit operands whose
// rows the global->LDS loads cannot read.
#include "general.hpp"
#include "grouped.hpp"

namespace brg {

namespace {

template <int KIND, int BM, int BN>
struct DutyShape {          // loading waves, sub-blocks in flight, workgroups on a CU: as duty_tile has them
    static constexpr bool WIDE = BN == 128;
    static constexpr int NLW = WIDE && KIND != KIND_F32 ? 8 : 4, DEPTH = WIDE || BM == 64 ? 4 : 3, PER_CU = WIDE ? 1 : 2;
    static constexpr int kThreads = (4 + NLW) * 64, kWaves = (4 + NLW) / 4 * PER_CU;
};

template <int KIND, bool B_KMAJ, int BM, int BN>
__global__ void __launch_bounds__((DutyShape<KIND, BM, BN>::kThreads), (DutyShape<KIND, BM, BN>::kWaves))
grouped_duty_kernel(GenArgs p, GroupArgs g)
{
    typedef DutyShape<KIND, BM, BN> D;
    constexpr int S = GenElem<KIND>::S;
    GroupTile t;
    if (!find_tile<BM>(g, p.tiles_n, p.walk, t))
        return;
    p.M = t.rows;
    select_piece(p.epi, g, t);
    general_duty_body<KIND, true, B_KMAJ, BM, BN, D::NLW, D::DEPTH>(p, p.A + (int64_t)t.first * p.lda * S, p.B + t.weights * g.stride_b * S, t.tm, t.tn, 0);
}

// (A reduction of one sub-block has no whole one for the loaders to repeat, and runs undivided.)
template <int KIND>
__global__ void __launch_bounds__(512, 4)
grouped_duty_wgrad_kernel(GenArgs p, GroupArgs g)
{
    typedef DutyShape<KIND, 64, 64> D;
    constexpr int S = GenElem<KIND>::S, SUB = GenElem<KIND>::SUB;
    static_assert(D::NLW == 4, "");
    GroupTile t;
    if (!find_reduction(g, p.tiles_m, p.tiles_n, p.walk, t))
        return;
    p.epi.C = (char *)p.epi.C + t.piece * g.stride_c * (p.epi.c_f32 ? 4 : 2);
    p.K = t.rows;
    p.walk.per = (p.K + SUB - 1) / SUB;
    const char *A = p.A + (int64_t)t.first * p.lda * S, *B = p.B + (int64_t)t.first * p.ldb * S;
    if (p.K == 0)
        store_empty_tile<64, 64, 512>(p.epi, p.M, p.N, t.tm, t.tn);
    else if (p.K <= SUB)
        general_body<KIND, false, false, 64, 64, 2, 2, 2, false, ROWS_NEAR>(p, A, B, t.tm, t.tn, 0);
    else
        general_duty_body<KIND, false, false, 64, 64, D::NLW, D::DEPTH>(p, A, B, t.tm, t.tn, 0);
}

template <int KIND, bool B_KMAJ, int BM, int BN>
hipError_t launch(const GroupedCall &c)
{
    typedef DutyConfig<KIND, BM, BN> Cfg;
    const Problem &p = c.p;
    GenArgs a = gen_args(p);
    a.tiles_n = (int)((p.N + BN - 1) / BN);
    a.walk = make_walk(1, a.tiles_n, 1, (p.K + GenElem<KIND>::SUB - 1) / GenElem<KIND>::SUB, 1, (int64_t)kWalkRows * a.tiles_n);
    GroupArgs g = c.g;
    g.max_tiles = (int)most_row_tiles(p.M, g.groups + 2 * g.cover, BM);
    auto kern = grouped_duty_kernel<KIND, B_KMAJ, BM, BN>;
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, Cfg::kLds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.max_tiles * a.tiles_n)), dim3(DutyShape<KIND, BM, BN>::kThreads), Cfg::kLds, p.stream, a, g);
    return hipGetLastError();
}

template <int KIND, bool B_KMAJ>
hipError_t launch_tile(const GroupedCall &c, int tile)
{
    return tile == GEN_128 ? launch<KIND, B_KMAJ, 128, 128>(c) : tile == GEN_MID ? launch<KIND, B_KMAJ, 128, 64>(c) : launch<KIND, B_KMAJ, 64, 64>(c);
}

template <int KIND>
hipError_t launch_wgrad(const GroupedCall &c)
{
    const Problem &p = c.p;
    GenArgs a = gen_args(p);
    a.tiles_m = (int)((p.M + 63) / 64);
    a.tiles_n = (int)((p.N + 63) / 64);
    a.walk = reduction_walk(a.tiles_m, a.tiles_n);
    const GroupArgs &g = c.g;
    constexpr size_t undivided = GenConfig<KIND, false, false, 64, 64, 2, 2, 2>::kLds, divided = DutyConfig<KIND, 64, 64>::kLds;
    constexpr size_t lds = undivided > divided ? undivided : divided;
    auto kern = grouped_duty_wgrad_kernel<KIND>;
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, lds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)reduction_grid((int64_t)a.tiles_m * a.tiles_n, g.groups)), dim3(512), lds, p.stream, a, g);
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_layout(const GroupedCall &c, int tile)
{
    return c.p.transB ? launch_tile<KIND, true>(c, tile) : launch_tile<KIND, false>(c, tile);
}

}  // namespace

hipError_t grouped_duty(const GroupedCall &c, int tile)
{
    return c.p.in_bf16 ? launch_layout<KIND_BF16>(c, tile) : c.p.in_f16 ? launch_layout<KIND_F16>(c, tile) : launch_layout<KIND_F32>(c, tile);
}

hipError_t grouped_duty_wgrad(const GroupedCall &c)
{
    return c.p.in_bf16 ? launch_wgrad<KIND_BF16>(c) : c.p.in_f16 ? launch_wgrad<KIND_F16>(c) : launch_wgrad<KIND_F32>(c);
}

}  // namespace brg
