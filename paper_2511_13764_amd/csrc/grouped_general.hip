// Grouped products of any size, alignment and type: the general kernel's 64 x 64 tile (general.hpp) on one piece's rows, its
// 32 x 32 tile for the narrow first product of adapters, and the 64 x 64 tile with both operands along m and n for the
// weight gradients.
#include "general.hpp"
#include "grouped.hpp"

namespace brg {

namespace {

struct Factor {
    static constexpr bool kSecond = false, kFactor = true;
    float factor;
};
struct Second {
    static constexpr bool kSecond = true, kFactor = false;
    const char *A, *B;
    int64_t lda, ldb, K;
};

constexpr int EXTRA_NONE = 0, EXTRA_FACTOR = 1, EXTRA_SECOND = 2;

template <int KIND, bool B_KMAJ, int BM, int ROWS, int EXTRA>
__global__ void __launch_bounds__(512, BM == 64 ? 4 : 2)
grouped_general_kernel(GenArgs p, GroupArgs g, const float *factors, LowRank low)
{
    constexpr int S = GenElem<KIND>::S, WG = BM == 64 ? 2 : 1, KW = BM == 64 ? 2 : 8;
    GroupTile t;
    if (!find_tile<BM>(g, p.tiles_n, p.walk, t))
        return;
    p.M = t.rows;
    select_piece(p.epi, g, t);
    const bool none = t.weights == kNoWeights;
    if (p.K == 0 || (none && EXTRA != EXTRA_SECOND)) {
        store_empty_tile<BM, BM, 512>(p.epi, p.M, p.N, t.tm, t.tn);
        return;
    }
    const char *A = p.A + (int64_t)t.first * p.lda * S, *B = p.B;
    if constexpr (EXTRA == EXTRA_SECOND) {
        const Second extra{low.H + (int64_t)t.first * low.ldh * S, low.up + (none ? 0 : t.weights) * low.stride_up * S, low.ldh,
                           low.ld_up, none ? 0 : low.R};
        general_body<KIND, true, B_KMAJ, BM, BM, WG, WG, KW, false, ROWS>(p, A, B, t.tm, t.tn, 0, extra);
    } else {
        B += t.weights * g.stride_b * S;
        if constexpr (EXTRA == EXTRA_FACTOR)
            general_body<KIND, true, B_KMAJ, BM, BM, WG, WG, KW, false, ROWS>(p, A, B, t.tm, t.tn, 0, Factor{factors ? factors[t.weights] : 1.0f});
        else
            general_body<KIND, true, B_KMAJ, BM, BM, WG, WG, KW, false, ROWS>(p, A, B, t.tm, t.tn, 0);
    }
}

template <int KIND, int ROWS>
__global__ void __launch_bounds__(512, 4)
grouped_general_wgrad_kernel(GenArgs p, GroupArgs g)
{
    constexpr int S = GenElem<KIND>::S;
    GroupTile t;
    if (!find_reduction(g, p.tiles_m, p.tiles_n, p.walk, t))
        return;
    p.epi.C = (char *)p.epi.C + t.piece * g.stride_c * (p.epi.c_f32 ? 4 : 2);
    p.K = t.rows;
    p.walk.per = (p.K + GenElem<KIND>::SUB - 1) / GenElem<KIND>::SUB;
    if (p.K == 0) {
        store_empty_tile<64, 64, 512>(p.epi, p.M, p.N, t.tm, t.tn);
        return;
    }
    general_body<KIND, false, false, 64, 64, 2, 2, 2, false, ROWS>(p, p.A + (int64_t)t.first * p.lda * S, p.B + (int64_t)t.first * p.ldb * S,
                                                                    t.tm, t.tn, 0);
}

template <int KIND, bool B_KMAJ, int BM, int ROWS, int EXTRA>
hipError_t launch(const GroupedCall &c)
{
    typedef GenConfig<KIND, true, B_KMAJ, BM, BM, BM == 64 ? 2 : 1, BM == 64 ? 2 : 1, BM == 64 ? 2 : 8> Cfg;
    static_assert(Cfg::NT == 512, "");
    const Problem &p = c.p;
    GenArgs a = gen_args(p);
    a.tiles_n = (int)((p.N + BM - 1) / BM);
    a.walk = make_walk(1, a.tiles_n, 1, (p.K + GenElem<KIND>::SUB - 1) / GenElem<KIND>::SUB, 1, (int64_t)kWalkRows * a.tiles_n);
    GroupArgs g = c.g;
    g.max_tiles = (int)most_row_tiles(p.M, g.groups + 2 * g.cover, BM);
    auto kern = grouped_general_kernel<KIND, B_KMAJ, BM, ROWS, EXTRA>;
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, Cfg::kLds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.max_tiles * a.tiles_n)), dim3(512), Cfg::kLds, p.stream, a, g, c.factors, c.low);
    return hipGetLastError();
}

// Runs shorter than a chunk are gathered, and rows far apart need 64-bit places: the same instances.
inline bool plain_rows(const GroupedCall &c, int tile)
{
    const Problem &p = c.p;
    const int64_t chunk = in_16bit(p) ? 8 : 4;
    Problem q = p;
    q.K = c.low.R; q.lda = c.low.ldh; q.ldb = c.low.ld_up;
    return !general_short_runs(p) && general_offsets_fit(p, tile) && (c.low.R == 0 || (c.low.R >= chunk && general_offsets_fit(q, tile)));
}

template <int KIND, bool B_KMAJ>
hipError_t launch_rows(const GroupedCall &c)
{
    if (c.low.R > 0)
        return plain_rows(c, GEN_64) ? launch<KIND, B_KMAJ, 64, ROWS_NEAR, EXTRA_SECOND>(c) : launch<KIND, B_KMAJ, 64, ROWS_SHORT, EXTRA_SECOND>(c);
    if (c.narrow)
        return plain_rows(c, GEN_32) ? launch<KIND, B_KMAJ, 32, ROWS_NEAR, EXTRA_FACTOR>(c) : launch<KIND, B_KMAJ, 32, ROWS_SHORT, EXTRA_FACTOR>(c);
    return plain_rows(c, GEN_64) ? launch<KIND, B_KMAJ, 64, ROWS_NEAR, EXTRA_NONE>(c) : launch<KIND, B_KMAJ, 64, ROWS_SHORT, EXTRA_NONE>(c);
}

template <int KIND, int ROWS>
hipError_t launch_wgrad(const GroupedCall &c)
{
    typedef GenConfig<KIND, false, false, 64, 64, 2, 2, 2> Cfg;
    const Problem &p = c.p;
    GenArgs a = gen_args(p);
    a.tiles_m = (int)((p.M + 63) / 64);
    a.tiles_n = (int)((p.N + 63) / 64);
    a.walk = reduction_walk(a.tiles_m, a.tiles_n);
    const GroupArgs &g = c.g;
    auto kern = grouped_general_wgrad_kernel<KIND, ROWS>;
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, Cfg::kLds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)reduction_grid((int64_t)a.tiles_m * a.tiles_n, g.groups)), dim3(512), Cfg::kLds, p.stream, a, g);
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_wgrad_rows(const GroupedCall &c)
{
    const bool plain = !general_short_runs(c.p) && general_offsets_fit(c.p, GEN_64);
    return plain ? launch_wgrad<KIND, ROWS_NEAR>(c) : launch_wgrad<KIND, ROWS_SHORT>(c);
}

template <int KIND>
hipError_t launch_layout(const GroupedCall &c)
{
    return c.p.transB ? launch_rows<KIND, true>(c) : launch_rows<KIND, false>(c);
}

}  // namespace

hipError_t grouped_general(const GroupedCall &c)
{
    return c.p.in_bf16 ? launch_layout<KIND_BF16>(c) : c.p.in_f16 ? launch_layout<KIND_F16>(c) : launch_layout<KIND_F32>(c);
}

hipError_t grouped_general_wgrad(const GroupedCall &c)
{
    return c.p.in_bf16 ? launch_wgrad_rows<KIND_BF16>(c) : c.p.in_f16 ? launch_wgrad_rows<KIND_F16>(c) : launch_wgrad_rows<KIND_F32>(c);
}

}  // namespace brg
