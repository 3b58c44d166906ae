// Grouped products on the tuned 16-bit kernels: their bodies on the tile that a workgroup finds in the offsets, with the piece's rows
// as the matrix.  A group whose rows end inside a tile costs a whole one, so the plan (grouped.hip) takes the tile by the
// rows a group has on average.  Sums are one chain of fp32 additions over all of K (or a group's rows), also with an incomplete block:
// the totals that plain calls close off there (bf16_stream128.hpp) are not among these instances.
#pragma once
#include "bf16_pingpong.hpp"
#include "bf16_stream128.hpp"
#include "grouped.hpp"

namespace brg {

// Point a forward product at its piece.
__device__ __forceinline__ void select_piece(Bf16Args &p, const GroupArgs &g, const GroupTile &t)
{
    p.M = t.rows;
    p.A += (int64_t)t.first * p.lda;
    p.B += t.weights * g.stride_b;
    select_piece(p.epi, g, t);
}
// Point a weight gradient at its group: the rows are the reduction.
__device__ __forceinline__ void select_reduction(Bf16Args &p, const GroupArgs &g, const GroupTile &t)
{
    p.K = t.rows;
    p.walk.per = (p.K + BK - 1) / BK;
    p.A += (int64_t)t.first * p.lda;
    p.B += (int64_t)t.first * p.ldb;
    p.epi.C = (char *)p.epi.C + t.piece * g.stride_c * (p.epi.c_f32 ? 4 : 2);
}

// 256 x 256 tiles, and a group's last one, where at most 128 of its rows are there, as 128 x 256 of the streaming kernel, 0.6 of the time
// (4096 rows in 8 groups, 11008 x 4096: 439 us without them).
template <int B_LAY, int KIND, bool TAIL>
__global__ void __launch_bounds__(512)
grouped_pingpong_kernel(Bf16Args p, GroupArgs g)
{
    MixedTile m;
    if (!find_mixed_tile(g, p.tiles_n, p.walk, m))
        return;
    const GroupTile &t = m.t;
    select_piece(p, g, t);
    if (m.small) {
        stream128_body<true, B_LAY, KIND, 256, TAIL, 128, false, NoOffsets>(p, t.tm, t.tn, 0);
        return;
    }
    // Experts start far apart and columns a block apart, which leaves neighbours A's blocks in L2 (4096 rows in 8 groups, 11008 x 4096: all at
    // block 0 410 us, experts apart 395, columns too 381; 3 blocks between columns 392).
    if (p.rotate && !TAIL)
        p.rotate = (int)((uint32_t)(t.weights * 11LL + t.tn) % (uint32_t)(p.K / BK));
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool edge = (w >> 2) ? (int64_t)(t.tm + 1) * PP_BM > p.M : (int64_t)(t.tn + 1) * PP_BN > p.N;
    if (!edge)
        pp_body<true, B_LAY, true, false, KIND, false, TAIL, NoOffsets>(p, t.tm, t.tn, NoOffsets{});
    else
        pp_body<true, B_LAY, true, true, KIND, false, TAIL, NoOffsets>(p, t.tm, t.tn, NoOffsets{});
}

template <int KIND>
__global__ void __launch_bounds__(512)
grouped_pingpong_wgrad_kernel(Bf16Args p, GroupArgs g)
{
    GroupTile t;
    if (!find_reduction(g, p.tiles_m, p.tiles_n, p.walk, t))
        return;
    select_reduction(p, g, t);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool edge = (w >> 2) ? (int64_t)(t.tm + 1) * PP_BM > p.M : (int64_t)(t.tn + 1) * PP_BN > p.N;
    if (p.K == 0)
        store_empty_tile<PP_BM, PP_BN, 512>(p.epi, p.M, p.N, t.tm, t.tn);
    else if (p.K % BK != 0) {
        if (!edge)
            pp_body<false, LAY_MN, true, false, KIND, false, TAIL_ROWS_OFF>(p, t.tm, t.tn);
        else
            pp_body<false, LAY_MN, true, true, KIND, false, TAIL_ROWS_OFF>(p, t.tm, t.tn);
    } else {
        if (!edge)
            pp_body<false, LAY_MN, true, false, KIND, false, TAIL_NO>(p, t.tm, t.tn);
        else
            pp_body<false, LAY_MN, true, true, KIND, false, TAIL_NO>(p, t.tm, t.tn);
    }
}

template <int BM, int BN, int B_LAY, int KIND, bool TAIL>
__global__ void __launch_bounds__(512, BN == 64 ? 4 : 2)
grouped_stream_kernel(Bf16Args p, GroupArgs g)
{
    GroupTile t;
    if (!find_tile<BM>(g, p.tiles_n, p.walk, t))
        return;
    select_piece(p, g, t);
    stream128_body<true, B_LAY, KIND, BN, TAIL, BM, false, NoOffsets>(p, t.tm, t.tn, 0);
}

template <int BM, int BN, int KIND>
__global__ void __launch_bounds__(512, BN == 64 ? 4 : 2)
grouped_stream_wgrad_kernel(Bf16Args p, GroupArgs g)
{
    GroupTile t;
    if (!find_reduction(g, p.tiles_m, p.tiles_n, p.walk, t))
        return;
    select_reduction(p, g, t);
    if (p.K == 0)
        store_empty_tile<BM, BN, 512>(p.epi, p.M, p.N, t.tm, t.tn);
    else if (p.K % BK != 0)
        stream128_body<false, LAY_MN, KIND, BN, true, BM, false, NoOffsets, true>(p, t.tm, t.tn, 0);
    else
        stream128_body<false, LAY_MN, KIND, BN, false, BM, false, NoOffsets>(p, t.tm, t.tn, 0);
}

// A projection with adapters: the matrix's own tiles, with the segments' blocks in front.
template <int B_LAY, int KIND, bool TAIL>
__global__ void __launch_bounds__(512)
adapters_pingpong_kernel(Bf16Args p, GroupArgs g, LowRank low)
{
    int tm, tn;
    tile_coords(blockIdx.x, p.tiles_m, p.tiles_n, p.walk, tm, tn);
    p.rotate = 0;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool edge = (w >> 2) ? (int64_t)(tm + 1) * PP_BM > p.M : (int64_t)(tn + 1) * PP_BN > p.N;
    if (!edge)
        pp_body<true, B_LAY, true, false, KIND, false, TAIL>(p, tm, tn, LowBlocks{g, low});
    else
        pp_body<true, B_LAY, true, true, KIND, false, TAIL>(p, tm, tn, LowBlocks{g, low});
}

template <int BM, int BN, int B_LAY, int KIND, bool TAIL>
__global__ void __launch_bounds__(512, BN == 64 ? 4 : 2)
adapters_stream_kernel(Bf16Args p, GroupArgs g, LowRank low)
{
    int tile, slice, tm, tn;
    slice_major_coords(p.tiles_m * p.tiles_n, 1, p.walk, tile, slice);
    group_walk(tile, p.tiles_m, p.tiles_n, p.walk, tm, tn);
    stream128_body<true, B_LAY, KIND, BN, TAIL, BM, false>(p, tm, tn, 0, LowBlocks{g, low});
}

template <int BM, int BN>
inline hipError_t launch_adapters(void (*kern)(Bf16Args, GroupArgs, LowRank), const GroupedCall &c, size_t lds)
{
    const Problem &p = c.p;
    Bf16Args a;
    fill_common_args(a, p);
    a.tiles_m = (int)((p.M + BM - 1) / BM);
    a.tiles_n = (int)((p.N + BN - 1) / BN);
    a.walk = make_walk(a.tiles_m, a.tiles_n, 1, (p.K + BK - 1) / BK, 1, (int64_t)kWalkRows * a.tiles_n);
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, lds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.tiles_m * a.tiles_n)), dim3(512), lds, p.stream, a, c.g, c.low);
    return hipGetLastError();
}

template <int BM, int BN>
inline hipError_t launch_tuned(void (*kern)(Bf16Args, GroupArgs), const GroupedCall &c, bool wgrad, size_t lds)
{
    const Problem &p = c.p;
    Bf16Args a;
    fill_common_args(a, p);
    a.tiles_m = (int)((p.M + BM - 1) / BM);
    a.tiles_n = (int)((p.N + BN - 1) / BN);
    a.walk = wgrad ? reduction_walk(a.tiles_m, a.tiles_n) : make_walk(1, a.tiles_n, 1, (p.K + BK - 1) / BK, 1, (int64_t)kWalkRows * a.tiles_n);
    // (as rotate_blocks, for the weights of all groups)
    a.rotate = !wgrad && p.transB == 1 && c.g.groups * p.N * p.K >= ((int64_t)32 << 20);
    GroupArgs g = c.g;
    if (!wgrad)
        g.max_tiles = (int)most_row_tiles(p.M, g.groups + 2 * g.cover, BM);
    const int64_t grid = wgrad ? reduction_grid((int64_t)a.tiles_m * a.tiles_n, g.groups) : (int64_t)g.max_tiles * a.tiles_n;
    static thread_local const void *configured[32] = {nullptr};
    const hipError_t e = raise_lds((const void *)kern, lds, configured);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(512), lds, p.stream, a, g);
    return hipGetLastError();
}

}  // namespace brg
