// Products whose rows do not share their weights: what the host and the kernels of the grouped calls agree on.
//
// Rows come in pieces that follow one another, their bounds in device memory: for piece e with rows a .. b - 1
//     C[a..b) = act(beta * C[a..b) + A[a..b) x B_id + bias_id)          (rows grouped by expert)
// or, with a second pair of operands, + H[a..b) x Up_id on weights B that all pieces share (adapters).  The weight gradient
// turns the pieces into the reduction: C_e = beta * C_e + A[a..b)^T x B[a..b).
//
// Bounds live in device memory, so the grid is the most tiles any bounds can give, every workgroup finds its own tile in
// them, and those left over end at once.  A bound outside 0 .. rows is moved to the nearer end and a piece that
// ends before it starts has no row, so whatever the offsets hold, no access leaves the matrices.
#pragma once
#include "bf16_tiles.hpp"
#include "launch_limits.hpp"
#include "variants.hpp"

namespace brg {

struct GroupArgs {
    int rows;                       // of A and C
    int groups;                     // bounds of group e: offsets[e], offsets[e + 1]; without offsets: e, e + 1
    const int64_t *offsets;
    const int64_t *ids;             // weights of group e: ids[e], or e itself
    int64_t weights;                // how many there are; a group whose number is outside them has none
    int cover;                      // 1: the rows before the first group and behind the last are pieces, too, without weights
    int max_tiles;                  // rows of tiles in the grid (forward)
    int64_t stride_b, stride_c, stride_bias;        // elements from one group's weights, result, bias to the next's
    int by_weights;                 // 1: adapters' own kernels take rows by their adapter (lowrank_first.hpp)
};

constexpr int kNoWeights = -1;

// Bounds i, i + 1, ... of the pieces, 0 <= i (any value behind the last).  All of them are requested together, under no
// condition of the lane's: one at a time they were 0.6 us each.
template <int COUNT>
__device__ __forceinline__ void piece_bounds(const GroupArgs &g, int i, int (&bound)[COUNT])
{
    i -= g.cover;
    int64_t v[COUNT];
    if (g.offsets) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            v[j] = g.offsets[i + j < 0 ? 0 : i + j < g.groups ? i + j : g.groups];
    } else {
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            v[j] = i + j < g.groups ? i + j : g.groups;
    }
#pragma unroll
    for (int j = 0; j < COUNT; ++j)
        bound[j] = i + j < 0 || v[j] < 0 ? 0 : v[j] >= g.rows || i + j > g.groups ? g.rows : (int)v[j];
}
__device__ __forceinline__ int pieces_of(const GroupArgs &g) { return g.groups + 2 * g.cover; }
// The number of a piece's weights, or kNoWeights.
__device__ __forceinline__ int piece_weights(const GroupArgs &g, int piece)
{
    const int e = piece - g.cover;
    if (e < 0 || e >= g.groups)
        return kNoWeights;
    const int64_t id = g.ids ? g.ids[e] : e;
    return id >= 0 && id < g.weights ? __builtin_amdgcn_readfirstlane((int)id) : kNoWeights;
}

// Sum of x over lanes 0 .. lane, without LDS (the row shifts and broadcasts of the data-parallel primitives).
__device__ __forceinline__ int wave_prefix_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);     // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);     // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);     // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);     // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);     // row_bcast:31 into rows 2 and 3
    return x;
}

struct GroupTile {
    int piece, weights;             // weights: their number, or kNoWeights
    int first, rows;                // of the piece
    int tm, tn;                     // tile of BM rows in it, tile of columns
};

// The tile of this workgroup.  Rows of tiles are numbered through all pieces; WALK: and walked as those of one matrix (tile_coords:
// every XCD has a contiguous run), else in the order of the grid, columns first.  False: there is none.  Every wave looks for
// itself, 256 pieces at a time, four in a lane: up to 256 of them cost one latency of memory and a prefix sum.
template <int BM, bool WALK = true>
__device__ __forceinline__ bool find_tile(const GroupArgs &g, int tiles_n, const Walk &walk, GroupTile &t, int block)
{
    const int lane = threadIdx.x & 63;
    const int pieces = pieces_of(g);
    int r = 0;
    auto place = [&](int total) {
        if (block >= total * tiles_n)
            return false;
        if constexpr (WALK) {
            tile_coords(block, total, tiles_n, walk, r, t.tn);
        } else {
            r = div_by(block, walk.by_tiles);       // (tiles_n of them)
            t.tn = block - r * tiles_n;
        }
        return true;
    };
    if (!g.offsets && !g.cover) {           // one row each
        if (!place(g.max_tiles))
            return false;
        t.piece = t.first = r;
        t.rows = 1;
        t.tm = 0;
        t.weights = piece_weights(g, r);
        return true;
    }
    int bound[5], tiles[4], own = 0, upto = 0;
    auto chunk = [&](int base) {
        piece_bounds(g, base + 4 * lane, bound);
        own = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            tiles[j] = base + 4 * lane + j < pieces && bound[j + 1] > bound[j] ? (bound[j + 1] - bound[j] + BM - 1) / BM : 0;
            own += tiles[j];
        }
        upto = wave_prefix_sum(own);
    };
    int total = 0;
    for (int base = 0; base < pieces; base += 256) {
        chunk(base);
        total += __builtin_amdgcn_readlane(upto, 63);
    }
    if (!place(total < g.max_tiles ? total : g.max_tiles))
        return false;
    int before = 0;
    for (int base = 0; base < pieces; base += 256) {
        if (pieces > 256)
            chunk(base);
        const int at = r - before - (upto - own);           // among this lane's tiles
        const uint64_t hit = __builtin_amdgcn_ballot_w64(at >= 0 && at < own);
        if (hit) {
            int piece = 0, first = bound[0], end = bound[1], tm = at;
#pragma unroll
            for (int j = 1; j < 4; ++j) {
                if (tm >= tiles[j - 1] && piece == j - 1) {
                    tm -= tiles[j - 1];
                    piece = j;
                    first = bound[j];
                    end = bound[j + 1];
                }
            }
            const int l = __builtin_ctzll(hit);
            t.piece = base + 4 * l + __builtin_amdgcn_readlane(piece, l);
            t.first = __builtin_amdgcn_readlane(first, l);
            t.rows = __builtin_amdgcn_readlane(end, l) - t.first;
            t.tm = __builtin_amdgcn_readlane(tm, l);
            t.weights = piece_weights(g, t.piece);
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}
template <int BM>
__device__ __forceinline__ bool find_tile(const GroupArgs &g, int tiles_n, const Walk &walk, GroupTile &t)
{
    return find_tile<BM>(g, tiles_n, walk, t, (int)blockIdx.x);
}

// The same for tiles of 256 rows of which a piece's last, where it holds at most 128, is a tile of 128 (`small`).  All tiles of 256 come
// first: they take longer, and the others fill the gaps at the end.
struct MixedTile {
    GroupTile t;
    bool small;                     // tm: in tiles of 128 rows, else of 256
};
// NARROW: tiles of 128 rows are also half as wide, 2 tiles_n of them in a row, in the order of the grid.
template <bool NARROW = false>
__device__ __forceinline__ bool find_mixed_tile(const GroupArgs &g, int tiles_n, const Walk &walk, MixedTile &out)
{
    const int lane = threadIdx.x & 63, pieces = pieces_of(g);
    int bound[5], big[4], own[2], upto[2];
    auto chunk = [&](int base) {
        piece_bounds(g, base + 4 * lane, bound);
        own[0] = own[1] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int rows = base + 4 * lane + j < pieces && bound[j + 1] > bound[j] ? bound[j + 1] - bound[j] : 0;
            big[j] = (rows + 127) / 256;
            own[0] += big[j];
            own[1] += rows > 256 * big[j];
        }
        upto[0] = wave_prefix_sum(own[0]);
        upto[1] = wave_prefix_sum(own[1]);
    };
    int total[2] = {0, 0};
    for (int base = 0; base < pieces; base += 256) {
        chunk(base);
        total[0] += __builtin_amdgcn_readlane(upto[0], 63);
        total[1] += __builtin_amdgcn_readlane(upto[1], 63);
    }
    total[0] = total[0] < g.max_tiles ? total[0] : g.max_tiles;
    total[1] = total[1] < g.max_tiles - total[0] ? total[1] : g.max_tiles - total[0];
    int block = (int)blockIdx.x, r;
    out.small = block >= total[0] * tiles_n;
    if (out.small)
        block -= total[0] * tiles_n;
    const int k = out.small ? 1 : 0;
    if (block >= total[k] * (NARROW && out.small ? 2 * tiles_n : tiles_n))
        return false;
    if (NARROW && out.small) {
        r = block / (2 * tiles_n);
        out.t.tn = block - r * (2 * tiles_n);
    } else {
        tile_coords(block, total[k], tiles_n, walk, r, out.t.tn);
    }
    int before = 0;
    for (int base = 0; base < pieces; base += 256) {
        if (pieces > 256)
            chunk(base);
        const int mine = out.small ? own[1] : own[0], at = r - before - ((out.small ? upto[1] : upto[0]) - mine);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(at >= 0 && at < mine);
        if (hit) {
            int piece = 0, first = 0, end = 0, tm = 0, left = at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int rows = bound[j + 1] - bound[j], tiles = base + 4 * lane + j >= pieces ? 0 : out.small ? rows > 256 * big[j] : big[j];
                if (left >= 0 && left < tiles) {
                    piece = j;
                    first = bound[j];
                    end = bound[j + 1];
                    tm = out.small ? 2 * big[j] : left;
                }
                left -= tiles;
            }
            const int l = __builtin_ctzll(hit);
            out.t.piece = base + 4 * l + __builtin_amdgcn_readlane(piece, l);
            out.t.first = __builtin_amdgcn_readlane(first, l);
            out.t.rows = __builtin_amdgcn_readlane(end, l) - out.t.first;
            out.t.tm = __builtin_amdgcn_readlane(tm, l);
            out.t.weights = piece_weights(g, out.t.piece);
            return true;
        }
        before += __builtin_amdgcn_readlane(out.small ? upto[1] : upto[0], 63);
    }
    return false;
}

// Weight gradients: the tile of group e's result, tiles_m x tiles_n of them a group, and the rows of its reduction.  Every XCD takes an
// eighth of every group's tiles, neighbours for its L2: groups are of different lengths, and a run of tiles that is one group leaves the XCDs
// of short groups idle (4096 rows in 8 groups, 4096 x 4096, a group for every XCD: 343 us).
__device__ __forceinline__ bool find_reduction(const GroupArgs &g, int tiles_m, int tiles_n, const Walk &walk, GroupTile &t)
{
    const int tiles = tiles_m * tiles_n, share = (tiles + 7) >> 3;
    const int at = (int)blockIdx.x >> 3;                // (walk.by_tiles divides by the share)
    t.piece = div_by(at, walk.by_tiles);
    const int xcd = (int)blockIdx.x & 7, tile = xcd * share + at - t.piece * share;
    if (t.piece >= g.groups || tile >= tiles)
        return false;
    // (every XCD begins at another group, so that they do not all multiply, and then all store, at the same time)
    t.piece += xcd * g.groups >> 3;
    t.piece -= t.piece >= g.groups ? g.groups : 0;
    group_walk(tile, tiles_m, tiles_n, walk, t.tm, t.tn);
    t.weights = t.piece;
    int bound[2];
    piece_bounds(g, t.piece, bound);
    t.first = __builtin_amdgcn_readfirstlane(bound[0]);
    const int end = __builtin_amdgcn_readfirstlane(bound[1]);
    t.rows = end > t.first ? end - t.first : 0;
    return true;
}

// A tile whose reduction is empty.
template <int BM, int BN, int NT>
__device__ __forceinline__ void store_empty_tile(const Epilogue &e, int64_t M, int64_t N, int tm, int tn)
{
    if (e.beta == 1.0f && !e.bias && !e.relu)
        return;
    for (int i = threadIdx.x; i < BM * BN; i += NT) {
        const int64_t m = (int64_t)tm * BM + i / BN, n = (int64_t)tn * BN + i % BN;
        if (m < M && n < N)
            epilogue_store(e, 0.0f, m, n);
    }
}

// Point an epilogue at a piece's rows and bias.
__device__ __forceinline__ void select_piece(Epilogue &e, const GroupArgs &g, const GroupTile &t)
{
    e.C = (char *)e.C + (int64_t)t.first * e.ldc * (e.c_f32 ? 4 : 2);
    if (e.bias)
        e.bias += (t.weights > 0 ? t.weights : 0) * g.stride_bias;
}

// ---- host side

// The second operands of a call with adapters, and what the first of its products is scaled with.
struct LowRank {
    const char *H;                  // rows x R
    int64_t ldh;
    const char *up;                 // R x N for every adapter, stored like the weights
    int64_t ld_up, stride_up;
    int64_t R;
};

struct GroupedCall {
    Problem p;                      // M: rows; B, bias and C of group 0
    GroupArgs g;
    bool narrow;                    // the first product of adapters: few columns,
    const float *factors;           // ... its sums scaled with the weights' own factor, or nullptr
    LowRank low;                    // R > 0: + H x up on weights that all rows share
};

// Raise a kernel's limit of dynamic LDS, once a thread.
inline hipError_t raise_lds(const void *kern, size_t lds, const void *(&configured)[32])
{
    for (const void *&k : configured) {
        if (k == kern)
            return hipSuccess;
        if (!k) {
            const hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e == hipSuccess)
                k = kern;
            return e;
        }
    }
    return hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

// What find_reduction takes from a launch's walk.
inline Walk reduction_walk(int tiles_m, int tiles_n)
{
    Walk w = make_walk(tiles_m, tiles_n, 1, 1, 1, (int64_t)kWalkRows * tiles_n);
    w.by_tiles = fastdiv(((int64_t)tiles_m * tiles_n + 7) / 8);
    return w;
}

// Most rows of tiles that pieces of `rows` rows in all can have.
inline int64_t most_row_tiles(int64_t rows, int64_t pieces, int bm)
{
    const int64_t by_piece = (rows + pieces * (bm - 1)) / bm;
    return rows < by_piece ? rows : by_piece;
}

// The kernels by what they take.  grouped_general.hip: any size, alignment and type.  grouped_duty.hip: the general kernel's divided
// tiles.  grouped_pingpong*.hip, grouped_stream*.hip: the tuned 16-bit kernels (tile: a GenTile).
hipError_t grouped_general(const GroupedCall &c);
hipError_t grouped_general_wgrad(const GroupedCall &c);
hipError_t grouped_duty(const GroupedCall &c, int tile);
hipError_t grouped_duty_wgrad(const GroupedCall &c);
hipError_t grouped_pingpong(const GroupedCall &c);
hipError_t grouped_pingpong_wgrad(const GroupedCall &c);
hipError_t grouped_stream(const GroupedCall &c, int tile);
hipError_t grouped_stream_wgrad(const GroupedCall &c, int tile);
hipError_t grouped_short_wgrad(const GroupedCall &c);       // grouped_wgrad.hip
constexpr int GEN_WIDE = GEN_TILES;     // 128 x 256
hipError_t adapters_pingpong(const GroupedCall &c);
hipError_t adapters_stream(const GroupedCall &c, int tile);
// lowrank.hip: the adapters' products as kernels of their own.
bool adapters_down_fits(const GroupedCall &c);
bool adapters_up_fits(const GroupedCall &c);
hipError_t adapters_down(const GroupedCall &c);
bool adapters_few_rows(const GroupedCall &c);
hipError_t adapters_down_and_sums(const GroupedCall &first, const GroupedCall &c, float *sums);
hipError_t adapters_up(const GroupedCall &c, const float *partial, int slices);
// adapters_beside.hip: H and the projection's sums (p) in one launch.
bool adapters_beside_fits(const GroupedCall &first, const Problem &p, const Plan &base);
hipError_t adapters_beside(const GroupedCall &first, const Problem &p, const Plan &base);

// grouped.hip.  The kernel a call takes, as the variant and form whose tile it has: V_BF16_PP256, V_BF16_STREAM128 (128 x 128),
// V_BF16_STREAM64 with form GEN_MID (128 x 64), V_BF16_STREAM32 with GEN_64 (64 x 64), V_BF16_128x128 (gradients:
// grouped_wgrad.hip), V_GENERIC with GEN_128, GEN_MID or GEN_64 (divided), GEN_32 (forward, rows that the tuned kernels do not
// take) or without a form (undivided).  Forced ones that do not take the call: BRGEMM_INVALID_ARG.
int plan_grouped(const GroupedCall &c, bool wgrad, int forced_variant, int forced_form, Plan *out);
hipError_t launch_grouped(GroupedCall &c, const Plan &plan);
hipError_t launch_grouped_wgrad(GroupedCall &c, const Plan &plan);
// A projection with adapters.  ADAPTERS_BLOCKS: the adapters as blocks of the projection's tiles (lowrank.hpp), whose kernel `base`
// is.  ADAPTERS_APART: the projection's sums into the workspace with the plan `base`, the adapters' behind it (lowrank.hip), H
// beside its tiles where those leave CUs free (adapters_beside.hip).  ADAPTERS_FEW_ROWS: the same, the sums from the launch that
// gives H (`base`: the general kernel, for want of a name).  ADAPTERS_GENERAL: both products in the general kernel.
enum AdaptersHow { ADAPTERS_BLOCKS, ADAPTERS_APART, ADAPTERS_FEW_ROWS, ADAPTERS_GENERAL };
struct AdaptersPlan {
    AdaptersHow how;
    Plan base;
};
int plan_adapters(const GroupedCall &c, size_t workspace_bytes, int forced_variant, int forced_form, AdaptersPlan *out);
// first: the call that gives H.
hipError_t launch_adapters_plan(GroupedCall &first, GroupedCall &c, const AdaptersPlan &plan, void *workspace, size_t workspace_bytes);

}  // namespace brg
