// The second product of adapters, Y += H x up_a, inside the tuned 16-bit kernels: every segment of rows that a tile holds is one
// or more blocks of the reduction, its rows of H (zeros for the tile's other rows) times its adapter's columns of up.  The blocks
// come first, through registers, in the LDS images that the kernel's own blocks have; so Y is summed in fp32 and rounded once, and
// nothing of size M x N is read or written for the adapters.
//
// A block's products reach its segment's rows alone (low_products): with zeros of H for the tile's other rows in one matrix product,
// an infinity or NaN in one adapter's up would be NaN in all of them.
//
// What it costs: a block of 64 of the rank for each segment in a tile, latency-bound (a load, a write to LDS, a barrier).  Segments
// of a few rows would make that most of the call: they go another way (lowrank.hip).
#pragma once
#include "grouped.hpp"

namespace brg {

struct NoLow {
    static constexpr bool kBlocks = false, kOffsets = true;         // the kernels' own calls may have tile offsets
};
struct NoOffsets {
    static constexpr bool kBlocks = false, kOffsets = false;        // rows grouped by their weights
};

// 8 consecutive 16-bit values of which `count` exist (zeros for the others); any alignment.
typedef uint32_t low_u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ gu32x4 low_chunk(const uint16_t *p, int count)
{
    gu32x4 v = {0, 0, 0, 0};
    if (count >= 8) {
        v = *(const low_u32x4_any2 *)p;
    } else if (count > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < count)
                v[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
    }
    return v;
}

// The blocks of one tile, in order.  Every wave keeps its own cursor: 64 segments at a time in its lanes.
struct LowBlocks {
    static constexpr bool kBlocks = true, kOffsets = false;
    const GroupArgs &g;
    const LowRank &low;
    int m0, m1;                     // rows of the tile
    int base;                       // segments base .. base + 63 are in the lanes
    uint64_t left;                  // those of them that are still to come
    int lo_l, hi_l, id_l;
    int lo, hi, id, r0;             // this block: rows lo .. hi - 1, adapter, first of the rank

    __device__ __forceinline__ void look(int first)
    {
        base = first;
        const int i = first + (int)(threadIdx.x & 63);
        const bool is = i < g.groups;
        int bound[2];
        piece_bounds(g, i + g.cover, bound);
        lo_l = bound[0];
        hi_l = bound[1];
        int64_t a = i;
        if (g.ids)
            a = g.ids[is ? i : 0];
        const bool has = a >= 0 && a < g.weights;
        id_l = has ? (int)a : 0;
        left = __builtin_amdgcn_ballot_w64(is && has && lo_l < hi_l && lo_l < m1 && hi_l > m0);
    }
    // How many blocks there are; leaves the cursor in front of the first.
    __device__ __forceinline__ int begin(int64_t tile_m0, int rows)
    {
        m0 = (int)tile_m0;
        m1 = (int)(tile_m0 + rows < g.rows ? tile_m0 + rows : g.rows);
        int segments = 0;
        left = 0;
        for (int first = 0; first < g.groups; first += 64) {
            look(first);
            segments += __builtin_popcountll(left);
        }
        if (g.groups > 64)
            look(0);
        r0 = (int)low.R;
        return segments * (int)((low.R + 63) / 64);
    }
    // On to the next block (there is one).
    __device__ __forceinline__ void next()
    {
        r0 += 64;
        if (r0 < (int)low.R)
            return;
        while (!left)
            look(base + 64);
        const int l = __builtin_ctzll(left);
        left &= left - 1;
        lo = __builtin_amdgcn_readlane(lo_l, l);
        hi = __builtin_amdgcn_readlane(hi_l, l);
        id = __builtin_amdgcn_readlane(id_l, l);
        r0 = 0;
    }
    // Before the first: a block of all rows that is not of these.
    __device__ __forceinline__ void take_all()
    {
        lo = 0;
        hi = g.rows;
    }
    // This block into the images of A (BM rows, k-contiguous) and B (BN columns from n0 on), by NT threads.
    template <int BM, int BN, int B_LAY, int NT, class BTile>
    __device__ __forceinline__ void stage(LDS_AS char *at, LDS_AS char *bt, int tid, int64_t n0, int64_t N) const
    {
        const uint16_t *H = (const uint16_t *)low.H, *up = (const uint16_t *)low.up + id * low.stride_up;
        const int ranks = (int)low.R - r0;          // of this block and those behind it
        gu32x4 a[BM * 8 / NT], b[BN * 8 / NT];
#pragma unroll
        for (int j = 0; j < BM * 8 / NT; ++j) {
            const int row = m0 + (j * NT + tid) / 8, c = (j * NT + tid) % 8;
            a[j] = low_chunk(H + (int64_t)row * low.ldh + r0 + 8 * c, row >= lo && row < hi ? ranks - 8 * c : 0);
        }
#pragma unroll
        for (int j = 0; j < BN * 8 / NT; ++j) {
            const int idx = j * NT + tid;
            if constexpr (B_LAY == LAY_K) {
                const int64_t n = n0 + idx / 8;
                b[j] = low_chunk(up + n * low.ld_up + r0 + 8 * (idx % 8), n < N ? ranks - 8 * (idx % 8) : 0);
            } else {
                const int kr = idx / (BN / 8);
                const int64_t n = n0 + 8 * (idx % (BN / 8)), cols = N - n;
                b[j] = low_chunk(up + (int64_t)(r0 + kr) * low.ld_up + n, kr < ranks && cols > 0 ? (cols < 8 ? (int)cols : 8) : 0);
            }
        }
#pragma unroll
        for (int j = 0; j < BM * 8 / NT; ++j) {
            const int row = (j * NT + tid) / 8, c = (j * NT + tid) % 8;
            *(LDS_AS gu32x4 *)(at + row * 128 + ((c ^ ((row >> 1) & 7)) << 4)) = a[j];
        }
#pragma unroll
        for (int j = 0; j < BN * 8 / NT; ++j) {
            const int idx = j * NT + tid;
            if constexpr (B_LAY == LAY_K) {
                const int row = idx / 8, c = idx % 8;
                *(LDS_AS gu32x4 *)(bt + row * 128 + ((c ^ ((row >> 1) & 7)) << 4)) = b[j];
            } else {
                const int kr = idx / (BN / 8), c = idx % (BN / 8);
                *(LDS_AS gu32x4 *)(bt + kr * BTile::kRowBytes + ((c ^ BTile::swz(kr)) << 4)) = b[j];
            }
        }
    }
};

// A staged block's products, added to a wave's sums: TM times 16 rows from `row` on, of the lane's row l % 16 of them each, TN times 16
// columns.  They are summed apart, four registers at a time, and added to the rows of the block's segment.  a_frag(i, h), b_frag(i, h):
// fragments from LDS; those of the shorter side stay, the others come one ahead, for the tiles' sums leave few registers: a second path
// that adds whole segments in the instruction spills up to 500.  What it costs against adding all rows in the instruction: 4096 x 11008 x 4096,
// 12 segments, rank 16 283 us against 277; 4096^3, 60 segments, rank 64 137 against 132.
template <int KIND, int TM, int TN, class FragA, class FragB>
__device__ __forceinline__ void low_products(const LowBlocks &low, int row, int lane, FragA a_frag, FragB b_frag, f32x4 (&acc)[TN][TM])
{
    constexpr bool BY_ROWS = TM >= TN;
    constexpr int STAY = BY_ROWS ? TN : TM, COME = BY_ROWS ? TM : TN;
    if (row >= low.hi || row + 16 * TM <= low.lo)
        return;                                     // none of this wave's rows
    bf16x8 stay[STAY][2], come[2][2];
#pragma unroll
    for (int i = 0; i < STAY; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            stay[i][h] = BY_ROWS ? b_frag(i, h) : a_frag(i, h);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        come[0][h] = BY_ROWS ? a_frag(0, h) : b_frag(0, h);
#pragma unroll
    for (int j = 0; j < COME; ++j) {
        if (j + 1 < COME) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                come[(j + 1) % 2][h] = BY_ROWS ? a_frag(j + 1, h) : b_frag(j + 1, h);
        }
#pragma unroll
        for (int i = 0; i < STAY; ++i) {
            const int a = BY_ROWS ? i : j, b = BY_ROWS ? j : i;
            const int own = row + 16 * b + (lane & 15);
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h)
                sum = mfma_16x16x32<KIND>(BY_ROWS ? stay[i][h] : come[j % 2][h], BY_ROWS ? come[j % 2][h] : stay[i][h], sum);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[a][b][e] += own >= low.lo && own < low.hi ? sum[e] : 0.0f;
            if (i % 2)
                __builtin_amdgcn_sched_barrier(0);
        }
    }
}

}  // namespace brg
