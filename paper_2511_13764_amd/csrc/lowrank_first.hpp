// The first product of adapters, H = scale_a * X x down_a, as the work of one workgroup (lowrank.hip says why it is divided so): in a
// launch of its own, or beside the projection's tiles.
#pragma once
#include "general.hpp"
#include "lowrank.hpp"

namespace brg {

namespace {

struct FirstArgs {
    const uint16_t *X, *down, *W;
    uint16_t *H;
    float *sums;                    // the projection's, M x N
    const float *factors;
    int64_t ldx, ld_down, ldh, ldw, N;
    int M, K, R, tiles_n;
    int first;                      // workgroups of H, in front of the projection's (they take longer to find their work)
    Walk walk;
};

constexpr int FIRST_WAVES = 8;

// Up to 16 rows with one adapter, and a tile of columns.  Lane l holds the number of the row l % 16 of them (the last one's where there are fewer).
struct RowTile {
    int weights, rows, tn, row_l;
    __device__ __forceinline__ int row(int r) const { return __builtin_amdgcn_ds_bpermute(4 * (r < rows ? r : rows - 1), row_l); }     // (all lanes)
};

// Rows with an adapter each, of which many have the same one (GroupArgs::by_weights): the rows of an adapter go together, 16 at a time, so
// that its weights are read once for them.  Adapters are taken in the order of their first rows, those without one together; every wave
// looks for itself.  Every turn is a comparison of 64 rows a register: at most 64 adapters, 256 rows.  list: 16 numbers of the wave's own.
__device__ __forceinline__ bool rows_of_adapter(const GroupArgs &g, int tile, RowTile &t, LDS_AS int *list)
{
    const int lane = threadIdx.x & 63;
    int id[4];
    uint64_t left[4], own[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = 64 * j + lane;
        const int64_t v = g.ids[i < g.rows ? i : 0];
        id[j] = v >= 0 && v < g.weights ? (int)v : kNoWeights;
        left[j] = __builtin_amdgcn_ballot_w64(i < g.rows);
    }
    while (left[0] | left[1] | left[2] | left[3]) {
        const int who = left[0]   ? __builtin_amdgcn_readlane(id[0], __builtin_ctzll(left[0]))
                        : left[1] ? __builtin_amdgcn_readlane(id[1], __builtin_ctzll(left[1]))
                        : left[2] ? __builtin_amdgcn_readlane(id[2], __builtin_ctzll(left[2]))
                                  : __builtin_amdgcn_readlane(id[3], __builtin_ctzll(left[3]));
        int count = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            own[j] = __builtin_amdgcn_ballot_w64(id[j] == who) & left[j];
            left[j] &= ~own[j];
            count += __builtin_popcountll(own[j]);
        }
        const int tiles = (count + 15) >> 4;
        if (tile >= tiles) {
            tile -= tiles;
            continue;
        }
        int before = -16 * tile;
        asm volatile("" ::: "memory");              // (a wave's LDS operations keep their order)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int rank = before + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(own[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)own[j], 0));
            if ((own[j] >> lane & 1) && rank >= 0 && rank < 16)
                list[rank] = 64 * j + lane;
            before += __builtin_popcountll(own[j]);
        }
        asm volatile("" ::: "memory");
        t.weights = who;
        t.rows = count - 16 * tile < 16 ? count - 16 * tile : 16;
        t.row_l = list[(lane & 15) < t.rows ? lane & 15 : t.rows - 1];
        return true;
    }
    return false;
}

// The rows and columns of workgroup `block`.
__device__ __forceinline__ bool find_rows(const GroupArgs &g, int tiles_n, const Walk &walk, RowTile &t, int block, LDS_AS int *list)
{
    if (g.by_weights) {
        const int tile = div_by(block, walk.by_tiles);
        t.tn = block - tile * tiles_n;
        return rows_of_adapter(g, tile, t, list);
    }
    GroupTile at;
    if (!find_tile<16, false>(g, tiles_n, walk, at, block))
        return false;
    t.weights = at.weights;
    t.tn = at.tn;
    t.rows = at.rows - 16 * at.tm < 16 ? at.rows - 16 * at.tm : 16;
    const int l = (int)(threadIdx.x & 15);
    t.row_l = at.first + 16 * at.tm + (l < t.rows ? l : t.rows - 1);
    return true;
}

// Most of these tiles that a call can have.
inline int64_t most_rows_tiles(const GroupedCall &c)
{
    const int64_t by_adapter = (c.p.M + 15 * (c.g.weights + 1)) / 16;
    return c.g.by_weights ? (by_adapter < c.p.M ? by_adapter : c.p.M) : most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16);
}


// LDS of one wave: a block of X and one of B.
template <int KIND, bool KMAJ, int MT, int RT>
struct FirstLds {
    static constexpr int COLS = 16 * RT, LD = COLS + 4;
    typedef GenImage<KIND, 16 * MT, true> ImageX;
    typedef GenImage<KIND, KMAJ ? COLS : COLS < 32 ? 32 : COLS, KMAJ> ImageB;
    static constexpr int kBlock = ImageX::BYTES + ImageB::BYTES, kSums = MT * 16 * LD * 4;
    static constexpr int kWave = kBlock > kSums ? kBlock : kSums;          // (the sums replace the blocks)
};

// 16 * MT rows of X, row_of(0) .. (those there are not repeat one) times 16 * RT columns of B (`limit` of them in all), over K: the waves' sums in LDS as
// sums[row][column] of every wave's part.  Rows and columns that are not there repeat one that is: their sums are nobody's.
// EXACT: chunks along a B stored along its columns are whole.
// Every wave's loads take whole lines of 128 bytes, eight rows of them, and go to the matrix instruction through images of its own in
// LDS.  (A lane's fragment straight from memory is 16 bytes of 16 rows next to each other in the wave, which the address unit takes line
// by line: 16 x 4096 x 4096 17.8 us.)
template <int KIND, bool KMAJ, int MT, int RT, bool EXACT, class RowOf>
__device__ __forceinline__ void first_sums(const uint16_t *X, int64_t ldx, RowOf row_of, const uint16_t *B, int64_t ldb, int64_t col0, int64_t limit, int K,
                                           LDS_AS char *lds, int lane, int w)
{
    typedef FirstLds<KIND, KMAJ, MT, RT> Lds;
    typedef typename Lds::ImageX ImageX;
    typedef typename Lds::ImageB ImageB;
    constexpr int LA = 2 * MT, LB = 2 * RT, DEPTH = LA + LB <= 4 ? 4 : 3;
    LDS_AS char *ximg = lds + w * Lds::kWave, *bimg = ximg + ImageX::BYTES;
    const uint16_t *x[LA], *b[KMAJ ? LB : 1];
#pragma unroll
    for (int j = 0; j < LA; ++j) {
        x[j] = X + (int64_t)row_of(8 * j + lane / 8) * ldx + 8 * (lane % 8);
    }
    int cols = 8;
    if constexpr (KMAJ) {
#pragma unroll
        for (int j = 0; j < LB; ++j) {
            const int64_t n = col0 + 8 * j + lane / 8;
            b[j] = B + (n < limit ? n : limit - 1) * ldb + 8 * (lane % 8);
        }
    } else {
        const int64_t n = col0 + 8 * (lane % ImageB::CPR), last = limit - 8;
        b[0] = B + (int64_t)(lane / ImageB::CPR) * ldb + (EXACT && n > last ? last : n);
        if constexpr (!EXACT)
            cols = limit - n < 8 ? (int)(limit - n) : 8;
    }
    constexpr int KR = 64 / ImageB::CPR;                // k-rows of one load of a B stored along its columns
    struct Set {
        gu32x4 a[LA], b[LB];
    };
    auto load = [&](Set &s, int kb) {
        const int64_t k0 = (int64_t)kb * 64;
#pragma unroll
        for (int j = 0; j < LA; ++j)
            s.a[j] = *(const low_u32x4_any2 *)(x[j] + k0);
#pragma unroll
        for (int j = 0; j < LB; ++j) {
            if constexpr (KMAJ) {
                s.b[j] = *(const low_u32x4_any2 *)(b[j] + k0);
            } else {
                const uint16_t *at = b[0] + (k0 + j * KR) * ldb;
                s.b[j] = EXACT ? (gu32x4)*(const low_u32x4_any2 *)at : low_chunk(at, cols);
            }
        }
    };
    auto load_tail = [&](Set &s, int kb) {
        const int k0 = kb * 64, there = K - k0 - 8 * (lane % 8);
#pragma unroll
        for (int j = 0; j < LA; ++j)
            s.a[j] = low_chunk(x[j] + k0, there);
#pragma unroll
        for (int j = 0; j < LB; ++j) {
            if constexpr (KMAJ)
                s.b[j] = low_chunk(b[j] + k0, there);
            else
                s.b[j] = low_chunk(b[0] + (int64_t)(k0 + j * KR) * ldb, k0 + j * KR + lane / ImageB::CPR < K ? cols : 0);
        }
    };
    f32x4 acc[RT][MT];
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            acc[a][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // (A wave's LDS operations keep their order: no wait between the images' writes, their reads and the next writes.)
    auto multiply = [&](const Set &s) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < LA; ++j)
            *(LDS_AS gu32x4 *)(ximg + ImageX::dst_byte(j * 64 + lane)) = s.a[j];
#pragma unroll
        for (int j = 0; j < LB; ++j)
            *(LDS_AS gu32x4 *)(bimg + ImageB::dst_byte(j * 64 + lane)) = s.b[j];
        asm volatile("" ::: "memory");
        bf16x8 fx[2][MT], fb[2][RT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                fx[h][m] = ImageX::frag16(ximg, 0, m, h, lane);
#pragma unroll
            for (int a = 0; a < RT; ++a)
                fb[h][a] = ImageB::frag16(bimg, 0, a, h, lane);
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int a = 0; a < RT; ++a)
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    acc[a][m] = mfma_16x16x32<KIND>(fb[h][a], fx[h][m], acc[a][m]);
    };
    // Whole turns of the sets request under no condition, so that the compiler knows how many loads are in flight; the rest of a
    // turn and its sums follow.
    const int whole = K / 64;
    const int n = whole > w ? (whole - w + FIRST_WAVES - 1) / FIRST_WAVES : 0;
    if (n > 0) {
        Set sets[DEPTH];
        auto step = [&](int i) { return w + FIRST_WAVES * (i < n ? i : n - 1); };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            load(sets[d], step(d));
        int i = 0;
        for (; i + 2 * DEPTH <= n; i += DEPTH) {
            static_for<0, DEPTH>([&](auto dc) {
                constexpr int d = decltype(dc)::value;
                __builtin_amdgcn_sched_barrier(0);
                multiply(sets[d]);
                __builtin_amdgcn_sched_barrier(0);
                load(sets[d], step(i + d + DEPTH));
            });
        }
        for (; i < n; i += DEPTH) {
            static_for<0, DEPTH>([&](auto dc) {
                constexpr int d = decltype(dc)::value;
                __builtin_amdgcn_sched_barrier(0);
                if (i + d < n)
                    multiply(sets[d]);
                if (i + d + DEPTH < n)
                    load(sets[d], step(i + d + DEPTH));
            });
        }
    }
    if (K % 64 != 0 && whole % FIRST_WAVES == w) {
        Set s;
        load_tail(s, whole);
        multiply(s);
    }
    asm volatile("" ::: "memory");
    LDS_AS float *sums = (LDS_AS float *)ximg;
#pragma unroll
    for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int m = 0; m < MT; ++m)
            *(LDS_AS f32x4 *)(sums + (16 * m + (lane & 15)) * Lds::LD + 16 * a + 4 * (lane >> 4)) = acc[a][m];
}

// Element (row, col) of all waves' sums, in wave order.
template <class Lds>
__device__ __forceinline__ float first_total(const LDS_AS char *lds, int row, int col)
{
    const LDS_AS float *at = (const LDS_AS float *)lds + row * Lds::LD + col;
    float v = at[0];
#pragma unroll
    for (int s = 1; s < FIRST_WAVES; ++s)
        v += at[s * (Lds::kWave / 4)];
    return v;
}
// One workgroup's part of H: 16 rows of a piece, 16 * RT of the rank.  lds: FIRST_WAVES * FirstLds::kWave bytes.
template <int KIND, bool KMAJ, int RT, bool EXACT>
__device__ __forceinline__ void first_tile(const FirstArgs &p, const GroupArgs &g, LDS_AS char *lds, int block)
{
    constexpr int COLS = 16 * RT;
    typedef FirstLds<KIND, KMAJ, 1, RT> Lds;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    RowTile t;
    if (!find_rows(g, p.tiles_n, p.walk, t, block, (LDS_AS int *)(lds + w * Lds::kWave)))
        return;
    const int col0 = t.tn * COLS;
    const bool none = t.weights == kNoWeights;
    if (!none)
        first_sums<KIND, KMAJ, 1, RT, EXACT>(p.X, p.ldx, [&](int r) { return t.row(r); }, p.down + t.weights * g.stride_b, p.ld_down, col0, p.R, p.K,
                                             lds, lane, w);
    __syncthreads();
    const float factor = !none && p.factors ? p.factors[t.weights] : 1.0f;
    for (int i = tid; i < 16 * COLS; i += FIRST_WAVES * 64) {
        const int row = i / COLS, col = i % COLS, at = t.row(row);
        if (row < t.rows && col0 + col < p.R) {
            const float v = none ? 0.0f : first_total<Lds>(lds, row, col) * factor;
            p.H[(int64_t)at * p.ldh + col0 + col] = KIND == KIND_F16 ? f32_to_f16_rne(v) : f32_to_bf16_rne(v);
        }
    }
}

// c: the first product's call (its B, N and C are down, R and H).
inline FirstArgs first_args(const GroupedCall &c)
{
    const Problem &p = c.p;
    FirstArgs a{};
    a.X = (const uint16_t *)p.A; a.down = (const uint16_t *)p.B; a.H = (uint16_t *)p.C; a.factors = c.factors;
    a.ldx = p.lda; a.ld_down = p.ldb; a.ldh = p.ldc;
    a.M = (int)p.M; a.K = (int)p.K; a.R = (int)p.N;
    return a;
}
// Workgroups of H, and what they need of the launch.
inline int first_grid(const GroupedCall &c, int rt, FirstArgs &a, GroupArgs &g)
{
    a.tiles_n = (a.R + 16 * rt - 1) / (16 * rt);
    a.walk = make_walk(1, a.tiles_n, 1, 1, 1, 1);
    g = c.g;
    g.max_tiles = (int)most_rows_tiles(c);
    return g.max_tiles * a.tiles_n;
}

}  // namespace

}  // namespace brg
