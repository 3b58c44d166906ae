// The two products of adapters as kernels of their own, for 16-bit operands of any size and alignment.
//
// H = scale_a * X x down_a (adapters_first_kernel).  R is 8 to 64 where K is thousands: X and the adapters are read once, nothing
// is reused but 16 rows' worth of down.  A workgroup owns 16 rows of a segment (or, of decode's rows with an adapter each, 16 with
// the same one: rows_of_adapter) and 16 * RT of the rank; its eight waves deal the blocks of 64 k among themselves, each with LDS
// of its own and DEPTH blocks ahead in registers, and add their sums in wave order.  Decode's projection is the same thing with
// more columns: for up to 32 rows and weights stored along k, workgroups of the same launch give X x W, 16 columns each, as fp32
// sums in the workspace.
//
// H's fp32 sums are rounded once, to the operands' type: that is what the call returns for the adapters' gradients, and the second
// product takes the same values, so that Y is what the returned H gives and the 16-bit matrix instruction can multiply it.  Against
// H kept in 32 bits Y differs by 5e-4 to 9e-4 of its size, where rounding Y to bf16 is 1.7e-3; a gradient made of a rounded G is
// 2.3e-3 off.
//
// Y = act(beta * Y + sum of partial sums + H x up_a + bias) (adapters_up_kernel), where the projection has left its fp32 sums, one set for every
// slice of its reduction, in the workspace.  For segments of a few rows, whose blocks would fill a projection's tiles with
// zeros (lowrank.hpp): decode with an adapter for every row costs 16 rows of up a row here, a whole block of a tile there.
#include "lowrank_first.hpp"

namespace brg {

namespace {
template <int KIND, bool KMAJ, int RT, bool EXACT, int OWN_MT>
__global__ void __launch_bounds__(FIRST_WAVES * 64, 2)
adapters_first_kernel(FirstArgs p, GroupArgs g)
{
    typedef FirstLds<KIND, KMAJ, 1, RT> Lds;
    typedef FirstLds<KIND, true, (OWN_MT > 0 ? OWN_MT : 1), 1> OwnLds;
    constexpr int BYTES = FIRST_WAVES * (OWN_MT > 0 && OwnLds::kWave > Lds::kWave ? OwnLds::kWave : Lds::kWave);
    __shared__ __attribute__((aligned(1024))) char lds_generic[BYTES];
    LDS_AS char *lds = (LDS_AS char *)lds_generic;
    if constexpr (OWN_MT > 0) {
        const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
        if ((int)blockIdx.x >= p.first) {
            const int64_t col0 = (int64_t)((int)blockIdx.x - p.first) * 16;
            first_sums<KIND, true, OWN_MT, 1, true>(p.X, p.ldx, [&](int r) { return r < p.M ? r : p.M - 1; }, p.W, p.ldw, col0, p.N, p.K, lds, lane, w);
            __syncthreads();
            for (int i = tid; i < 16 * 16 * OWN_MT; i += FIRST_WAVES * 64) {
                const int row = i / 16, col = i % 16;
                if (row < p.M && col0 + col < p.N)
                    p.sums[row * p.N + col0 + col] = first_total<OwnLds>(lds, row, col);
            }
            return;
        }
    }
    first_tile<KIND, KMAJ, RT, EXACT>(p, g, lds, (int)blockIdx.x);
}

struct UpArgs {
    const float *partial;           // slices x M x N
    int64_t M, N;
    int slices, tiles_n;
    Epilogue epi;
    Walk walk;
};

constexpr int UP_COLS = 256;        // of a workgroup: 64 a wave

// RC: ranks that a step takes (16, 32 or 64).  A wave's part of up, 64 columns by RC ranks, is read in whole lines and goes through an
// image of its own in LDS (first_sums says why); what the partial sums hold is requested with it.
template <int KIND, bool KMAJ, int RC>
__global__ void __launch_bounds__(256)
adapters_up_kernel(UpArgs p, GroupArgs g, LowRank low)
{
    constexpr int LD = 64 + 4, HALVES = RC == 64 ? 2 : 1, LOADS = RC / 8;
    typedef GenImage<KIND, 64, KMAJ> Image;
    __shared__ __attribute__((aligned(1024))) char lds_generic[4 * Image::BYTES];
    static_assert(Image::BYTES >= 16 * LD * 4, "the sums replace the image");
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    RowTile t;
    if (!find_rows(g, p.tiles_n, p.walk, t, (int)blockIdx.x, (LDS_AS int *)((LDS_AS char *)lds_generic + w * (int)Image::BYTES)))
        return;
    const int rows = t.rows;
    const int64_t n0 = (int64_t)t.tn * UP_COLS + 64 * w;
    if (n0 >= p.N)
        return;
    LDS_AS char *image = (LDS_AS char *)lds_generic + w * (int)Image::BYTES;
    const int64_t slice = p.M * p.N;
    // Four columns of four rows a lane: row 4 * i + lane / 16, columns 4 * (lane % 16) .. + 3.
    const int64_t n = n0 + 4 * (lane % 16), left = p.N - n;
    int at_row[4];
    f32x4 first[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        at_row[i] = t.row(4 * i + lane / 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * i + lane / 16 < rows && left >= 4)
            first[i] = *(const f32x4_any4 *)(p.partial + at_row[i] * p.N + n);
    f32x4 acc[4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
        acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int r = lane & 15, q = lane >> 4;
    if (t.weights != kNoWeights) {
        // (a row that is not there repeats one that is; ranks that are not there are zeros of both operands)
        const uint16_t *H = (const uint16_t *)low.H + (int64_t)t.row_l * low.ldh;
        const uint16_t *up = (const uint16_t *)low.up + t.weights * low.stride_up;
        const int R = (int)low.R;
        if constexpr (RC == 16) {                   // the other half of an instruction's 32 ranks
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int idx = j * 64 + lane;
                *(LDS_AS gu32x4 *)(image + Image::dst_byte(KMAJ ? idx / 2 * 8 + 2 + idx % 2 : 128 + idx)) = gu32x4{0, 0, 0, 0};
            }
        }
        for (int r0 = 0; r0 < R; r0 += RC) {
            gu32x4 v[LOADS], x[HALVES];
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int idx = j * 64 + lane;
                if constexpr (KMAJ) {
                    const int64_t col = n0 + idx / LOADS;
                    const int k = r0 + 8 * (idx % LOADS);
                    v[j] = low_chunk(up + col * low.ld_up + k, col < p.N ? R - k : 0);
                } else {
                    const int k = r0 + idx / 8;
                    const int64_t col = n0 + 8 * (idx % 8), cols = p.N - col < 8 ? p.N - col : 8;
                    v[j] = low_chunk(up + (int64_t)k * low.ld_up + col, k < R ? (int)cols : 0);
                }
            }
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int k = r0 + 32 * h + 8 * q;
                x[h] = low_chunk(H + k, RC == 16 && q > 1 ? 0 : R - k);
            }
            asm volatile("" ::: "memory");          // (a wave's LDS operations keep their order)
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int idx = j * 64 + lane;
                *(LDS_AS gu32x4 *)(image + Image::dst_byte(KMAJ ? idx / LOADS * 8 + idx % LOADS : idx)) = v[j];
            }
            asm volatile("" ::: "memory");
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    acc[a] = mfma_16x16x32<KIND>(Image::frag16(image, 0, a, h, lane), __builtin_bit_cast(bf16x8, x[h]), acc[a]);
        }
    }
    // Row by row through this wave's LDS: whole lines of the partial sums and of Y.
    asm volatile("" ::: "memory");
    LDS_AS float *sums = (LDS_AS float *)image;
#pragma unroll
    for (int a = 0; a < 4; ++a)
        *(LDS_AS f32x4 *)(sums + r * LD + 16 * a + 4 * q) = acc[a];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    const bool vec = (p.epi.ldc & 3) == 0 && (((uintptr_t)p.epi.C) & 15) == 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 4 * i + lane / 16;
        if (row >= rows || left <= 0)
            continue;
        f32x4 v = *(LDS_AS f32x4 *)(sums + row * LD + 4 * (lane % 16));
        const float *at = p.partial + at_row[i] * p.N + n;
        if (left >= 4) {
            v += first[i];
            // (four slices' loads at a time are under way)
            for (int z = 1; z < p.slices; z += 4) {
                f32x4 o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[e] = *(const f32x4_any4 *)(at + (z + e < p.slices ? z + e : z) * slice);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (z + e < p.slices)
                        v += o[e];
            }
        } else {
            for (int z = 0; z < p.slices; ++z)
                for (int e = 0; e < left; ++e)
                    v[e] += at[z * slice + e];
        }
        store4_epilogue(p.epi, at_row[i], n, left, vec, v[0], v[1], v[2], v[3]);
    }
}

template <int KIND, bool KMAJ, int RT, bool EXACT, int OWN_MT>
hipError_t launch_first(const GroupedCall &c, FirstArgs &a)
{
    GroupArgs g;
    a.first = first_grid(c, RT, a, g);
    const unsigned grid = (unsigned)(a.first + (OWN_MT > 0 ? (a.N + 15) / 16 : 0));
    hipLaunchKernelGGL((adapters_first_kernel<KIND, KMAJ, RT, EXACT, OWN_MT>), dim3(grid), dim3(FIRST_WAVES * 64), 0, c.p.stream, a, g);
    return hipGetLastError();
}

// The widest tile that R fills, halved while that leaves CUs without work.
template <int KIND>
hipError_t launch_first_of(const GroupedCall &c, FirstArgs &a)
{
    const int64_t rows = most_rows_tiles(c);
    int rt = a.R > 32 ? 4 : a.R > 16 ? 2 : 1;
    while (rt > 1 && rows * ((a.R + 16 * rt - 1) / (16 * rt)) < 256)
        rt /= 2;
    if (c.p.transB) {
        if (a.sums == nullptr)
            return rt == 4 ? launch_first<KIND, true, 4, true, 0>(c, a) : rt == 2 ? launch_first<KIND, true, 2, true, 0>(c, a)
                           : launch_first<KIND, true, 1, true, 0>(c, a);
        if (a.M <= 16)
            return rt > 1 ? launch_first<KIND, true, 2, true, 1>(c, a) : launch_first<KIND, true, 1, true, 1>(c, a);
        return rt > 1 ? launch_first<KIND, true, 2, true, 2>(c, a) : launch_first<KIND, true, 1, true, 2>(c, a);
    }
    if (a.R % 8 != 0)
        return launch_first<KIND, false, 2, false, 0>(c, a);
    return rt == 4 ? launch_first<KIND, false, 4, true, 0>(c, a) : launch_first<KIND, false, 2, true, 0>(c, a);
}

template <int KIND, bool KMAJ, int RC>
hipError_t launch_up(const GroupedCall &c, const UpArgs &a, unsigned grid)
{
    hipLaunchKernelGGL((adapters_up_kernel<KIND, KMAJ, RC>), dim3(grid), dim3(256), 0, c.p.stream, a, c.g, c.low);
    return hipGetLastError();
}
template <int KIND, bool KMAJ>
hipError_t launch_up_of(const GroupedCall &c, const UpArgs &a, unsigned grid)
{
    return c.low.R > 32 ? launch_up<KIND, KMAJ, 64>(c, a, grid) : c.low.R > 16 ? launch_up<KIND, KMAJ, 32>(c, a, grid) : launch_up<KIND, KMAJ, 16>(c, a, grid);
}

}  // namespace

// Grids are 32-bit counts of threads.
bool adapters_down_fits(const GroupedCall &c)
{
    return in_16bit(c.p) && first_product_fits(most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16), c.p.N, 0);
}
bool adapters_up_fits(const GroupedCall &c)
{
    return in_16bit(c.p) && c.low.R <= (1 << 20) && most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16) * ((c.p.N + UP_COLS - 1) / UP_COLS) <= 0xffffffffLL / 256;
}

hipError_t adapters_down(const GroupedCall &c)
{
    FirstArgs a = first_args(c);
    return c.p.in_f16 ? launch_first_of<KIND_F16>(c, a) : launch_first_of<KIND_BF16>(c, a);
}

// Few rows and weights stored along k: the projection's sums come with H from one launch.
bool adapters_few_rows(const GroupedCall &c)
{
    return in_16bit(c.p) && c.p.transB == 1 && c.p.M <= 32 && c.p.K >= 64 &&
           first_product_fits(most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16), c.low.R, (c.p.N + 15) / 16);
}
hipError_t adapters_down_and_sums(const GroupedCall &first, const GroupedCall &c, float *sums)
{
    FirstArgs a = first_args(first);
    a.W = (const uint16_t *)c.p.B; a.ldw = c.p.ldb; a.N = c.p.N;
    a.sums = sums;
    return c.p.in_f16 ? launch_first_of<KIND_F16>(first, a) : launch_first_of<KIND_BF16>(first, a);
}

hipError_t adapters_up(const GroupedCall &call, const float *partial, int slices)
{
    GroupedCall c = call;
    const Problem &p = c.p;
    UpArgs a;
    a.partial = partial; a.M = p.M; a.N = p.N; a.slices = slices;
    a.tiles_n = (int)((p.N + UP_COLS - 1) / UP_COLS);
    a.epi.beta = p.beta; a.epi.C = p.C; a.epi.ldc = p.ldc; a.epi.c_f32 = p.c_f32; a.epi.c_f16 = p.in_f16; a.epi.c_i32 = 0;
    a.epi.bias = p.bias; a.epi.relu = p.relu;
    a.walk = make_walk(1, a.tiles_n, 1, 1, 1, 1);
    c.g.max_tiles = (int)most_rows_tiles(c);
    const unsigned grid = (unsigned)(c.g.max_tiles * a.tiles_n);
    if (p.in_f16)
        return p.transB ? launch_up_of<KIND_F16, true>(c, a, grid) : launch_up_of<KIND_F16, false>(c, a, grid);
    return p.transB ? launch_up_of<KIND_BF16, true>(c, a, grid) : launch_up_of<KIND_BF16, false>(c, a, grid);
}

}  // namespace brg
