// The two products of adapters as kernels of their own, for 16-bit operands of any size and alignment.
//
// H = scale_a * X x down_a (adapters_down_kernel).  R is 8 to 64 where K is thousands: X and the adapters are read once, nothing is
// reused but 16 rows' worth of down, so there is nothing for LDS to do (but turn a down that is stored along the rank).  A workgroup
// owns 16 rows of a segment and 16 * RT of the rank; its eight waves deal the blocks of 64 k among themselves, load fragments
// straight into registers, DEPTH blocks ahead, and add their sums in LDS in wave order.
//
// Y = act(beta * Y + sum of partial sums + H x up_a + bias) (adapters_up_kernel), where the projection has left its fp32 sums, one set for every
// slice of its reduction, in the workspace.  For segments of a few rows, whose blocks would fill a projection's tiles with
// zeros (lowrank.hpp): decode with an adapter for every row costs 16 rows of up a row here, a whole block of a tile there.
#include "general.hpp"
#include "lowrank.hpp"

namespace brg {

namespace {

struct DownArgs {
    const uint16_t *X, *down;
    uint16_t *H;
    const float *factors;
    int64_t ldx, ld_down, ldh;
    int K, R, tiles_n;
    Walk walk;
};

constexpr int DOWN_WAVES = 8;

template <int KIND, bool KMAJ, int RT>
__global__ void __launch_bounds__(DOWN_WAVES * 64)
adapters_down_kernel(DownArgs p, GroupArgs g)
{
    constexpr int COLS = 16 * RT, LD = COLS + 4, DEPTH = RT == 4 ? 2 : 4;
    typedef GenImage<KIND, COLS < 32 ? 32 : COLS, false> Image;          // down stored along the rank: 64 k-rows of COLS
    static_assert(KMAJ || RT > 1, "");
    __shared__ __attribute__((aligned(1024))) char turn_generic[KMAJ ? 16 : DOWN_WAVES * Image::BYTES];
    __shared__ float sums[DOWN_WAVES][16][LD];

    GroupTile t;
    if (!find_tile<16>(g, p.tiles_n, p.walk, t))
        return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col0 = t.tn * COLS, row0 = t.first + 16 * t.tm, rows = t.rows - 16 * t.tm < 16 ? t.rows - 16 * t.tm : 16;
    const bool none = t.weights == kNoWeights;
    f32x4 acc[RT];
#pragma unroll
    for (int a = 0; a < RT; ++a)
        acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (!none) {
        const int r = lane & 15, q = lane >> 4;
        const bool row_is = r < rows;
        const uint16_t *x = p.X + (int64_t)(row0 + (row_is ? r : 0)) * p.ldx;
        const uint16_t *down = p.down + t.weights * g.stride_b;
        LDS_AS char *turn = (LDS_AS char *)turn_generic + (KMAJ ? 0 : w * (int)Image::BYTES);
        struct Set {
            gu32x4 a[2], b[2 * RT];
        };
        // Block kb: 64 k from 64 * kb on.  WHOLE: all of them exist.
        auto load = [&](Set &s, int kb, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            const int k0 = kb * 64;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + 32 * h + 8 * q;
                s.a[h] = low_chunk(x + k, !row_is ? 0 : WHOLE ? 8 : p.K - k);
                if constexpr (KMAJ) {
#pragma unroll
                    for (int a = 0; a < RT; ++a) {
                        const int n = col0 + 16 * a + r;
                        s.b[2 * a + h] = low_chunk(down + (int64_t)n * p.ld_down + k, n >= p.R ? 0 : WHOLE ? 8 : p.K - k);
                    }
                }
            }
            if constexpr (!KMAJ) {
#pragma unroll
                for (int j = 0; j < 2 * RT; ++j) {
                    const int idx = j * 64 + lane, kr = idx / Image::CPR, n = col0 + 8 * (idx % Image::CPR);
                    const int cols = p.R - n < 8 ? p.R - n : 8;
                    s.b[j] = low_chunk(down + (int64_t)(k0 + kr) * p.ld_down + n, WHOLE || k0 + kr < p.K ? cols : 0);
                }
            }
        };
        auto multiply = [&](const Set &s) {
            if constexpr (!KMAJ) {
                asm volatile("" ::: "memory");          // (this wave's own image: its LDS operations keep their order)
#pragma unroll
                for (int j = 0; j < 2 * RT; ++j)
                    *(LDS_AS gu32x4 *)(turn + Image::dst_byte(j * 64 + lane)) = s.b[j];
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int a = 0; a < RT; ++a) {
                    bf16x8 b;
                    if constexpr (KMAJ)
                        b = __builtin_bit_cast(bf16x8, s.b[2 * a + h]);
                    else
                        b = Image::frag16(turn, 0, a, h, lane);
                    acc[a] = mfma_16x16x32<KIND>(b, __builtin_bit_cast(bf16x8, s.a[h]), acc[a]);
                }
        };
        const int whole = p.K / 64;
        Set sets[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (w + DOWN_WAVES * d < whole)
                load(sets[d], w + DOWN_WAVES * d, std::true_type{});
        for (int kb = w; kb < whole; kb += DOWN_WAVES * DEPTH) {
            static_for<0, DEPTH>([&](auto dc) {
                constexpr int d = decltype(dc)::value;
                const int at = kb + DOWN_WAVES * d;
                if (at < whole) {
                    multiply(sets[d]);
                    if (at + DOWN_WAVES * DEPTH < whole)
                        load(sets[d], at + DOWN_WAVES * DEPTH, std::true_type{});
                }
            });
        }
        if (p.K % 64 != 0 && whole % DOWN_WAVES == w) {
            load(sets[0], whole, std::false_type{});
            multiply(sets[0]);
        }
    }
#pragma unroll
    for (int a = 0; a < RT; ++a)
        *(LDS_AS f32x4 *)&((LDS_AS float *)sums)[(w * 16 + (lane & 15)) * LD + 16 * a + 4 * (lane >> 4)] = acc[a];
    __syncthreads();
    const float factor = !none && p.factors ? p.factors[t.weights] : 1.0f;
    for (int i = tid; i < 16 * COLS; i += DOWN_WAVES * 64) {
        const int row = i / COLS, col = i % COLS;
        if (row < rows && col0 + col < p.R) {
            float v = sums[0][row][col];
#pragma unroll
            for (int s = 1; s < DOWN_WAVES; ++s)
                v += sums[s][row][col];
            v = none ? 0.0f : v * factor;
            p.H[(int64_t)(row0 + row) * p.ldh + col0 + col] = KIND == KIND_F16 ? f32_to_f16_rne(v) : f32_to_bf16_rne(v);
        }
    }
}

struct UpArgs {
    const float *partial;           // slices x M x N
    int64_t M, N;
    int slices, tiles_n;
    Epilogue epi;
    Walk walk;
};

constexpr int UP_COLS = 256;        // of a workgroup: 64 a wave

template <int KIND, bool KMAJ>
__global__ void __launch_bounds__(256)
adapters_up_kernel(UpArgs p, GroupArgs g, LowRank low)
{
    constexpr int LD = 64 + 4;
    typedef GenImage<KIND, 64, false> Image;
    __shared__ __attribute__((aligned(1024))) char turn_generic[KMAJ ? 16 : 4 * Image::BYTES];
    __shared__ float sums[4][16][LD];
    GroupTile t;
    if (!find_tile<16>(g, p.tiles_n, p.walk, t))
        return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row0 = t.first + 16 * t.tm, rows = t.rows - 16 * t.tm < 16 ? t.rows - 16 * t.tm : 16;
    const int64_t n0 = (int64_t)t.tn * UP_COLS + 64 * w;
    const int r = lane & 15, q = lane >> 4;
    f32x4 acc[4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
        acc[a] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (t.weights != kNoWeights) {
        const uint16_t *H = (const uint16_t *)low.H + (int64_t)(row0 + r) * low.ldh;
        const uint16_t *up = (const uint16_t *)low.up + t.weights * low.stride_up;
        LDS_AS char *turn = (LDS_AS char *)turn_generic + (KMAJ ? 0 : w * (int)Image::BYTES);
        const int R = (int)low.R;
        for (int r0 = 0; r0 < R; r0 += 64) {
            const int halves = R - r0 > 32 ? 2 : 1;
            if constexpr (!KMAJ) {
                asm volatile("" ::: "memory");
                gu32x4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int kr = j * 8 + lane / 8;
                    const int64_t n = n0 + 8 * (lane % 8), cols = p.N - n < 8 ? p.N - n : 8;
                    v[j] = low_chunk(up + (int64_t)(r0 + kr) * low.ld_up + n, r0 + kr < R ? (int)cols : 0);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *(LDS_AS gu32x4 *)(turn + Image::dst_byte(j * 64 + lane)) = v[j];
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h < halves) {
                    const int k = r0 + 32 * h + 8 * q;
                    const bf16x8 x = __builtin_bit_cast(bf16x8, low_chunk(H + k, r < rows ? R - k : 0));
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        bf16x8 b;
                        if constexpr (KMAJ) {
                            const int64_t n = n0 + 16 * a + r;
                            b = __builtin_bit_cast(bf16x8, low_chunk(up + n * low.ld_up + k, n < p.N ? R - k : 0));
                        } else {
                            b = Image::frag16(turn, 0, a, h, lane);
                        }
                        acc[a] = mfma_16x16x32<KIND>(b, x, acc[a]);
                    }
                }
            }
        }
    }
    // Row by row through this wave's LDS: whole lines of the partial sums and of Y.
#pragma unroll
    for (int a = 0; a < 4; ++a)
        *(LDS_AS f32x4 *)&((LDS_AS float *)sums)[(w * 16 + r) * LD + 16 * a + 4 * q] = acc[a];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    const bool vec = (p.epi.ldc & 3) == 0 && (((uintptr_t)p.epi.C) & 15) == 0;
    const int64_t slice = p.M * p.N;
    for (int i = lane; i < rows * 16; i += 64) {
        const int64_t m = row0 + i / 16, n = n0 + 4 * (i % 16), left = p.N - n;
        if (left <= 0)
            continue;
        f32x4 v = *(LDS_AS f32x4 *)&((LDS_AS float *)sums)[(w * 16 + i / 16) * LD + 4 * (i % 16)];
        const float *part = p.partial + m * p.N + n;
        if (left >= 4) {
            // (four slices' loads at a time are under way)
            for (int z = 0; z < p.slices; z += 4) {
                f32x4 o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[e] = *(const f32x4_any4 *)(part + (z + e < p.slices ? z + e : z) * slice);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (z + e < p.slices)
                        v += o[e];
            }
        } else {
            for (int z = 0; z < p.slices; ++z)
                for (int e = 0; e < left; ++e)
                    v[e] += part[z * slice + e];
        }
        store4_epilogue(p.epi, m, n, left, vec, v[0], v[1], v[2], v[3]);
    }
}

template <int KIND, bool KMAJ, int RT>
hipError_t launch_down(const GroupedCall &c)
{
    const Problem &p = c.p;
    const int tiles_n = (int)((p.N + 16 * RT - 1) / (16 * RT));
    DownArgs a{(const uint16_t *)p.A, (const uint16_t *)p.B, (uint16_t *)p.C, c.factors, p.lda, p.ldb, p.ldc, (int)p.K, (int)p.N, tiles_n,
               make_walk(1, tiles_n, 1, 1, 1, (int64_t)kWalkRows * tiles_n)};
    GroupArgs g = c.g;
    g.max_tiles = (int)most_row_tiles(p.M, g.groups + 2 * g.cover, 16);
    hipLaunchKernelGGL((adapters_down_kernel<KIND, KMAJ, RT>), dim3((unsigned)(g.max_tiles * tiles_n)), dim3(DOWN_WAVES * 64), 0, p.stream, a, g);
    return hipGetLastError();
}

// The widest tile that R fills, halved while that leaves CUs without work.
template <int KIND>
hipError_t launch_down_of(const GroupedCall &c)
{
    const int64_t rows = most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16);
    int rt = c.p.N > 32 ? 4 : c.p.N > 16 ? 2 : 1;
    while (rt > 1 && rows * ((c.p.N + 16 * rt - 1) / (16 * rt)) < 128)
        rt /= 2;
    if (c.p.transB)
        return rt == 4 ? launch_down<KIND, true, 4>(c) : rt == 2 ? launch_down<KIND, true, 2>(c) : launch_down<KIND, true, 1>(c);
    return rt == 4 ? launch_down<KIND, false, 4>(c) : launch_down<KIND, false, 2>(c);
}

template <int KIND>
hipError_t launch_up(const GroupedCall &c, const UpArgs &a, unsigned grid)
{
    if (c.p.transB)
        hipLaunchKernelGGL((adapters_up_kernel<KIND, true>), dim3(grid), dim3(256), 0, c.p.stream, a, c.g, c.low);
    else
        hipLaunchKernelGGL((adapters_up_kernel<KIND, false>), dim3(grid), dim3(256), 0, c.p.stream, a, c.g, c.low);
    return hipGetLastError();
}

}  // namespace

// Grids are 32-bit counts of threads.
bool adapters_down_fits(const GroupedCall &c)
{
    return in_16bit(c.p) && most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16) * ((c.p.N + 15) / 16) <= 0xffffffffLL / 512;
}
bool adapters_up_fits(const GroupedCall &c)
{
    return in_16bit(c.p) && c.low.R <= (1 << 20) && most_row_tiles(c.p.M, c.g.groups + 2 * c.g.cover, 16) * ((c.p.N + UP_COLS - 1) / UP_COLS) <= 0xffffffffLL / 256;
}

hipError_t adapters_down(const GroupedCall &c) { return c.p.in_f16 ? launch_down_of<KIND_F16>(c) : launch_down_of<KIND_BF16>(c); }

hipError_t adapters_up(const GroupedCall &call, const float *partial, int slices)
{
    GroupedCall c = call;
    const Problem &p = c.p;
    UpArgs a;
    a.partial = partial; a.M = p.M; a.N = p.N; a.slices = slices;
    a.tiles_n = (int)((p.N + UP_COLS - 1) / UP_COLS);
    a.epi.beta = p.beta; a.epi.C = p.C; a.epi.ldc = p.ldc; a.epi.c_f32 = p.c_f32; a.epi.c_f16 = p.in_f16; a.epi.c_i32 = 0;
    a.epi.bias = p.bias; a.epi.relu = p.relu;
    a.walk = make_walk(1, a.tiles_n, 1, 1, 1, (int64_t)kWalkRows * a.tiles_n);
    c.g.max_tiles = (int)most_row_tiles(p.M, c.g.groups + 2 * c.g.cover, 16);
    const unsigned grid = (unsigned)(c.g.max_tiles * a.tiles_n);
    return p.in_f16 ? launch_up<KIND_F16>(c, a, grid) : launch_up<KIND_BF16>(c, a, grid);
}

}  // namespace brg
