// Weight gradients whose reductions are short: 128 x 128 x 64 tiles, four waves of 64 x 64, one LDS stage, and three workgroups on
// a CU (144 registers).
//
// What bounds them is not the reduction but the result, G x N x K values for a few hundred rows a group: a workgroup of the 256 x 256
// kernel has its CU to itself, and while it waits for its group's bounds, its first loads and the old values the CU stores nothing (64
// rows a group, 64 groups of 1024 x 2048: 12 us for a tile of 128 KiB).  Here one workgroup's chain of latencies is hidden by two others';
// a block of the reduction is requested, waited for and multiplied with nothing in flight beside it, which the others hide as well.
#include "grouped_tuned.hpp"

namespace brg {

namespace {

constexpr int SW_PITCH = 64 + 4;            // floats of a staged row: 32 rows of a wave's 64 columns
constexpr int SW_STAGE = 32 * SW_PITCH * 4;
constexpr int SW_LDS = 4 * SW_STAGE > 2 * 128 * BK * 2 ? 4 * SW_STAGE : 2 * 128 * BK * 2;

template <int KIND>
__global__ void __launch_bounds__(256, 3)
grouped_short_wgrad_kernel(Bf16Args p, GroupArgs g)
{
    typedef MNMajorTile<128, 4> Tile;
    constexpr uint32_t HALF = 128 * BK * 2;
    __shared__ __attribute__((aligned(1024))) char lds_generic[SW_LDS];
    LDS_AS char *lds = (LDS_AS char *)lds_generic;
    GroupTile t;
    if (!find_reduction(g, p.tiles_m, p.tiles_n, p.walk, t))
        return;
    select_reduction(p, g, t);
    if (p.K == 0) {
        store_empty_tile<128, 128, 256>(p.epi, p.M, p.N, t.tm, t.tn);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = w >> 1, wn = w & 1;
    const int64_t m0 = (int64_t)t.tm * 128, n0 = (int64_t)t.tn * 128;
    uint32_t a_src[4], b_src[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        a_src[j] = Tile::src_rel_bytes(w, j, lane, m0, p.M, p.lda);
        b_src[j] = Tile::src_rel_bytes(w, j, lane, n0, p.N, p.ldb);
    }
    const char *A = (const char *)uniform_ptr(p.A + m0), *B = (const char *)uniform_ptr(p.B + n0);
    f32x4 acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&]() {
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            bf16x8 fa[4], fb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fa[i] = Tile::read_frag16(lds, wm * 64, i, st, lane);
                fb[i] = Tile::read_frag16(lds + HALF, wn * 64, i, st, lane);
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    acc[a][b] = mfma_16x16x32<KIND>(fb[a], fa[b], acc[a][b]);
        }
        wait_lgkmcnt0();
        block_sync();                               // nobody reads this block any more
    };
    const int64_t a_step = Tile::kstep(p.lda) * 2, b_step = Tile::kstep(p.ldb) * 2;
    auto block = [&](auto partial, int rows) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // (of an incomplete block: rows past its end are switched off and zeros in their place; through registers, as in the other
            // kernels, 63 rows took 1.4 times what 64 take)
            if (!decltype(partial)::value || 4 * (4 * w + j) + lane / 16 < rows) {
                load16_to_lds_saddr(A, a_src[j], (uint32_t)(size_t)(lds + Tile::dst_byte(w, j)));
                load16_to_lds_saddr(B, b_src[j], (uint32_t)(size_t)(lds + HALF + Tile::dst_byte(w, j)));
            } else {
                *(LDS_AS s16x8 *)(lds + Tile::dst_byte(w, j) + lane * 16) = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
                *(LDS_AS s16x8 *)(lds + HALF + Tile::dst_byte(w, j) + lane * 16) = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
        }
        A += a_step;
        B += b_step;
        wait_vmcnt0();
        wait_lgkmcnt0();
        block_sync();
        multiply();
    };
    const int whole = (int)(p.K / BK);
    for (int kb = 0; kb < whole; ++kb)
        block(std::false_type{}, BK);
    if (p.K % BK != 0)
        block(std::true_type{}, (int)(p.K % BK));

    // Epilogue: 32 rows x 64 columns of a wave at a time through its part of LDS, stored in whole lines.
    const int64_t row0 = m0 + wm * 64, col0 = n0 + wn * 64;
    if (col0 >= p.N)
        return;
    LDS_AS char *stage = lds + w * SW_STAGE;
    const bool whole_cols = col0 + 64 <= p.N;
    if (!p.epi.c_f32 && p.epi.beta == 0.0f && (p.epi.ldc & 7) == 0 && (((uintptr_t)p.epi.C) & 15) == 0 && whole_cols) {
        uint16_t *C = (uint16_t *)p.epi.C + row0 * p.epi.ldc + col0;
        static_for<0, 2>([&](auto hc) {
            constexpr int h = decltype(hc)::value;
            asm volatile("" ::: "memory");
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const f32x4 v = acc[a][2 * h + b];
                    *(LDS_AS gu32x2 *)(stage + (16 * b + (lane & 15)) * 136 + (16 * a + 4 * (lane >> 4)) * 2) =
                        gu32x2{KIND == KIND_F16 ? pack_f16x2(v[0], v[1]) : pack_bf16x2(v[0], v[1]),
                               KIND == KIND_F16 ? pack_f16x2(v[2], v[3]) : pack_bf16x2(v[2], v[3])};
                }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 8 * i + lane / 8, c = lane % 8;
                const gu32x2 lo = *(LDS_AS gu32x2 *)(stage + row * 136 + c * 16), hi = *(LDS_AS gu32x2 *)(stage + row * 136 + c * 16 + 8);
                if (row0 + 32 * h + row < p.M)
                    __builtin_nontemporal_store(gu32x4{lo[0], lo[1], hi[0], hi[1]}, (gu32x4 *)(C + (32 * h + row) * p.epi.ldc + 8 * c));
            }
            __builtin_amdgcn_wave_barrier();
        });
        return;
    }
    const bool vec = (p.epi.ldc & 3) == 0 && (((uintptr_t)p.epi.C) & 15) == 0;
    const bool fast_f32 = p.epi.c_f32 && vec && whole_cols;
    static_for<0, 2>([&](auto hc) {
        constexpr int h = decltype(hc)::value;
        const int64_t m = row0 + 32 * h + lane / 16, n = col0 + 4 * (lane % 16);
        float *C = (float *)p.epi.C + m * p.epi.ldc + n;
        f32x4 old[8];
        if (fast_f32 && p.epi.beta != 0.0f) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                old[i] = *(const f32x4 *)((const float *)p.epi.C + (m + 4 * i < p.M ? m + 4 * i : p.M - 1) * p.epi.ldc + n);
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(LDS_AS f32x4 *)(stage + ((16 * b + (lane & 15)) * SW_PITCH + 16 * a + 4 * (lane >> 4)) * 4) = acc[a][2 * h + b];
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f32x4 v = *(LDS_AS f32x4 *)(stage + ((4 * i + lane / 16) * SW_PITCH + 4 * (lane % 16)) * 4);
            if (m + 4 * i < p.M) {
                if (fast_f32) {
                    if (p.epi.beta != 0.0f) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = fmaf(p.epi.beta, old[i][e], v[e]);
                    }
                    __builtin_nontemporal_store(v, (f32x4 *)(C + 4 * i * p.epi.ldc));
                } else {
                    store4_epilogue(p.epi, m + 4 * i, n, p.N - n, vec, v[0], v[1], v[2], v[3]);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    });
}

}  // namespace

hipError_t grouped_short_wgrad(const GroupedCall &c)
{
    const Problem &p = c.p;
    Bf16Args a;
    fill_common_args(a, p);
    a.tiles_m = (int)((p.M + 127) / 128);
    a.tiles_n = (int)((p.N + 127) / 128);
    a.walk = reduction_walk(a.tiles_m, a.tiles_n);
    const dim3 grid((unsigned)reduction_grid((int64_t)a.tiles_m * a.tiles_n, c.g.groups));
    if (p.in_f16)
        hipLaunchKernelGGL(grouped_short_wgrad_kernel<KIND_F16>, grid, dim3(256), 0, p.stream, a, c.g);
    else
        hipLaunchKernelGGL(grouped_short_wgrad_kernel<KIND_BF16>, grid, dim3(256), 0, p.stream, a, c.g);
    return hipGetLastError();
}

}  // namespace brg
