// What the 256 x 256 kernels of 4-bit images share: tile, phases, loads and the epilogue.
#pragma once
#include "mx4_stream.hpp"

namespace brg {

namespace {

constexpr int PP_BM = 256, PP_BN = 256;
constexpr int PP_TM = 8, PP_TN = 4;             // 16 x 16 tiles of a wave: 128 x 64; waves 0-3 above 4-7

__device__ __forceinline__ void phase_sync() { block_sync(); }

// Tile of a workgroup: 256 x 256, or `small`, of at most 128 rows, for which 128 x 128 tiles are faster than half of a large one: with groups one of those
// (tm, tn: in tiles of that), behind all others, which take longer; without them two.  (4096 rows in 8 groups, 4096 x 11008, images: 128 us with
// small tiles of 128 x 256, so 107; 11008 x 4096, bf16 rows: 342 and 324, 2048 rows 241 and 196.)
template <bool GROUPED>
__device__ __forceinline__ bool mx4_large_tile(Mx4Args &p, const GroupArgs &g, int &tm, int &tn, bool &small)
{
    if constexpr (GROUPED) {
        MixedTile m;
        if (!find_mixed_tile<true>(g, p.tiles_n, p.walk, m))
            return false;
        select_piece(p, g, m.t);
        tm = m.t.tm;
        tn = m.t.tn;
        small = m.small;
    } else {
        tile_coords(blockIdx.x, p.tiles_m, p.tiles_n, p.walk, tm, tn);
        small = p.M - (int64_t)tm * PP_BM <= PP_BM / 2;
    }
    return true;
}

// A small one.
template <int LEFT, bool GROUPED>
__device__ __forceinline__ void mx4_small_tile(const Mx4Args &p, int tm, int tn)
{
    if constexpr (GROUPED) {
        if ((int64_t)tn * 128 < p.N)
            mx4_stream_tile<LEFT, 128, 128>(p, tm, tn, 0);
    } else {
#pragma unroll 1
        for (int i = 2 * tn; i < 2 * tn + 2 && (int64_t)i * 128 < p.N; ++i) {
            block_sync();                       // (the last one's sums have been read)
            mx4_stream_tile<LEFT, 128, 128>(p, 2 * tm, i, 0);
        }
    }
}

// Sums of a wave, 128 x 64 from (m0, n0) on, in `acc` (lane l: row l % 16, columns 4 (l / 16) .. + 3 of every 16 x 16), to C: 32 rows at
// a time, staged in its own MX4_STAGED bytes of LDS at `staged`, stored in whole lines.
constexpr uint32_t MX4_STAGED = 32 * (64 + 4) * 4;
__device__ __forceinline__ void mx4_store(const Mx4Args &p, f32x4 (&acc)[PP_TN][PP_TM], LDS_AS char *staged, int64_t m0, int64_t n0)
{
    constexpr int TN = PP_TN;
    const int lane = threadIdx.x & 63;
    const bool has_bias = p.epi.bias != nullptr, relu = p.epi.relu != 0;
    if (!p.epi.c_f32 && p.epi.beta == 0.0f && (p.epi.ldc & 7) == 0 && (((uintptr_t)p.epi.C) & 15) == 0 && n0 + 16 * TN <= p.N) {
        constexpr int PITCH = 32 * TN + 8, LANES = 2 * TN;          // bytes, and lanes, of a row
        uint16_t *crow = (uint16_t *)p.epi.C + m0 * p.epi.ldc + n0;
        f32x4 add[TN];
#pragma unroll
        for (int a = 0; a < TN; ++a)
            add[a] = bias4(p.epi, n0 + 16 * a + 4 * (lane >> 4));
        static_for<0, PP_TM / 2>([&](auto bc) {
            constexpr int b2 = decltype(bc)::value;
            asm volatile("" ::: "memory");
            static_for<0, 2 * TN>([&](auto aq) {
                constexpr int bb = decltype(aq)::value / TN, a = decltype(aq)::value % TN;
                f32x4 v = acc[a][2 * b2 + bb];
                if (has_bias)
                    v += add[a];
                if (relu) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = v[e] < 0.0f ? 0.0f : v[e];           // NaN stays NaN
                }
                *(LDS_AS u32x2 *)(staged + (16 * bb + (lane & 15)) * PITCH + (16 * a + 4 * (lane >> 4)) * 2) =
                    u32x2{pack_c16x2(v[0], v[1], p.epi.c_f16), pack_c16x2(v[2], v[3], p.epi.c_f16)};
            });
            asm volatile("" ::: "memory");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < LANES / 2; ++i) {
                const int row = i * (64 / LANES) + lane / LANES, c8 = lane % LANES;
                const u32x2 lo = *(LDS_AS u32x2 *)(staged + row * PITCH + c8 * 16), hi = *(LDS_AS u32x2 *)(staged + row * PITCH + c8 * 16 + 8);
                if (m0 + b2 * 32 + row < p.M)
                    __builtin_nontemporal_store(u32x4{lo[0], lo[1], hi[0], hi[1]}, (u32x4 *)(crow + (int64_t)(b2 * 32 + row) * p.epi.ldc + c8 * 8));
            }
            __builtin_amdgcn_wave_barrier();
        });
        return;
    }
    constexpr int LD = 16 * TN + 4, LANES = 4 * TN;
    LDS_AS float *stage = (LDS_AS float *)staged;
    static_for<0, PP_TM / 2>([&](auto bc) {
        constexpr int b2 = decltype(bc)::value;
        asm volatile("" ::: "memory");
        static_for<0, 2 * TN>([&](auto aq) {
            constexpr int bb = decltype(aq)::value / TN, a = decltype(aq)::value % TN;
            *(LDS_AS f32x4 *)(stage + (16 * bb + (lane & 15)) * LD + 16 * a + 4 * (lane >> 4)) = acc[a][2 * b2 + bb];
        });
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int i = 0; i < LANES / 2; ++i) {
            const int row = i * (64 / LANES) + lane / LANES, c4 = lane % LANES;
            const f32x4 v = *(LDS_AS f32x4 *)(stage + row * LD + c4 * 4);
            const int64_t m = m0 + b2 * 32 + row, n = n0 + c4 * 4;
            if (m < p.M && n < p.N)
                gen_store4(p.epi, m, n, p.N - n, v);
        }
        __builtin_amdgcn_wave_barrier();
    });
}

}  // namespace

}  // namespace brg
