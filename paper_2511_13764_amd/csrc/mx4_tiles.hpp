// What the 256 x 256 kernels of 4-bit images share: tile, phases, loads and the epilogue.
#pragma once
#include "mx4.hpp"

namespace brg {

namespace {

constexpr int PP_BM = 256, PP_BN = 256;
constexpr int PP_TM = 8, PP_TN = 4;             // 16 x 16 tiles of a wave: 128 x 64; waves 0-3 above 4-7

__device__ __forceinline__ void phase_sync() { block_sync(); }

// First row and column tile of a workgroup's 256 x 256.  With groups all tiles of more than 128 rows come first: they take longer.
template <bool GROUPED>
__device__ __forceinline__ bool mx4_large_tile(Mx4Args &p, const GroupArgs &g, int64_t &m0, int &tn)
{
    if constexpr (GROUPED) {
        MixedTile m;
        if (!find_mixed_tile(g, p.tiles_n, p.walk, m))
            return false;
        select_piece(p, g, m.t);
        m0 = (int64_t)m.t.tm * (m.small ? PP_BM / 2 : PP_BM);
        tn = m.t.tn;
    } else {
        int tm;
        tile_coords(blockIdx.x, p.tiles_m, p.tiles_n, p.walk, tm, tn);
        m0 = (int64_t)tm * PP_BM;
    }
    return true;
}

// load16_to_lds_saddr with 4 bytes a lane.
__device__ __forceinline__ void load4_to_lds_saddr(const char *base, uint32_t lane_off, uint32_t lds_addr)
{
    const uint64_t b = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    const uint64_t ub = ((uint64_t)hi << 32) | lo;
    const uint32_t la = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :
                 : "s"(la), "v"(lane_off), "s"(ub)
                 : "m0");
}

// Sums of a wave, 128 x 16 TN from (m0, n0) on, in `acc` (lane l: row l % 16, columns 4 (l / 16) .. + 3 of every 16 x 16), to C: 32 rows at
// a time, staged in its own MX4_STAGED bytes of LDS at `staged`, stored in whole lines.
constexpr uint32_t MX4_STAGED = 32 * (64 + 4) * 4;
template <int TN>
__device__ __forceinline__ void mx4_store(const Mx4Args &p, f32x4 (&acc)[TN][PP_TM], LDS_AS char *staged, int64_t m0, int64_t n0)
{
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
