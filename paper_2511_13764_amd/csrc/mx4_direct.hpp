// A tile of a product with a 4-bit image whose operands go from memory to registers (mx4_direct.hip; mx4_half.hip for the weights that binary16
// does not hold).
#pragma once
#include "mx4.hpp"

namespace brg {

namespace {

// Eight 16-bit values of a row at k, zeros from K on.
__device__ __forceinline__ s16x8 load_left(const char *row, int64_t k, int64_t K)
{
    const uint16_t *x = (const uint16_t *)row + k;
    if (k + 8 <= K)
        return *(const s16x8_any2 *)x;
    s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K)
            v[i] = (short)x[i];
    return v;
}

// W waves share the reduction.  sums: W * 16 TM * (16 TN + 4).
template <int LEFT, int TM, int TN, int W>
__device__ __forceinline__ void direct_body(const Mx4Args &p, int tm, int tn, int slice, LDS_AS float *sums)
{
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)tm * 16 * TM, n0 = (int64_t)tn * 16 * TN;
    const int r = lane & 15, q = lane >> 4;

    const char *a_row[TM], *a_pow[TM], *b_row[TN], *b_pow[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + 16 * i + r < p.M ? m0 + 16 * i + r : p.M - 1;
        a_row[i] = p.A + m * p.lda;
        a_pow[i] = p.a_powers + m * 8 + 2 * q;
    }
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        const int64_t n = n0 + 16 * i + r < p.N ? n0 + 16 * i + r : p.N - 1;
        b_row[i] = p.B + n * p.ldb + 16 * q;
        b_pow[i] = p.b_powers + n * 8 + 2 * q;
    }
    f32x4 acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i)
            acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int end = (slice + 1) * p.per < p.blocks ? (slice + 1) * p.per : p.blocks;
    for (int kb = slice * p.per + w; kb < end; kb += W) {
        i32x4 b[TN][2];
        uint32_t bp[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            b[j][0] = *(const i32x4 *)(b_row[j] + (int64_t)kb * MX_ROW);
            b[j][1] = *(const i32x4 *)(b_row[j] + (int64_t)kb * MX_ROW + 64);
            bp[j] = *(const uint16_t *)(b_pow[j] + kb * p.b_plane);
        }
        if constexpr (LEFT == LEFT_MX4) {
            i32x4 a[TM][2];
            uint32_t ap[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                a[i][0] = *(const i32x4 *)(a_row[i] + (int64_t)kb * MX_ROW + 16 * q);
                a[i][1] = *(const i32x4 *)(a_row[i] + (int64_t)kb * MX_ROW + 16 * q + 64);
                ap[i] = *(const uint16_t *)(a_pow[i] + kb * p.a_plane);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    acc[j][i] = mfma_mx4<0, 0>(b[j][0], a[i][0], acc[j][i], (int)bp[j], (int)ap[i]);
                    acc[j][i] = mfma_mx4<1, 1>(b[j][1], a[i][1], acc[j][i], (int)bp[j], (int)ap[i]);
                }
        } else {
            const int64_t k0 = (int64_t)kb * MX_K;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                bool narrow = true;             // the powers are such that binary16 holds the weights
                if constexpr (LEFT == LEFT_F16) {
                    bool in = true;
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const uint32_t e = (bp[j] >> (8 * s)) & 255;
                        in = in && e >= MX_F16_LEAST && e <= MX_F16_MOST;
                    }
                    narrow = __builtin_amdgcn_ballot_w64(!in) == 0;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    s16x8 a[TM];
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        a[i] = load_left(a_row[i], k0 + 32 * (4 * s + q) + 8 * c, p.K);
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const float power = mx4_power((bp[j] >> (8 * s)) & 255);
                        const uint32_t codes = (uint32_t)b[j][s][c];
                        if constexpr (LEFT == LEFT_BF16) {
                            const bf16x8 v = widen_bf16(codes, power);
#pragma unroll
                            for (int i = 0; i < TM; ++i)
                                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, a[i]), acc[j][i], 0, 0, 0);
                        } else if (narrow) {
                            const f16x8 v = widen_f16(codes, power);
#pragma unroll
                            for (int i = 0; i < TM; ++i)
                                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(f16x8, a[i]), acc[j][i], 0, 0, 0);
                        } else {
                            const bf16x8 v = widen_bf16(codes, power);
#pragma unroll
                            for (int i = 0; i < TM; ++i) {
                                bf16x8 high, low;
                                split_f16(__builtin_bit_cast(f16x8, a[i]), high, low);
                                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low, acc[j][i], 0, 0, 0);
                                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high, acc[j][i], 0, 0, 0);
                            }
                        }
                    }
                }
            }
        }
    }

    // A lane has row l % 16 and four neighbouring columns of every 16 x 16.
    constexpr int LD = 16 * TN + 4, SLICE = 16 * TM * LD;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i)
            *(LDS_AS f32x4 *)(sums + w * SLICE + (16 * i + r) * LD + 16 * j + 4 * q) = acc[j][i];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * TM * 4 * TN; i += 64 * W) {
        const int row = i / (4 * TN), col = i % (4 * TN) * 4;
        f32x4 v = *(LDS_AS f32x4 *)(sums + row * LD + col);
#pragma unroll
        for (int s = 1; s < W; ++s)
            v += *(LDS_AS f32x4 *)(sums + s * SLICE + row * LD + col);
        if (m0 + row >= p.M || n0 + col >= p.N)
            continue;
        if (p.split > 1)
            store4_partial(p.partial + ((int64_t)slice * p.M + m0 + row) * p.N + n0 + col, p.N - n0 - col, (p.N & 3) == 0, v[0], v[1], v[2], v[3]);
        else
            gen_store4(p.epi, m0 + row, n0 + col, p.N - n0 - col, v);
    }
}

// Workgroups of 512: true in all threads where every power of the tile's weights is one that binary16 takes (or of a block of zeros).
template <int BN>
__device__ __forceinline__ bool powers_fit(const Mx4Args &p, int tn, LDS_AS char *smem)
{
    bool fit = true;
    const int64_t n = (int64_t)tn * BN + (threadIdx.x % BN);
    if (n < p.N) {
        for (int kb = threadIdx.x / BN; kb < p.blocks; kb += 512 / BN) {
            const u32x2 v = *(const u32x2 *)(p.b_powers + kb * p.b_plane + n * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t e = (v[i >> 2] >> (8 * (i & 3))) & 255;
                if (e == 0) {                   // place i: block 4 (i % 2) + i / 2
                    const u32x4 c = *(const u32x4 *)(p.B + n * p.ldb + (int64_t)kb * MX_ROW + (4 * (i & 1) + (i >> 1)) * 16);
                    fit = fit && ((c[0] | c[1] | c[2] | c[3]) & 0x77777777u) == 0;
                } else {
                    fit = fit && e >= MX_F16_LEAST && e <= MX_F16_MOST;
                }
            }
        }
    }
    LDS_AS int *vote = (LDS_AS int *)smem;
    if ((threadIdx.x & 63) == 0)
        vote[threadIdx.x >> 6] = 1;
    if (!fit)
        vote[threadIdx.x >> 6] = 0;             // (behind the store of 1: LDS keeps a wave's order)
    __syncthreads();
    int all = 1;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        all &= vote[i];
    __syncthreads();
    return all != 0;
}

// A tile of other weights beside binary16 rows, 32 x 32 at a time, by 512 threads (37 KB of LDS).
template <int BM, int BN>
__device__ __forceinline__ void direct_tile(const Mx4Args &p, int tm, int tn, int slice, LDS_AS float *sums)
{
    for (int i = 0; i < BM * BN / 1024; ++i) {
        const int m = tm * (BM / 32) + i % (BM / 32), n = tn * (BN / 32) + i / (BM / 32);
        if ((int64_t)m * 32 < p.M && (int64_t)n * 32 < p.N)
            direct_body<LEFT_F16, 2, 2, 8>(p, m, n, slice, sums);
        __syncthreads();
    }
}

}  // namespace

}  // namespace brg
