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

// Four registers of four groups of 16 lanes: word c of group q becomes word q of group c.
__device__ __forceinline__ void turn_over(i32x4 &x)
{
    const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)x[0], (uint32_t)x[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)x[1], (uint32_t)x[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    x = i32x4{(int)c[0], (int)c[1], (int)d[0], (int)d[1]};
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
        b_pow[i] = p.b_powers + n * 8 + (LEFT == LEFT_MX4 ? 2 * q : 0);
    }
    f32x4 acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i)
            acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int end = (slice + 1) * p.per < p.blocks ? (slice + 1) * p.per : p.blocks;
    // Images: a lane has the codes and powers of blocks q and 4 + q.  16-bit rows: of every block e the codes 8 q .. + 7, and its power.
    constexpr int PER = LEFT == LEFT_MX4 ? 2 : 8;
    struct Weights {
        i32x4 codes[TN][2];
        u32x2 powers[TN];
    };
    struct Rows {
        i32x4 v[TM][PER];
        uint32_t powers[TM];
    };
    auto load_weights = [&](int kb, Weights &x) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            x.codes[j][0] = *(const mx4_codes *)(b_row[j] + (int64_t)kb * MX_ROW);
            x.codes[j][1] = *(const mx4_codes *)(b_row[j] + (int64_t)kb * MX_ROW + 64);
            if constexpr (LEFT == LEFT_MX4)
                x.powers[j][0] = *(const uint16_t *)(b_pow[j] + kb * p.b_plane);
            else
                x.powers[j] = *(const u32x2 *)(b_pow[j] + kb * p.b_plane);
        }
    };
    auto load_rows = [&](int kb, Rows &x) {
        if constexpr (LEFT == LEFT_MX4) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                x.v[i][0] = *(const mx4_codes *)(a_row[i] + (int64_t)kb * MX_ROW + 16 * q);
                x.v[i][1] = *(const mx4_codes *)(a_row[i] + (int64_t)kb * MX_ROW + 16 * q + 64);
                x.powers[i] = *(const uint16_t *)(a_pow[i] + kb * p.a_plane);
            }
        } else {
            const int64_t k0 = (int64_t)kb * MX_K;
            if (k0 + MX_K <= p.K) {             // (no branch of the lane's between the requests)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        x.v[i][e] = __builtin_bit_cast(i32x4, (s16x8)*(const s16x8_any2 *)((const uint16_t *)a_row[i] + k0 + 32 * e + 8 * q));
            } else {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        x.v[i][e] = __builtin_bit_cast(i32x4, load_left(a_row[i], k0 + 32 * e + 8 * q, p.K));
            }
        }
    };
    auto multiply = [&](Weights &wt, const Rows &x) {
        if constexpr (LEFT == LEFT_MX4) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    acc[j][i] = mfma_mx4<0, 0>(wt.codes[j][0], x.v[i][0], acc[j][i], (int)wt.powers[j][0], (int)x.powers[i]);
                    acc[j][i] = mfma_mx4<1, 1>(wt.codes[j][1], x.v[i][1], acc[j][i], (int)wt.powers[j][0], (int)x.powers[i]);
                }
        } else {
            // Lane group q read block 4 s + q whole, 16 bytes; now word c is its part of block 4 s + c: the four groups' four words turned over.
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    turn_over(wt.codes[j][s]);
            // Power of block e: place 2 (e % 4) + e / 4, turned to where an exponent is (the conversion looks at that alone).
            auto factor = [&](int j, int e) {
                const int place = 2 * (e & 3) + (e >> 2);
                const uint32_t word = wt.powers[j][place >> 2];
                return __builtin_amdgcn_alignbit(word, word, 9 + 8 * (place & 3));
            };
            bool narrow = true;                 // the powers are such that binary16 holds the weights
            if constexpr (LEFT == LEFT_F16) {
                bool in = true;
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t e = (wt.powers[j][i >> 2] >> (8 * (i & 3))) & 255;
                        in = in && e >= MX_F16_LEAST && e <= MX_F16_MOST;
                    }
                narrow = __builtin_amdgcn_ballot_w64(!in) == 0;
            }
            if (narrow) {
#pragma unroll
                for (int e = 0; e < PER; ++e)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const float power = __uint_as_float(factor(j, e));
                        const uint32_t codes = (uint32_t)wt.codes[j][e >> 2][e & 3];
                        const bf16x8 v = LEFT == LEFT_F16 ? __builtin_bit_cast(bf16x8, widen_f16(codes, power)) : widen_bf16(codes, power);
#pragma unroll
                        for (int i = 0; i < TM; ++i)
                            acc[j][i] = mfma_16x16x32<LEFT == LEFT_F16 ? KIND_F16 : KIND_BF16>(v, __builtin_bit_cast(bf16x8, x.v[i][e]), acc[j][i]);
                    }
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e)
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        bf16x8 high, low;
                        split_f16(__builtin_bit_cast(f16x8, x.v[i][e]), high, low);
#pragma unroll
                        for (int j = 0; j < TN; ++j) {
                            const bf16x8 v = widen_bf16((uint32_t)wt.codes[j][e >> 2][e & 3], __uint_as_float(factor(j, e)));
                            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, low, acc[j][i], 0, 0, 0);
                            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, high, acc[j][i], 0, 0, 0);
                        }
                    }
            }
        }
    };
    // The next block's weights are requested before this one's products.
    const int first = slice * p.per + w;
    Weights wt;
    if (first < end)
        load_weights(first, wt);
    for (int kb = first; kb < end; kb += W) {
        Weights next;
        Rows rows;
        load_rows(kb, rows);
        load_weights(kb + W < end ? kb + W : kb, next);
        multiply(wt, rows);
        wt = next;
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
        for (int kb0 = threadIdx.x / BN; kb0 < p.blocks; kb0 += 4 * (512 / BN)) {
            u32x2 four[4];                      // (requested together)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int kb = kb0 + i * (512 / BN);
                four[i] = *(const u32x2 *)(p.b_powers + (kb < p.blocks ? kb : kb0) * p.b_plane + n * 8);
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int kb = kb0 + h * (512 / BN) < p.blocks ? kb0 + h * (512 / BN) : kb0;
                const u32x2 v = four[h];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t e = (v[i >> 2] >> (8 * (i & 3))) & 255;
                    if (e == 0) {                   // place i: block 4 (i % 2) + i / 2
                        const mx4_codes c = *(const mx4_codes *)(p.B + n * p.ldb + (int64_t)kb * MX_ROW + (4 * (i & 1) + (i >> 1)) * 16);
                        fit = fit && ((c[0] | c[1] | c[2] | c[3]) & 0x77777777u) == 0;
                    } else {
                        fit = fit && e >= MX_F16_LEAST && e <= MX_F16_MOST;
                    }
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

// A tile of other weights beside binary16 rows, 16 x 16 at a time, by 512 threads (10 KB of LDS; larger ones need more registers than the kernels
// that call this).
template <int BM, int BN>
__device__ __forceinline__ void direct_tile(const Mx4Args &p, int64_t m0, int tn, int slice, LDS_AS float *sums)
{
    for (int i = 0; i < BM / 16 * (BN / 16); ++i) {
        const int m = (int)(m0 / 16) + i % (BM / 16), n = tn * (BN / 16) + i / (BM / 16);
        if ((int64_t)m * 16 < p.M && (int64_t)n * 16 < p.N)
            direct_body<LEFT_F16, 1, 1, 8>(p, m, n, slice, sums);
        __syncthreads();
    }
}

}  // namespace

}  // namespace brg
