// A tile of a product with a 4-bit image whose operands go from memory to registers (mx4_direct.hip; the other kernels of binary16 rows for
// weights that binary16 does not hold), and results beside weights that bf16 does not hold either.
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

// Weights under 2^126 and 2^127 (images that others quantised) may be beyond bf16, and widen_bf16 makes infinities of them.  Then all
// results of that column are none that is finite, whatever the row holds: one row of a wave's results tells whether to look at the powers.
template <int TN, int TM>
__device__ __forceinline__ bool not_finite(const f32x4 (&acc)[TN][TM])
{
    uint64_t none = 0;
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            none |= __builtin_amdgcn_ballot_w64(!__builtin_isfinite(acc[a][0][i]));
    return none != 0;
}

// Whether one of `columns` weights from n0 on has such a power in one of the blocks from, from + step, .. before end (a wave's question).
__device__ __forceinline__ bool far_powers(const Mx4Args &p, int64_t n0, int columns, int from, int end, int step)
{
    const int lane = threadIdx.x & 63;
    bool far = false;
#pragma unroll 1
    for (int i = lane & 15; i < columns; i += 16) {
        const char *at = p.b_powers + (n0 + i < p.N ? n0 + i : p.N - 1) * 8;
#pragma unroll 1
        for (int kb = from + (lane >> 4) * step; kb < end; kb += 4 * step) {
            const u32x2 v = *(const u32x2 *)(at + kb * p.b_plane);
#pragma unroll
            for (int b = 0; b < 8; ++b)
                far = far || ((v[b >> 2] >> (8 * (b & 3))) & 255) - 253u < 2u;
        }
    }
    return __builtin_amdgcn_ballot_w64(far) != 0;
}

// 16 x 16 results from (m0, n0) on of those blocks beside 16-bit rows, whatever the powers are, in the accumulators' layout.  Weights that may be beyond
// bf16 are widened under a power 2^8 lower, and meet the row's value times 2^8, clamped to where that does not overflow (from 2^119 on every
// product with such a weight is an infinity).  Weights under other powers, and what is not finite in a row, have instructions of their own, so that
// no zero that fills a gap meets an infinity.  Takes few registers, so that its callers keep theirs, and its time.
template <int LEFT>
__device__ __forceinline__ f32x4 far_sum(const Mx4Args &p, int64_t m0, int64_t n0, int from, int end, int step)
{
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int64_t m = m0 + r < p.M ? m0 + r : p.M - 1, n = n0 + r < p.N ? n0 + r : p.N - 1;
    const char *a_row = p.A + m * p.lda, *b_row = p.B + n * p.ldb + 4 * q, *b_pow = p.b_powers + n * 8;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int i = 0; from + (i >> 3) * step < end; ++i) {
        const int kb = from + (i >> 3) * step, e = i & 7;
        const uint32_t codes = *(const uint32_t *)(b_row + (int64_t)kb * MX_ROW + e * 16);
        const uint32_t power = (uint8_t)b_pow[kb * p.b_plane + 2 * (e & 3) + (e >> 2)];
        const s16x8 x = load_left(a_row, (int64_t)kb * MX_K + 32 * e + 8 * q, p.K);
        const bool far = power - 253u < 2u;
        const i32x4 all = __builtin_bit_cast(i32x4, widen_bf16(codes, __uint_as_float((far ? power - 8 : power) << 23)));
        const i32x4 near_ones = far ? i32x4{0, 0, 0, 0} : all, far_ones = far ? all : i32x4{0, 0, 0, 0};
        auto add = [&](bf16x8 v) {
            bf16x8 finite, lifted, other;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float f = (float)v[k];
                const bool is = __builtin_isfinite(f);
                finite[k] = is ? v[k] : (__bf16)0.0f;
                other[k] = is ? (__bf16)0.0f : v[k];
                lifted[k] = (__bf16)(is ? 256.0f * fminf(fmaxf(f, -0x1p119f), 0x1p119f) : 0.0f);
            }
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, near_ones), finite, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, far_ones), lifted, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, all), other, acc, 0, 0, 0);
        };
        if constexpr (LEFT == LEFT_F16) {
            bf16x8 high, low;
            split_f16(__builtin_bit_cast(f16x8, x), high, low);
            add(low);
            add(high);
        } else {
            add(__builtin_bit_cast(bf16x8, x));
        }
    }
    return acc;
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
    // The next block's weights are requested before this one's products.  (Behind the last none: registers that a request holds are waited for at the
    // end, 16 x 4096 x 4096 7.4 us instead of 7.1.)
    const int first = slice * p.per + w;
    Weights wt;
    if (first < end)
        load_weights(first, wt);
    for (int kb = first; kb < end; kb += W) {
        Weights next;
        Rows rows;
        load_rows(kb, rows);
        if (kb + W < end)
            load_weights(kb + W, next);
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
    if constexpr (LEFT != LEFT_MX4) {
        if (__builtin_expect(not_finite(acc), 0) && far_powers(p, n0, 16 * TN, first, end, W)) {
#pragma unroll 1
            for (int i = 0; i < TM * TN; ++i)
                *(LDS_AS f32x4 *)(sums + w * SLICE + (16 * (i % TM) + r) * LD + 16 * (i / TM) + 4 * q) =
                    far_sum<LEFT>(p, m0 + 16 * (i % TM), n0 + 16 * (i / TM), first, end, W);
        }
    }
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
