// Tiles of 16 to 128 rows and 64 or 128 columns of a product with a 4-bit image: four waves load, four multiply (bf16_stream128.hpp says why).
//
// Two images: a stage is 256 columns, A, B and the powers of both.  16-bit rows (mx4_half.hip has the fragments): with 64 rows the same, four blocks of 64 columns of A beside
// the weights (with a stage for each block the barrier and the way through LDS bound it: 512 x 4096 x 4096 25.7 us); with 128 rows LDS does not hold that, a stage is one block, and the
// weights come in a ring of three long blocks of their own, a quarter of one with each stage.  Every loading wave makes the same number of
// loads a stage, rows past an edge being the last one again, so the loads can be counted; what there is nothing to load for any more is loaded
// again, to where nobody reads.
// Binary16: the conversion is exact for powers 2^-23 .. 2^13.  A multiplying wave looks at the powers as it gets them, and where one is outside the tile
// is taken again as mx4_direct does, which splits A's values instead (all powers looked through first: 512 x 4096 x 4096 21.3 us, so 20.1; 16 x 11008 x 4096 12.3 and
// 11.3).  In bf16 it is for powers up to 2^125 (not_finite).
// One barrier a stage publishes it and frees the slot of the one before; a multiplying wave reads the first half of a block while the matrix pipe works
// on the second half of the last.
#pragma once
#include "mx4_direct.hpp"

namespace brg {

namespace {

// A stage holds SUBS blocks of A, and B beside it unless that has a ring of its own.
template <int LEFT, int BM, int BN>
struct Mx4Ring {
    static constexpr bool IMAGE = LEFT == LEFT_MX4, APART = !IMAGE && BM == 128;
    static constexpr int SUBS = IMAGE || APART ? 1 : 4;
    static constexpr uint32_t A_BYTES = BM * MX_ROW, B_BYTES = BN * MX_ROW, POWERS = IMAGE ? (BM + BN) * 8 : 0;
    static constexpr uint32_t STAGE = SUBS * A_BYTES + (APART ? 0 : B_BYTES) + POWERS;
    // (16 rows: three workgroups a CU; with five stages two, 32 rows of 7 experts, 11008 x 4096 out of memory, 43 us instead of 38, with two 40)
    static constexpr int STAGES = APART ? 5 : !IMAGE || (BM == 64 && BN == 128) ? 3 : 4;
    static constexpr uint32_t LONG = STAGE * STAGES;            // APART: where the three long blocks are
    static constexpr uint32_t SUMS = BM * (BN + 4) * 4;
    static constexpr uint32_t BYTES = LONG + (APART ? 3 * B_BYTES : 0);
    static constexpr uint32_t VOTES = BYTES - 64;
    static_assert(SUMS <= VOTES, "the sums end before the votes");
    static constexpr size_t LDS = BYTES;
};

// Not 0 where one of 8 powers is outside 2^-23 .. 2^13.
__device__ __forceinline__ uint32_t beyond_f16(u32x2 powers)
{
    uint32_t out = 0;                           // of two bytes at a time, e + 255 - most and e + 256 - least
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t e = (powers[i >> 1] >> (8 * (i & 1))) & 0x00ff00ffu;
        out |= (e + 0x00010001u * (255 - MX_F16_MOST)) | ~(e + 0x00010001u * (256 - MX_F16_LEAST));
    }
    return out & 0x01000100u;
}

// False where binary16 does not hold the tile's weights; nothing is stored then.
template <int LEFT, int BM, int BN>
__device__ __forceinline__ bool mx4_stream_body(const Mx4Args &p, int tm, int tn, int slice)
{
    typedef Mx4Ring<LEFT, BM, BN> R;
    constexpr bool IMAGE = R::IMAGE, APART = R::APART;
    constexpr int SUBS = R::SUBS;
    typedef KMajorTile<BM, 4> ATile;
    typedef KMajorTile<BN, 4> BTile;
    // (16-bit rows: no column by two waves, see widen_bf16)
    constexpr int WAVES_M = IMAGE ? 2 : 1, WM = BM / WAVES_M, WN = BN * WAVES_M / 4, TM = WM / 16, TN = WN / 16;
    // (of four blocks of A a loading wave has one)
    constexpr int LA = SUBS == 4 ? BM / 8 : ATile::kPerWave, LB = BTile::kPerWave, L = IMAGE ? LA + LB + 2 : APART ? LA + 1 : LA + LB;
    constexpr int stages = R::STAGES, ahead = stages - 1;
    static_assert((stages - 2) * L <= 63, "outstanding loads must fit vmcnt");

    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    LDS_AS char *smem = (LDS_AS char *)smem_generic;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    // This slice's long blocks, and its blocks.
    const int begin = slice * p.per, end = begin + p.per < p.blocks ? begin + p.per : p.blocks;
    const int n_long = end > begin ? end - begin : 0;
    const int last = (int)((p.K + 63) / 64) - begin * 4;
    const int n_iter = IMAGE ? n_long : n_long * 4 < last ? n_long * 4 : last;
    const int n_stages = APART ? n_iter : n_long;

    if (w >= 4) {
        // ---------------- loading waves ----------------
        const int wl = w - 4;
        uint32_t a_src[LA];
#pragma unroll
        for (int j = 0; j < LA; ++j)
            a_src[j] = ATile::src_rel_bytes(SUBS == 4 ? 0 : wl, j, lane, m0, p.M, p.lda / 2);
        // APART: wave-load 4 q + wl in quarter q
        auto b_load = [&](int j) { return APART ? 4 * j + wl : wl * LB + j; };
        constexpr int LBQ = APART ? 4 : LB;
        uint32_t b_src[LBQ];
        static_assert(!APART || BN == 128, "a wave-load for every loading wave in every quarter");
#pragma unroll
        for (int j = 0; j < LBQ; ++j)
            b_src[j] = BTile::src_rel_bytes(0, b_load(j), lane, n0, p.N, p.ldb / 2);
        const char *a_ptr = p.A + m0 * p.lda + (int64_t)begin * (IMAGE ? MX_ROW : 4 * MX_ROW);
        const char *b_ptr = p.B + n0 * p.ldb + (int64_t)begin * MX_ROW;
        const char *ap_ptr = p.a_powers + m0 * 8 + begin * p.a_plane, *bp_ptr = p.b_powers + n0 * 8 + begin * p.b_plane;
        // Powers of 32 rows a wave-load, A's first.
        uint32_t power_src[2] = {0, 0}, power_dst[2] = {0, 0};
        bool power_of_a[2] = {false, false};
        if constexpr (IMAGE) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int i = (2 * wl + k) % ((BM + BN) / 32);
                power_of_a[k] = i < BM / 32;
                const int row = (power_of_a[k] ? i : i - BM / 32) * 32 + (lane >> 1);
                const int64_t left = power_of_a[k] ? p.M - m0 : p.N - n0;
                power_src[k] = (uint32_t)(row < left ? row : (int)left - 1) * 8 + (lane & 1) * 4;
                power_dst[k] = R::A_BYTES + R::B_BYTES + (uint32_t)i * 256u;
            }
        }
        int slot = 0, buffer = 1;
        auto issue_block = [&](int t) {
            const uint32_t base = (uint32_t)slot * R::STAGE;
            if constexpr (!APART) {
#pragma unroll
                for (int j = 0; j < LB; ++j)
                    load16_to_lds_saddr(b_ptr, b_src[j], (uint32_t)(size_t)(smem + base + SUBS * R::A_BYTES + (uint32_t)b_load(j) * 1024u));
                b_ptr += MX_ROW;
                if constexpr (IMAGE) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        load4_to_lds_saddr(power_of_a[k] ? ap_ptr : bp_ptr, power_src[k], (uint32_t)(size_t)(smem + base + power_dst[k]));
                    ap_ptr += p.a_plane;
                    bp_ptr += p.b_plane;
                }
            } else {
                // a quarter of the next long block, or, behind the last, of that one again
                const int q = t & 3;
                const char *from = b_ptr + ((t >> 2) + 1 < n_long ? MX_ROW : 0);
                const uint32_t to = R::LONG + (uint32_t)buffer * R::B_BYTES;
                static_for<0, 4>([&](auto qc) {
                    constexpr int k = decltype(qc)::value;
                    if (q == k)
                        load16_to_lds_saddr(from, b_src[k], (uint32_t)(size_t)(smem + to + (uint32_t)b_load(k) * 1024u));
                });
                if (q == 3) {
                    b_ptr = from;
                    buffer = buffer == 2 ? 0 : buffer + 1;
                }
            }
            // (behind the last block of A, that one again)
            const char *from = a_ptr + (SUBS == 1 ? 0 : (SUBS * t + wl < n_iter ? wl : n_iter - 1 - SUBS * t) * MX_ROW);
#pragma unroll
            for (int j = 0; j < LA; ++j)
                load16_to_lds_saddr(from, a_src[j], (uint32_t)(size_t)(smem + base + (SUBS == 4 ? (uint32_t)wl * R::A_BYTES + (uint32_t)j * 1024u : ATile::dst_byte(wl, j))));
            a_ptr += SUBS * MX_ROW;
            slot = slot + 1 == stages ? 0 : slot + 1;
        };
        if constexpr (APART) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n_iter > 0)
                    load16_to_lds_saddr(b_ptr, b_src[k], (uint32_t)(size_t)(smem + R::LONG + (uint32_t)b_load(k) * 1024u));
        }
        for (int t = 0; t < ahead && t < n_stages; ++t)
            issue_block(t);
        for (int t = 0; t < n_stages; ++t) {
            // Stage t has landed once only the stages - 2 younger ones are outstanding.
            if (t + ahead - 1 < n_stages)
                wait_vmcnt_le<(stages - 2) * L>();
            else
                wait_vmcnt0();
            block_sync();
            if (t + ahead < n_stages)
                issue_block(t + ahead);
        }
        block_sync();
    } else {
        // ---------------- multiplying waves ----------------
        const int wm = IMAGE ? w >> 1 : 0, wn = IMAGE ? w & 1 : w;
        f32x4 acc[TN][TM];
#pragma unroll
        for (int a = 0; a < TN; ++a)
#pragma unroll
            for (int b = 0; b < TM; ++b)
                acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        bf16x8 fa[2][TM];
        i32x4 fb[2][TN];                        // IMAGE
        uint32_t codes[2][TN], factor[2][TN];   // 16-bit rows
        uint32_t pa[2][(TM + 1) / 2], pb[2][(TN + 1) / 2];      // IMAGE: powers of two fragments each
        u32x2 powers[TN], next[TN];             // 16-bit rows: of a long block
        uint32_t beyond = 0;
        const int r = lane & 15, q = lane >> 4;
        const uint32_t lane_pair = lane & 16 ? 0x07060302u : 0x05040100u;
        const char *bp_row[TN];
        if constexpr (!IMAGE) {
#pragma unroll
            for (int a = 0; a < TN; ++a) {
                const int64_t n = n0 + wn * WN + 16 * a + r;
                bp_row[a] = p.b_powers + (n < p.N ? n : p.N - 1) * 8 + begin * p.b_plane;
                if (n_iter > 0)
                    next[a] = *(const u32x2 *)bp_row[a];
            }
        }
        // Powers of fragments i and i + 1.
        auto powers_of = [&](LDS_AS char *at) {
            return __builtin_amdgcn_perm(*(LDS_AS uint32_t *)(at + 128), *(LDS_AS uint32_t *)at, lane_pair);
        };
        auto read_half = [&](auto hc, int slot, const int u, int buffer) {
            constexpr int h = decltype(hc)::value;
            LDS_AS char *at = smem + (uint32_t)slot * R::STAGE;
            if constexpr (IMAGE) {
                LDS_AS char *pw = at + R::A_BYTES + R::B_BYTES + r * 8 + (q >> 1) * 4;
                if constexpr (h == 0) {
#pragma unroll
                    for (int i = 0; i < TN; i += 2)
                        pb[0][i / 2] = powers_of(pw + BM * 8 + (wn * WN + 16 * i) * 8);
#pragma unroll
                    for (int i = 0; i < TM; i += 2)
                        pa[0][i / 2] = powers_of(pw + (wm * WM + 16 * i) * 8);
                } else {
                    // (those of the first half are read while the second half of the last block still needs its own)
#pragma unroll
                    for (int i = 0; i < TN / 2; ++i)
                        pb[1][i] = pb[0][i];
#pragma unroll
                    for (int i = 0; i < TM / 2; ++i)
                        pa[1][i] = pa[0][i];
                }
#pragma unroll
                for (int i = 0; i < TN; ++i)
                    fb[h][i] = __builtin_bit_cast(i32x4, BTile::read_frag16(at + R::A_BYTES, wn * WN, i, h, lane));
            } else {
                LDS_AS char *bt = (APART ? smem + R::LONG + (uint32_t)buffer * R::B_BYTES : at + SUBS * R::A_BYTES) + (wn * WN + r) * MX_ROW + 4 * q;
                const uint32_t chunk = (uint32_t)((2 * u + h) ^ (r >> 1)) << 4;
                const uint32_t turn = (uint32_t)(9 + 4 * (u & 2) + 16 * h);
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    codes[h][i] = *(LDS_AS uint32_t *)(bt + chunk + i * 16 * MX_ROW);
                    const uint32_t word = u & 1 ? powers[i][1] : powers[i][0];
                    factor[h][i] = __builtin_amdgcn_alignbit(word, word, turn);
                }
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[h][i] = ATile::read_frag16(at + (SUBS == 1 ? 0 : (uint32_t)u * R::A_BYTES), wm * WM, i, h, lane);
        };
        auto mfma_half = [&](auto hc) {
            constexpr int h = decltype(hc)::value;
            static_for<0, TN>([&](auto ac) {
                constexpr int a = decltype(ac)::value;
                if constexpr (IMAGE) {
                    static_for<0, TM>([&](auto bc) {
                        constexpr int b = decltype(bc)::value;
                        acc[a][b] = mfma_mx4<2 * (a & 1) + h, 2 * (b & 1) + h>(fb[h][a], __builtin_bit_cast(i32x4, fa[h][b]), acc[a][b],
                                                                              (int)pb[h][a / 2], (int)pa[h][b / 2]);
                    });
                } else {
                    const float f = __uint_as_float(factor[h][a]);
                    const bf16x8 v = LEFT == LEFT_F16 ? __builtin_bit_cast(bf16x8, widen_f16(codes[h][a], f)) : widen_bf16(codes[h][a], f);
#pragma unroll
                    for (int b = 0; b < TM; ++b)
                        acc[a][b] = mfma_16x16x32<LEFT == LEFT_F16 ? KIND_F16 : KIND_BF16>(v, fa[h][b], acc[a][b]);
                }
            });
        };
        constexpr std::integral_constant<int, 0> H0{};
        constexpr std::integral_constant<int, 1> H1{};
        int slot = 0, buffer = 0;
        // Block u of a long one (IMAGE: u = 0).
        auto block = [&](auto first, auto uc) {
            constexpr int u = decltype(uc)::value;
            if constexpr (SUBS == 1 || u == 0)
                block_sync();                   // its stage is in LDS
            read_half(H0, slot, u, buffer);
            if constexpr (!decltype(first)::value)
                mfma_half(H1);                  // second half of the block before
            __builtin_amdgcn_sched_barrier(0);
            read_half(H1, slot, u, buffer);
            mfma_half(H0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (SUBS == 1 || u == 3) {
                wait_lgkmcnt0();                // before the loaders may overwrite the slot
                slot = slot + 1 == stages ? 0 : slot + 1;
            }
        };
        if constexpr (IMAGE) {
            if (n_iter > 0) {
                block(std::true_type{}, H0);
                for (int t = 1; t < n_iter; ++t)
                    block(std::false_type{}, H0);
                mfma_half(H1);
            }
        } else {
            // (The first half of all adds zeros.  Four blocks are written out: in a loop over blocks the compiler waits for `next` in every
            // one, 1 us for each long block.)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[1][i] = __builtin_bit_cast(bf16x8, i32x4{0, 0, 0, 0});
#pragma unroll
            for (int i = 0; i < TN; ++i)
                codes[1][i] = factor[1][i] = 0;
            auto long_block = [&](int i, auto whole, int blocks) {
#pragma unroll
                for (int a = 0; a < TN; ++a) {
                    powers[a] = next[a];
                    if constexpr (LEFT == LEFT_F16)
                        beyond |= beyond_f16(powers[a]);
                    bp_row[a] += i + 1 < n_long ? p.b_plane : 0;
                    next[a] = *(const u32x2 *)bp_row[a];
                }
                static_for<0, 4>([&](auto uc) {
                    if (decltype(whole)::value || decltype(uc)::value < blocks)
                        block(std::false_type{}, uc);
                });
                buffer = buffer == 2 ? 0 : buffer + 1;
            };
            int i = 0;
            for (; 4 * i + 4 <= n_iter; ++i)
                long_block(i, std::true_type{}, 4);
            if (4 * i < n_iter)
                long_block(i, std::false_type{}, n_iter - 4 * i);
            if (n_iter > 0)
                mfma_half(H1);
            wait_lgkmcnt0();
        }
        block_sync();                           // nobody reads fragments any more
        LDS_AS float *stage = (LDS_AS float *)smem;
#pragma unroll
        for (int a = 0; a < TN; ++a)
#pragma unroll
            for (int b = 0; b < TM; ++b)
                *(LDS_AS f32x4 *)(stage + (wm * WM + 16 * b + r) * (BN + 4) + wn * WN + 16 * a + 4 * q) = acc[a][b];
        if constexpr (LEFT == LEFT_BF16) {
            if (__builtin_expect(not_finite(acc), 0) && far_powers(p, n0 + wn * WN, WN, begin, end, 1)) {
#pragma unroll 1
                for (int i = 0; i < TM * TN; ++i)
                    *(LDS_AS f32x4 *)(stage + (16 * (i % TM) + r) * (BN + 4) + wn * WN + 16 * (i / TM) + 4 * q) =
                        far_sum<LEFT>(p, m0 + 16 * (i % TM), n0 + wn * WN + 16 * (i / TM), begin, end, 1);
            }
        }
        if constexpr (LEFT == LEFT_F16) {
            const bool any = __builtin_amdgcn_ballot_w64(beyond != 0) != 0;
            if (lane == 0)
                *(LDS_AS int *)(smem + R::VOTES + w * 4) = any;
        }
        wait_lgkmcnt0();
    }
    block_sync();
    if constexpr (LEFT == LEFT_F16) {
        LDS_AS int *vote = (LDS_AS int *)(smem + R::VOTES);
        const int any = vote[0] | vote[1] | vote[2] | vote[3];
        block_sync();
        // (a block of zeros has the least power)
        if (any && !powers_fit<BN>(p, tn, smem + R::VOTES))
            return false;
    }
    // Whole rows of the tile, by all waves.
    LDS_AS float *stage = (LDS_AS float *)smem;
    float *part = p.split > 1 ? p.partial + (int64_t)slice * p.M * p.N : nullptr;
    for (int i = tid; i < BM * BN / 4; i += 512) {
        const int row = i / (BN / 4), col = i % (BN / 4) * 4;
        const int64_t m = m0 + row, n = n0 + col;
        if (m >= p.M || n >= p.N)
            continue;
        const f32x4 v = *(LDS_AS f32x4 *)(stage + row * (BN + 4) + col);
        if (part)
            store4_partial(part + m * p.N + n, p.N - n, (p.N & 3) == 0, v[0], v[1], v[2], v[3]);
        else
            gen_store4(p.epi, m, n, p.N - n, v);
    }
    return true;
}

// The tile, whatever its weights are.
template <int LEFT, int BM, int BN>
__device__ __forceinline__ void mx4_stream_tile(const Mx4Args &p, int tm, int tn, int slice)
{
    const bool stored = mx4_stream_body<LEFT, BM, BN>(p, tm, tn, slice);
    if constexpr (LEFT == LEFT_F16) {
        extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
        if (!stored)
            direct_tile<BM, BN>(p, (int64_t)tm * BM, tn, slice, (LDS_AS float *)(LDS_AS char *)smem_generic);
    }
}

}  // namespace

}  // namespace brg
