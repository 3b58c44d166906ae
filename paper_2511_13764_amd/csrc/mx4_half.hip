// 256 x 256 tiles of 16-bit rows with a 4-bit image: two wavefronts a SIMD in alternating phases.
//
// Phases, fragments of A and accumulators are those of the 16-bit kernel (bf16_pingpong.hpp), a block being 64 columns of A.  The weights stay 4 bits wide
// up to the registers: 256 columns of them are 128 bytes a row, so they come in blocks four times as long, a lane reads 4 bytes a
// fragment instead of 16, and four conversions, which also apply the power, make a fragment of those.  A fragment is 32 columns, one block of
// the image, of which lane l has the codes 8 (l / 16) .. + 7, so every lane needs one power a fragment.  The conversion looks at the exponent of
// its factor alone, so a byte among others becomes one by a rotation.
//   LDS: A in a ring of ten units of 64 rows, two blocks and a half; two of the long blocks of weights; two of their powers.
//   Waves 4-7 request the first half of A's block t + 2, waves 0-3 the second half of block t + 1; either takes a quarter of the next long block of weights
//   in each of the first two of the four blocks that it lasts.
// 16-bit weights of the same size would be 64 KB a block through LDS and 96 KB of fragments a phase; here it is 40 and 72.
// Binary16: the conversion is exact for powers 2^-23 .. 2^13.  A workgroup looks through its weights' powers first (2 KB for each 256 columns, about
// 1 us at K = 4096), and where one is outside takes its tile as mx4_direct does, which splits A's values instead.  In bf16 it is for powers up to 2^125
// (not_finite).
#include "mx4_tiles.hpp"

namespace brg {

namespace {

constexpr int BM = PP_BM, BN = PP_BN, TM = PP_TM, TN = PP_TN;
constexpr uint32_t UNIT = 8192, UNITS = 10;     // 64 rows x 64 columns of A
constexpr uint32_t WEIGHTS = UNIT * UNITS, LONG = 32768;        // 256 rows x 256 columns
constexpr uint32_t POWERS = WEIGHTS + 2 * LONG;
constexpr size_t LDS = POWERS + 2 * 2048;
static_assert(Mx4Ring<LEFT_BF16, 128, 128>::LDS <= LDS, "small tiles");
typedef KMajorTile<256, 4> Tile;                // rows of 128 bytes, both operands

template <bool F16, bool EDGE>
__device__ __forceinline__ void body(const Mx4Args &p, int64_t m0, int tn)
{
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    LDS_AS char *smem = (LDS_AS char *)smem_generic;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = w >> 2, wl = w & 3;       // waves w and w + 4 share a SIMD
    const int wm = group, wn = wl;
    const int64_t n0 = (int64_t)tn * BN;
    const int n_iter = (int)((p.K + 63) / 64);

    // Of a unit's eight wave-loads (8 rows each) wave wl takes 2 wl and 2 wl + 1.
    const int64_t a_step = 8 * p.lda, b_step = 8 * p.ldb;
    const char *a_ptr = (const char *)uniform_ptr((const uint16_t *)(p.A + (m0 + (group ? 0 : 128) + 16 * wl) * p.lda));
    // (unit 2 u + group of the weights in the long block's block u = 0, 1)
    const char *b_ptr = (const char *)uniform_ptr((const uint16_t *)(p.B + (n0 + 64 * group + 16 * wl) * p.ldb));
    const char *bp_ptr = p.b_powers + n0 * 8;
    const uint32_t a_lane0 = Tile::lane_off_bytes(0, lane, p.lda / 2), a_lane1 = Tile::lane_off_bytes(1, lane, p.lda / 2);
    const uint32_t b_lane0 = Tile::lane_off_bytes(0, lane, p.ldb / 2), b_lane1 = Tile::lane_off_bytes(1, lane, p.ldb / 2);
    const int a_left = (int)((p.M < m0 + 256 ? p.M : m0 + 256) - m0) - (group ? 0 : 128) - 16 * wl;
    const int b_left = (int)((p.N < n0 + 256 ? p.N : n0 + 256) - n0) - 64 * group - 16 * wl;
    auto slot_of = [](int first, int u) { return first + u >= (int)UNITS ? first + u - (int)UNITS : first + u; };
    // Wave-load j of 4 of the wave's two units of A, the first of which has slot `first`.
    auto issue_a = [&](int j, int first) {
        const uint32_t dst = (uint32_t)slot_of(first, j / 2) * UNIT + (uint32_t)(2 * wl + j % 2) * 1024u;
        if (!EDGE || (lane >> 3) < a_left - 64 * (j / 2) - 8 * (j % 2))
            load16_to_lds_saddr(a_ptr + (8 * (j / 2) + j % 2) * a_step, j % 2 ? a_lane1 : a_lane0, (uint32_t)(size_t)(smem + dst));
    };
    // Wave-load j of 2 of the next long block's unit 2 u + group.
    auto issue_b = [&](int j, int u, uint32_t buffer) {
        const uint32_t dst = WEIGHTS + buffer * LONG + (uint32_t)(2 * u + group) * UNIT + (uint32_t)(2 * wl + j) * 1024u;
        if (!EDGE || (lane >> 3) < b_left - 128 * u - 8 * j)
            load16_to_lds_saddr(b_ptr + (16 * u + j) * b_step, j ? b_lane1 : b_lane0, (uint32_t)(size_t)(smem + dst));
    };
    // Its powers, by waves 0 and 1; at an edge 4 bytes a lane, so that none behind the last row's are touched.
    auto issue_powers = [&](uint32_t buffer) {
        if constexpr (!EDGE) {
            if (wl < 2)
                load16_to_lds_saddr(bp_ptr + wl * 1024, (uint32_t)lane * 16, (uint32_t)(size_t)(smem + POWERS + buffer * 2048u + (uint32_t)wl * 1024u));
        } else {
#pragma unroll
            for (int i = 2 * wl; i < 2 * wl + 2; ++i)
                if (n0 + 32 * i + (lane >> 1) < p.N)
                    load4_to_lds_saddr(bp_ptr + i * 256, (uint32_t)lane * 4, (uint32_t)(size_t)(smem + POWERS + buffer * 2048u + (uint32_t)i * 256u));
        }
    };

    f32x4 acc[TN][TM];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b)
            acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    bf16x8 fa[2][TM], fb[2][TN];
    uint32_t codes[2][TN];
    u32x2 powers[TN];                           // of this lane's rows of weights, a long block's
    uint32_t factor[2][TN];                     // the exponent is the power
    const uint32_t lane_frag = (uint32_t)((lane & 15) * 128 + (((lane >> 4) ^ ((lane & 15) >> 1)) << 4));
    const uint32_t lane_code = WEIGHTS + (uint32_t)(wn * UNIT) + (uint32_t)((lane & 15) * 128 + (((lane & 15) >> 1) << 4) + 4 * (lane >> 4));
    const uint32_t lane_power = POWERS + (uint32_t)((wn * 64 + (lane & 15)) * 8);
    // first: slot of A's unit 0; u: block of the long block, `buffer` where that is; ld_first: slot of the first unit requested.
    auto memory_phase = [&](auto gc, bool request_a, bool request_b, int first, int u, uint32_t buffer, int ld_first) {
        constexpr int GROUP = decltype(gc)::value;
        const uint32_t at_a0 = (uint32_t)slot_of(first, 2 * wm) * UNIT + lane_frag, at_a1 = (uint32_t)slot_of(first, 2 * wm + 1) * UNIT + lane_frag;
        LDS_AS char *a0 = smem + at_a0, *a1 = smem + at_a1, *a0s = smem + (at_a0 ^ 64u), *a1s = smem + (at_a1 ^ 64u);
        const uint32_t at_b = (lane_code ^ (uint32_t)(u << 5)) + buffer * LONG;
        LDS_AS char *b0 = smem + at_b, *b1 = smem + (at_b ^ 16u);
        if (u == 0) {
#pragma unroll
            for (int a = 0; a < TN; ++a)
                powers[a] = *(LDS_AS u32x2 *)(smem + lane_power + buffer * 2048u + a * 128);
        }
#pragma unroll
        for (int a = 0; a < TN; ++a) {
            codes[0][a] = *(LDS_AS uint32_t *)(b0 + a * 2048);
            codes[1][a] = *(LDS_AS uint32_t *)(b1 + a * 2048);
        }
        static_for<0, TM>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            fa[0][i] = *(LDS_AS bf16x8 *)((i < 4 ? a0 : a1) + (i & 3) * 2048);
            fa[1][i] = *(LDS_AS bf16x8 *)((i < 4 ? a0s : a1s) + (i & 3) * 2048);
            if constexpr (i < 4) {
                if (request_a)
                    issue_a(i, ld_first);
            } else if constexpr (i < 6) {
                if (request_b && u < 2)
                    issue_b(i - 4, u, buffer ^ 1);
            } else if constexpr (i == 6 && GROUP == 0) {
                if (request_b && u == 2)
                    issue_powers(buffer ^ 1);
            }
        });
        // Blocks 2 u and 2 u + 1 of the long block: bytes u / 2 and u / 2 + 2 of word u % 2, turned to where an exponent is.
        const uint32_t turn = (uint32_t)(9 + 4 * (u & 2));
#pragma unroll
        for (int a = 0; a < TN; ++a) {
            const uint32_t word = u & 1 ? powers[a][1] : powers[a][0];
            factor[0][a] = __builtin_amdgcn_alignbit(word, word, turn);
            factor[1][a] = __builtin_amdgcn_alignbit(word, word, turn + 16);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int a = 0; a < TN; ++a)
                fb[j][a] = F16 ? __builtin_bit_cast(bf16x8, widen_f16(codes[j][a], __uint_as_float(factor[j][a])))
                               : widen_bf16(codes[j][a], __uint_as_float(factor[j][a]));
        if (request_a)
            a_ptr += 128;
        if (request_b && u == 3)
            b_ptr += MX_ROW;
        if (GROUP == 0 && request_b && u == 3)
            bp_ptr += p.b_plane;
    };
    auto compute_block = [&]() {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int a = 0; a < TN; ++a)
#pragma unroll
                for (int b = 0; b < TM; ++b)
                    acc[a][b] = mfma_16x16x32<F16 ? KIND_F16 : KIND_BF16>(fb[j][a], fa[j][b], acc[a][b]);
    };

    auto run = [&](auto gc) {
        constexpr int GROUP = decltype(gc)::value;
        constexpr int AHEAD = GROUP == 0 ? 1 : 2, FIRST = GROUP == 0 ? 2 : 0;
        // The first long block, and A up to where the loop goes on.
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            issue_b(0, u, 0);
            issue_b(1, u, 0);
        }
        b_ptr += MX_ROW;
        if constexpr (GROUP == 0) {
            issue_powers(0);
            bp_ptr += p.b_plane;
        }
        for (int t = 0; t < AHEAD && t < n_iter; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                issue_a(j, FIRST + 4 * t);
            a_ptr += 128;
        }
        wait_vmcnt0();
        phase_sync();
        if constexpr (GROUP == 1)
            phase_sync();                       // waves 4-7 run one phase behind
        int first = 0;                          // slot of block t's unit 0
        for (int t = 0; t < n_iter; ++t) {
            const int u = t & 3;
            const bool request_a = t + AHEAD < n_iter, request_b = t - u + 4 < n_iter;
            if constexpr (EDGE && GROUP == 1)
                wait_vmcnt0();                  // what was requested before this phase is there
            memory_phase(gc, request_a, request_b, first, u, (uint32_t)(t >> 2) & 1u, slot_of(first, FIRST + 4 * AHEAD - (FIRST + 4 * AHEAD >= (int)UNITS ? (int)UNITS : 0)));
            first = slot_of(first, 4);
            wait_lgkmcnt0();
            if constexpr (!EDGE && GROUP == 1) {
                if (!request_a)
                    wait_vmcnt0();
                else if (request_b && u < 2)
                    wait_vmcnt_le<6>();
                else
                    wait_vmcnt_le<4>();
            }
            phase_sync();
            compute_block();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (GROUP == 0)
                wait_vmcnt0();                  // requested a phase ago
            phase_sync();
        }
        if constexpr (GROUP == 0)
            phase_sync();
    };
    if (n_iter > 0) {
        if (group == 0)
            run(std::integral_constant<int, 0>{});
        else
            run(std::integral_constant<int, 1>{});
    }
    if constexpr (!F16) {
        if (__builtin_expect(not_finite(acc), 0) && far_powers(p, n0 + wn * 64, 16 * TN, 0, p.blocks, 1)) {
#pragma unroll 1
            for (int i = 0; i < TM * TN; ++i) {
                const int64_t row = m0 + wm * 128 + 16 * (i % TM), col = n0 + wn * 64 + 16 * (i / TM);
                if (row >= p.M || col >= p.N)
                    continue;
                const f32x4 v = far_sum<LEFT_BF16>(p, row, col, 0, p.blocks, 1);
                const int64_t m = row + (lane & 15), n = col + 4 * (lane >> 4);
                if (m < p.M && n < p.N)
                    gen_store4(p.epi, m, n, p.N - n, v);
            }
            return;
        }
    }
    mx4_store(p, acc, smem + (uint32_t)w * MX4_STAGED, m0 + wm * 128, n0 + wn * 64);
}

template <bool F16, bool GROUPED>
__global__ void __launch_bounds__(512)
mx4_half_kernel(Mx4Args p, GroupArgs g)
{
    int tm, tn;
    bool small;
    if (!mx4_large_tile<GROUPED>(p, g, tm, tn, small))
        return;
    if (small) {
        mx4_small_tile<F16 ? LEFT_F16 : LEFT_BF16, GROUPED>(p, tm, tn);
        return;
    }
    const int64_t m0 = (int64_t)tm * BM;
    if constexpr (F16) {
        extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
        LDS_AS char *smem = (LDS_AS char *)smem_generic;
        if (!powers_fit<BN>(p, tn, smem)) {
            direct_tile<BM, BN>(p, m0, tn, 0, (LDS_AS float *)smem);
            return;
        }
    }
    if (m0 + BM <= p.M && (int64_t)(tn + 1) * BN <= p.N)
        body<F16, false>(p, m0, tn);
    else
        body<F16, true>(p, m0, tn);
}

}  // namespace

hipError_t mx4_half(const Mx4Call &c)
{
    void (*kern)(Mx4Args, GroupArgs) = c.left == LEFT_F16 ? (c.grouped ? mx4_half_kernel<true, true> : mx4_half_kernel<true, false>)
                                                          : (c.grouped ? mx4_half_kernel<false, true> : mx4_half_kernel<false, false>);
    return mx4_launch<BM, BN, true>(kern, c, 512, LDS);
}

}  // namespace brg
