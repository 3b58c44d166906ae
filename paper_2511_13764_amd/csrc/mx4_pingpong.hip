// 256 x 256 tiles of a product of two 4-bit images: two wavefronts a SIMD in alternating phases.
//
// A block of 256 columns is 128 bytes a row, as 64 columns of a 16-bit operand are, and its 64 matrix instructions a wave take the same
// 1024 cycles (16 x 16 x 128 and 16 x 16 x 32 both take 16), so loads, LDS image and phases are those of the 16-bit kernel (bf16_pingpong.hpp): while four waves
// multiply, the other four read the fragments of their block and request a later one, and a barrier swaps them.  What is new is the
// powers, 8 bytes a row and block.  They need 8 KB of LDS, two blocks of them, so the operands' ring is one of 19 units of 64 rows
// instead of five half-blocks.  That is enough for either half of the waves to request four units a block, because half of A's rows are read by
// waves 0-3 alone and free a phase before the rest.
// A lane reads the powers of two fragments at once, keeps its two bytes of each, and the instruction takes its byte of the four by itself.
// Why 16 x 16 x 128: on random operands the register-only rate is 7.3 PFLOP/s, with 32 x 32 x 64 5.4 (both 10 by the clock; power).
#include "mx4_tiles.hpp"

namespace brg {

namespace {

constexpr uint32_t UNIT = 8192, UNITS = 19;     // 64 rows of a block
constexpr uint32_t POWERS = UNIT * UNITS;       // 2 x (A, B) x 256 rows x 8 bytes
constexpr size_t LDS = POWERS + 8192;
static_assert(Mx4Ring<LEFT_MX4, 128, 128>::LDS <= LDS, "small tiles");
constexpr int BM = PP_BM, BN = PP_BN, TM = PP_TM, TN = PP_TN;
typedef KMajorTile<256, 4> Tile;                // rows of 128 bytes

// EDGE: the tile overhangs the matrix; lanes outside are switched off (what LDS holds in their place reaches rows and columns that are not
// stored), and as a wave-load without lanes is skipped, loads are then not counted but all waited for before the next.
template <bool EDGE>
__device__ __forceinline__ void body(const Mx4Args &p, int64_t m0, int tn)
{
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    LDS_AS char *smem = (LDS_AS char *)smem_generic;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = w >> 2, wl = w & 3;       // waves w and w + 4 share a SIMD
    const int wm = group, wn = wl;
    const int64_t n0 = (int64_t)tn * BN;
    const int n_iter = p.blocks;

    // Loads.  Units of a block in the order in which they are done with: rows 0 .. 127 of A, which waves 0-3 alone read, B, and the rest of A,
    // which waves 4-7 read a phase later.  Unit u of block t has slot (8 t + u) % 19.  Waves 4-7 take units 0 .. 3 (A, B) of the block that their
    // cursor stands at, waves 0-3 units 4 .. 7 (B, A); of a unit's eight wave-loads (8 rows each) wave wl takes 2 wl and 2 wl + 1.  Both
    // images have one pitch: two pointers, two lane offsets (the swizzle's), a step.
    const int64_t step = 8 * p.lda;             // bytes from one wave-load to the next
    const char *a_ptr = p.A + (m0 + (group ? 0 : 128)) * p.lda, *b_ptr = p.B + (n0 + (group ? 0 : 128)) * p.lda;
    const char *first_ptr = (const char *)uniform_ptr((const uint16_t *)((group ? a_ptr : b_ptr) + 2 * wl * step));
    const char *other_ptr = (const char *)uniform_ptr((const uint16_t *)((group ? b_ptr : a_ptr) + 2 * wl * step));
    const char *ap_ptr = p.a_powers + m0 * 8, *bp_ptr = p.b_powers + n0 * 8;
    const uint32_t lane0 = Tile::lane_off_bytes(0, lane, p.lda / 2), lane1 = Tile::lane_off_bytes(1, lane, p.lda / 2);
    auto slot_of = [](int first, int u) { return first + u >= (int)UNITS ? first + u - (int)UNITS : first + u; };
    // EDGE: rows that there are, counted from the wave's first.
    const int a_left = (int)((p.M < m0 + 256 ? p.M : m0 + 256) - m0) - (group ? 0 : 128) - 16 * wl;
    const int b_left = (int)((p.N < n0 + 256 ? p.N : n0 + 256) - n0) - (group ? 0 : 128) - 16 * wl;
    // Wave-load j of 8 of this wave: half j % 2 of its unit j / 2, which has the slot `first` + j / 2.
    auto issue = [&](auto jc, const char *&at, int first) {
        constexpr int j = decltype(jc)::value;
        const uint32_t dst = (uint32_t)slot_of(first, j / 2) * UNIT + (uint32_t)(2 * wl + j % 2) * 1024u;
        const int left = ((j < 4) == (group == 1) ? a_left : b_left) - 64 * (j / 2 % 2) - 8 * (j % 2);
        if (!EDGE || (lane >> 3) < left)
            load16_to_lds_saddr(at, j % 2 ? lane1 : lane0, (uint32_t)(size_t)(smem + dst));
        at = j == 3 ? other_ptr : at + (j % 2 ? 7 * step : step);
    };
    // Powers of a block, by waves 0-3: a lane takes those of two rows, or, at an edge, half of those of one, so that none behind the last is
    // touched.  (4 bytes a lane everywhere, sixteen wave-loads instead of four, are level: 8192^3 246.)
    auto issue_powers = [&](uint32_t ld_parity) {
        if constexpr (!EDGE) {
            load16_to_lds_saddr((wl < 2 ? ap_ptr : bp_ptr) + (wl & 1) * 1024, (uint32_t)lane * 16, (uint32_t)(size_t)(smem + POWERS + ld_parity + (uint32_t)wl * 1024u));
        } else {
#pragma unroll
            for (int i = 2 * wl; i < 2 * wl + 2; ++i) {
                const uint32_t dst = POWERS + ld_parity + (uint32_t)i * 256u;
                if (m0 + 32 * i + (lane >> 1) < p.M)
                    load4_to_lds_saddr(ap_ptr + i * 256, (uint32_t)lane * 4, (uint32_t)(size_t)(smem + dst));
                if (n0 + 32 * i + (lane >> 1) < p.N)
                    load4_to_lds_saddr(bp_ptr + i * 256, (uint32_t)lane * 4, (uint32_t)(size_t)(smem + dst + 2048));
            }
        }
    };
    auto next_block = [&]() {
        first_ptr += MX_ROW;
        other_ptr += MX_ROW;
        ap_ptr += p.a_plane;
        bp_ptr += p.b_plane;
    };

    f32x4 acc[TN][TM];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b)
            acc[a][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Memory phase: the block's 24 fragments and their powers; between them, the requests.
    i32x4 fa[2][TM], fb[2][TN];
    uint32_t pa[TM / 2], pb[TN / 2];            // powers of two fragments each
    const uint32_t lane_frag = (uint32_t)((lane & 15) * 128 + ((((lane >> 4) ^ (((lane & 15) >> 1) & 7))) << 4));
    const uint32_t lane_power = POWERS + (uint32_t)((lane & 15) * 8 + (lane >> 5) * 4);
    const uint32_t lane_pair = lane & 16 ? 0x07060302u : 0x05040100u;
    // Powers of fragments i and i + 1, 16 rows apart: two words in one read, of each the lane's half.
    auto powers_of = [&](LDS_AS char *at) {
        return __builtin_amdgcn_perm(*(LDS_AS uint32_t *)(at + 128), *(LDS_AS uint32_t *)at, lane_pair);
    };
    auto memory_phase = [&](auto gc, bool request, int rd_first, uint32_t rd_parity, int ld_first) {
        constexpr int GROUP = decltype(gc)::value;
        const char *at = first_ptr;
        const uint32_t at_a0 = (uint32_t)slot_of(rd_first, GROUP * 6) * UNIT + lane_frag, at_a1 = (uint32_t)slot_of(rd_first, GROUP * 6 + 1) * UNIT + lane_frag;
        const uint32_t at_b0 = (uint32_t)slot_of(rd_first, 2 + wn) * UNIT + lane_frag;
        // (the second half of a row's chunks is 64 bytes away, up or down)
        LDS_AS char *a0 = smem + at_a0, *a1 = smem + at_a1, *b0 = smem + at_b0;
        LDS_AS char *a0s = smem + (at_a0 ^ 64u), *a1s = smem + (at_a1 ^ 64u), *b0s = smem + (at_b0 ^ 64u);
        LDS_AS char *pw = smem + rd_parity + lane_power;
        static_for<0, 12>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            if constexpr (j < 4) {
                fb[0][j] = *(LDS_AS i32x4 *)(b0 + j * 2048);
                fb[1][j] = *(LDS_AS i32x4 *)(b0s + j * 2048);
            } else {
                constexpr int i = j - 4;
                fa[0][i] = *(LDS_AS i32x4 *)((i < 4 ? a0 : a1) + (i & 3) * 2048);
                fa[1][i] = *(LDS_AS i32x4 *)((i < 4 ? a0s : a1s) + (i & 3) * 2048);
            }
            if (request) {
                if constexpr (j < 8)
                    issue(jc, at, ld_first);
                else if constexpr (GROUP == 0 && j == 8)
                    issue_powers(rd_parity ^ 4096);
            }
        });
        // (the powers last: between the fragments 8192^3 takes 3 % longer)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TN / 2; ++i)
            pb[i] = powers_of(pw + 2048 + wn * 512 + i * 256);
#pragma unroll
        for (int i = 0; i < TM / 2; ++i)
            pa[i] = powers_of(pw + wm * 1024 + i * 256);
        if (request)
            next_block();
    };
    auto compute_block = [&]() {
        static_for<0, 2>([&](auto sc) {
            constexpr int s = decltype(sc)::value;
            static_for<0, TN>([&](auto ac) {
                constexpr int a = decltype(ac)::value;
                static_for<0, TM>([&](auto bc) {
                    constexpr int b = decltype(bc)::value;
                    acc[a][b] = mfma_mx4<2 * (a & 1) + s, 2 * (b & 1) + s>(fb[s][a], fa[s][b], acc[a][b], (int)pb[a / 2], (int)pa[b / 2]);
                });
            });
        });
    };

    // Waves 4-7 run one phase behind.
    auto run = [&](auto gc) {
        constexpr int GROUP = decltype(gc)::value;
        constexpr int LOADS = 8, AHEAD = GROUP == 0 ? 1 : 2, FIRST = GROUP == 0 ? 4 : 0;
        for (int t = 0; t < AHEAD && t < n_iter; ++t) {
            const char *at = first_ptr;
            static_for<0, LOADS>([&](auto jc) { issue(jc, at, FIRST + 8 * t); });
            if constexpr (GROUP == 0)
                issue_powers(0);
            next_block();
        }
        wait_vmcnt0();
        phase_sync();
        if constexpr (GROUP == 1)
            phase_sync();
        int first = 0;                          // slot of block t's unit 0
        for (int t = 0; t < n_iter; ++t) {
            const bool request = t + AHEAD < n_iter;
            if constexpr (EDGE && GROUP == 1)
                wait_vmcnt0();                  // block t + 1's units, requested a block ago, are there
            memory_phase(gc, request, first, (uint32_t)(t & 1) * 4096u, slot_of(first, FIRST + 8 * AHEAD));
            first = slot_of(first, 8);
            wait_lgkmcnt0();
            if constexpr (!EDGE && GROUP == 1) {
                if (request)
                    wait_vmcnt_le<LOADS>();
                else
                    wait_vmcnt0();
            }
            phase_sync();
            compute_block();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (GROUP == 0)
                wait_vmcnt0();                  // block t + 1's, requested a phase ago
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

    mx4_store(p, acc, smem + (uint32_t)w * MX4_STAGED, m0 + wm * 128, n0 + wn * 64);
}

template <bool GROUPED>
__global__ void __launch_bounds__(512)
mx4_pingpong_kernel(Mx4Args p, GroupArgs g)
{
    int tm, tn;
    bool small;
    if (!mx4_large_tile<GROUPED>(p, g, tm, tn, small))
        return;
    if (small)
        mx4_small_tile<LEFT_MX4, GROUPED>(p, tm, tn);
    else if ((int64_t)(tm + 1) * BM <= p.M && (int64_t)(tn + 1) * BN <= p.N)
        body<false>(p, (int64_t)tm * BM, tn);
    else
        body<true>(p, (int64_t)tm * BM, tn);
}

}  // namespace

hipError_t mx4_pingpong(const Mx4Call &c)
{
    return mx4_launch<BM, BN, true>(c.grouped ? mx4_pingpong_kernel<true> : mx4_pingpong_kernel<false>, c, 512, LDS);
}

}  // namespace brg
