// Plan and launches of the grouped products (grouped.hpp).
#include "../../include/brgemm.h"
#include "grouped.hpp"
#include <cmath>

namespace brg {

namespace {

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// True when the tuned 16-bit kernels can read the operands.
bool rows_eligible(const GroupedCall &c)
{
    Problem q = c.p;
    q.ms_b = c.g.stride_b;
    return in_16bit(q) && c.low.R == 0 && !c.narrow && (c.p.transA || q.K >= 8) && bf16_rows_eligible(q);
}

// True when the divided tiles can (duty_eligible, on the rows of a group; a gradient's short groups run undivided by themselves).
bool divided_eligible(const GroupedCall &c, int tile)
{
    Problem q = c.p;
    if (q.transA)
        q.K = q.K > 256 ? q.K : 256;                // (the length of a reduction is the kernel's own matter)
    return c.low.R == 0 && !c.narrow && general_offsets_fit(q, tile) && duty_eligible(q);
}

bool takes(const GroupedCall &c, bool wgrad, int variant, int form)
{
    switch (variant) {
    case V_GENERIC: return form < 0 || (form == GEN_32 && !wgrad && c.low.R == 0 && !rows_eligible(c)) || (form < GEN_32 && (!wgrad || form == GEN_64) && divided_eligible(c, form));
    case V_BF16_PP256:
    case V_BF16_STREAM128: return form < 0 && rows_eligible(c);
    case V_BF16_128x128: return wgrad && form < 0 && rows_eligible(c);
    case V_BF16_STREAM64: return form == GEN_MID && rows_eligible(c);
    case V_BF16_STREAM32: return form == GEN_64 && rows_eligible(c);
    default: return false;
    }
}

// A kernel a plan may take, and what it costs in a rough model of time, in microseconds.  Forward: workgroups that run at once, a
// tile's fixed part and a block of its reduction, with that many running.  The sizes of the groups are known to the device
// alone: the model takes them as spread exponentially around their mean, what a router leaves at worst.
struct Candidate {
    Plan plan;
    int bm, bn, at_once;
    double fixed, block;
};

// Tiles of bm rows that `groups` groups of `rows` rows in all are expected to have.
double expected_row_tiles(double rows, double groups, int bm)
{
    const double used = rows < groups ? rows : groups;
    return used / (1.0 - std::exp(-bm * used / rows));
}

// Fitted to sweeps of the four tuned kernels over 4 to 64 groups of 1 to 1024 rows, 1024 x 1024 to 11008 x 4096 weights in both layouts (a
// block: 64 k), and of the general kernel's three divided tiles over odd sizes (1001 x 1301 to 4001 x 1003; fp32: a block is 32 k).  The 32 x 32
// tile, whose eight waves share the reduction, for both: 4 groups of 512 x 2048 in fp32, 16 to 200 rows in all, 16 us where 64 x 64 takes 39 and
// leaves most CUs without a tile, 8 groups of 701 x 3333 in bf16 15 and 24; from two rounds on the larger tiles' reuse wins (fp32, 600 rows,
// 2 groups of 1024 x 1024 30 and 23; bf16, 64 rows, 8 groups of 2003 x 1001 14.5 and 12).
// How far the choice is from the best tile: fp32, 120 calls, 2 % on average and 11 % at most; 16-bit rows off 16 bytes, 150 calls of 4 to
// 800 rows, 3.8 % on average, up to 35 % where 64 x 64 is taken for 128 x 64 (800 rows, 2 groups of 2001 x 4099: 56 us and 41.6) and up to 19 %
// where it is taken for 32 x 32 (64 and 200 rows, 32 groups of 701 x 3333: 63 us and 53).
// The choice within them: 8 groups of 4096 x 4096 take 49 us in 64 x 64 tiles and 80 in 256 x 256 with a row each, 164 and 111 with 256;
// 4 groups of 1024 x 1024 8 and 23, 11 and 27.
Plan choose_forward(const GroupedCall &c)
{
    static const Candidate tuned[] = {{{V_BF16_STREAM32, 1, GEN_64}, 64, 64, 512, 2.0, 0.47}, {{V_BF16_STREAM64, 1, GEN_MID}, 128, 64, 512, 2.0, 0.66},
                                      {{V_BF16_STREAM128, 1, -1}, 128, 128, 256, 3.0, 0.58}, {{V_BF16_PP256, 1, -1}, 256, 256, 256, 9.0, 1.42}};
    static const Candidate divided16[] = {{{V_GENERIC, 1, GEN_64}, 64, 64, 512, 2.0, 0.72}, {{V_GENERIC, 1, GEN_MID}, 128, 64, 512, 2.0, 1.4},
                                          {{V_GENERIC, 1, GEN_128}, 128, 128, 256, 3.0, 0.95}, {{V_GENERIC, 1, GEN_32}, 32, 32, 256, 3.0, 0.22}};
    static const Candidate divided32[] = {{{V_GENERIC, 1, GEN_64}, 64, 64, 512, 2.0, 1.1}, {{V_GENERIC, 1, GEN_MID}, 128, 64, 512, 2.0, 1.95},
                                          {{V_GENERIC, 1, GEN_128}, 128, 128, 256, 3.0, 1.95}, {{V_GENERIC, 1, GEN_32}, 32, 32, 256, 4.5, 0.165}};
    const Problem &p = c.p;
    const bool rows = rows_eligible(c);
    const Candidate *list = rows ? tuned : in_16bit(p) ? divided16 : divided32;
    const double esz = in_16bit(p) ? 2.0 : 4.0, groups = c.g.groups < p.M ? c.g.groups : (double)p.M;
    const double bytes = esz * (groups * p.N * p.K + (double)p.M * (p.K + p.N));
    const double blocks = (double)((p.K + (in_16bit(p) ? 63 : 31)) / (in_16bit(p) ? 64 : 32));
    Plan best{V_GENERIC, 1, -1};
    double best_t = 1e30;
    for (int i = 0; i < 4; ++i) {
        const Candidate &k = list[i];
        if (!takes(c, false, k.plan.variant, k.plan.form))
            continue;
        const double tiles = expected_row_tiles((double)p.M, (double)c.g.groups, k.bm) * (double)((p.N + k.bn - 1) / k.bn);
        // A workgroup that has its CU to itself takes a block in about half the time of two that share it.
        const bool alone = k.at_once == 512 && tiles <= 256.0;
        const bool once = tiles <= 1.03 * k.at_once;            // (the expected number is never quite a whole one)
        const double rounds = once ? 1.0 : tiles / k.at_once + 0.4;
        const double again = k.bm != 32 || once ? 1.0 : in_16bit(p) ? 1.6 : 1.12;          // (what neighbouring tiles share is read by more of them)
        const double work = again * rounds * (k.fixed + blocks * k.block * (alone ? 0.55 : 1.0)), memory = bytes / 5.5e6;
        const double t = (work > memory ? work : memory) + 0.1 * work;
        if (t < best_t) {
            best_t = t;
            best = k.plan;
        }
    }
    return best;
}

// Weight gradients.  A tile's fixed part (the result's bytes among it), a block of its reduction, and the time of that block however few
// workgroups run, which counts for the longest group: 1 + 0.8 ln(groups) times the mean.  Fitted to sweeps of 1 to 64 groups of 4 to 2500
// rows, results of 16 x 4096 to 4096 x 4096.  256 x 256 tiles come in rounds, of the others several share a CU.
Plan choose_wgrad(const GroupedCall &c)
{
    const Problem &p = c.p;
    if (!rows_eligible(c))
        return takes(c, true, V_GENERIC, GEN_64) ? Plan{V_GENERIC, 1, GEN_64} : Plan{V_GENERIC, 1, -1};
    const int bytes = (p.c_f32 ? 4 : 2) * (p.c_f32 && p.beta != 0.0f ? 2 : 1);        // of a result, read ones twice
    struct Kernel {
        Plan plan;
        int bm, bn;
        double start, fixed, block, alone;
    };
    const Kernel kernels[] = {{{V_BF16_128x128, 1, -1}, 128, 128, 4.5, bytes == 2 ? 1.4 : bytes == 4 ? 2.6 : 6.0, 0.47, 0.95},
                              {{V_BF16_STREAM64, 1, GEN_MID}, 128, 64, 3.0, 2.4, 0.42, 0.35}, {{V_BF16_STREAM32, 1, GEN_64}, 64, 64, 2.0, 1.95, 0.21, 0.30},
                              {{V_BF16_PP256, 1, -1}, 256, 256, 2.5, bytes == 2 ? 7.5 : bytes == 4 ? 14.0 : 22.5, 1.5, 1.5}};
    const double blocks = (double)p.K / c.g.groups / 64.0 + 0.5, longest = 1.0 + 0.8 * std::log((double)c.g.groups);
    Plan best{};
    double best_t = 1e30;
    for (const Kernel &k : kernels) {
        const double tiles = (double)((p.M + k.bm - 1) / k.bm) * (double)((p.N + k.bn - 1) / k.bn) * c.g.groups;
        double n = tiles / 256.0;
        if (k.bm == 256)
            n = std::ceil(n);
        const double shared = n * k.block, alone = longest * k.alone;
        const double results = n * k.fixed, sums = blocks * (shared > alone ? shared : alone);
        const bool hides = k.plan.variant == V_BF16_128x128;         // one workgroup's sums behind another's results
        const double t = k.start + results + sums - (hides ? 0.4 * (results < sums ? results : sums) : 0.0);
        if (t < best_t) {
            best_t = t;
            best = k.plan;
        }
    }
    return best;
}

}  // namespace

int plan_grouped(const GroupedCall &c, bool wgrad, int forced_variant, int forced_form, Plan *out)
{
    if (forced_variant >= 0 || forced_form >= 0) {
        *out = Plan{forced_variant < 0 ? V_GENERIC : forced_variant, 1, forced_form};
        return takes(c, wgrad, out->variant, out->form) ? BRGEMM_OK : BRGEMM_INVALID_ARG;
    }
    *out = wgrad ? choose_wgrad(c) : choose_forward(c);
    return BRGEMM_OK;
}

hipError_t launch_grouped(GroupedCall &c, const Plan &plan)
{
    Problem &p = c.p;
    const int64_t rows = most_row_tiles(p.M, c.g.groups + 2 * c.g.cover, 32);
    if (rows > kMostTiles)
        return hipErrorInvalidValue;                // (the caller refuses these)
    if (rows * ((p.N + 31) / 32) > kMostTiles) {
        const int64_t n = p.N <= 256 ? round_up(p.N / 2, 32) : round_up(p.N / 2, 256);
        const int64_t esz = in_16bit(p) ? 2 : 4;
        GroupedCall rest = c;
        p.N = n;
        rest.p.N -= n;
        rest.p.B = (const char *)p.B + n * (p.transB ? p.ldb : 1) * esz;
        rest.p.C = (char *)p.C + n * (p.c_f32 ? 4 : 2);
        rest.p.bias = p.bias ? p.bias + n : nullptr;
        rest.low.up = c.low.up ? c.low.up + n * (p.transB ? c.low.ld_up : 1) * esz : nullptr;
        const hipError_t e = launch_grouped(c, plan);
        return e == hipSuccess ? launch_grouped(rest, plan) : e;
    }
    if (plan.variant == V_GENERIC && plan.form == GEN_32) {
        c.narrow = true;                            // (the tile of adapters' first product, without a factor)
        return grouped_general(c);
    }
    if (plan.variant == V_GENERIC)
        return plan.form < 0 ? grouped_general(c) : grouped_duty(c, plan.form);
    if (plan.variant == V_BF16_PP256)
        return grouped_pingpong(c);
    return grouped_stream(c, plan.variant == V_BF16_STREAM128 ? GEN_128 : plan.form);
}

// The kernel that takes adapters as blocks for a projection's plan, under the names by which one is forced: a plan's reduced tile
// (Plan::form) is the general kernel's or has no instance with blocks.
static Plan blocks_plan(const Plan &projection)
{
    switch (projection.variant) {
    case V_BF16_PP256:
    case V_BF16_128x128:                            // (128 x 256)
    case V_BF16_STREAM128: return Plan{projection.variant, 1, -1};
    case V_BF16_STREAM64: return Plan{V_BF16_STREAM64, 1, GEN_MID};
    default: return Plan{V_BF16_STREAM32, 1, GEN_64};
    }
}

// Which way the adapters of a projection take.
static AdaptersPlan choose_adapters(const GroupedCall &c, size_t workspace_bytes)
{
    const Problem &p = c.p;
    AdaptersPlan out{ADAPTERS_GENERAL, Plan{V_GENERIC, 1, -1}};
    if (!in_16bit(p) || p.K < 8 || ((p.M + 63) / 64) * ((p.N + 63) / 64) > kMostTiles)
        return out;
    Problem q = p;
    const size_t sums = (size_t)p.M * (size_t)p.N * sizeof(float);
    const bool apart = adapters_up_fits(c) && sums <= workspace_bytes;
    const bool blocks = bf16_rows_eligible(p) && c.low.R <= 4096;
    const int64_t each = c.g.groups > 0 ? p.M / c.g.groups : p.M;
    // What the projection's sums would take on their own, a split of the reduction among them.
    Plan sums_plan{V_GENERIC, 1, -1};
    if (apart) {
        q.c_f32 = 1; q.beta = 0.0f; q.bias = nullptr; q.relu = 0; q.ldc = p.N;
        if (choose_plan(q, workspace_bytes, -1, 0, -1, &sums_plan) == BRGEMM_OK)
            prefer_small_tiles(q, workspace_bytes, &sums_plan);
    }
    if (apart && each < 64 && adapters_few_rows(c)) {
        out.how = ADAPTERS_FEW_ROWS;
    } else if (blocks && ((each >= 64 && sums_plan.split == 1 && sums_plan.form != GEN_32) || !apart)) {
        // (Blocks know neither a split nor tiles of 32 x 32: 458 rows in 2 segments, 704 x 6784, 54 us in 88 unsplit tiles and 32 apart;
        // 200 rows in one, 1024 x 8192, 61 and 31.)
        out.how = ADAPTERS_BLOCKS;
        q = p;
        q.K = round_up(p.K, BK);                    // (the tiles take an incomplete block)
        if (choose_plan(q, 0, -1, 0, -1, &out.base) == BRGEMM_OK)
            prefer_small_tiles(q, 0, &out.base);
        out.base = blocks_plan(out.base);
    } else if (apart) {
        out.how = ADAPTERS_APART;
        out.base = sums_plan;
    }
    return out;
}

int plan_adapters(const GroupedCall &c, size_t workspace_bytes, int forced_variant, int forced_form, AdaptersPlan *out)
{
    if (forced_variant < 0 && forced_form < 0) {
        *out = choose_adapters(c, workspace_bytes);
        return BRGEMM_OK;
    }
    // A forced variant names the projection's kernel with the adapters as its blocks, the general one both products in it.
    *out = AdaptersPlan{forced_variant <= V_GENERIC ? ADAPTERS_GENERAL : ADAPTERS_BLOCKS, Plan{forced_variant < 0 ? V_GENERIC : forced_variant, 1, forced_form}};
    if (out->how == ADAPTERS_GENERAL)
        return forced_form < 0 ? BRGEMM_OK : BRGEMM_INVALID_ARG;
    const bool is = forced_variant == V_BF16_STREAM64 ? forced_form == GEN_MID : forced_variant == V_BF16_STREAM32 ? forced_form == GEN_64
                    : forced_form < 0 && forced_variant != V_F32_128x128;
    return is && in_16bit(c.p) && c.p.K >= 8 && c.low.R <= 4096 && bf16_rows_eligible(c.p) ? BRGEMM_OK : BRGEMM_INVALID_ARG;
}

hipError_t launch_adapters_plan(GroupedCall &first, GroupedCall &c, const AdaptersPlan &plan, void *workspace, size_t workspace_bytes)
{
    const Problem &p = c.p;
    hipError_t e;
    if (plan.how == ADAPTERS_FEW_ROWS) {
        e = adapters_down_and_sums(first, c, (float *)workspace);
        return e == hipSuccess ? adapters_up(c, (const float *)workspace, 1) : e;
    }
    const auto down = [&] { return adapters_down_fits(first) ? adapters_down(first) : launch_grouped(first, Plan{V_GENERIC, 1, -1}); };
    if (plan.how == ADAPTERS_APART && p.N > 0) {
        Problem q = p;
        q.c_f32 = 1; q.beta = 0.0f; q.bias = nullptr; q.relu = 0;
        q.split = plan.base.split; q.form = plan.base.form;
        if (q.split > 1) {
            q.partial = (float *)workspace;
        } else {
            const size_t sums = (size_t)round_up(p.M * p.N * (int64_t)sizeof(float), 256);
            q.C = workspace; q.ldc = p.N;
            if (sums < workspace_bytes) {
                q.scratch = (char *)workspace + sums;
                q.scratch_bytes = workspace_bytes - sums;
            }
        }
        if (adapters_beside_fits(first, q, plan.base)) {
            e = adapters_beside(first, q, plan.base);
        } else {
            e = down();
            e = e == hipSuccess ? launch_variant(plan.base.variant, q) : e;
        }
        return e == hipSuccess ? adapters_up(c, (const float *)workspace, q.split) : e;
    }
    e = down();
    if (e != hipSuccess || p.N == 0)
        return e;
    if (plan.how == ADAPTERS_BLOCKS) {
        switch (plan.base.variant) {
        case V_BF16_PP256: return adapters_pingpong(c);
        case V_BF16_128x128: return adapters_stream(c, GEN_WIDE);
        case V_BF16_STREAM128: return adapters_stream(c, GEN_128);
        case V_BF16_STREAM64: return adapters_stream(c, GEN_MID);
        default: return adapters_stream(c, GEN_64);
        }
    }
    return launch_grouped(c, Plan{V_GENERIC, 1, -1});
}

hipError_t launch_grouped_wgrad(GroupedCall &c, const Plan &plan)
{
    Problem &p = c.p;
    const ReductionPart part = reduction_part(p.M, p.N, c.g.groups);
    if (part.m == p.M && part.n == p.N && part.groups == c.g.groups) {
        if (plan.variant == V_GENERIC)
            return plan.form < 0 ? grouped_general_wgrad(c) : grouped_duty_wgrad(c);
        if (plan.variant == V_BF16_PP256)
            return grouped_pingpong_wgrad(c);
        if (plan.variant == V_BF16_128x128)
            return grouped_short_wgrad(c);
        return grouped_stream_wgrad(c, plan.variant == V_BF16_STREAM128 ? GEN_128 : plan.form);
    }
    const int64_t esz = in_16bit(p) ? 2 : 4, csz = p.c_f32 ? 4 : 2;
    GroupedCall rest = c;
    if (part.m < p.M) {
        rest.p.M -= part.m;
        rest.p.A = (const char *)p.A + part.m * esz;
        rest.p.C = (char *)p.C + part.m * p.ldc * csz;
    } else if (part.n < p.N) {
        rest.p.N -= part.n;
        rest.p.B = (const char *)p.B + part.n * esz;
        rest.p.C = (char *)p.C + part.n * csz;
    } else {
        rest.g.groups -= (int)part.groups;
        rest.g.offsets += part.groups;
        rest.p.C = (char *)p.C + part.groups * c.g.stride_c * csz;
    }
    p.M = part.m;
    p.N = part.n;
    c.g.groups = (int)part.groups;
    const hipError_t e = launch_grouped_wgrad(c, plan);
    return e == hipSuccess ? launch_grouped_wgrad(rest, plan) : e;
}

}  // namespace brg
