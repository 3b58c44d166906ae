// Plan and launches of the grouped products (grouped.hpp).
#include "../../include/brgemm.h"
#include "grouped.hpp"

namespace brg {

namespace {

// HIP keeps the grid of a launch as 32-bit counts of threads: larger ones are launched in halves, as elsewhere.
constexpr int64_t kMostTiles = 0xffffffffLL / 512;

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
    case V_GENERIC: return form < 0 || (form < GEN_32 && (!wgrad || form == GEN_64) && divided_eligible(c, form));
    case V_BF16_PP256:
    case V_BF16_STREAM128: return form < 0 && rows_eligible(c);
    case V_BF16_128x128: return wgrad && form < 0 && rows_eligible(c);
    case V_BF16_STREAM64: return form == GEN_MID && rows_eligible(c);
    case V_BF16_STREAM32: return form == GEN_64 && rows_eligible(c);
    default: return false;
    }
}

}  // namespace

int plan_grouped(const GroupedCall &c, bool wgrad, int forced_variant, int forced_form, Plan *out)
{
    const Problem &p = c.p;
    if (forced_variant >= 0 || forced_form >= 0) {
        *out = Plan{forced_variant < 0 ? V_GENERIC : forced_variant, 1, forced_form};
        return takes(c, wgrad, out->variant, out->form) ? BRGEMM_OK : BRGEMM_INVALID_ARG;
    }
    *out = Plan{V_GENERIC, 1, -1};
    if (rows_eligible(c)) {
        if (wgrad) {
            const int64_t tiles = ((p.M + 255) / 256) * ((p.N + 255) / 256) * c.g.groups;
            *out = tiles >= 256 ? Plan{V_BF16_PP256, 1, -1} : Plan{V_BF16_STREAM128, 1, -1};
        } else {
            const int64_t each = p.M / (c.g.groups > 0 ? c.g.groups : 1);
            *out = each > 128 ? Plan{V_BF16_PP256, 1, -1} : each > 48 ? Plan{V_BF16_STREAM128, 1, -1} : Plan{V_BF16_STREAM32, 1, GEN_64};
        }
    } else if (takes(c, wgrad, V_GENERIC, GEN_64)) {
        *out = Plan{V_GENERIC, 1, GEN_64};
    }
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
    if (plan.variant == V_GENERIC)
        return plan.form < 0 ? grouped_general(c) : grouped_duty(c, plan.form);
    if (plan.variant == V_BF16_PP256)
        return grouped_pingpong(c);
    return grouped_stream(c, plan.variant == V_BF16_STREAM128 ? GEN_128 : plan.form);
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
    if (apart && each < 64 && adapters_few_rows(c)) {
        out.how = ADAPTERS_FEW_ROWS;
    } else if (blocks && (each >= 64 || !apart)) {
        out.how = ADAPTERS_BLOCKS;
        q.K = round_up(p.K, BK);                    // (the tiles take an incomplete block)
        if (choose_plan(q, 0, -1, 0, -1, &out.base) == BRGEMM_OK)
            prefer_small_tiles(q, 0, &out.base);
    } else if (apart) {
        out.how = ADAPTERS_APART;
        q.c_f32 = 1; q.beta = 0.0f; q.bias = nullptr; q.relu = 0; q.ldc = p.N;
        if (choose_plan(q, workspace_bytes, -1, 0, -1, &out.base) == BRGEMM_OK)
            prefer_small_tiles(q, workspace_bytes, &out.base);
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
    e = adapters_down_fits(first) ? adapters_down(first) : launch_grouped(first, Plan{V_GENERIC, 1, -1});
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
    if (plan.how == ADAPTERS_GENERAL)
        return launch_grouped(c, Plan{V_GENERIC, 1, -1});
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
    e = launch_variant(plan.base.variant, q);
    return e == hipSuccess ? adapters_up(c, (const float *)workspace, q.split) : e;
}

hipError_t launch_grouped_wgrad(GroupedCall &c, const Plan &plan)
{
    Problem &p = c.p;
    const int64_t tiles = ((p.M + 63) / 64) * ((p.N + 63) / 64);
    GroupedCall rest = c;
    const int64_t csz = p.c_f32 ? 4 : 2;
    if (reduction_grid(tiles, 1) > kMostTiles) {
        const int64_t m = round_up(p.M / 2, 256);
        p.M = m;
        rest.p.M -= m;
        rest.p.A = (const char *)p.A + m * (in_16bit(p) ? 2 : 4);
        rest.p.C = (char *)p.C + m * p.ldc * csz;
    } else if (reduction_grid(tiles, c.g.groups) > kMostTiles && c.g.groups > 1) {
        const int half = c.g.groups / 2;
        c.g.groups = half;
        rest.g.groups -= half;
        rest.g.offsets += half;
        rest.p.C = (char *)p.C + half * c.g.stride_c * csz;
    } else {
        if (plan.variant == V_GENERIC)
            return plan.form < 0 ? grouped_general_wgrad(c) : grouped_duty_wgrad(c);
        if (plan.variant == V_BF16_PP256)
            return grouped_pingpong_wgrad(c);
        if (plan.variant == V_BF16_128x128)
            return grouped_short_wgrad(c);
        return grouped_stream_wgrad(c, plan.variant == V_BF16_STREAM128 ? GEN_128 : plan.form);
    }
    const hipError_t e = launch_grouped_wgrad(c, plan);
    return e == hipSuccess ? launch_grouped_wgrad(rest, plan) : e;
}

}  // namespace brg
