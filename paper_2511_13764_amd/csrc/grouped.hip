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

hipError_t launch_grouped_wgrad(GroupedCall &c, const Plan &plan)
{
    Problem &p = c.p;
    const int64_t tiles = ((p.M + 63) / 64) * ((p.N + 63) / 64);
    GroupedCall rest = c;
    const int64_t csz = p.c_f32 ? 4 : 2;
    if (tiles > kMostTiles) {
        const int64_t m = round_up(p.M / 2, 256);
        p.M = m;
        rest.p.M -= m;
        rest.p.A = (const char *)p.A + m * (in_16bit(p) ? 2 : 4);
        rest.p.C = (char *)p.C + m * p.ldc * csz;
    } else if (tiles * c.g.groups > kMostTiles) {
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
        return grouped_stream_wgrad(c, plan.variant == V_BF16_STREAM128 ? GEN_128 : plan.form);
    }
    const hipError_t e = launch_grouped_wgrad(c, plan);
    return e == hipSuccess ? launch_grouped_wgrad(rest, plan) : e;
}

}  // namespace brg
