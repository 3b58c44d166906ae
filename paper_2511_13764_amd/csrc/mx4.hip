// Plan and launches of the products with 4-bit images (mx4.hpp).
#include "../../include/brgemm.h"
#include "mx4.hpp"

namespace brg {

namespace {

// (Rows of an image that are 2^29 bytes apart and more leave the lanes' 32-bit offsets.)
bool near_rows(const Mx4Call &c) { return c.a.K <= (int64_t)1 << 29; }

// 16-bit rows that global->LDS loads can read.
bool whole_rows(const Mx4Call &c)
{
    return ((uintptr_t)c.a.A & 15) == 0 && c.a.lda % 16 == 0 && c.a.lda <= (int64_t)1 << 29 && c.a.K % 64 == 0;
}

// (A lane's offset reaches over the 128 rows of a tile.)
bool near_tile(const Mx4Call &c)
{
    return c.a.ldb <= (int64_t)1 << 24 && c.a.lda <= (int64_t)1 << 24 && (c.left == LEFT_MX4 || whole_rows(c));
}

// Most groups have at most 16 rows.
bool few_rows(const Mx4Call &c) { return c.grouped ? c.a.M <= 12 * c.g.groups : c.a.M <= 16; }

bool takes(const Mx4Call &c, int variant, int form)
{
    switch (variant) {
    case V_GENERIC: return form < 0;
    case V_BF16_PP256: return form < 0 && near_rows(c) && (c.left == LEFT_MX4 || whole_rows(c));
    case V_BF16_STREAM128:
    case V_BF16_STREAM64: return form < 0 && near_tile(c);
    case V_BF16_STREAM32: return (form == GEN_64 || (form < 0 && c.left != LEFT_MX4)) && near_tile(c);
    default: return false;
    }
}

Plan choose(const Mx4Call &c)
{
    if (takes(c, V_BF16_PP256, -1) && c.a.M >= 512)
        return Plan{V_BF16_PP256, 1, -1};
    return Plan{V_GENERIC, 1, -1};
}

}  // namespace

int plan_mx4(const Mx4Call &c, int forced_variant, int forced_form, Plan *out)
{
    if (forced_variant >= 0 || forced_form >= 0) {
        *out = Plan{forced_variant < 0 ? V_GENERIC : forced_variant, 1, forced_form};
        return takes(c, out->variant, out->form) ? BRGEMM_OK : BRGEMM_INVALID_ARG;
    }
    *out = choose(c);
    return BRGEMM_OK;
}

hipError_t launch_mx4(const Mx4Call &c, const Plan &plan)
{
    if (!c.grouped && (c.a.M + 15) / 16 > kMostTiles) {
        // More rows of tiles than a launch holds: the rows in two parts.
        const int64_t m = c.a.M / 2 / 256 * 256;
        Mx4Call first = c, rest = c;
        first.a.M = m;
        rest.a.M -= m;
        rest.a.A += m * c.a.lda;
        rest.a.a_powers += m * 8;
        rest.a.epi.C = (char *)c.a.epi.C + m * c.a.epi.ldc * (c.a.epi.c_f32 ? 4 : 2);
        const hipError_t e = launch_mx4(first, plan);
        return e == hipSuccess ? launch_mx4(rest, plan) : e;
    }
    const int64_t rows = c.grouped ? most_row_tiles(c.a.M, c.g.groups, 16) : (c.a.M + 15) / 16;
    if (rows * ((c.a.N + 15) / 16) > kMostTiles && c.a.N > 16) {
        // More tiles than a launch holds: the columns in two parts.
        const int64_t n = (c.a.N / 2 + 255) / 256 * 256 < c.a.N ? (c.a.N / 2 + 255) / 256 * 256 : (c.a.N / 2 + 15) / 16 * 16;
        Mx4Call first = c, rest = c;
        first.a.N = n;
        rest.a.N -= n;
        rest.a.B += n * c.a.ldb;
        rest.a.b_powers += n * 8;
        rest.a.epi.C = (char *)c.a.epi.C + n * (c.a.epi.c_f32 ? 4 : 2);
        rest.a.epi.bias = c.a.epi.bias ? c.a.epi.bias + n : nullptr;
        const hipError_t e = launch_mx4(first, plan);
        return e == hipSuccess ? launch_mx4(rest, plan) : e;
    }
    if (plan.variant == V_BF16_STREAM128)
        return mx4_stream(c, 128, 128);
    if (plan.variant == V_BF16_STREAM64)
        return mx4_stream(c, 64, 128);
    if (plan.variant == V_BF16_STREAM32)
        return mx4_stream(c, plan.form == GEN_64 ? 64 : few_rows(c) ? 16 : 32, 64);
    return plan.variant != V_BF16_PP256 ? mx4_direct(c) : c.left == LEFT_MX4 ? mx4_pingpong(c) : mx4_half(c);
}

}  // namespace brg
