// Plan and launches of the products with 4-bit images (mx4.hpp).
#include "../../include/brgemm.h"
#include "mx4.hpp"
#include <cmath>

namespace brg {

namespace {

// 16-bit rows that tiles can read: global->LDS loads, and a lane's offset that reaches over 128 of them.
bool whole_rows(const Mx4Call &c)
{
    return ((uintptr_t)c.a.A & 15) == 0 && c.a.lda % 16 == 0 && c.a.lda <= (int64_t)1 << 24 && c.a.K % 64 == 0;
}

bool near_tile(const Mx4Call &c)
{
    return c.a.ldb <= (int64_t)1 << 24 && (c.left == LEFT_MX4 || whole_rows(c));
}

// Most groups have at most 16 rows.
bool few_rows(const Mx4Call &c) { return c.grouped ? c.a.M <= 12 * c.g.groups : c.a.M <= 16; }

bool takes(const Mx4Call &c, int variant, int form)
{
    switch (variant) {
    case V_GENERIC: return form < 0;
    case V_BF16_PP256:
    case V_BF16_STREAM128:
    case V_BF16_STREAM64: return form < 0 && near_tile(c);
    case V_BF16_STREAM32: return (form == GEN_64 || (form < 0 && c.left != LEFT_MX4)) && near_tile(c);
    default: return false;
    }
}

// A split of the reduction needs its slices' sums in the workspace.
size_t split_bytes(const Mx4Call &c, int split) { return (size_t)split * (size_t)c.a.M * (size_t)c.a.N * sizeof(float); }
bool splits(const Mx4Call &c, int variant, int split)
{
    return split == 1 || (!c.grouped && variant != V_BF16_PP256 && split <= kMaxSplit && split <= c.a.blocks && split_bytes(c, split) <= c.workspace_bytes &&
                          split_bytes(c, 1) <= (size_t)1 << 33);
}

// A kernel a plan may take, and what a call of it costs in a rough model of time, in microseconds: what every call has, a tile's fixed part, 256
// columns of its reduction where the tile has a CU to itself and where two share one (at_once == 512), and bytes a microsecond.
struct Candidate {
    Plan plan;
    int bm, bn, at_once;
    double call, fixed, alone, shared, rate;
};

// Fitted to sweeps of all tiles over 600 calls of either kind (1 to 8192 rows, 2 to 64 groups or none, weights 256 x 256 to 11008 x 8192); the choice is
// behind the best of them by 2 % on average, 3 % for many rows in groups, and by up to 57 % (1556 rows, 2496 x 2816: 45 us in 128 x 128
// tiles and 29 in 64 x 128).
const Candidate kRows[] = {{{V_GENERIC, 1, -1}, 16, 16, 512, 5.9, 0.0, 0.095, 0.227, 1e12}, {{V_BF16_STREAM32, 1, -1}, 32, 64, 512, 2.8, 2.2, 0.287, 0.533, 5.1e6},
                           {{V_BF16_STREAM32, 1, GEN_64}, 64, 64, 256, 1.5, 3.3, 0.482, 0.482, 2.4e6}, {{V_BF16_STREAM64, 1, -1}, 64, 128, 256, 0.4, 4.7, 0.761, 0.761, 2.7e6},
                           {{V_BF16_STREAM128, 1, -1}, 128, 128, 256, 0.0, 5.75, 1.516, 1.516, 1.9e6}, {{V_BF16_PP256, 1, -1}, 256, 256, 256, 1.0, 9.2, 5.16, 5.16, 1.6e6}};
const Candidate kImages[] = {{{V_GENERIC, 1, -1}, 16, 16, 512, 6.0, 0.0, 0.025, 0.08, 1e12}, {{V_BF16_STREAM32, 1, GEN_64}, 64, 64, 512, 1.95, 3.3, 0.119, 0.326, 5.3e6},
                             {{V_BF16_STREAM64, 1, -1}, 64, 128, 512, 1.6, 3.9, 0.221, 0.611, 5.5e6}, {{V_BF16_STREAM128, 1, -1}, 128, 128, 256, 0.0, 6.1, 0.378, 0.378, 4.7e6},
                             {{V_BF16_PP256, 1, -1}, 256, 256, 256, 7.2, 3.2, 1.337, 1.337, 2.3e6}};

// Tiles of bm rows that groups of `rows` rows in all are expected to have (sizes spread exponentially, as in choose_forward of gemm_grouped).
// Of 256 rows, the last of a group where it has at most 128 rows (two of 128 x 128) counts as `half` of one.
double row_tiles(const Mx4Call &c, int bm, double half = 1.0)
{
    if (!c.grouped)
        return (double)((c.a.M + bm - 1) / bm);
    const double rows = (double)c.a.M, groups = (double)c.g.groups, used = rows < groups ? rows : groups;
    const double more = std::exp(-bm * used / rows);
    return used / (1.0 - more) * (1.0 - (1.0 - half) * (1.0 - std::sqrt(more)));
}

double model(const Mx4Call &c, const Candidate &k, int split)
{
    const Mx4Args &a = c.a;
    const int bm = k.plan.variant == V_BF16_STREAM32 && k.plan.form < 0 && few_rows(c) ? 16 : k.bm;
    const double half = bm < 256 ? 1.0 : 0.7;
    const double tiles = row_tiles(c, bm, half) * (double)((a.N + k.bn - 1) / k.bn) * split;
    const double blocks = split > 1 ? (double)((a.blocks + split - 1) / split) : (double)((a.K + 63) / 64) / 4.0;
    double work;
    if (tiles <= 260.0) {
        work = k.fixed + blocks * k.alone;
    } else {
        const double n = tiles / k.at_once, rounds = n <= 1.02 ? 1.0 : !c.grouped ? std::ceil(n) : n > 1.4 ? n + 0.4 : 1.8;
        work = rounds * (k.fixed + blocks * (k.at_once == 512 ? k.shared : k.alone));
    }
    const double groups = !c.grouped ? 1.0 : (double)(c.g.groups < a.M ? c.g.groups : a.M);
    const double bytes = groups * a.N * a.K / 2 + (double)a.M * a.K * (c.left == LEFT_MX4 ? 0.5 : 2.0) + 2.0 * a.M * a.N;
    const double memory = bytes / k.rate;
    // (a split's second launch, and its sums)
    return k.call + (work > memory ? work : memory) + (split > 1 ? 3.5 + 8e-7 * (double)a.M * (double)a.N * split : 0.0);
}

Plan choose(const Mx4Call &c)
{
    const bool images = c.left == LEFT_MX4;
    const int64_t rows = c.grouped ? (c.a.M + c.g.groups - 1) / c.g.groups : c.a.M;
    Plan best{V_GENERIC, 1, -1};
    double best_t = 1e30;
    for (int i = 0; i < (images ? 5 : 6); ++i) {
        const Candidate &k = images ? kImages[i] : kRows[i];
        // (the first is fitted to 16 rows and up to 1024 tiles; beyond them it is for what the others do not read)
        if (!takes(c, k.plan.variant, k.plan.form) || (k.plan.variant == V_GENERIC && (rows > 16 || row_tiles(c, 16) * (double)((c.a.N + 15) / 16) > 1024.0)))
            continue;
        // Splits of long reductions on few tiles: 16-bit rows in the smallest tiles (16 x 4096 x 11008 21.8 us without).
        static const int most[] = {1, 2, 3, 4, 6, 8};
        for (int split : most) {
            if (split > 1 && (images || k.plan.variant != V_BF16_STREAM32 || k.plan.form >= 0 || c.a.blocks < 2 * split || !splits(c, k.plan.variant, split)))
                break;
            const double t = model(c, k, split);
            if (t < best_t) {
                best_t = t;
                best = k.plan;
                best.split = split;
            }
        }
    }
    return best;
}

}  // namespace

int plan_mx4(const Mx4Call &c, int forced_variant, int forced_split, int forced_form, Plan *out)
{
    if (forced_variant >= 0 || forced_form >= 0 || forced_split > 0) {
        *out = Plan{forced_variant < 0 ? V_GENERIC : forced_variant, forced_split > 0 ? forced_split : 1, forced_form};
        if (!takes(c, out->variant, out->form))
            return BRGEMM_INVALID_ARG;
        return splits(c, out->variant, out->split) ? BRGEMM_OK : out->split > kMaxSplit || c.grouped || out->variant == V_BF16_PP256 || out->split > c.a.blocks ? BRGEMM_INVALID_ARG : BRGEMM_WORKSPACE_TOO_SMALL;
    }
    *out = choose(c);
    return BRGEMM_OK;
}

// Rows that the tiles cannot read (off 16 bytes, or a K that ends inside 64 columns) are copied into the workspace first, with zeros
// behind K: 2.5 us and a read and a write of them, where 512 x 4096 x 4096 takes 45 us in mx4_direct and 18 in tiles.
static size_t copy_bytes(const Mx4Call &c) { return (size_t)c.a.M * (size_t)((c.a.K + 63) / 64) * 128; }
bool mx4_copies(const Mx4Call &c)
{
    const int64_t rows = c.grouped ? (c.a.M + c.g.groups - 1) / c.g.groups : c.a.M;
    return c.left != LEFT_MX4 && rows > 16 && c.a.K > 0 && !whole_rows(c) && copy_bytes(c) <= c.workspace_bytes && copy_bytes(c) <= (size_t)1 << 32;
}
hipError_t mx4_copy(Mx4Call &c)
{
    const int64_t pitch = (c.a.K + 63) / 64 * 128;
    const hipError_t e = launch_mx4_rows((const char *)c.a.A, c.a.lda, c.a.M, c.a.K, (char *)c.workspace, pitch, c.stream);
    const size_t used = (copy_bytes(c) + 255) / 256 * 256;
    c.a.A = (const char *)c.workspace;
    c.a.lda = pitch;
    c.a.K = pitch / 2;
    c.workspace = (char *)c.workspace + used;
    c.workspace_bytes = c.workspace_bytes > used ? c.workspace_bytes - used : 0;
    return e;
}

// The slices' sums added up.
static hipError_t reduce(const Mx4Call &c)
{
    Problem p{};
    p.M = c.a.M; p.N = c.a.N;
    p.C = c.a.epi.C; p.ldc = c.a.epi.ldc; p.c_f32 = c.a.epi.c_f32; p.in_f16 = c.a.epi.c_f16; p.in_bf16 = !p.in_f16;
    p.beta = c.a.epi.beta; p.bias = c.a.epi.bias; p.relu = c.a.epi.relu;
    p.split = c.a.split; p.partial = c.a.partial;
    p.nmat = 1;
    p.stream = c.stream;
    return launch_reduce(p);
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
    if (plan.split > 1) {
        Mx4Call part = c;
        part.a.split = plan.split;
        part.a.partial = (float *)c.workspace;
        const hipError_t e = launch_mx4(part, Plan{plan.variant, 1, plan.form});
        return e == hipSuccess ? reduce(part) : e;
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
