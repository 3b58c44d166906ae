// Which experts a row takes, how many rows each expert has and where they go, and the loss that keeps experts level.
//
//   p_t = softmax(logits_t);  ids_t: the largest logits, of equal ones the lower expert;  gates: p at them, or that over their sum
//   counts_e: rows that took e;  offsets: their running sum;  place: where row t's j-th choice stands among all, by expert, then by row
//   loss = E sum_e f_e P_e,  f_e = counts_e / sum counts,  P_e = mean of p_te over the rows counted (those that took an expert)
//   dlogits_te = p_te (d_te - sum p_t d_t) + dloss E / n p_te (f_e - sum p_t f),  d: dgates at the chosen (level: p among the chosen)
//
// A row is 8 to 64 lanes with 1 to 16 logits each, in registers from one read to the last use; what rows share (counts, sums of p) goes
// workgroup by workgroup to the workspace, a second launch adds those up in the order of the rows, so that results do not depend on which
// workgroup was first, and a third places the rows.  Few rows are one workgroup and one launch.  Bound by launches and latencies: the data are a few MB.
#include "../../include/brgemm.h"
#include "grouped.hpp"
#include "numbers.hpp"
#include "route.hpp"

namespace brg {

namespace {

constexpr int NT = 512, NW = NT / 64;           // threads and waves of a workgroup
constexpr int SCAN_PARTS = 32, SCAN_EACH = 16;  // of route_scan_kernel: parts of all workgroups, workgroups of a part
constexpr int MOST_BLOCKS = SCAN_PARTS * SCAN_EACH;
constexpr int UNSCANNED = 32;                   // so few workgroups the third launch adds up by itself (300 rows, 64 experts: 10.9 us with the second)
constexpr float kNone = -INFINITY;

// f over the LANES lanes of a row, in every one of them (all lanes of the wave active).
template <int LANES, class F>
__device__ __forceinline__ uint32_t across(uint32_t x, F f)
{
    x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));       // lanes 1 0 3 2
    x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));       // lanes 2 3 0 1
    x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));      // 8 lanes mirrored
    if constexpr (LANES > 8)
        x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true));  // 16 lanes mirrored
    if constexpr (LANES > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = f(r[0], r[1]);
    }
    if constexpr (LANES > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = f(r[0], r[1]);
    }
    return x;
}
template <int LANES>
__device__ __forceinline__ float sum_across(float v)
{
    return __uint_as_float(across<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int LANES>
__device__ __forceinline__ float max_across(float v)
{
    return __uint_as_float(across<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int LANES>
__device__ __forceinline__ uint32_t min_across(uint32_t v)
{
    return across<LANES>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

// NV logits that follow one another, at their own alignment.
template <class T, int NV> struct Run { typedef T type __attribute__((ext_vector_type(NV), aligned(sizeof(T)))); };

// A row's logits: lane l of its LANES has experts NV l .. NV l + NV - 1; where there is no expert -inf.
template <int DT, int LANES, int NV>
struct Row {
    float x[NV], p[NV];
    float largest, sum;                         // sum of exp(x - largest)

    __device__ __forceinline__ void load(const typename Num<DT>::type *logits, int lane, int experts, bool is)
    {
        typedef typename Num<DT>::type T;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            x[v] = kNone;
        if (!is)
            return;
        if constexpr (NV > 1) {
            if (lane * NV + NV <= experts) {
                const auto run = *(const typename Run<T, NV>::type *)(logits + lane * NV);
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    x[v] = Num<DT>::wide(run[v]);
                return;
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (lane * NV + v < experts)
                x[v] = Num<DT>::wide(logits[lane * NV + v]);
    }
    __device__ __forceinline__ void drop()      // (the row takes no expert)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            x[v] = kNone;
    }
    // p = softmax(x), zeros where no expert is to be had.  (fmaxf drops NaN; its row then has a sum of NaN.)
    __device__ __forceinline__ void softmax()
    {
        float m = kNone, s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            m = fmaxf(m, x[v]);
        largest = max_across<LANES>(m);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            p[v] = largest == kNone ? 0.0f : expf(x[v] - largest);
            s += p[v];
        }
        sum = sum_across<LANES>(s);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            p[v] = largest == kNone ? 0.0f : p[v] / sum;
    }
};

struct RouteArgs {
    int64_t M, ld, ldd;
    int experts, chosen, level;
    int64_t per;                                // rows of a workgroup
    int blocks;                                 // workgroups
    const void *logits;
    const uint8_t *valid;
    int64_t *ids;
    float *gates;
    int64_t *offsets, *rows, *place;
    float *balance;
    const float *dgates, *dloss;
    void *dlogits;
    int *counts;                                // blocks x E
    float *sums;                                // blocks x (E + 1): of p, and the rows counted
    int *totals;                                // E
    float *sums_of_all;                         // E + 1
};

// ids and gates of rows first .. end - 1, and of those rows, in LDS when this returns to all threads: counts[e] and
// sums[e] (of p), sums[E] the rows counted.  `parts`: NW * (LANES * NV + 1) floats; `picks`: NT / LANES * kMostChosen.
template <int DT, int LANES, int NV>
__device__ __forceinline__ void choose_rows(const RouteArgs &a, int64_t first, int64_t end, int *counts, float *sums, float *parts, int *picks)
{
    typedef typename Num<DT>::type T;
    constexpr int AT_ONCE = NT / LANES;
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, E = a.experts;
    for (int e = threadIdx.x; e < E; e += NT)
        counts[e] = 0;
    __syncthreads();
    float mine[NV] = {};
    int counted = 0;
    auto pass = [&](int64_t t0) {
        const int64_t t = t0 + slot, at_t = t < end ? t : first;
        const uint8_t valid = a.valid ? a.valid[at_t] : 1;
        Row<DT, LANES, NV> row;
        row.load((const T *)a.logits + at_t * a.ld, lane, E, t < end);      // (beside `valid`, not after it)
        const bool is = t < end && valid != 0;
        if (!is)
            row.drop();
        row.softmax();
        // Choice by choice: the largest logit left, in the first lane that has it (its experts are the lowest), which notes it in LDS.
        uint32_t taken = 0;                     // bit v: this lane's v-th expert is chosen
        float chosen = kNone;                   // of choice `lane`
        int *const pick = picks + slot * (int)kMostChosen;
        for (int j = 0; j < a.chosen; ++j) {
            float own = kNone;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                own = fmaxf(own, (taken >> v) & 1 ? kNone : row.x[v]);
            const float best = max_across<LANES>(own);
            const uint64_t with = __builtin_amdgcn_ballot_w64(own == best && best != kNone) >> (threadIdx.x & (64 - LANES));
            chosen = lane == j ? best : chosen;
            if (with != 0 && lane == __builtin_ctzll(with)) {
                int at = 0;
#pragma unroll
                for (int v = NV - 1; v >= 0; --v)
                    at = row.x[v] == best && !((taken >> v) & 1) ? v : at;
                taken |= 1u << at;
                pick[j] = lane * NV + at;
            }
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        const int id = lane < a.chosen && chosen != kNone ? pick[lane] : -1;
        float gate = id >= 0 ? expf(chosen - row.largest) / row.sum : 0.0f;
        if (a.level) {
            const float total = sum_across<LANES>(gate);
            gate = id >= 0 ? gate / total : 0.0f;
        }
        if (t < end && lane < a.chosen) {
            a.ids[t * a.chosen + lane] = id;
            a.gates[t * a.chosen + lane] = gate;
            if (id >= 0)
                atomicAdd(&counts[id], 1);
        }
        if (is && row.largest != kNone) {
            ++counted;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                mine[v] += row.p[v];
        }
    };
    constexpr int64_t MOST = 256 * AT_ONCE;     // rows whose p are added up in 32 bits
    if (end - first <= MOST) {
        for (int64_t t0 = first; t0 < end; t0 += AT_ONCE)
            pass(t0);
    } else {                                    // (one workgroup may have 2^31)
        double all[NV] = {};
        for (int64_t from = first; from < end; from += MOST) {
            for (int64_t t0 = from; t0 < end && t0 < from + MOST; t0 += AT_ONCE)
                pass(t0);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                all[v] += mine[v];
                mine[v] = 0.0f;
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
            mine[v] = (float)all[v];
    }
    // Sums over the rows of a wave, then of all waves: always in this order.
#pragma unroll
    for (int apart = LANES; apart < 64; apart *= 2) {
        counted += __shfl_xor(counted, apart);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            mine[v] += __shfl_xor(mine[v], apart);
    }
    const int w = threadIdx.x >> 6;
    float *part = parts + w * (LANES * NV + 1);
    if ((threadIdx.x & 63) < LANES) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
            part[lane * NV + v] = mine[v];
        if (lane == 0)
            part[LANES * NV] = __int_as_float(counted);
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += NT) {
        float s = 0.0f;
        uint32_t n = 0;                         // (of whole numbers, e == E)
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const float part = parts[i * (LANES * NV + 1) + (e < E ? e : LANES * NV)];
            s += part;
            n += __float_as_uint(part);
        }
        sums[e] = e < E ? s : (float)n;
    }
    __syncthreads();
}

// The places of the choices of rows first .. end - 1, which follow `before` choices of earlier rows; total: of all rows, E counts in LDS that
// become where every expert starts.  running: NW x E.  Writes the offsets where `writes`.  Returns how many choices there are in all.
struct Slots {
    int64_t from, to;                           // of a wave , 64 at a time
    int id;                                     // the first 64
    __device__ __forceinline__ Slots(const RouteArgs &a, int64_t first, int64_t end)
    {
        const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const int64_t begin = first * a.chosen, stop = end * a.chosen;
        const int64_t share = ((stop - begin + NW - 1) / NW + 63) / 64 * 64;
        from = begin + w * share < stop ? begin + w * share : stop;
        to = from + share < stop ? from + share : stop;
        id = from + lane < to ? (int)a.ids[from + lane] : -1;
    }
};
__device__ __forceinline__ int place_rows(const RouteArgs &a, const Slots &slots, int *before, int *total, int *running, bool writes)
{
    const int E = a.experts, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t from = slots.from, to = slots.to;
    for (int i = threadIdx.x; i < NW * E; i += NT)
        running[i] = 0;
    __syncthreads();
    for (int64_t s = from + lane; s < to; s += 64) {
        const int id = s < from + 64 ? slots.id : (int)a.ids[s];
        if (id >= 0)
            atomicAdd(&running[w * E + id], 1);
    }
    __shared__ int all;
    if (w == 0) {                               // counts to where every expert starts
        int carry = 0;
        for (int e0 = 0; e0 < E; e0 += 64) {
            const int c = e0 + lane < E ? total[e0 + lane] : 0, upto = wave_prefix_sum(c);
            if (e0 + lane < E) {
                total[e0 + lane] = carry + upto - c;
                if (writes)
                    a.offsets[e0 + lane] = carry + upto - c;
            }
            carry += __builtin_amdgcn_readlane(upto, 63);
        }
        if (lane == 0) {
            all = carry;
            if (writes)
                a.offsets[E] = carry;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += NT) {
        int at = total[e] + before[e];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int c = running[i * E + e];
            running[i * E + e] = at;
            at += c;
        }
    }
    __syncthreads();
    const int bits = 32 - __builtin_clz((unsigned)E);
    for (int64_t s0 = from; s0 < to; s0 += 64) {
        const int64_t s = s0 + lane;
        const int id = s0 == from ? slots.id : s < to ? (int)a.ids[s] : -1;
        uint64_t same = __builtin_amdgcn_ballot_w64(id >= 0);
        for (int b = 0; b < bits; ++b) {
            const bool set = (id >> b) & 1;
            const uint64_t with = __builtin_amdgcn_ballot_w64(set);
            same &= set ? with : ~with;
        }
        const uint64_t lower = ((uint64_t)1 << lane) - 1;
        if (id >= 0) {
            const int at = running[w * E + id] + __builtin_popcountll(same & lower);
            a.place[s] = at;
            a.rows[at] = s / a.chosen;
            asm volatile("" ::: "memory");
            if ((same & ~lower) >> 1 >> lane == 0)          // the last of its expert
                running[w * E + id] = at + 1;
        } else if (s < to) {
            a.place[s] = -1;
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
    return all;
}

// Loss, rows counted and mean probabilities: where every expert starts and sums (E + 1) in LDS, `all` choices.
__device__ __forceinline__ void write_balance(const RouteArgs &a, const int *starts, const float *sums, int all, float *parts)
{
    const int E = a.experts;
    __syncthreads();
    const float n = sums[E];
    float s = 0.0f;
    for (int e = threadIdx.x; e < E; e += NT) {
        const float mean = n > 0.0f ? sums[e] / n : 0.0f;
        a.balance[2 + e] = mean;
        s += all > 0 ? (float)((e + 1 < E ? starts[e + 1] : all) - starts[e]) / (float)all * mean : 0.0f;
    }
    s = sum_across<64>(s);
    if ((threadIdx.x & 63) == 0)
        parts[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        float loss = 0.0f;
        for (int i = 0; i < NW; ++i)
            loss += parts[i];
        a.balance[0] = (float)E * loss;
        a.balance[1] = n;
    }
}

// Rows without a choice in `rows`, behind the last.
__device__ __forceinline__ void clear_rest(const RouteArgs &a, int all, int block, int blocks)
{
    for (int64_t s = all + (int64_t)block * NT + threadIdx.x; s < a.M * a.chosen; s += (int64_t)blocks * NT)
        a.rows[s] = -1;
}

struct Shared {
    int counts[kMostExperts], total[kMostExperts];
    float sums[kMostExperts + 1];
    union {
        float parts[NW * (kMostExperts + 1)];
        int running[NW * kMostExperts];
    };
    int picks[NT / 8 * kMostChosen];
};

// All rows in one workgroup.
template <int DT, int LANES, int NV>
__global__ void __launch_bounds__(NT)
route_few_kernel(RouteArgs a)
{
    __shared__ Shared s;
    choose_rows<DT, LANES, NV>(a, 0, a.M, s.counts, s.sums, s.parts, s.picks);
    for (int e = threadIdx.x; e < a.experts; e += NT)
        s.total[e] = s.counts[e];
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += NT)
        s.counts[e] = 0;                        // (no earlier rows)
    const int all = place_rows(a, Slots(a, 0, a.M), s.counts, s.total, s.running, true);
    clear_rest(a, all, 0, 1);
    write_balance(a, s.total, s.sums, all, s.parts);
}

// Many rows, first launch: a workgroup's rows, their counts and sums.
template <int DT, int LANES, int NV>
__global__ void __launch_bounds__(NT)
route_choose_kernel(RouteArgs a)
{
    __shared__ Shared s;
    const int64_t first = blockIdx.x * a.per, end = first + a.per < a.M ? first + a.per : a.M;
    choose_rows<DT, LANES, NV>(a, first, end, s.counts, s.sums, s.parts, s.picks);
    for (int e = threadIdx.x; e <= a.experts; e += NT) {
        if (e < a.experts)
            a.counts[(int64_t)blockIdx.x * a.experts + e] = s.counts[e];
        a.sums[(int64_t)blockIdx.x * (a.experts + 1) + e] = s.sums[e];
    }
}

// Second launch, a lane for each expert (and one for the rows counted) and every 32nd of the workgroups: counts become those of the rows
// before each workgroup's, with their total and the sum of p beside them.  (Without it every workgroup of the third adds up what all
// have: 4099 rows, 160 experts 19 us.  With an expert's counts next to each other every one is a store of its own: 2048 rows, 1024 experts 17.8 us in the
// first launch, 13.1 as it is.)
__global__ void __launch_bounds__(32 * SCAN_PARTS)
route_scan_kernel(RouteArgs a)
{
    __shared__ int counts[SCAN_PARTS][32];
    __shared__ float sums[SCAN_PARTS][32];
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, e = (int)blockIdx.x * 32 + lane, E = a.experts;
    const int each = (a.blocks + SCAN_PARTS - 1) / SCAN_PARTS, first = part * each;
    const int end = first + each < a.blocks ? first + each : a.blocks;
    int *const count = a.counts + (e < E ? e : 0);
    const float *const sum = a.sums + (e <= E ? e : 0);
    int c[SCAN_EACH], own = 0;
    float p = 0.0f;
    auto read = [&](auto nc) {                  // (all loads at once; what is not this part's own, the last one's)
        constexpr int n = decltype(nc)::value;
        float v[n];
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int b = first + i < a.blocks ? first + i : a.blocks - 1;
            c[i] = count[b * E];
            v[i] = sum[b * (E + 1)];
        }
#pragma unroll
        for (int i = 0; i < n; ++i) {
            c[i] = first + i < end ? c[i] : 0;
            own += c[i];
            p += first + i < end ? v[i] : 0.0f;
        }
    };
    if (each <= SCAN_EACH / 2)
        read(std::integral_constant<int, SCAN_EACH / 2>{});
    else
        read(std::integral_constant<int, SCAN_EACH>{});
    counts[part][lane] = own;
    sums[part][lane] = p;
    __syncthreads();
    int before = 0, total = 0;
    p = 0.0f;
#pragma unroll
    for (int i = 0; i < SCAN_PARTS; ++i) {
        before += i < part ? counts[i][lane] : 0;
        total += counts[i][lane];
        p += sums[i][lane];
    }
    if (e < E) {
#pragma unroll
        for (int i = 0; i < SCAN_EACH; ++i) {
            if (i < each) {
                if (first + i < end)
                    count[(first + i) * E] = before;
                before += c[i];
            }
        }
    }
    if (part == 0 && e <= E) {
        a.sums_of_all[e] = p;
        if (e < E)
            a.totals[e] = total;
    }
}

// Third launch: the places of a workgroup's rows; one more workgroup has the offsets and the balance.
__global__ void __launch_bounds__(NT)
route_place_kernel(RouteArgs a)
{
    __shared__ Shared s;
    const int E = a.experts, block = (int)blockIdx.x;
    const bool last = block == a.blocks;
    const int64_t first = last ? 0 : block * a.per, end = last ? 0 : first + a.per < a.M ? first + a.per : a.M;
    const Slots slots(a, first, end);           // (requested first)
    for (int e = threadIdx.x; e <= E; e += NT) {
        if (a.blocks <= UNSCANNED) {
            const int *const count = a.counts + (e < E ? e : 0);
            int before = 0, total = 0;
            float sum = 0.0f;
#pragma unroll 8
            for (int b = 0; b < a.blocks; ++b) {
                const int c = count[b * E];
                before += b < block ? c : 0;
                total += c;
                sum += last ? a.sums[b * (E + 1) + e] : 0.0f;
            }
            if (e < E) {
                s.counts[e] = last ? 0 : before;
                s.total[e] = total;
            }
            s.sums[e] = sum;
        } else {
            if (e < E) {
                s.counts[e] = last ? 0 : a.counts[(int64_t)block * E + e];
                s.total[e] = a.totals[e];
            }
            if (last)
                s.sums[e] = a.sums_of_all[e];
        }
    }
    __syncthreads();
    const int all = place_rows(a, slots, s.counts, s.total, s.running, last);
    if (last)
        write_balance(a, s.total, s.sums, all, s.parts);
    else
        clear_rest(a, all, block, a.blocks);
}

constexpr int GRAD_NT = 512;

template <int DT, int LANES, int NV>
__global__ void __launch_bounds__(GRAD_NT)
route_grad_kernel(RouteArgs a)
{
    typedef typename Num<DT>::type T;
    constexpr int AT_ONCE = GRAD_NT / LANES;
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES, E = a.experts;
    // What all rows need, requested beside the first row: used in turn, every one of these loads is 1 us.
    const int64_t all = a.offsets[E];
    const float n = a.balance[1], dloss = a.dloss ? *a.dloss : 0.0f;
    int64_t bounds[NV + 1] = {};
    if (lane * NV + NV <= E) {
        const auto run = *(const typename Run<int64_t, NV>::type *)(a.offsets + lane * NV);
#pragma unroll
        for (int v = 0; v < NV; ++v)
            bounds[v] = run[v];
        bounds[NV] = a.offsets[lane * NV + NV];
    } else if (lane * NV < E) {
#pragma unroll
        for (int v = 0; v <= NV; ++v)
            bounds[v] = a.offsets[lane * NV + v < E ? lane * NV + v : E];
    }
    for (int64_t t0 = (int64_t)blockIdx.x * AT_ONCE; t0 < a.M; t0 += (int64_t)gridDim.x * AT_ONCE) {
        const int64_t t = t0 + slot, at_t = t < a.M ? t : a.M - 1;
        int64_t i = -1;                         // of choice `lane`
        float d = 0.0f;
        if (t < a.M && lane < a.chosen) {
            i = a.ids[t * a.chosen + lane];
            d = a.dgates ? a.dgates[t * a.chosen + lane] : 0.0f;
        }
        Row<DT, LANES, NV> row;
        row.load((const T *)a.logits + at_t * a.ld, lane, E, t < a.M);
        const int id = i >= 0 && i < E ? (int)i : -1;
        d = id >= 0 ? d : 0.0f;
        const bool is = min_across<LANES>(id >= 0 ? 0u : 1u) == 0;
        if (!is)
            row.drop();
        row.softmax();
        const float weight = all > 0 && n > 0.0f ? dloss * (float)E / n : 0.0f;
        float f[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v)
            f[v] = weight != 0.0f ? (float)(bounds[v + 1] - bounds[v]) / (float)all : 0.0f;
        float dp[NV] = {};
        uint32_t taken = 0;
        for (int j = 0; j < a.chosen; ++j) {
            const int ij = __shfl(id, j, LANES);
            const float dj = __shfl(d, j, LANES);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const bool hit = ij == lane * NV + v;
                dp[v] += hit ? dj : 0.0f;
                taken |= hit ? 1u << v : 0u;
            }
        }
        // The gates' own probabilities: p, or p among the chosen.
        float g[NV], dot = 0.0f, even = 0.0f, among = 1.0f;
        if (a.level) {
            float s = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                s += (taken >> v) & 1 ? row.p[v] : 0.0f;
            among = sum_across<LANES>(s);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            g[v] = !a.level ? row.p[v] : (taken >> v) & 1 ? row.p[v] / among : 0.0f;
            dot += g[v] * dp[v];
            even += row.p[v] * f[v];
        }
        dot = sum_across<LANES>(dot);
        even = sum_across<LANES>(even);
        if (t < a.M) {
            T *to = (T *)a.dlogits + t * a.ldd + lane * NV;
            typename Run<T, NV>::type out;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                out[v] = Num<DT>::narrow(is ? g[v] * (dp[v] - dot) + weight * (row.p[v] * (f[v] - even)) : 0.0f);
            if (lane * NV + NV <= E) {
                *(typename Run<T, NV>::type *)to = out;
            } else {
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    if (lane * NV + v < E)
                        to[v] = out[v];
            }
        }
    }
}

// Lanes and values a lane by the number of experts: few lanes mean few steps across them, and 16 suffice for the choices.
template <class F>
hipError_t by_experts(int64_t experts, F f)
{
    if (experts <= 8) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (experts <= 16) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    if (experts <= 32) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    if (experts <= 64) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
    if (experts <= 128) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 4>{});
    if (experts <= 256) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 8>{});
    if (experts <= 512) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 16>{});
}
int lanes_of(int64_t experts) { return experts <= 8 ? 8 : experts <= 64 ? 16 : experts <= 256 ? 32 : 64; }

// Workgroups of the first launch, of whole passes over as many rows as they take at once.
int64_t blocks_of(int64_t M, int64_t experts)
{
    const int64_t at_once = NT / lanes_of(experts);
    if (M <= 4 * at_once)
        return 1;
    const int64_t n = (M + at_once - 1) / at_once, passes = (n + MOST_BLOCKS - 1) / MOST_BLOCKS;
    return (n + passes - 1) / passes;
}
size_t block_bytes(int64_t experts) { return (size_t)(2 * experts + 1) * 4; }

RouteArgs args_of(const RouteCall &c)
{
    return RouteArgs{c.M, c.ld, c.ldd, c.experts, c.chosen, c.level, c.M, 1, c.logits, c.valid, c.ids, c.gates, c.offsets, c.rows, c.place,
                     c.balance, c.dgates, c.dloss, c.dlogits, nullptr, nullptr, nullptr, nullptr};
}

template <int DT>
hipError_t route(const RouteCall &c)
{
    RouteArgs a = args_of(c);
    int64_t blocks = blocks_of(c.M, c.experts);
    const int64_t fit = (int64_t)(c.workspace_bytes / block_bytes(c.experts)) - 1;         // (one for what all have)
    blocks = blocks < fit ? blocks : fit;
    return by_experts(c.experts, [&](auto lanes, auto values) {
        constexpr int L = decltype(lanes)::value, V = decltype(values)::value;
        if (blocks <= 1) {
            hipLaunchKernelGGL((route_few_kernel<DT, L, V>), dim3(1), dim3(NT), 0, c.stream, a);
            return hipGetLastError();
        }
        constexpr int64_t at_once = NT / L;
        a.per = (c.M + blocks * at_once - 1) / (blocks * at_once) * at_once;
        a.blocks = (int)((c.M + a.per - 1) / a.per);
        a.counts = (int *)c.workspace;
        a.sums = (float *)(a.counts + (int64_t)a.blocks * c.experts);
        a.totals = (int *)(a.sums + (int64_t)a.blocks * (c.experts + 1));
        a.sums_of_all = (float *)(a.totals + c.experts);
        hipLaunchKernelGGL((route_choose_kernel<DT, L, V>), dim3((unsigned)a.blocks), dim3(NT), 0, c.stream, a);
        if (a.blocks > UNSCANNED)
            hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)(c.experts / 32 + 1)), dim3(32 * SCAN_PARTS), 0, c.stream, a);
        hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)a.blocks + 1), dim3(NT), 0, c.stream, a);
        return hipGetLastError();
    });
}

template <int DT>
hipError_t route_grad(const RouteCall &c)
{
    const RouteArgs a = args_of(c);
    return by_experts(c.experts, [&](auto lanes, auto values) {
        constexpr int L = decltype(lanes)::value, V = decltype(values)::value;
        const int64_t groups = (c.M + GRAD_NT / L - 1) / (GRAD_NT / L);
        hipLaunchKernelGGL((route_grad_kernel<DT, L, V>), dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(GRAD_NT), 0, c.stream, a);
        return hipGetLastError();
    });
}

}  // namespace

size_t route_workspace(int64_t M, int64_t experts)
{
    const int64_t blocks = blocks_of(M, experts);
    return blocks > 1 ? (size_t)(blocks + 1) * block_bytes(experts) : 0;
}

hipError_t launch_route(const RouteCall &c)
{
    return c.dtype == BRGEMM_DTYPE_F32 ? route<BRGEMM_DTYPE_F32>(c) : c.dtype == BRGEMM_DTYPE_BF16 ? route<BRGEMM_DTYPE_BF16>(c)
                                                                                              : route<BRGEMM_DTYPE_F16>(c);
}

hipError_t launch_route_grad(const RouteCall &c)
{
    return c.dtype == BRGEMM_DTYPE_F32 ? route_grad<BRGEMM_DTYPE_F32>(c) : c.dtype == BRGEMM_DTYPE_BF16 ? route_grad<BRGEMM_DTYPE_BF16>(c)
                                                                                                   : route_grad<BRGEMM_DTYPE_F16>(c);
}

}  // namespace brg
