// attn_paged_plan.h -- how a call over the paged cache is cut into units of work, and how partial results are merged.
//
// The host knows the number of rows and sequences, not the lengths, so the workgroups work the cut out for themselves, all of
// them alike, from start and kv_len (a load, a sum over the wave, one more load for every 64 sequences); for a batch of
// many sequences one workgroup does it before them (attn_paged_plan_kernel) and they look theirs up.  A unit
// is (sequence, key head, tile of BM rows, range of keys).  A row is a query head of a token: the G query heads that
// share a key head lie side by side (row = token * G + head in group), so that a key is fetched once for all of them.
//
// No range of a call is longer than L blocks of 64 keys, and the ranges of a sequence are alike: L is what
// lets about `target` units (what the chip holds at once), or a few times that, share all the keys that the call has to walk,
// so a long sequence among short ones is walked by many workgroups.  A sequence of one range is finished by its unit;
// the units of the others leave normalised fp32 rows and their log-sum-exp, which attn_paged_merge_kernel joins.
// Working a cut out takes 0.5 us of a workgroup for one sequence, 1.2 for 64.  The merge of decoding steps is a launch of 4 us,
// most of it its own latency; that of chunks reads more: at D = 128, 32 heads over 8, 512 new tokens at 8000 leave 34 MB of
// partial rows (13.3 us), 3 x 200 at 2000 49 MB (14.4), 4 x 200 26 MB (17.3).  It is launched wherever the table could hold a sequence of
// two ranges: with nothing to merge it takes 4.4 us over 1000 tokens of 32 heads, 9.4 over 4096.
#pragma once
#include <type_traits>

#include "attn_cache_rows.h"
#include "attn_common.h"

namespace attn {

constexpr int kPlanBlock = 64;          // keys of a block

struct PagedParams {
    CacheParams c;
    // [B + 1] or NULL: the cut, worked out once for a batch of many sequences.  [0] = (units, Plan::per_block), [1 + b] = units
    // and slots of the sequences before b.  (Asked for first: here it is in the same line as what the plan begins with.)
    int2 *cut;
    const void *q;
    void *o;
    float *lse;
    const void *k, *v;
    const unsigned char *k_scale, *v_scale;
    long long q_st, q_sh;               // strides of q in elements
    int H_q, G;                         // G = H_q / H_kv
    uint32_t g_mul, g_shift;            // row / G without a division (token_of)
    int causal;
    float c_log2;                       // scale * log2(e)
    // units of this kernel: sequences of rows in (rows_above, rows_upto], cut for `target` workgroups at once that take up to
    // `rounds` units each; what a unit costs besides its keys and what a merge costs, in blocks
    int rows_above, rows_upto, target, rounds, min_range, overhead, merging;
    int halve;                          // a chunk's rows see half of the chunk's own keys (causal)
    int most_units;                     // no batch has more (starts that decrease may claim to)
    int slots;                          // partial results that the workspace holds for this kernel
    int kernel;                         // 0: attn_paged_rows.h, 1: attn_paged_tiles.h
    // partial results, of either kernel
    struct Parts {
        float *o;                       // [slots][BM][D]
        float *lse;                     // [slots][BM]
        int slots, BM;
        int2 *cut;                      // see cut
    } parts[2];
    int4 *merge;                        // [T]: see MergeNote

    // token of a row of the sequence, row >= 0: row / G = row * ceil(2^(31 + s) / G) / 2^(31 + s), s = ceil(log2 G), exact
    // below 2^31
    __device__ __forceinline__ int token_of(int row) const
    {
        return G == 1 ? row : (int)((uint32_t)(((uint64_t)(uint32_t)row * g_mul) >> 32) >> g_shift);
    }
};

// The same with a tree of drafted tokens: which of its sequence's new tokens a row sees, [T][mask_words] words of 32 bits.
struct TreeParams : PagedParams {
    const uint32_t *mask;
    int mask_words;
};
template <bool TREE>
using ParamsOf = typename std::conditional<TREE, TreeParams, PagedParams>::type;

// What the merge kernel needs to know of a token: x = first slot of its sequence, y = row tiles of the sequence,
// z = its ranges, w = first row of the token in its sequence * 2 + kernel.  Only sequences of several ranges have a
// meaningful x and w.
typedef int4 MergeNote;

struct Unit {
    int b, h, tile, range, n_ranges, n_tiles;
    int row0, n_rows;                   // start[b], rows of the sequence (tokens * G)
    int n, kv;                          // new tokens, cached positions
    int key0, key1, len;                // this range; keys of a range
    int slot0, slot;                    // first slot of the sequence, slot of this unit (n_ranges > 1)
};

// Inclusive prefix sum over the wave (the sum: lane 63), in the vector unit's own lane exchange: 16 lanes, then a row's
// last lane to the next row and the first two rows' to the last two.  Through LDS (shuffles) the six steps of every
// sum would take most of a microsecond of a launch that takes a few.
template <typename T>
__device__ __forceinline__ T wave_prefix(T x)
{
    auto from = [](T v, auto ctrl, auto rows) -> T {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    x += from(x, std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1
    x += from(x, std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    x += from(x, std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    x += from(x, std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    x += from(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15
    x += from(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast 31
    return x;
}

template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_prefix(x)), 63));
}

template <typename T>
__device__ __forceinline__ T wave_first(T x)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

__device__ __forceinline__ int wave_max(int x)              // of numbers >= 0
{
    auto from = [](int v, auto ctrl, auto rows) { return __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    x = max(x, from(x, std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{}));
    x = max(x, from(x, std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{}));
    x = max(x, from(x, std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{}));
    x = max(x, from(x, std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{}));
    x = max(x, from(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));
    x = max(x, from(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));
    return __builtin_amdgcn_readlane(x, 63);
}

// Units of one range of a sequence, H heads x n tiles: which one number w is.  Workgroups go to the 8 XCDs in turn; the tiles
// of a head, which stream the same keys, belong to one XCD (its L2) as far as heads go evenly into XCDs, or to as many as share
// the head.  Heavier tiles (the last ones, causal) come first and every XCD gets its share of them.
__host__ __device__ __forceinline__ void place_in_layer(int w, int H, int n, int &h, int &tile)
{
    if (n == 1) {
        h = w, tile = 0;
        return;
    }
    const int whole = H / kNumXcd * kNumXcd;                // heads that have an XCD to themselves
    int t;
    if (w < whole * n) {
        const int x = w % kNumXcd, i = w / kNumXcd, k = quotient(i, n);
        h = k * kNumXcd + x;
        t = i - k * n;
    } else {
        const int rest = H - whole;
        const int log_rest = rest == 4 ? 2 : rest == 2 ? 1 : 0, log_share = 3 - log_rest;     // XCDs of a head
        const bool shared = rest <= 2 || rest == 4;
        w -= whole * n;
        const int done = shared ? n >> log_share << log_share : 0;      // tiles dealt out to the XCDs of their head
        if (w < done * rest) {
            const int x = w % kNumXcd, i = w / kNumXcd;
            h = x & (rest - 1);
            t = (i << log_share) + (x >> log_rest);
        } else {
            w -= done * rest;
            const int k = quotient(w, rest);
            h = w - k * rest;
            t = done + k;
        }
        h += whole;
    }
    tile = n - 1 - t;
}

// Rows and positions of a sequence as a kernel of BM-row tiles sees them.
struct PlanSeq {
    int tiles, blocks, n, kv, start;
};

template <int BM>
__device__ __forceinline__ PlanSeq plan_sequence(const PagedParams &p, int b)
{
    PlanSeq s = {0, 0, 0, 0, 0};
    if (b < p.c.B) {
        s.start = p.c.start_of(b);
        s.n = max(p.c.start_of(b + 1) - s.start, 0);
        s.kv = p.c.length_of(b);
        const long long rows = (long long)s.n * p.G;
        if (rows > p.rows_above && rows <= p.rows_upto) {
            s.tiles = (int)((rows + BM - 1) / BM);
            s.blocks = s.kv > 0 ? (s.kv - 1) / kPlanBlock + 1 : 1;
        }
    }
    return s;
}

// The cut of a call: units, and 1 / (blocks of a range), 0 for whole sequences.
struct Plan {
    int total;
    float per_block;

    // (to the rounding of a product, the same one everywhere)
    __device__ __forceinline__ int ranges(const PlanSeq &s) const
    {
        return s.tiles ? max(1, (int)ceilf((float)s.blocks * per_block)) : 0;
    }
};

// Unit that a workgroup of a launch of `slots` (fewer than units: a multiple of the XCD count) takes in pass k: odd passes
// run through an XCD's workgroups in reverse, so that who had the heaviest tile of one pass gets the lightest of the next.
__device__ __forceinline__ int unit_of_pass(int slots, int k)
{
    const int wg = blockIdx.x, x = wg % kNumXcd, m = wg / kNumXcd;
    return k * slots + (k & 1 ? (slots / kNumXcd - 1 - m) * kNumXcd + x : wg);
}

// Who works a cut out together: a wave, or (GroupScope) a workgroup of sixteen.
struct WaveScope {
    static constexpr int kLanes = 64;
    bool one;                           // a batch of one sequence: lane 0 has it
    __device__ __forceinline__ int lane() const { return threadIdx.x & 63; }
    template <typename T>
    __device__ __forceinline__ T sum(T x) const
    {
        return one ? wave_first(x) : wave_sum(x);
    }
    __device__ __forceinline__ int most(int x) const { return one ? wave_first(x) : wave_max(x); }
    // x of the lanes before this one, and of all
    __device__ __forceinline__ int before(int x, int &all) const
    {
        const int upto = wave_prefix(x);
        all = __builtin_amdgcn_readlane(upto, 63);
        return upto - x;
    }
};
struct GroupScope {
    static constexpr int kLanes = 1024;
    int *lds;                           // [16]
    __device__ __forceinline__ int lane() const { return threadIdx.x; }
    template <typename T, typename F>
    __device__ __forceinline__ T join(T of_wave, F f) const
    {
        __syncthreads();                // what lay there has been read
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6] = __builtin_bit_cast(int, of_wave);
        __syncthreads();
        T all = __builtin_bit_cast(T, lds[0]);
        for (int w = 1; w < 16; ++w)
            all = f(w, all, __builtin_bit_cast(T, lds[w]));
        return all;
    }
    template <typename T>
    __device__ __forceinline__ T sum(T x) const
    {
        return join(wave_sum(x), [](int, T a, T b) { return a + b; });
    }
    __device__ __forceinline__ int most(int x) const
    {
        return join(wave_max(x), [](int, int a, int b) { return max(a, b); });
    }
    __device__ __forceinline__ int before(int x, int &all) const
    {
        const int upto = wave_prefix(x), wave = threadIdx.x >> 6;
        int first = 0;                  // of this wave
        all = join(__builtin_amdgcn_readlane(upto, 63), [&](int w, int a, int b) {
            first = w == wave ? a : first;
            return a + b;
        });
        return first + upto - x;
    }
};

// s: plan_sequence of this lane, for find_unit.
template <int BM, typename Scope>
__device__ __forceinline__ Plan plan_cut(const PagedParams &p, const Scope &scope, PlanSeq &s)
{
    constexpr int N = Scope::kLanes;
    const int lane = scope.lane(), B = p.c.B;
    Plan plan;
    // f(s) for every N sequences; up to N of them stay in their registers from one pass to the next
    s = plan_sequence<BM>(p, lane);
    auto pass = [&](auto f) {
        f();
        if (B > N) {
            for (int b = N; b < B; b += N) {
                s = plan_sequence<BM>(p, b + lane);
                f();
            }
            s = plan_sequence<BM>(p, lane);
        }
    };
    auto sum = [&](auto x) { return scope.sum(x); };
    // work of the call, in (row tile, block, key head)
    float work = 0.f;
    int tiles = 0, most = 0;
    pass([&] {
        const float seen = (float)s.blocks - (p.halve ? (float)min(s.n, s.kv) * (0.5f / kPlanBlock) : 0.f);
        work += sum((float)s.tiles * fmaxf(seen, 1.f));
        tiles += sum(s.tiles);
        most = max(most, scope.most(s.blocks));
    });
    work *= (float)p.c.H_kv;
    int total, held;                            // units of a key head, and slots of those that share their rows with others
    int longest;                                // range
    constexpr bool kFit = BM > 64;              // the tile kernels, whose units are long
    auto count = [&](int L) {
        plan.per_block = (1.f - 0x1p-22f) / (float)L;
        total = held = longest = 0;
        pass([&] {
            const int nr = plan.ranges(s);
            total += sum(s.tiles * nr);
            held += sum(nr > 1 ? s.tiles * nr : 0);
            if (kFit)
                longest = max(longest, scope.most(s.tiles ? quotient(s.blocks + nr - 1, nr) : 0));
            else
                longest = L;
        });
        return (long long)held * p.c.H_kv <= p.slots;
    };
    // Whole sequences, or a cut into as many units as workgroups run at once, or a few times that many (a number that just
    // exceeds them leaves most idle in the last round): what ends soonest, each unit with its share of the work and its
    // overhead, none sooner than the longest, and a cut with the merge behind it.
    auto ends = [&](int n, int longest) {
        const float units = (float)n * (float)p.c.H_kv;
        return fmaxf(ceilf(units / (float)p.target) * (work / fmaxf(units, 1.f) + (float)p.overhead), (float)(longest + p.overhead));
    };
    float soonest = ends(tiles, most);
    int L = 0;                                  // whole sequences
    for (int k = 1; k <= p.rounds; ++k) {
        int l = max(p.min_range, (int)fminf(ceilf(work / (float)(k * p.target)), 0x1p24f));
        const bool last = l == p.min_range;
        // ranges are whole blocks and a sequence's are alike, so the units may be a good deal more than k rounds: then so much
        // longer ranges too
        for (int again = 0; again < (kFit ? 2 : 1) && l < most; ++again) {
            const bool fits = count(l);
            const float e = ends(total, longest) + (float)p.merging;
            if (fits && e < soonest)
                L = l, soonest = e;
            if (!kFit)
                break;
            const float over = (float)total * (float)p.c.H_kv / (float)(k * p.target);
            if (over <= 1.f)
                break;
            l = (int)fminf(ceilf((float)l * over), 0x1p24f);
        }
        if (last)
            break;
    }
    if (L == 0)
        plan.per_block = 0.f, total = tiles;
    else if (p.rounds > 1)
        count(L);
    plan.total = __builtin_amdgcn_readfirstlane(min(total * p.c.H_kv, p.most_units));
    plan.per_block = wave_first(plan.per_block);
    return plan;
}

// Every wave of a workgroup calls this.
template <int BM>
__device__ __forceinline__ Plan plan_call(const PagedParams &p, PlanSeq &s)
{
    if (__builtin_expect(p.cut != nullptr, 0)) {
        const int2 known = p.cut[0];
        return Plan{__builtin_amdgcn_readfirstlane(known.x), __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(known.y))};
    }
    return plan_cut<BM>(p, WaveScope{p.c.B == 1}, s);
}

// The cut of a batch of many sequences, left in p.cut.
template <int BM, typename Scope>
__device__ __forceinline__ void leave_cut(const PagedParams &p, const Scope &scope)
{
    PlanSeq s;
    const Plan plan = plan_cut<BM>(p, scope, s);
    if (scope.lane() == 0)
        p.cut[0] = int2{plan.total, __builtin_bit_cast(int, plan.per_block)};
    int units = 0, slots = 0;
    for (int b = scope.lane(); b - scope.lane() < p.c.B; b += Scope::kLanes) {
        s = plan_sequence<BM>(p, b);
        const int nr = plan.ranges(s), mine = s.tiles * nr * p.c.H_kv;
        int all, all_slots;
        const int2 before = {units + scope.before(mine, all), slots + scope.before(nr > 1 ? mine : 0, all_slots)};
        if (b < p.c.B)
            p.cut[1 + b] = before;
        units += all, slots += all_slots;
    }
}

template <int BM, bool TREE>
__global__ __launch_bounds__(1024) void attn_paged_plan_kernel(const ParamsOf<TREE> p)
{
    __shared__ int lds[16];
    leave_cut<BM>(p, GroupScope{lds});
}

// Unit `wg` of the call (every wave of a workgroup calls this); false: there is none.  s: plan_sequence of this lane.
template <int BM>
__device__ __forceinline__ bool find_unit(const PagedParams &p, const Plan &plan, PlanSeq s, int wg, Unit &u)
{
    const int lane = threadIdx.x & 63, B = p.c.B;
    if (wg >= plan.total)
        return false;
    // the unit is number w of sequence u.b, which x describes
    PlanSeq x;
    int nr, w;
    auto scalar = [](int &x) { x = __builtin_amdgcn_readfirstlane(x); };
    if (__builtin_expect(p.cut != nullptr, 0)) {
        // the last sequence with no more than wg units before it: 64 of them are compared at a time
        int lo = 0, n = B;
        while (n > 64) {
            const int step = (n + 63) / 64;
            const int below = __popcll(__ballot(lane * step < n && p.cut[1 + lo + min(lane * step, n - 1)].x <= wg));
            if (below == 0)
                return false;
            const int next = (below - 1) * step;
            lo += next;
            n = min(step, n - next);
        }
        const int below = __popcll(__ballot(lane < n && p.cut[1 + lo + min(lane, n - 1)].x <= wg));
        if (below == 0)
            return false;
        u.b = __builtin_amdgcn_readfirstlane(lo + below - 1);
        const int2 before = p.cut[1 + u.b];
        x = plan_sequence<BM>(p, u.b);
        scalar(x.tiles), scalar(x.blocks), scalar(x.n), scalar(x.kv), scalar(x.start);
        nr = __builtin_amdgcn_readfirstlane(plan.ranges(x));
        w = __builtin_amdgcn_readfirstlane(wg - before.x), u.slot0 = __builtin_amdgcn_readfirstlane(before.y);
    } else {
        int units0 = 0, slots0 = 0;
        for (int b = 0;; b += 64) {
            const int ranges = plan.ranges(s);
            const int mine = s.tiles * ranges * p.c.H_kv, kept = ranges > 1 ? mine : 0;
            const int after = units0 + (B == 1 ? mine : wave_prefix(mine)), after_slots = slots0 + (B == 1 ? kept : wave_prefix(kept));
            const unsigned long long behind = __ballot(after > wg);
            if (behind) {
                const int l = __ffsll(behind) - 1;
                auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
                u.b = b + l;
                x = PlanSeq{of(s.tiles), of(s.blocks), of(s.n), of(s.kv), of(s.start)};
                nr = of(ranges), w = wg - of(after - mine), u.slot0 = of(after_slots - kept);
                break;
            }
            if (b + 64 >= B)
                return false;
            units0 = __builtin_amdgcn_readlane(after, 63);
            slots0 = __builtin_amdgcn_readlane(after_slots, 63);
            s = plan_sequence<BM>(p, b + 64 + lane);
        }
    }
    if (w < 0 || w >= x.tiles * nr * p.c.H_kv)             // starts that decrease can count more units than an int holds
        return false;
    u.n = x.n, u.kv = x.kv, u.row0 = x.start;
    u.n_tiles = x.tiles, u.n_ranges = nr;
    const int layer = u.n_tiles * p.c.H_kv;
    u.range = u.n_ranges == 1 ? 0 : quotient(w, layer);
    place_in_layer(w - u.range * layer, p.c.H_kv, u.n_tiles, u.h, u.tile);
    u.slot = u.slot0 + (u.range * p.c.H_kv + u.h) * u.n_tiles + u.tile;
    u.len = (u.n_ranges == 1 ? x.blocks : quotient(x.blocks + u.n_ranges - 1, u.n_ranges)) * kPlanBlock;
    u.n_rows = u.n * p.G;
    u.key0 = min(u.range * u.len, u.kv);
    u.key1 = min(u.key0 + u.len, u.kv);
    // the same in all lanes: scalars from here on
    scalar(u.row0), scalar(u.b), scalar(u.h), scalar(u.tile), scalar(u.range), scalar(u.key0), scalar(u.key1), scalar(u.slot0);
    scalar(u.slot), scalar(u.n), scalar(u.kv), scalar(u.n_rows), scalar(u.n_tiles), scalar(u.n_ranges);
    // starts that decrease can count rows twice: a slot behind the workspace's last is not written
    return u.n_ranges == 1 || (unsigned)u.slot < (unsigned)p.slots;
}

// The first unit of every row tile tells the merge kernel about the tokens whose first row lies in the tile.
template <int BM, int THREADS>
__device__ __forceinline__ void leave_note(const PagedParams &p, const Unit &u)
{
    if (u.range != 0 || u.h != 0 || !p.merge)
        return;
    const int first = p.token_of(u.tile * BM + p.G - 1), behind = min(p.token_of((u.tile + 1) * BM + p.G - 1), u.n);
    for (int i = first + threadIdx.x; i < behind; i += THREADS)
        p.merge[u.row0 + i] = MergeNote{u.slot0, u.n_tiles, u.n_ranges, i * p.G * 2 + p.kernel};
}

// Partial results -> o and lse.  D/4 lanes hold a row (token, query head), four elements each; `walkers` such groups take
// a row's ranges in turn, eight at a time with their loads in flight together, and meet in LDS.  Few rows: a
// workgroup to a row, for the bound is then the latency of the walk.  Many: a workgroup to as many rows as it holds, since
// most of them will have nothing to merge.
template <int D, typename OUT, bool TREE>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(const ParamsOf<TREE> p, int walkers)
{
    constexpr int TPR = D / 4, U = 8;
    __shared__ f32x4 s_acc[256];
    __shared__ f32x2 s_ml[256 / TPR];
    const int group = threadIdx.x / TPR, sub = threadIdx.x % TPR, walker = group & (walkers - 1);
    const int log_walkers = __builtin_ctz(walkers);            // powers of two, both, and T H_q < 2^30
    const int at = (int)blockIdx.x * (256 / TPR >> log_walkers) + (group >> log_walkers);
    const int t = quotient(at, p.H_q), hq = at - t * p.H_q;
    int n_ranges = 0;
    long long slot = 0, step = 0;
    const float *part_o = nullptr, *part_lse = nullptr;
    const bool exists = at < p.c.T * p.H_q;
    const MergeNote note = p.merge[exists ? t : 0];
    // a token of no sequence has no note: what lies there is old
    if (exists && t >= p.c.start_of(0) && t < p.c.start_of(p.c.B)) {
        const bool tiles = note.w & 1;
        const int h = quotient(hq, p.G), row = (note.w >> 1) + hq - h * p.G, n_tiles = note.y;
        const int slots = tiles ? p.parts[1].slots : p.parts[0].slots, BM = tiles ? p.parts[1].BM : p.parts[0].BM;
        part_o = tiles ? p.parts[1].o : p.parts[0].o, part_lse = tiles ? p.parts[1].lse : p.parts[0].lse;
        const int log_bm = __builtin_ctz(BM);
        if (note.z > 1 && note.z <= slots && n_tiles >= 1 && row >= 0 && row >> log_bm < n_tiles && note.x >= 0) {
            step = (long long)p.c.H_kv * n_tiles;
            slot = note.x + (long long)h * n_tiles + (row >> log_bm);
            n_ranges = slot + (note.z - 1) * step < slots ? note.z : 0;
            slot = (slot << log_bm) + (row & (BM - 1));
            step <<= log_bm;
        }
    }
    float m = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = walker; s0 < n_ranges; s0 += U * walkers) {
        float l[U];
        f32x4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long long k = slot + min(s0 + i * walkers, n_ranges - 1) * step;
            l[i] = part_lse[k];
            x[i] = *reinterpret_cast<const f32x4 *>(part_o + k * D + 4 * sub);
        }
        float m_new = m;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (s0 + i * walkers >= n_ranges)
                l[i] = -INFINITY;
            m_new = fmaxf(m_new, l[i]);
        }
        if (m_new == -INFINITY)     // no key of these ranges is visible
            continue;
        const float keep = expf(m - m_new);
        sum *= keep;
        acc *= keep;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (l[i] == -INFINITY)  // its row of partial results was not written
                continue;
            const float w = expf(l[i] - m_new);
            sum += w;
            acc += w * x[i];
        }
        m = m_new;
    }
    if (walkers > 1) {
        s_acc[threadIdx.x] = acc;
        if (sub == 0)
            s_ml[group] = f32x2{m, sum};
        __syncthreads();
        for (int d = walkers / 2; d > 0; d /= 2) {
            if (walker < d) {
                const f32x2 ml = s_ml[group + d];
                const float m_new = fmaxf(m, ml[0]);
                const float a = m == -INFINITY ? 0.f : expf(m - m_new), b = ml[0] == -INFINITY ? 0.f : expf(ml[0] - m_new);
                acc = a * acc + b * s_acc[threadIdx.x + d * TPR];
                sum = a * sum + b * ml[1];
                m = m_new;
                if (d > 1) {
                    s_acc[threadIdx.x] = acc;
                    if (sub == 0)
                        s_ml[group] = f32x2{m, sum};
                }
            }
            if (d > 1)
                __syncthreads();
        }
    }
    if (n_ranges < 1 || walker != 0)
        return;
    acc *= sum > 0.f ? 1.f / sum : 0.f;
    typedef OUT out4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<out4 *>(static_cast<OUT *>(p.o) + (size_t)at * D + 4 * sub) = __builtin_convertvector(acc, out4);
    if (sub == 0)
        p.lse[at] = m + logf(sum);       // -inf where there is no key
}

}  // namespace attn
