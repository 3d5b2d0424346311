// attn_paged_plan.h -- how a call over the paged cache is cut into units of work, and how partial results are merged.
//
// The host knows the number of rows and sequences, not the lengths, so the workgroups work the cut out for themselves, all of
// them alike, from start and kv_len (a load, a sum over the wave, one more load for every 64 sequences).  A unit
// is (sequence, key head, tile of BM rows, range of keys).  A row is a query head of a token: the G query heads that
// share a key head lie side by side (row = token * G + head in group), so that a key is fetched once for all of them.
//
// All ranges of a call have the same length L, in blocks of 64 keys, whatever the lengths of the sequences: L is what
// lets about `target` units (what the chip holds at once) share all the keys that the call has to walk, so a long
// sequence among short ones is walked by many workgroups.  A sequence of one range is finished by its unit;
// the units of the others leave normalised fp32 rows and their log-sum-exp, which attn_paged_merge_kernel joins.
#pragma once
#include "attn_cache_rows.h"
#include "attn_common.h"

namespace attn {

constexpr int kPlanBlock = 64;          // keys of a block

struct PagedParams {
    CacheParams c;
    const void *q;
    void *o;
    float *lse;
    const void *k, *v;
    const unsigned char *k_scale, *v_scale;
    long long q_st, q_sh;               // strides of q in elements
    int H_q, G;                         // G = H_q / H_kv
    int causal;
    float c_log2;                       // scale * log2(e)
    // units of this kernel: sequences of rows in (rows_above, rows_upto], cut for `target` units
    int rows_above, rows_upto, target, min_range;
    int n_slots;                        // partial results that the workspace holds
    float *part_o;                      // [n_slots][BM][D]
    float *part_lse;                    // [n_slots][BM]
    int4 *merge;                        // [T]: see MergeNote
};

// What the merge kernel needs to know of a token: x = first slot of its sequence, y = row tiles of the sequence,
// z = its ranges, w = first row of the token in its sequence; w < 0 with z = 1: nothing to merge.
typedef int4 MergeNote;

struct Unit {
    int b, h, tile, range, n_ranges, n_tiles;
    int row0, n_rows;                   // start[b], rows of the sequence (tokens * G)
    int n, kv;                          // new tokens, cached positions
    int key0, key1;                     // this range
    int slot0, slot;                    // first slot of the sequence, slot of this unit (n_ranges > 1)
};

__device__ __forceinline__ int wave_sum(int x)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2)
        x += __shfl_xor(x, m, 64);
    return x;
}

__device__ __forceinline__ int wave_prefix(int x)   // inclusive
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int y = __shfl_up(x, m, 64);
        x += lane >= m ? y : 0;
    }
    return x;
}

// Every wave of workgroup `wg` calls this; false: the launch has no unit for it.
template <int BM>
__device__ __forceinline__ bool plan_unit(const PagedParams &p, int wg, Unit &u)
{
    const int lane = threadIdx.x & 63;
    struct Seq {
        int tiles, blocks, n, kv;
    };
    auto sequence = [&](int b) -> Seq {
        Seq s = {0, 0, 0, 0};
        if (b < p.c.B) {
            s.n = p.c.rows_of(b);
            s.kv = p.c.length_of(b);
            const long long rows = (long long)s.n * p.G;
            if (rows > p.rows_above && rows <= p.rows_upto) {
                s.tiles = (int)((rows + BM - 1) / BM);
                s.blocks = s.kv > 0 ? (s.kv - 1) / kPlanBlock + 1 : 1;
            }
        }
        return s;
    };
    const bool one = p.c.B <= 64;
    Seq s = sequence(lane);
    // work of the call, in (row tile, block, key head); more than 2^40 units of it cannot be
    float work = 0.f;
    for (int b = 0;; b += 64) {
        float w = (float)s.tiles * (float)s.blocks;
#pragma unroll
        for (int m = 1; m < 64; m *= 2)
            w += __shfl_xor(w, m, 64);
        work += w;
        if (b + 64 >= p.c.B)
            break;
        s = sequence(b + 64 + lane);
    }
    // (a float is enough: the same one in every workgroup, and the margin of one block covers its rounding)
    const float share = ceilf(work * (float)p.c.H_kv * (1.0f + 0x1p-20f) / (float)p.target);
    const int L = max(p.min_range, (int)fminf(share, 0x1p25f));
    // units and slots in front of every sequence
    auto ranges = [&](const Seq &x) { return x.tiles ? (x.blocks + L - 1) / L : 0; };
    if (!one)
        s = sequence(lane);
    int total = 0;
    if (one) {
        total = wave_sum(s.tiles * ranges(s));
    } else {
        for (int b = 0;; b += 64) {
            total += wave_sum(s.tiles * ranges(s));
            if (b + 64 >= p.c.B)
                break;
            s = sequence(b + 64 + lane);
        }
        s = sequence(lane);
    }
    total *= p.c.H_kv;
    if (wg >= total)
        return false;
    const int v = xcd_remap(wg, total);
    int units0 = 0, slots0 = 0;
    for (int b = 0;; b += 64) {
        const int nr = ranges(s);
        const int mine = s.tiles * nr * p.c.H_kv, held = nr > 1 ? mine : 0;
        const int after = units0 + wave_prefix(mine), after_slots = slots0 + wave_prefix(held);
        const unsigned long long behind = __ballot(after > v);
        if (behind) {
            const int l = __ffsll(behind) - 1;
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
            u.b = b + l;
            u.n = of(s.n), u.kv = of(s.kv);
            u.n_tiles = of(s.tiles), u.n_ranges = of(nr);
            const int w = v - of(after - mine);
            if (w < 0 || w >= of(mine))        // starts that decrease can count more units than an int holds
                return false;
            u.slot0 = of(after_slots - held);
            u.slot = u.slot0 + w;
            u.tile = w % u.n_tiles;
            const int hr = w / u.n_tiles;
            u.h = hr % p.c.H_kv;
            u.range = hr / p.c.H_kv;
            break;
        }
        units0 = __builtin_amdgcn_readlane(after, 63);
        slots0 = __builtin_amdgcn_readlane(after_slots, 63);
        if (b + 64 >= p.c.B)
            return false;
        s = sequence(b + 64 + lane);
    }
    u.row0 = __builtin_amdgcn_readfirstlane(p.c.start_of(u.b));
    u.n_rows = u.n * p.G;
    u.key0 = min((long long)u.range * L * kPlanBlock, (long long)u.kv);
    u.key1 = min((long long)(u.range + 1) * L * kPlanBlock, (long long)u.kv);
    // starts that decrease can count rows twice: a slot behind the workspace's last is not written
    return u.n_ranges == 1 || (unsigned)u.slot < (unsigned)p.n_slots;
}

// The first unit of every row tile tells the merge kernel about the tokens whose first row lies in the tile.
template <int BM, int THREADS>
__device__ __forceinline__ void leave_note(const PagedParams &p, const Unit &u)
{
    if (u.range != 0 || u.h != 0 || !p.merge)
        return;
    const int first = (u.tile * BM + p.G - 1) / p.G, behind = min(((u.tile + 1) * BM + p.G - 1) / p.G, u.n);
    for (int i = first + threadIdx.x; i < behind; i += THREADS)
        p.merge[u.row0 + i] = MergeNote{u.slot0, u.n_tiles, u.n_ranges, u.n_ranges > 1 ? i * p.G : -1};
}

// Partial results -> o and lse.  A workgroup takes 256 / (D / 4) (token, query head) rows; D/4 lanes hold a row, four
// elements each, and walk its ranges four at a time with their loads in flight together.
template <int D, typename OUT>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(const PagedParams p, int BM)
{
    constexpr int TPR = D / 4, U = 4;
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) / TPR;
    const int sub = threadIdx.x % TPR;
    if (at >= (long long)p.c.T * p.H_q)
        return;
    const int t = (int)(at / p.H_q), hq = (int)(at % p.H_q);
    // a token of no sequence has no note: what lies there is old
    if (t < p.c.start_of(0) || t >= p.c.start_of(p.c.B))
        return;
    const MergeNote note = p.merge[t];
    const int n_tiles = note.y, n_ranges = note.z;
    if (n_ranges <= 1 || note.w < 0 || n_tiles < 1)
        return;
    const int row = note.w + hq % p.G, h = hq / p.G;
    const int tile = row / BM, in_tile = row % BM;
    const long long step = (long long)p.c.H_kv * n_tiles;
    const long long slot = note.x + (long long)h * n_tiles + tile;
    if (note.x < 0 || tile >= n_tiles || n_ranges > p.n_slots || slot + (n_ranges - 1) * step >= p.n_slots)
        return;
    float m = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n_ranges; s0 += U) {
        float l[U];
        f32x4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const long long k = (slot + min(s0 + i, n_ranges - 1) * step) * BM + in_tile;
            l[i] = p.part_lse[k];
            x[i] = *reinterpret_cast<const f32x4 *>(p.part_o + k * D + 4 * sub);
        }
        float m_new = m;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (s0 + i >= n_ranges)
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
            const float w = expf(l[i] - m_new);
            sum += w;
            acc += w * x[i];
        }
        m = m_new;
    }
    acc *= sum > 0.f ? 1.f / sum : 0.f;
    typedef OUT out4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<out4 *>(static_cast<OUT *>(p.o) + at * D + 4 * sub) = __builtin_convertvector(acc, out4);
    if (sub == 0)
        p.lse[at] = m + logf(sum);       // -inf where there is no key
}

}  // namespace attn
