// attn_evict.hip -- which places of the paged cache to keep, and moving them together: kernels and entry points
// (include/attn_evict.h).
//
// Select: the keep-th largest weight is found digit by digit (11, 11 and 10 bits of the order-preserving integer of a float) from counts
// in LDS, which no order of additions can change; what a wave has of free and of kept places is then counted, and the lists are written in
// the places' order.  Up to kSelectWhole places a workgroup has a list, its ranks in registers from the first reading on: 512 lists of
// 2176 places in 12 us.  Longer ones are shared out to workgroups, in four launches: a digit's counts of every part, which the next launch
// adds up.  32 lists of 131072 places in 52 us (a workgroup to a list: 150, bound by its vector unit).
//
// Move: a copy of rows; 16 bytes to a lane.  Dropped places before the new end are filled from kept ones behind it, so that as
// little as possible moves and nothing depends on an order: a longer list is as many independent copies.  Short lists,
// whose places may be source and destination at once, are read whole by a workgroup before it writes.  512 lists of 120 rows of 256
// bytes: 63 MB in 14.8 us (4.3 TB/s); registers kept to six waves to a SIMD, with two 24.8 us.
#include <hip/hip_runtime.h>

#include "attn_cache.h"
#include "attn_cache_rows.h"
#include "attn_common.h"
#include "attn_evict.h"
#include "attn_fwd.h"
#include "attn_launch.h"
#include "attn_paged_plan.h"

namespace attn {

struct SelectParams {
    const float *weights;
    const int *stamps, *seen, *kv_len, *keep;
    int *dst, *src, *new_len;
    int sinks, recent, B, H_kv, width, moves;
    // lists in parts: the counts of the digits [lists][parts][kBins] each, then what is known of a list and of its parts
    int parts, part_places;             // of a list at most, of a part (a multiple of kPartChunk)
    int *counts[3];
    int2 *known;                        // [lists]: leading bits of the keep-th largest rank, how many that have them are kept
    int *kept;                          // [lists][parts]: kept ones that are known so far
};

// Floats, by their bits, in the order of unsigned integers: NaN below everything, the zeros alike.
__device__ __forceinline__ uint32_t rank_of(uint32_t x)
{
    const float f = __builtin_bit_cast(float, x) + 0.f;
    const uint32_t bits = __builtin_bit_cast(uint32_t, f);
    return f != f ? 0u : bits ^ ((uint32_t)((int)bits >> 31) | 0x80000000u);
}
constexpr uint32_t kAlways = 0xffffffffu;                   // above the rank of +infinity

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kBins = 2048;
constexpr int digit_bits(int pass) { return pass == 2 ? 10 : 11; }
constexpr int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }

constexpr int kHeld = 8;                // vectors of four ranks that a thread holds
constexpr int kSelectThreads = 512, kSelectWhole = kSelectThreads * 4 * kHeld;     // (256 for lists of up to half of that)
static_assert(kBins == 4 * 512, "a thread of a part has four bins");
constexpr int kPartThreads = 512, kPartChunk = kPartThreads * 4 * kHeld, kMostParts = 64;

// What a workgroup shares.
template <int THREADS>
struct SelectShared {
    __attribute__((aligned(16))) int count[kBins];
    int of_wave[2][THREADS / 64];
    int of_vector[3][kHeld * THREADS / 64];                // of a wave's part of a vector: equal ranks, free places, kept ones behind
    int of_part[2][kMostParts + 2];
    int found[2];
};

// One list, or a part of it, as the threads of a workgroup see it.
template <int THREADS>
struct SelectList {
    static constexpr int WAVES = THREADS / 64, STRIDE = THREADS * 4;
    typedef SelectShared<THREADS> Shared;
    const SelectParams &p;
    Shared &sh;
    const int tid, lane, wave;
    int b, h, kv, keep;
    bool whole;                         // nothing is dropped
    size_t row;
    u32x4 held[kHeld];

    __device__ __forceinline__ SelectList(const SelectParams &p_, Shared &sh_, int list)
        : p(p_), sh(sh_), tid(threadIdx.x), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6))
    {
        b = quotient(list, p.H_kv), h = list - b * p.H_kv;
        kv = min(max(p.kv_len[b], 0), p.width), keep = min(kv, max(p.keep[b], 0));
        row = (size_t)b * p.H_kv + h;
        // (more moves than the lists may hold, or none)
        whole = min(keep, kv - keep) > p.moves || keep == 0 || keep == kv;
    }
    __device__ __forceinline__ int new_len() const { return min(keep, kv - keep) > p.moves ? kv : keep; }

    // Ranks of the places [lo, hi), no more than a vector of four for each of the kHeld turns from lo & ~3 on: asked for (all on their way
    // before the first is looked at; behind hi the last ones once more), and made.  seen: the sequence's, if there are stamps
    i32x4 number[kHeld];
    int seen;
    __device__ __forceinline__ void ask(int lo, int hi)
    {
        const float *const weights = p.weights + row * p.width;
        const int base = (lo & ~3) + 4 * tid, last = (hi - 1) & ~3;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if ((lo & ~3) + i * STRIDE < hi)
                held[i] = *reinterpret_cast<const u32x4 *>(weights + min(base + i * STRIDE, last));
        if (p.stamps) {
            const int *const stamps = p.stamps + row * p.width;
            seen = p.seen[b];
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if ((lo & ~3) + i * STRIDE < hi)
                    number[i] = *reinterpret_cast<const i32x4 *>(stamps + min(base + i * STRIDE, last));
        }
    }
    __device__ __forceinline__ void make(int lo)
    {
        const long long late = (long long)(p.stamps ? seen : kv) - p.recent;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int j = (lo & ~3) + 4 * tid + i * STRIDE, of_wave = __builtin_amdgcn_readfirstlane(j);   // first place of the wave
#pragma unroll
            for (int k = 0; k < 4; ++k)
                held[i][k] = rank_of(held[i][k]);
            if (p.stamps) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    held[i][k] = number[i][k] < p.sinks || number[i][k] >= late ? kAlways : held[i][k];
            } else if (of_wave < p.sinks || of_wave + 255 >= late) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    held[i][k] = j + k < p.sinks || j + k >= late ? kAlways : held[i][k];
            }
        }
    }
    // f(first place of the lane's four, their ranks), lanes behind hi take part
    template <typename F>
    __device__ __forceinline__ void each(int lo, int hi, F f)
    {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if ((lo & ~3) + i * STRIDE < hi)
                f((lo & ~3) + i * STRIDE + 4 * tid, held[i]);
    }
    __device__ __forceinline__ void clear()
    {
        for (int i = tid; i < kBins / 4; i += THREADS)
            reinterpret_cast<i32x4 *>(sh.count)[i] = i32x4{0, 0, 0, 0};
        __syncthreads();
    }
    // counts of a digit among the ranks of [lo, hi) whose bits above it are `top`
    __device__ __forceinline__ void tally(int pass, uint32_t top, int lo, int hi)
    {
        const int shift = digit_shift(pass), bits = digit_bits(pass);
        const uint32_t known = pass == 0 ? 0u : ~0u << (shift + bits);
        each(lo, hi, [&](int j, u32x4 r) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const bool mine = j + k >= lo && j + k < hi && (r[k] & known) == top;
                // (one value everywhere: 64 additions to one place, some 7 us of a part of 16384)
                if (mine)
                    atomicAdd(&sh.count[r[k] >> shift & ((1 << bits) - 1)], 1);
            }
        });
    }
    // x of the waves before this one, and of all
    __device__ __forceinline__ int join(int x, int k, int &all)
    {
        if (lane == 0)
            sh.of_wave[k][wave] = x;
        __syncthreads();
        int s = 0;
        all = 0;
        for (int w = 0; w < WAVES; ++w) {
            s += w < wave ? sh.of_wave[k][w] : 0;
            all += sh.of_wave[k][w];
        }
        return s;
    }
    // the digit in which the left-th largest lies, by the counts; left: how many of its elements are kept
    __device__ __forceinline__ int find(int &left)
    {
        constexpr int PER = kBins / THREADS;                // from the largest digit down, neighbouring ones to a thread
        __syncthreads();
        const int first = kBins - (tid + 1) * PER;
        int mine = 0, all;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            mine += sh.count[first + i];
        const int upto = wave_prefix(mine);
        int before = upto - mine + join(__builtin_amdgcn_readlane(upto, 63), 0, all);
        if (before < left && left <= before + mine) {
            int digit = first + PER - 1;
            while (before + sh.count[digit] < left)
                before += sh.count[digit--];
            sh.found[0] = digit, sh.found[1] = left - before;
        }
        __syncthreads();
        const int digit = sh.found[0];
        left = sh.found[1];
        __syncthreads();                                    // (before anything of it is written again)
        return digit;
    }
    // The lists' elements of the places [lo, hi), whose ranks are held: kept are the ranks above top, and of those that equal it the first
    // `left`.  at_dst, at_src: elements of the places before; all three go on to what follows.  What a wave's part of a vector holds is
    // counted, summed in the order of the places, and written.  all_same: how many equal it, -1 if that is to be counted.
    __device__ __forceinline__ void emit(int lo, int hi, uint32_t top, int all_same, int &left, int &at_dst, int &at_src)
    {
        constexpr int N = kHeld * WAVES;
        static_assert(N <= 64, "a lane to a wave's part of a vector");
        int *const dst = p.dst + row * p.moves, *const src = p.src + row * p.moves;
        auto lower = [](unsigned long long x) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0u)); };
        // x of the parts before part i of this wave (lane i * WAVES + wave has it), and of all
        auto sums = [&](int k, int &all) {
            const int x = lane < N ? sh.of_vector[k][lane] : 0, upto = wave_prefix(x);
            all = __builtin_amdgcn_readlane(upto, 63);
            return upto - x;
        };
        const bool takes = lo < keep, gives = hi > keep;    // (a part of a list has one of the two)
        int before_same = 0;
        if (all_same < 0 || (left > 0 && left < all_same)) {
            int n_same[kHeld] = {};
            each(lo, hi, [&, i = 0](int j, u32x4 r) mutable {
                int n = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    n += __popcll(__ballot(j + k >= lo && j + k < hi && r[k] == top));
                n_same[i++] = n;
            });
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (lane == 0)
                    sh.of_vector[0][i * WAVES + wave] = n_same[i];
            __syncthreads();
            before_same = sums(0, all_same);
        }
        // (all of the last rank, or none: no order among them)
        const bool some = left > 0 && left < all_same;
        uint32_t hole = 0, mover = 0;                       // bit 4 i + k
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            int holes = 0, movers = 0;
            if ((lo & ~3) + i * STRIDE < hi) {
                const int j = (lo & ~3) + i * STRIDE + 4 * tid;
                bool kept[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    kept[k] = held[i][k] > top || (held[i][k] == top && left > 0);
                if (some) {
                    int rank = __builtin_amdgcn_readlane(before_same, i * WAVES + wave);
                    bool same[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        same[k] = j + k >= lo && j + k < hi && held[i][k] == top;
                        rank += lower(__ballot(same[k]));
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        kept[k] = same[k] ? rank < left : kept[k];
                        rank += same[k];
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool there = j + k >= lo && j + k < hi;
                    if (takes) {
                        const bool x = there && !kept[k] && (!gives || j + k < keep);
                        hole |= (uint32_t)x << (4 * i + k);
                        holes += __popcll(__ballot(x));
                    }
                    if (gives) {
                        const bool y = there && kept[k] && (!takes || j + k >= keep);
                        mover |= (uint32_t)y << (4 * i + k);
                        movers += __popcll(__ballot(y));
                    }
                }
            }
            if (lane == 0)
                sh.of_vector[1][i * WAVES + wave] = holes, sh.of_vector[2][i * WAVES + wave] = movers;
        }
        __syncthreads();
        int all_holes, all_movers;
        const int before_holes = sums(1, all_holes), before_movers = sums(2, all_movers);
        auto write = [&](int *list, uint32_t which, int before) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                if (__ballot(which >> (4 * i) & 15) == 0)
                    continue;
                int at = __builtin_amdgcn_readlane(before, i * WAVES + wave);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    at += lower(__ballot(which >> (4 * i + k) & 1));
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (which >> (4 * i + k) & 1)
                        list[at++] = (lo & ~3) + i * STRIDE + 4 * tid + k;
            }
        };
        if (takes)
            write(dst, hole, at_dst + before_holes);
        if (gives)
            write(src, mover, at_src + before_movers);
        at_dst += all_holes, at_src += all_movers, left -= min(left, all_same);
        __syncthreads();                                    // the counts have been read
    }
    // the elements of the lists from n on
    __device__ __forceinline__ void fill(int n, int part, int parts)
    {
        int *const dst = p.dst + row * p.moves, *const src = p.src + row * p.moves;
        for (long long i = (long long)n + part * THREADS + tid; i < p.moves; i += (long long)parts * THREADS)
            dst[i] = src[i] = -1;
    }
};

// A list to a workgroup.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void attn_select_kernel(const SelectParams p)
{
    __shared__ SelectShared<THREADS> sh;
    SelectList<THREADS> l(p, sh, blockIdx.x);
    if (l.h == 0 && l.tid == 0)
        p.new_len[l.b] = l.new_len();
    int at_dst = 0, at_src = 0;
    if (!l.whole) {
        l.ask(0, l.kv);
        l.make(0);
        uint32_t top = 0;
        int left = l.keep;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            l.clear();
            l.tally(pass, top, 0, l.kv);
            top |= (uint32_t)l.find(left) << digit_shift(pass);
        }
        l.emit(0, l.kv, top, -1, left, at_dst, at_src);
    }
    l.fill(at_dst, 0, 1);
}

// The parts of a list: [0, keep) in stretches of part_places, then [keep, kv) in stretches that begin at a multiple of four.
struct SelectPart {
    int below, all;                     // parts before keep, and of the list
    __device__ __forceinline__ SelectPart(const SelectParams &p, int kv, int keep)
    {
        below = (keep + p.part_places - 1) / p.part_places;
        all = below + (kv - (keep & ~3) + p.part_places - 1) / p.part_places;
    }
    __device__ __forceinline__ int lo(const SelectParams &p, int keep, int i) const
    {
        return i < below ? i * p.part_places : max(keep, (keep & ~3) + (i - below) * p.part_places);
    }
    __device__ __forceinline__ int hi(const SelectParams &p, int kv, int keep, int i) const
    {
        return i < below ? min((i + 1) * p.part_places, keep) : min((keep & ~3) + (i - below + 1) * p.part_places, kv);
    }
};

// One of four launches over the parts of the lists.  Launch 0 counts the first digit; 1 and 2 add up the parts' counts of the digit
// before and count the next one; 3 adds up the last ones and writes the lists.
template <int PASS>
__global__ __launch_bounds__(kPartThreads, 4) void attn_select_part_kernel(const SelectParams p)
{
    __shared__ SelectShared<kPartThreads> sh;
    const int list = quotient((int)blockIdx.x, p.parts), part = blockIdx.x - list * p.parts;
    SelectList<kPartThreads> l(p, sh, list);
    if (l.whole) {
        if (PASS == 3) {
            if (l.h == 0 && part == 0 && l.tid == 0)
                p.new_len[l.b] = l.new_len();
            l.fill(0, part, p.parts);
        }
        return;
    }
    const SelectPart parts(p, l.kv, l.keep);
    if (part >= parts.all)
        return;
    const int lo = parts.lo(p, l.keep, part), hi = parts.hi(p, l.kv, l.keep, part);
    uint32_t top = 0;
    int left = l.keep;
    int *const kept = p.kept + (size_t)list * p.parts;
    l.ask(lo, min((lo & ~3) + kPartChunk, hi));             // (on their way while the counts are added up)
    // f(from, upto) with the ranks of those places, a chunk at a time
    auto chunks = [&](auto f) {
        for (int from = lo; from < hi;) {
            const int upto = min((from & ~3) + kPartChunk, hi);
            if (from != lo)
                l.ask(from, upto);
            l.make(from);
            f(from, upto);
            from = upto;
        }
    };
    if constexpr (PASS > 0) {
        if (PASS > 1) {
            const int2 known = p.known[(size_t)(PASS - 2) * gridDim.x / p.parts + list];
            top = (uint32_t)known.x, left = known.y;
        }
        const int *const counts = p.counts[PASS - 1] + (size_t)list * p.parts * kBins;
        for (int i = l.tid; i < kBins / 4; i += kPartThreads) {
            i32x4 sum = {0, 0, 0, 0};
            for (int k0 = 0; k0 < parts.all; k0 += 8) {     // eight rows on their way
                i32x4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    x[k] = *reinterpret_cast<const i32x4 *>(counts + (size_t)min(k0 + k, parts.all - 1) * kBins + 4 * i);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    sum += k0 + k < parts.all ? x[k] : i32x4{0, 0, 0, 0};
            }
            reinterpret_cast<i32x4 *>(sh.count)[i] = sum;
        }
        const int digit = l.find(left);
        top |= (uint32_t)digit << digit_shift(PASS - 1);
        if (PASS < 3) {
            if (part == 0 && l.tid == 0)
                p.known[(size_t)(PASS - 1) * gridDim.x / p.parts + list] = int2{(int)top, left};
            // this part's ranks above the digit are kept
            int more = 0, all;
            const i32x4 own = *reinterpret_cast<const i32x4 *>(counts + (size_t)part * kBins + 4 * l.tid);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                more += 4 * l.tid + j > digit ? own[j] : 0;
            l.join(wave_sum(more), 1, all);
            if (l.tid == 0)
                kept[part] = (PASS > 1 ? kept[part] : 0) + all;
        } else {
            // kept ones of every part: so far, above the last digit, and of those that equal it as many as the parts before leave
            int *const of_part = sh.of_part[0], *const same = sh.of_part[1];
            for (int k = l.wave; k < parts.all; k += kPartThreads / 64) {
                constexpr int N = (1 << digit_bits(2)) / 256;
                i32x4 x[N];
                int more = 0;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[i] = *reinterpret_cast<const i32x4 *>(counts + (size_t)k * kBins + 256 * i + 4 * l.lane);
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        more += 256 * i + 4 * l.lane + j > digit ? x[i][j] : 0;
                more = wave_sum(more);
                if (l.lane == 0)
                    of_part[k] = kept[k] + more, same[k] = counts[(size_t)k * kBins + digit];
            }
            __syncthreads();
            int at_dst = 0, at_src = 0, all = 0, of_last = left;
            for (int k = 0; k < parts.all; ++k) {
                const int taken = min(of_last, same[k]), n = of_part[k] + taken;
                const int holes = k < parts.below ? parts.hi(p, l.kv, l.keep, k) - parts.lo(p, l.keep, k) - n : 0;
                if (k < part)
                    at_dst += holes, at_src += k < parts.below ? 0 : n, left -= taken;
                of_last -= taken, all += holes;
            }
            if (l.h == 0 && part == 0 && l.tid == 0)
                p.new_len[l.b] = l.new_len();
            const int equal = hi - (lo & ~3) <= kPartChunk ? same[part] : -1;
            __syncthreads();
            chunks([&](int from, int upto) { l.emit(from, upto, top, equal, left, at_dst, at_src); });
            l.fill(all, part, parts.all);
            return;
        }
        __syncthreads();                                    // the sums have been read
    }
    l.clear();
    chunks([&](int from, int upto) { l.tally(PASS, top, from, upto); });
    __syncthreads();
    int *const mine = p.counts[PASS < 3 ? PASS : 0] + ((size_t)list * p.parts + part) * kBins;
    for (int i = l.tid; i < kBins / 4; i += kPartThreads)
        reinterpret_cast<i32x4 *>(mine)[i] = reinterpret_cast<const i32x4 *>(sh.count)[i];
}

// Sizes of a call: parts of a list, places of a part, bytes of workspace.
struct SelectSizes {
    int parts, part_places;
    long long bytes;
};
inline SelectSizes select_sizes(int B, int H_kv, int width)
{
    SelectSizes s = {1, kPartChunk, 0};
    if (width > kSelectWhole) {
        const long long chunks = ((long long)width + kPartChunk - 1) / kPartChunk;
        s.part_places = (int)((chunks + kMostParts - 1) / kMostParts * kPartChunk);
        s.parts = (int)(((long long)width + s.part_places - 1) / s.part_places) + 2;      // (both stretches may end in a short one)
        s.bytes = (long long)B * H_kv * ((3LL * kBins + 1) * s.parts * 4 + 2 * (long long)sizeof(int2));
        s.bytes = (s.bytes + 15) / 16 * 16;
    }
    return s;
}

struct MoveParams {
    const int *page_table, *dst, *src;
    unsigned char *pool[2], *scale[2];
    float *weights;
    int *stamps;
    int list_heads, moves, B, H_kv, n_pages, page_log2, table_width;

    // row of the pool (page, h, place) of a place of sequence b; -1: there is none
    __device__ __forceinline__ long long row_of(int b, int h, int place) const
    {
        if (place < 0 || place >> page_log2 >= table_width)
            return -1;
        const int id = page_table[(size_t)b * table_width + (place >> page_log2)];
        return (unsigned)id < (unsigned)n_pages ? (long long)((((size_t)id * H_kv + h) << page_log2) + (place & ((1 << page_log2) - 1))) : -1;
    }
};

constexpr int kMoveTogether = 128;      // elements of a list that are read before any is written

// One list, or kMoveTogether elements of a longer one, of a sequence and key head; blockIdx.y: keys or values.  RB: bytes of a row.
template <int RB>
__global__ __launch_bounds__(256, RB == 512 ? 4 : 6) void attn_move_kernel(const MoveParams p, int parts)
{
    constexpr int LPR = RB / 16, RPP = 256 / LPR, N = kMoveTogether / RPP;    // lanes of a row, rows of a pass, passes
    const int w = blockIdx.y, tid = threadIdx.x;
    const long long list = quotient((long long)blockIdx.x, parts);
    const int part = (int)(blockIdx.x - list * parts);
    const int b = (int)quotient(list, p.H_kv), h = (int)(list - (long long)b * p.H_kv);
    const size_t first = ((size_t)b * p.list_heads + (p.list_heads == 1 ? 0 : h)) * p.moves;
    const int e0 = part * kMoveTogether, n = min(p.moves - e0, kMoveTogether);
    __shared__ long long s_to[kMoveTogether], s_from[kMoveTogether];
    bool any = false;
    if (tid < kMoveTogether) {
        long long to = -1, from = -1;
        int d = -1, s = -1;
        if (tid < n) {
            d = p.dst[first + e0 + tid], s = p.src[first + e0 + tid];
            to = p.row_of(b, h, d), from = p.row_of(b, h, s);
        }
        any = to >= 0 && from >= 0;
        s_to[tid] = any ? to : -1, s_from[tid] = any ? from : -1;
    }
    if (!__syncthreads_or(any))
        return;
    // ---- scales, weights and stamps: one element to a thread
    unsigned char unit = 0;
    float weight = 0.f;
    int stamp = 0;
    const size_t place0 = ((size_t)b * p.H_kv + h) * ((size_t)p.table_width << p.page_log2);
    if (any) {
        if (p.scale[w])
            unit = p.scale[w][s_from[tid]];
        if (w == 0 && p.weights)
            weight = p.weights[place0 + p.src[first + e0 + tid]];
        if (w == 0 && p.stamps)
            stamp = p.stamps[place0 + p.src[first + e0 + tid]];
    }
    // ---- rows
    unsigned char *const pool = p.pool[w];
    const int column = tid % LPR * 16;
    u32x4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long from = s_from[i * RPP + tid / LPR];
        if (from >= 0)
            x[i] = *reinterpret_cast<const u32x4 *>(pool + from * RB + column);
    }
    __syncthreads();                    // all sources have been read
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long to = s_to[i * RPP + tid / LPR];
        if (to >= 0)
            *reinterpret_cast<u32x4 *>(pool + to * RB + column) = x[i];
    }
    if (any) {
        if (p.scale[w])
            p.scale[w][s_to[tid]] = unit;
        if (w == 0 && p.weights)
            p.weights[place0 + p.dst[first + e0 + tid]] = weight;
        if (w == 0 && p.stamps)
            p.stamps[place0 + p.dst[first + e0 + tid]] = stamp;
    }
}

}  // namespace attn

namespace {

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

template <int RB>
int launch_move(const attn::MoveParams &p, hipStream_t st)
{
    const long long parts = ((long long)p.moves + attn::kMoveTogether - 1) / attn::kMoveTogether;
    const long long blocks = parts * p.B * p.H_kv;
    if (blocks > attn::most_workgroups(256))
        return ATTN_ERR_SHAPE;
    hipLaunchKernelGGL((attn::attn_move_kernel<RB>), dim3((unsigned)blocks, 2), dim3(256), 0, st, p, (int)parts);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

}  // namespace

extern "C" long long attn_cache_select_workspace_bytes(int B, int H_kv, int width)
{
    if (B < 1 || H_kv < 1 || width < 1 || width % 16 || width > (1 << 30) || (long long)B * H_kv >= 1 << 22)
        return -1;
    return attn::select_sizes(B, H_kv, width).bytes;
}

extern "C" int attn_cache_select(const float *weights, const int *stamps, const int *seen, const int *kv_len, const int *keep,
                                 int *dst, int *src, int *new_len, int sinks, int recent, void *workspace, long long workspace_bytes,
                                 int B, int H_kv, int width, int moves_width, void *stream)
{
    if (!weights || !kv_len || !keep || !dst || !src || !new_len || !stamps != !seen)
        return ATTN_ERR_NULL;
    if (B < 1 || H_kv < 1 || width < 1 || width % 16 || width > (1 << 30) || moves_width < 1 || sinks < 0 || recent < 0 ||
        (long long)B * H_kv >= 1 << 22)
        return ATTN_ERR_SHAPE;
    const long long longer = width > moves_width ? width : moves_width;
    if ((long long)B * H_kv > (1LL << 40) / longer)
        return ATTN_ERR_SHAPE;
    for (const int *p : {kv_len, keep, seen})
        if (p && (uintptr_t)new_len < (uintptr_t)(p + B) && (uintptr_t)p < (uintptr_t)(new_len + B))
            return ATTN_ERR_SHAPE;
    const attn::SelectSizes s = attn::select_sizes(B, H_kv, width);
    const long long lists = (long long)B * H_kv, groups = lists * s.parts;
    if (groups > attn::most_workgroups(attn::kPartThreads) || lists > attn::most_workgroups(attn::kSelectThreads))
        return ATTN_ERR_SHAPE;
    if (s.bytes && !workspace)
        return ATTN_ERR_NULL;
    if (misaligned(weights, 16) || misaligned(stamps, 16) || misaligned(seen, 4) || misaligned(kv_len, 4) || misaligned(keep, 4) ||
        misaligned(dst, 4) || misaligned(src, 4) || misaligned(new_len, 4) || (s.bytes && misaligned(workspace, 16)))
        return ATTN_ERR_ALIGN;
    if (workspace_bytes < s.bytes)
        return ATTN_ERR_WORKSPACE;
    attn::SelectParams p;
    p.weights = weights, p.stamps = stamps, p.seen = seen, p.kv_len = kv_len, p.keep = keep;
    p.dst = dst, p.src = src, p.new_len = new_len;
    p.sinks = sinks, p.recent = recent, p.B = B, p.H_kv = H_kv, p.width = width, p.moves = moves_width;
    p.parts = s.parts, p.part_places = s.part_places;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (s.bytes == 0) {
        constexpr int half = attn::kSelectThreads / 2;
        if (width <= attn::kSelectWhole / 2)
            hipLaunchKernelGGL((attn::attn_select_kernel<half>), dim3((unsigned)lists), dim3(half), 0, st, p);
        else
            hipLaunchKernelGGL((attn::attn_select_kernel<attn::kSelectThreads>), dim3((unsigned)lists), dim3(attn::kSelectThreads), 0, st, p);
        return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
    }
    int *const ws = static_cast<int *>(workspace);
    for (int i = 0; i < 3; ++i)
        p.counts[i] = ws + i * groups * attn::kBins;
    p.known = reinterpret_cast<int2 *>(ws + 3 * groups * attn::kBins);
    p.kept = reinterpret_cast<int *>(p.known + 2 * lists);
    const dim3 grid((unsigned)groups), block(attn::kPartThreads);
    hipLaunchKernelGGL((attn::attn_select_part_kernel<0>), grid, block, 0, st, p);
    hipLaunchKernelGGL((attn::attn_select_part_kernel<1>), grid, block, 0, st, p);
    hipLaunchKernelGGL((attn::attn_select_part_kernel<2>), grid, block, 0, st, p);
    hipLaunchKernelGGL((attn::attn_select_part_kernel<3>), grid, block, 0, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

extern "C" int attn_cache_move(void *k_pages, void *v_pages, unsigned char *k_scale, unsigned char *v_scale, const int *page_table,
                               const int *dst, const int *src, int kind, float *weights, int *stamps, int list_heads,
                               int moves_width, int B, int H_kv, int D, int n_pages, int page_size, int table_width, void *stream)
{
    if (!k_pages || !v_pages || !page_table || !dst || !src || (kind == ATTN_CACHE_E4M3 && (!k_scale || !v_scale)))
        return ATTN_ERR_NULL;
    if (B < 1 || H_kv < 1 || n_pages < 1 || table_width < 1 || moves_width < 1 || B > attn::kMostSequences ||
        (list_heads != 1 && list_heads != H_kv))
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    if ((kind != ATTN_CACHE_16BIT && kind != ATTN_CACHE_E4M3) || page_size < 16 || page_size > 256 ||
        (page_size & (page_size - 1)))
        return ATTN_ERR_UNSUPPORTED;
    const long long most = (1LL << 40) / D, width = (long long)table_width * page_size;
    if ((long long)n_pages * H_kv > most / page_size || H_kv > (1 << 24) || width > (1 << 30) ||
        (long long)B * H_kv > (1LL << 40) / (width > moves_width ? width : moves_width))
        return ATTN_ERR_SHAPE;
    if (misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(page_table, 4) || misaligned(dst, 4) || misaligned(src, 4) ||
        misaligned(weights, 4) || misaligned(stamps, 4) ||
        (kind == ATTN_CACHE_E4M3 && (misaligned(k_scale, 16) || misaligned(v_scale, 16))))
        return ATTN_ERR_ALIGN;
    attn::MoveParams p;
    const bool e4m3 = kind == ATTN_CACHE_E4M3;
    p.page_table = page_table, p.dst = dst, p.src = src;
    p.pool[0] = static_cast<unsigned char *>(k_pages), p.pool[1] = static_cast<unsigned char *>(v_pages);
    p.scale[0] = e4m3 ? k_scale : nullptr, p.scale[1] = e4m3 ? v_scale : nullptr;
    p.weights = weights, p.stamps = stamps;
    p.list_heads = list_heads, p.moves = moves_width, p.B = B, p.H_kv = H_kv, p.n_pages = n_pages;
    p.page_log2 = __builtin_ctz((unsigned)page_size), p.table_width = table_width;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (D * (e4m3 ? 1 : 2)) {
    case 64: return launch_move<64>(p, st);
    case 128: return launch_move<128>(p, st);
    case 256: return launch_move<256>(p, st);
    default: return launch_move<512>(p, st);
    }
}
