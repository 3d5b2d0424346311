// attn_evict.hip -- which places of the paged cache to keep, and moving them together: kernels and entry points
// (include/attn_evict.h).
//
// Select: a workgroup to a sequence and key head.  The keep-th largest weight is found digit by digit (11, 11 and 10 bits of the
// order-preserving integer of a float) from counts in LDS, which no order of additions can change; then every wave
// counts what its stretch of places has to give and take, and after one sum over the waves writes its part of the lists.
//
// Move: a copy of rows; 16 bytes to a lane.  Dropped places before the new end are filled from kept ones behind it, so that as
// little as possible moves and nothing depends on an order: a longer list is as many independent copies.  Short lists,
// whose places may be source and destination at once, are read whole by a workgroup before it writes.
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
};

// Floats in the order of unsigned integers: NaN below everything, the zeros alike.
__device__ __forceinline__ uint32_t rank_of(float x)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, x + 0.f);
    return x != x ? 0u : bits >> 31 ? ~bits : bits | 0x80000000u;
}
constexpr uint32_t kAlways = 0xffffffffu;                   // above the rank of +infinity

typedef __attribute__((ext_vector_type(4))) int i32x4;

// THREADS of a workgroup; HELD: ranks stay in registers from the first reading on, in so many vectors of four to a thread (a list of up to
// THREADS * 4 * HELD places), 0: every pass reads anew, which the L2 serves.
template <int THREADS, int HELD>
struct SelectTiling {
    static constexpr int DIGIT = THREADS == 256 ? 11 : 12;  // bits of the first digit; the second one has half of the rest
    static constexpr int BINS = 1 << DIGIT, WAVES = THREADS / 64;
    static constexpr int STRIDE = THREADS * 4;              // places of a vector of all threads
    static constexpr int SEGMENT = HELD ? STRIDE * HELD : 131072;     // places whose outcome lies in LDS at once, bit by bit
};

template <int THREADS, int HELD>
__global__ __launch_bounds__(THREADS) void attn_select_kernel(const SelectParams p)
{
    typedef SelectTiling<THREADS, HELD> T;
    constexpr int WAVES = T::WAVES;
    __shared__ __attribute__((aligned(16))) int count[T::BINS];
    // of every 256 places four words: bit l of word k is place 4 l + k, kept in any case and as one of the last rank
    __shared__ unsigned long long above[T::SEGMENT / 64], equal[T::SEGMENT / 64];
    __shared__ int of_wave[3][WAVES];
    __shared__ int found[2];                                // digit, how many are to be kept of its elements
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = quotient((int)blockIdx.x, p.H_kv), h = blockIdx.x - b * p.H_kv;
    const int kv = min(max(p.kv_len[b], 0), p.width), keep = min(kv, max(p.keep[b], 0));
    const size_t row = (size_t)b * p.H_kv + h;
    int *const dst = p.dst + row * p.moves, *const src = p.src + row * p.moves;
    const bool whole = min(keep, kv - keep) > p.moves;      // more moves than the lists may hold
    if (h == 0 && tid == 0)
        p.new_len[b] = whole ? kv : keep;
    int at_dst = 0, at_src = 0;
    if (!whole && keep > 0 && keep < kv) {
        const float *const weights = p.weights + row * p.width;
        const int *const stamps = p.stamps ? p.stamps + row * p.width : nullptr;
        const long long late = (long long)(p.stamps ? p.seen[b] : kv) - p.recent;
        // four ranks from place j on (a multiple of four; the rows end on one)
        auto read = [&](int j) -> u32x4 {
            const f32x4 w = *reinterpret_cast<const f32x4 *>(weights + j);
            i32x4 number = {j, j + 1, j + 2, j + 3};
            if (stamps)
                number = *reinterpret_cast<const i32x4 *>(stamps + j);
            u32x4 r;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                r[k] = number[k] < p.sinks || number[k] >= late ? kAlways : rank_of(w[k]);
            return r;
        };
        u32x4 held[HELD ? HELD : 1];
        if constexpr (HELD != 0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i * T::STRIDE < kv) {
                    const int j = i * T::STRIDE + 4 * tid;
                    if (j < kv)
                        held[i] = read(j);
                }
        }
        // f(first place of the lane's four, their ranks) for the places from `from` to `upto`; lanes behind kv take part
        auto each = [&](int from, int upto, auto f) {
            if constexpr (HELD != 0) {
#pragma unroll
                for (int i = 0; i < HELD; ++i)
                    if (i * T::STRIDE < kv)
                        f(i * T::STRIDE + 4 * tid, held[i]);
            } else {
                constexpr int U = 4;
                for (int j0 = from + 4 * tid; j0 - 4 * tid < upto; j0 += U * T::STRIDE) {
                    u32x4 r[U];
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        r[u] = read(min(j0 + u * T::STRIDE, (kv - 1) & ~3));
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (j0 - 4 * tid + u * T::STRIDE < upto)
                            f(j0 + u * T::STRIDE, r[u]);
                }
            }
        };
        // ---- the keep-th largest rank, digit by digit: its leading bits, and how many of those that have them are kept
        uint32_t top = 0;
        int left = keep, shift = 32;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass == 0 ? T::DIGIT : pass == 1 ? (33 - T::DIGIT) / 2 : (32 - T::DIGIT) / 2;
            const uint32_t known = pass == 0 ? 0u : ~0u << shift;
            shift -= bits;
            for (int i = tid; i < T::BINS / 4; i += THREADS)
                reinterpret_cast<i32x4 *>(count)[i] = i32x4{0, 0, 0, 0};
            __syncthreads();
            each(0, kv, [&](int j, u32x4 r) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool mine = j + k < kv && (r[k] & known) == top;
                    const int digit = r[k] >> shift & ((1 << bits) - 1);
                    // the first lane counts for all that have its digit: one value may be everywhere
                    const unsigned long long with = __ballot(mine);
                    if (with == 0)
                        continue;
                    const int lead = __ffsll(with) - 1;
                    const bool same = mine && digit == __builtin_amdgcn_readlane(digit, lead);
                    const unsigned long long all = __ballot(same);
                    if (mine && (!same || lane == lead))
                        atomicAdd(&count[digit], same ? __popcll(all) : 1);
                }
            });
            __syncthreads();
            // from the largest digit down, PER neighbouring ones to a thread
            constexpr int PER = T::BINS / THREADS;
            const int first = T::BINS - (tid + 1) * PER;
            int mine = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                mine += count[first + i];
            const int upto = wave_prefix(mine);
            if (lane == 63)
                of_wave[0][wave] = upto;
            __syncthreads();
            int before = upto - mine;
            for (int w = 0; w < wave; ++w)
                before += of_wave[0][w];
            if (before < left && left <= before + mine) {
                int digit = first + PER - 1;
                while (before + count[digit] < left)
                    before += count[digit--];
                found[0] = digit, found[1] = left - before;
            }
            __syncthreads();
            top |= (uint32_t)found[0] << shift;
            left = found[1];
            __syncthreads();                                // (before anything of it is written again)
        }
        // ---- kept: above `top`, and the first `left` of those that equal it; a segment at a time
        for (int seg = 0; seg < kv; seg += T::SEGMENT) {
            const int n = min(kv - seg, T::SEGMENT), blocks = (n + 255) / 256;
            each(seg, seg + n, [&](int j, u32x4 r) {
                const int at = (j - seg) / 256 * 4;         // (a wave's 256 places are a block)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned long long more = __ballot(j + k < kv && r[k] > top), same = __ballot(j + k < kv && r[k] == top);
                    if (lane == k && at < 4 * blocks)
                        above[at + k] = more, equal[at + k] = same;
                }
            });
            __syncthreads();
            // a wave has a stretch of blocks
            const int stretch = (blocks + WAVES - 1) / WAVES;
            const int first = min(wave * stretch, blocks), behind = min(first + stretch, blocks);
            auto join = [&](int x, int k, int &all) {       // of the waves before this one, and of all
                if (lane == 0)
                    of_wave[k][wave] = x;
                __syncthreads();
                int s = 0;
                all = 0;
                for (int w = 0; w < WAVES; ++w) {
                    s += w < wave ? of_wave[k][w] : 0;
                    all += of_wave[k][w];
                }
                return s;
            };
            int same = 0, all_same, all_holes, all_movers;
            for (int i = 4 * first + lane; i - lane < 4 * behind; i += 64)
                same += wave_sum(i < 4 * behind ? __popcll(equal[i]) : 0);
            int e = join(same, 0, all_same);
            // what is kept of the last rank joins the others; free places before the end and kept ones behind it are counted
            int holes = 0, movers = 0;
            auto lower = [&](unsigned long long x) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0u)); };
            for (int i = first; i < behind; ++i) {
                unsigned long long m[4], q[4];
                int rank = e;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    m[k] = above[4 * i + k], q[k] = equal[4 * i + k];
                    rank += lower(q[k]);
                    e += __popcll(q[k]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool mine = q[k] >> lane & 1;
                    m[k] |= __ballot(mine && rank < left);
                    rank += mine;
                    if (lane == k)
                        above[4 * i + k] = m[k];
                    const int j = seg + 256 * i + 4 * lane + k;
                    const bool kept = m[k] >> lane & 1;
                    holes += __popcll(__ballot(!kept && j < keep));
                    movers += __popcll(__ballot(kept && j >= keep));
                }
            }
            int d = at_dst + join(holes, 1, all_holes), s = at_src + join(movers, 2, all_movers);
            for (int i = first; i < behind; ++i) {
                const int j = seg + 256 * i + 4 * lane;
                bool hole[4], mover[4];
                int to = d, from = s;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool kept = above[4 * i + k] >> lane & 1;
                    hole[k] = !kept && j + k < keep, mover[k] = kept && j + k >= keep;
                    const unsigned long long x = __ballot(hole[k]), y = __ballot(mover[k]);
                    to += lower(x), from += lower(y);
                    d += __popcll(x), s += __popcll(y);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (hole[k])
                        dst[to++] = j + k;
                    if (mover[k])
                        src[from++] = j + k;
                }
            }
            at_dst += all_holes, at_src += all_movers, left -= min(left, all_same);
            __syncthreads();                                // the segment's words have been read
        }
    }
    for (int i = at_dst + tid; i < p.moves; i += THREADS)
        dst[i] = src[i] = -1;
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

// One list, or 64 elements of a longer one, of a sequence and key head; blockIdx.y: keys or values.  RB: bytes of a row.
template <int RB>
__global__ __launch_bounds__(256) void attn_move_kernel(const MoveParams p, int parts)
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

extern "C" int attn_cache_select(const float *weights, const int *stamps, const int *seen, const int *kv_len, const int *keep,
                                 int *dst, int *src, int *new_len, int sinks, int recent, int B, int H_kv, int width,
                                 int moves_width, void *stream)
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
    if (misaligned(weights, 16) || misaligned(stamps, 16) || misaligned(seen, 4) || misaligned(kv_len, 4) || misaligned(keep, 4) ||
        misaligned(dst, 4) || misaligned(src, 4) || misaligned(new_len, 4))
        return ATTN_ERR_ALIGN;
    attn::SelectParams p;
    p.weights = weights, p.stamps = stamps, p.seen = seen, p.kv_len = kv_len, p.keep = keep;
    p.dst = dst, p.src = src, p.new_len = new_len;
    p.sinks = sinks, p.recent = recent, p.B = B, p.H_kv = H_kv, p.width = width, p.moves = moves_width;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(B * H_kv));
    if (width <= attn::SelectTiling<256, 8>::SEGMENT)
        hipLaunchKernelGGL((attn::attn_select_kernel<256, 8>), grid, dim3(256), 0, st, p);
    else if (width <= attn::SelectTiling<1024, 8>::SEGMENT)
        hipLaunchKernelGGL((attn::attn_select_kernel<1024, 8>), grid, dim3(1024), 0, st, p);
    else
        hipLaunchKernelGGL((attn::attn_select_kernel<1024, 0>), grid, dim3(1024), 0, st, p);
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
