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

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

__global__ __launch_bounds__(kSelectThreads) void attn_select_kernel(const SelectParams p)
{
    __shared__ int count[2048];
    __shared__ int wave_sum_lds[3][kSelectWaves];
    __shared__ int found[2];                                // digit, how many are to be kept of its elements
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = quotient((int)blockIdx.x, p.H_kv), h = blockIdx.x - b * p.H_kv;
    const int kv = min(max(p.kv_len[b], 0), p.width), keep = min(kv, max(p.keep[b], 0));
    const size_t row = (size_t)b * p.H_kv + h;
    int *const dst = p.dst + row * p.moves, *const src = p.src + row * p.moves;
    const bool whole = min(keep, kv - keep) > p.moves;      // more moves than the lists may hold
    if (h == 0 && tid == 0)
        p.new_len[b] = whole ? kv : keep;
    int n_moves = 0;
    if (!whole && keep > 0 && keep < kv) {
        const float *const weights = p.weights + row * p.width;
        const int *const stamps = p.stamps ? p.stamps + row * p.width : nullptr;
        const int seen = p.stamps ? p.seen[b] : kv;
        const long long late = (long long)seen - p.recent;
        auto rank = [&](int j) -> uint32_t {
            const int stamp = stamps ? stamps[j] : j;
            return stamp < p.sinks || stamp >= late ? kAlways : rank_of(weights[j]);
        };
        // ---- the keep-th largest rank: its leading bits, and how many of those that have them are kept
        uint32_t top = 0;
        int left = keep;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            const uint32_t above = pass == 0 ? 0u : ~0u << (shift + bits);    // bits that are known
            for (int i = tid; i < 2048; i += kSelectThreads)
                count[i] = 0;
            __syncthreads();
            for (int j = tid; j < kv; j += kSelectThreads) {
                const uint32_t r = rank(j);
                if ((r & above) == top)
                    atomicAdd(&count[r >> shift & ((1 << bits) - 1)], 1);
            }
            __syncthreads();
            // from the largest digit down: thread t has digits 2047 - 2t and 2046 - 2t
            const int c0 = count[2047 - 2 * tid], c1 = count[2046 - 2 * tid];
            const int upto = wave_prefix(c0 + c1);
            if (lane == 63)
                wave_sum_lds[0][wave] = upto;
            __syncthreads();
            int before = upto - c0 - c1;
            for (int w = 0; w < wave; ++w)
                before += wave_sum_lds[0][w];
            if (before < left && left <= before + c0 + c1) {
                const bool second = left > before + c0;
                found[0] = 2047 - 2 * tid - second;
                found[1] = left - before - (second ? c0 : 0);
            }
            __syncthreads();
            top |= (uint32_t)found[0] << shift;
            left = found[1];
            __syncthreads();
        }
        // ---- kept: above `top`, and the first `left` of those that equal it.  A wave has a stretch of places
        const int stretch = ((kv + kSelectWaves - 1) / kSelectWaves + 63) & ~63;
        const int first = min(wave * stretch, kv), behind = min(first + stretch, kv);
        auto sum_before = [&](int x, int k) {               // of the waves before this one
            if (lane == 0)
                wave_sum_lds[k][wave] = x;
            __syncthreads();
            int s = 0;
            for (int w = 0; w < wave; ++w)
                s += wave_sum_lds[k][w];
            return s;
        };
        int equal = 0;
        for (int j = first; j < behind; j += 64)
            equal += __popcll(__ballot(j + lane < behind && rank(j + lane) == top));
        equal = sum_before(equal, 0);
        const unsigned long long lower = (1ull << lane) - 1;
        auto walk = [&](auto f) {                           // f(place, is a free place before the end, is a kept one behind it)
            int e = equal;
            for (int j = first; j < behind; j += 64) {
                const bool there = j + lane < behind;
                const uint32_t r = there ? rank(j + lane) : 0u;
                const unsigned long long same = __ballot(there && r == top);
                const bool kept = there && (r > top || (r == top && e + __popcll(same & lower) < left));
                e += __popcll(same);
                f(j + lane, there && !kept && j + lane < keep, kept && j + lane >= keep);
            }
        };
        int gives = 0, takes = 0;
        walk([&](int, bool hole, bool mover) {
            takes += __popcll(__ballot(hole));
            gives += __popcll(__ballot(mover));
        });
        int at_dst = sum_before(takes, 1), at_src = sum_before(gives, 2);
        for (int w = 0; w < kSelectWaves; ++w)
            n_moves += wave_sum_lds[1][w];
        walk([&](int j, bool hole, bool mover) {
            const unsigned long long holes = __ballot(hole), movers = __ballot(mover);
            if (hole)
                dst[at_dst + __popcll(holes & lower)] = j;
            if (mover)
                src[at_src + __popcll(movers & lower)] = j;
            at_dst += __popcll(holes), at_src += __popcll(movers);
        });
    }
    for (int i = n_moves + tid; i < p.moves; i += kSelectThreads)
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
    hipLaunchKernelGGL(attn::attn_select_kernel, dim3((unsigned)(B * H_kv)), dim3(attn::kSelectThreads), 0,
                       static_cast<hipStream_t>(stream), p);
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
