// attn_paged.hip -- entry points of the attention over the paged cache (include/attn_cache.h).
#include <hip/hip_runtime.h>

#include <math.h>

#include "attn_cache.h"
#include "attn_fwd.h"
#include "attn_paged_rows.h"

namespace attn {

// What the chip holds at once: two workgroups of the row kernel on each of 256 compute units.
constexpr int kRowTarget = 512;
// A range of fewer keys than this costs more to merge than its walk by other workgroups saves.
constexpr int kRowMinRange = 2;                        // blocks of kPlanBlock keys

constexpr long long kSlack = 64;                       // units and slots that rounding can add

// 16-row tiles of a workgroup: as few as hold a sequence's rows, up to what the registers hold
inline int row_tiles(int D, long long rows)
{
    return rows <= 16 ? 1 : rows <= 32 || D == 256 ? 2 : 4;
}

struct Workspace {
    long long slots, part_o, part_lse, merge, bytes;   // offsets in bytes
};

// Any BM the entry point may choose fits: the slots' rows are what it is laid out for.
inline Workspace workspace_of(int T, int D)
{
    constexpr long long kMaxRows = 64;
    Workspace w;
    // a sequence of two ranges or more has at most twice its share of the target's units
    w.slots = 2 * kRowTarget + kSlack;
    w.part_o = 0;
    w.part_lse = w.slots * kMaxRows * D * 4;
    w.merge = w.part_lse + w.slots * kMaxRows * 4;
    w.bytes = w.merge + (long long)T * (long long)sizeof(MergeNote);
    return w;
}

}  // namespace attn

namespace {

using attn::PagedParams;

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

template <int D, int MT, typename E, bool E4M3>
int launch_rows(PagedParams &p, hipStream_t st)
{
    constexpr int BM = 16 * MT;
    // sequences' tiles are at most one more than their rows fill, ranges at most one more than their share of the target
    const long long tiles = (long long)p.c.T * p.G / BM + (p.c.B < p.c.T ? p.c.B : p.c.T);
    const long long grid = tiles * p.c.H_kv + p.target + attn::kSlack;
    if (grid > 0x7fffffffLL)
        return ATTN_ERR_SHAPE;
    hipLaunchKernelGGL((attn::attn_paged_rows_kernel<D, MT, E, E4M3>), dim3((unsigned)grid), dim3(256), 0, st, p);
    if (hipGetLastError() != hipSuccess)
        return ATTN_ERR_LAUNCH;
    // no sequence can be longer than one range: nothing to merge
    if (((long long)p.c.table_width << p.c.page_log2) <= (long long)p.min_range * attn::kPlanBlock)
        return ATTN_OK;
    const long long blocks = ((long long)p.c.T * p.H_q * (D / 4) + 255) / 256;
    if (blocks > 0x7fffffffLL)
        return ATTN_ERR_SHAPE;
    hipLaunchKernelGGL((attn::attn_paged_merge_kernel<D, typename E::t>), dim3((unsigned)blocks), dim3(256), 0, st, p, BM);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <int D, typename E, bool E4M3>
int launch(PagedParams &p, int max_q, hipStream_t st)
{
    p.rows_above = 0, p.rows_upto = 0x7fffffff;
    p.target = attn::kRowTarget, p.min_range = attn::kRowMinRange;
    switch (attn::row_tiles(D, (long long)max_q * p.G)) {
    case 1: return launch_rows<D, 1, E, E4M3>(p, st);
    case 2: return launch_rows<D, 2, E, E4M3>(p, st);
    default:
        if constexpr (D != 256)
            return launch_rows<D, 4, E, E4M3>(p, st);
        return ATTN_ERR_UNSUPPORTED;
    }
}

template <typename E>
int paged_fwd(const void *q, const long long *strides, void *o, float *lse, const void *k_pages, const void *v_pages,
              const unsigned char *k_scale, const unsigned char *v_scale, const int *page_table, const int *start,
              const int *kv_len, int kind, void *workspace, long long workspace_bytes, int max_q, int T, int B, int H_q,
              int H_kv, int D, int n_pages, int page_size, int table_width, int causal, float scale, void *stream)
{
    if (!q || !strides || !o || !lse || !k_pages || !v_pages || !page_table || !start || !kv_len || !workspace ||
        (kind == ATTN_CACHE_E4M3 && (!k_scale || !v_scale)))
        return ATTN_ERR_NULL;
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || n_pages < 1 || table_width < 1 || max_q < 1 || B == 0x7fffffff)
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    if ((kind != ATTN_CACHE_16BIT && kind != ATTN_CACHE_E4M3) || page_size < 16 || page_size > 256 ||
        (page_size & (page_size - 1)))
        return ATTN_ERR_UNSUPPORTED;
    if ((long long)T * H_q > 0x7fffffffLL || (long long)n_pages * H_kv > (1LL << 40) / D / page_size || H_kv > (1 << 24) ||
        (long long)table_width * page_size > (1 << 30))
        return ATTN_ERR_SHAPE;
    for (int i = 0; i < 2; ++i) {
        const long long n = i ? H_q : T;
        if (n > 1 && (strides[i] < 0 || strides[i] % 8 || strides[i] > (1LL << 40) / n))
            return ATTN_ERR_SHAPE;
    }
    if (misaligned(q, 16) || misaligned(o, 16) || misaligned(lse, 4) || misaligned(k_pages, 16) || misaligned(v_pages, 16) ||
        misaligned(workspace, 16) || misaligned(page_table, 4) || misaligned(start, 4) || misaligned(kv_len, 4) ||
        (kind == ATTN_CACHE_E4M3 && (misaligned(k_scale, 16) || misaligned(v_scale, 16))))
        return ATTN_ERR_ALIGN;
    if (!(scale > 0.f) || !(scale < INFINITY))
        return ATTN_ERR_SCALE;
    const attn::Workspace w = attn::workspace_of(T, D);
    if (workspace_bytes < w.bytes)
        return ATTN_ERR_WORKSPACE;
    PagedParams p;
    p.c.page_table = page_table, p.c.start = start, p.c.kv_len = kv_len;
    p.c.T = T, p.c.B = B, p.c.H_kv = H_kv, p.c.n_pages = n_pages, p.c.table_width = table_width;
    p.c.page_log2 = __builtin_ctz((unsigned)page_size);
    p.q = q, p.o = o, p.lse = lse, p.k = k_pages, p.v = v_pages, p.k_scale = k_scale, p.v_scale = v_scale;
    p.q_st = strides[0], p.q_sh = strides[1];
    p.H_q = H_q, p.G = H_q / H_kv;
    p.causal = causal != 0;
    p.c_log2 = (float)((double)scale * 1.44269504088896340736);
    unsigned char *const ws = static_cast<unsigned char *>(workspace);
    p.n_slots = (int)w.slots;
    p.part_o = reinterpret_cast<float *>(ws + w.part_o);
    p.part_lse = reinterpret_cast<float *>(ws + w.part_lse);
    p.merge = reinterpret_cast<attn::MergeNote *>(ws + w.merge);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool e4m3 = kind == ATTN_CACHE_E4M3;
    switch (D) {
    case 64: return e4m3 ? launch<64, E, true>(p, max_q, st) : launch<64, E, false>(p, max_q, st);
    case 128: return e4m3 ? launch<128, E, true>(p, max_q, st) : launch<128, E, false>(p, max_q, st);
    default: return e4m3 ? launch<256, E, true>(p, max_q, st) : launch<256, E, false>(p, max_q, st);
    }
}

}  // namespace

extern "C" long long attn_paged_fwd_workspace_bytes(int T, int B, int H_q, int H_kv, int D)
{
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || (D != 64 && D != 128 && D != 256) ||
        (long long)T * H_q > 0x7fffffffLL)
        return -1;
    return attn::workspace_of(T, D).bytes;
}

extern "C" int attn_paged_fwd(const void *q, const long long *strides, void *o, float *lse, const void *k_pages,
                              const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                              const int *page_table, const int *start, const int *kv_len, int kind, void *workspace,
                              long long workspace_bytes, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages,
                              int page_size, int table_width, int causal, float scale, void *stream)
{
    return paged_fwd<attn::PagedBF16>(q, strides, o, lse, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind,
                                      workspace, workspace_bytes, max_q, T, B, H_q, H_kv, D, n_pages, page_size, table_width,
                                      causal, scale, stream);
}

extern "C" int attn_paged_fwd_f16(const void *q, const long long *strides, void *o, float *lse, const void *k_pages,
                                  const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,
                                  const int *page_table, const int *start, const int *kv_len, int kind, void *workspace,
                                  long long workspace_bytes, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages,
                                  int page_size, int table_width, int causal, float scale, void *stream)
{
    return paged_fwd<attn::PagedF16>(q, strides, o, lse, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind,
                                     workspace, workspace_bytes, max_q, T, B, H_q, H_kv, D, n_pages, page_size, table_width,
                                     causal, scale, stream);
}
