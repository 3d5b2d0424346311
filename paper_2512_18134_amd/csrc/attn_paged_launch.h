// attn_paged_launch.h -- host side of the attention over the paged cache: which kernels a call takes, its workspace, its checks.
// TREE: the new tokens see each other by a mask (include/attn_tree.h), otherwise by their order.
#pragma once
#include <hip/hip_runtime.h>

#include <math.h>

#include "attn_cache.h"
#include "attn_fwd.h"
#include "attn_launch.h"
#include "attn_paged_asm.h"
#include "attn_paged_tiles.h"

namespace attn {

// Workgroups that the chip holds at once: on each of 256 compute units two of the tile kernel for e4m3 chunks and for trees (three for trees of
// up to 128 rows at D < 256: PagedTilesTiling::PER_CU), one of the scheduled one for 16-bit chunks, and of the row kernel what its tiling
// promises the compiler.  (16 sequences of four drafted tokens and 512 .. 4100
// positions, D = 256: 26.0 us cut for 512, 22.0 for 256.)
constexpr int kTarget = 512;
template <int D, int MT>
constexpr int row_slots()
{
    return kTarget / 2 * PagedRowsTiling<D, MT, 4>::PER_CU;
}
// Cuts that a launch may choose from (PagedParams::rounds).  Four for tiles gain nothing: four sequences of 200 new tokens at 2000
// 62.6 us, with two 59.9; a chunk of 2048 at 32768 823 and 817.
constexpr int kRowsRounds = 1, kTilesRounds = 2;
// what a unit costs besides its keys (the plan, the first loads, the exchange or the write), and a merge, in blocks' time
constexpr int kRowsOverhead = 1, kTilesOverhead = 4, kRowsMerging = 1, kTilesMerging = 12;
// A range of fewer blocks (of kPlanBlock keys) costs more to merge than its walk by another workgroup saves.
constexpr int kRowsMinRange = 2, kTilesMinRange = 4;
// Bytes of K and V of one key head up to which a sequence is walked by one workgroup, of kWaves waves, without a cut and without
// a merge.  One sequence of 8 key heads, D = 128, 500 keys: 9.0 us whole, 9.6 cut; 16 of them 10.0 and 13.2; of twice the
// keys 13.6 whole, 9.9 cut.
constexpr long long kWholeBytes = 1 << 18;
constexpr int kWaves = 8;
// Bytes of K and V, counted for every 16-row tile that reads them, up to which a tree's rows are taken 16 at a time; K and V as many as the table
// can hold.  32 heads over 8, D = 128, us by 16 rows and by what is chosen otherwise: 15 drafts at 1000 in e4m3 (8 MB) 11.7 and 17.0, in 16 bits
// (16 MB) 11.9 and 17.6, at 2000 (33 MB) 12.6 and 16.4; beyond the bound 40 at 1000 (45 MB) 14.8 and 47.7, 15 at 4000 (66 MB) 17.2 and 21.4,
// four of 15 at 1000 (78 MB) 16.5 and 22.4; 16 of 8 at 8000, 16 heads over 4 (786 MB) 83.6 and 58.1.  8 of 6 at 300, 8 heads over 2, D = 256 (12 MB)
// 13.6 and 21.9.
constexpr long long kFewBytes = 32 << 20;
constexpr int kSlots = 2 * kTarget + 64;
// words of 64 bits of a row's mask, at most: as many new tokens as a tree of drafts will not have
constexpr int kMostMaskWords = 1 << 10;

// Sequences up to which every workgroup works the cut out for itself, 64 of them at a time; of more, a launch of its own does,
// which takes some 3 us: 128 sequences of up to 2000 keys 102.8 us each for itself, 107.4 that way; 256 of up to 200 32.2 and
// 28.5; 1024 213 and 103; 4096 2245 and 379.
constexpr int kOwnCut = 128;

// rows of a sequence up to which the row kernel takes it
constexpr int rows_kernel_most(int D) { return D == 256 ? 64 : 128; }
// 16-row tiles of its workgroup: as few as hold the rows
inline int row_tiles(int D, long long rows) { return rows <= 16 ? 1 : rows <= 32 || D == 256 ? 2 : 4; }

struct Workspace {
    long long part_o[2], part_lse[2], merge, cut[2], bytes;   // offsets in bytes
};

// D = 128: 9, 18 or 36 MB for the row kernel, by the tiles that T tokens can need (no max_q asks for taller ones), and 143 MB for
// the tile kernels of calls with more rows than it takes.  How many slots a call uses is up to lengths that the host
// does not see.
inline Workspace workspace_of(int T, int B, int G, int D)
{
    Workspace w;
    long long at = 0;
    const long long most = rows_kernel_most(D), call = (long long)T * G;
    for (int kernel = 0; kernel < 2; ++kernel) {
        const long long rows = kernel ? (D == 256 ? 128 : 256) : 16 * row_tiles(D, call < most ? call : most);
        const long long slots = kernel && call <= most ? 0 : kSlots;
        w.part_o[kernel] = at;
        at += slots * rows * D * 4;
        w.part_lse[kernel] = at;
        at += slots * rows * 4;
    }
    w.merge = at;
    at += (long long)T * (long long)sizeof(MergeNote);
    for (int kernel = 0; kernel < 2; ++kernel) {
        w.cut[kernel] = at;
        at += B > kOwnCut ? (B + 1LL) * (long long)sizeof(int2) : 0;
    }
    w.bytes = at;
    return w;
}

// A call of trees has one kernel at a time: kSlots partial results of the tallest tiles that its rows can ask for.
inline int tree_rows(int D, long long rows) { return rows <= 16 ? 16 : D == 256 || rows <= 128 ? 128 : 256; }
inline Workspace tree_workspace_of(int T, int B, int G, int D)
{
    Workspace w = {};
    w.merge = (long long)kSlots * tree_rows(D, (long long)T * G) * (D + 1) * 4;
    w.cut[0] = w.cut[1] = w.merge + (long long)T * (long long)sizeof(MergeNote);
    w.bytes = w.cut[0] + (B > kOwnCut ? (B + 1LL) * (long long)sizeof(int2) : 0);
    return w;
}

inline bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// The cut of a batch of many sequences, before the kernel that takes its units.
template <int BM, bool TREE>
int launch_cut(ParamsOf<TREE> &p, hipStream_t st)
{
    p.cut = p.parts[p.kernel].cut;
    if (p.cut)
        hipLaunchKernelGGL((attn_paged_plan_kernel<BM, TREE>), dim3(1), dim3(1024), 0, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

// Workgroups that a kernel of tiles of BM rows may have units for: a sequence's tiles are at most one more than its rows
// fill; ranges are one for every tile and head, and the target's (twice that where rows are taken to see half).
inline long long most_units(const PagedParams &p, int BM)
{
    const long long tiles = (long long)p.c.T * p.G / BM + (p.c.B < p.c.T ? p.c.B : p.c.T);
    const long long blocks = (((long long)p.c.table_width << p.c.page_log2) + kPlanBlock - 1) / kPlanBlock;
    const long long most_ranges = (blocks + p.min_range - 1) / p.min_range;
    const long long units = tiles * p.c.H_kv + (long long)p.target * p.rounds * (p.halve ? 2 : 1) + 64;
    return units < tiles * p.c.H_kv * most_ranges ? units : tiles * p.c.H_kv * most_ranges;
}

template <int D, int MT, typename E, bool E4M3, bool TREE, int NW = 4>
int launch_rows(ParamsOf<TREE> p, int upto, hipStream_t st)
{
    p.kernel = 0, p.slots = p.parts[0].slots, p.rows_above = 0, p.rows_upto = upto;
    p.target = row_slots<D, MT>(), p.rounds = kRowsRounds, p.min_range = kRowsMinRange, p.overhead = kRowsOverhead;
    p.merging = kRowsMerging;
    p.halve = 0;
    if (NW > 4)
        p.rounds = 0;                                      // whole sequences
    const long long grid = most_units(p, 16 * MT);
    if (grid > most_workgroups(NW * 64))
        return ATTN_ERR_SHAPE;
    p.most_units = (int)grid;
    if (const int rc = launch_cut<16 * MT, TREE>(p, st))
        return rc;
    constexpr int lds = PagedRowsTiling<D, MT, NW>::LDS_BYTES;
    if (!allow_lds(reinterpret_cast<const void *>(attn_paged_rows_kernel<D, MT, E, E4M3, NW, TREE>), lds))
        return ATTN_ERR_LAUNCH;
    hipLaunchKernelGGL((attn_paged_rows_kernel<D, MT, E, E4M3, NW, TREE>), dim3((unsigned)grid), dim3(NW * 64), lds, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <int D, typename E, bool E4M3, bool TREE>
int launch_rows(const ParamsOf<TREE> &p, int MT, int upto, hipStream_t st)
{
    if (MT == 1)
        return launch_rows<D, 1, E, E4M3, TREE>(p, upto, st);
    if constexpr (D != 256)
        if (MT == 4)
            return launch_rows<D, 4, E, E4M3, TREE>(p, upto, st);
    return launch_rows<D, 2, E, E4M3, TREE>(p, upto, st);
}

// QB (TREE): 32-row blocks of a wave of the tile kernel
template <int D, typename E, bool E4M3, bool TREE, int QB = PagedTilesTiling<D>::QB>
int launch_tiles(ParamsOf<TREE> p, int above, hipStream_t st)
{
    p.kernel = 1, p.slots = p.parts[1].slots, p.rows_above = above, p.rows_upto = 0x7fffffff;
    p.rounds = kTilesRounds, p.min_range = kTilesMinRange, p.overhead = kTilesOverhead;
    p.merging = kTilesMerging;
    p.halve = p.causal;
    const void *kern;
    int lds, threads;
    if constexpr (E4M3 || TREE) {
        typedef PagedTilesTiling<D, QB> T;
        p.target = kTarget / 2 * T::PER_CU;
        kern = reinterpret_cast<const void *>(attn_paged_tiles_kernel<D, E, E4M3, TREE, QB>);
        lds = T::LDS_BYTES, threads = T::THREADS;
    } else {
        typedef PagedAsmTiling<D> T;
        p.target = kTarget / 2;
        kern = reinterpret_cast<const void *>(attn_paged_asm_kernel<D, std::is_same<E, PagedF16>::value>);
        lds = T::LDS_BYTES, threads = T::THREADS;
    }
    const long long units = most_units(p, p.parts[1].BM), grid = units < p.target ? units : p.target;   // (a multiple of 8 if less)
    if (units > 0x7fffffffLL)
        return ATTN_ERR_SHAPE;
    p.most_units = (int)units;
    if (!allow_lds(kern, lds))
        return ATTN_ERR_LAUNCH;
    if constexpr (E4M3 || TREE) {
        if (const int rc = launch_cut<PagedTilesTiling<D, QB>::BM, TREE>(p, st))
            return rc;
        hipLaunchKernelGGL((attn_paged_tiles_kernel<D, E, E4M3, TREE, QB>), dim3((unsigned)grid), dim3(threads), lds, st, p);
    } else {
        if (const int rc = launch_cut<PagedAsmTiling<D>::BM, TREE>(p, st))
            return rc;
        hipLaunchKernelGGL((attn_paged_asm_kernel<D, std::is_same<E, PagedF16>::value>), dim3((unsigned)grid), dim3(threads), lds, st, p);
    }
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

// The merge behind a call's kernels: workgroups, 0 where no sequence can be longer than one range.
struct Merge {
    int walkers;
    long long blocks;
};

// many: the tile kernel's partial results are most of them; shortest: blocks of the shortest range
template <int D>
Merge merge_of(const PagedParams &p, bool many, int shortest)
{
    Merge m = {1, 0};
    if (((long long)p.c.table_width << p.c.page_log2) <= (long long)shortest * kPlanBlock)
        return m;
    constexpr int kGroups = 256 / (D / 4);
    const long long o_rows = (long long)p.c.T * p.H_q;
    // eight ranges to a walker, of as many as a sequence may be expected to have: a launch has one for each head and row tile,
    // and what the target leaves (twice that, for batches of uneven lengths)
    const long long most_ranges = ((long long)p.c.table_width << p.c.page_log2) / (shortest * kPlanBlock) + 1;
    const long long tiles = (long long)p.c.T * p.G / p.parts[many].BM + 1;
    const long long alone = (p.c.B > tiles ? p.c.B : tiles) * p.c.H_kv;
    const long long expected = 1 + 2 * kTarget / alone;
    while (m.walkers < kGroups && 8 * m.walkers < expected && 8 * m.walkers < most_ranges)
        m.walkers *= 2;
    m.blocks = (o_rows * m.walkers + kGroups - 1) / kGroups;
    return m;
}

template <int D, typename E, bool TREE>
int launch_merge(const ParamsOf<TREE> &p, const Merge &m, hipStream_t st)
{
    if (m.blocks)
        hipLaunchKernelGGL((attn_paged_merge_kernel<D, typename E::t, TREE>), dim3((unsigned)m.blocks), dim3(256), 0, st, p, m.walkers);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <int D, typename E, bool E4M3>
int launch(PagedParams &p, int max_q, hipStream_t st)
{
    // Sequences of few rows and of many may be in one batch; each kernel takes its own.  One launch where max_q, or a
    // single sequence, says that there is one kind (and then for whatever the batch holds).
    const int most = rows_kernel_most(D);
    const long long rows = (long long)(max_q < p.c.T ? max_q : p.c.T) * p.G;
    const bool few = rows <= most, many = !few, both = many && p.c.B > 1;
    const int MT = row_tiles(D, rows < most ? rows : most);
    p.parts[0].BM = 16 * MT, p.parts[1].BM = E4M3 ? PagedTilesTiling<D>::BM : PagedAsmTiling<D>::BM;
    int rc = ATTN_OK;
    // Short sequences, and no more of them than compute units.  (The bound is what the page table can hold.)
    if constexpr (D != 256)
        if (few && MT == 1 && ((long long)p.c.T * p.G / 16 + (p.c.B < p.c.T ? p.c.B : p.c.T)) * p.c.H_kv <= kTarget / 2 &&
            ((long long)p.c.table_width << p.c.page_log2) * D * (E4M3 ? 2 : 4) <= kWholeBytes)
            return launch_rows<D, 1, E, E4M3, false, kWaves>(p, 0x7fffffff, st);
    static_assert(kRowsMinRange <= kTilesMinRange, "the row kernel's ranges are the shorter ones");
    const Merge merge = merge_of<D>(p, many, few || both ? kRowsMinRange : kTilesMinRange);
    if (merge.blocks > most_workgroups(256))               // (before anything is launched)
        return ATTN_ERR_SHAPE;
    if (few || both)
        rc = launch_rows<D, E, E4M3, false>(p, MT, both ? most : 0x7fffffff, st);
    if (rc == ATTN_OK && many)
        rc = launch_tiles<D, E, E4M3, false>(p, both ? most : 0, st);
    return rc == ATTN_OK ? launch_merge<D, E, false>(p, merge, st) : rc;
}

// Trees of drafted tokens: few rows of many heads, or some hundreds.  One kernel takes all sequences of a call:
//   * the row kernel by 16 rows where no sequence has more, or where K and V are so small that reading them for every such tile
//     takes no time (kFewBytes)
//   * the row kernel by 32 or 64 rows where no sequence has more: 16 sequences of 8 drafts at 8000, 16 heads over 4, D = 128, 58.1 us
//     and in e4m3 31.5, by the tile kernel 64.4 and 42.7; of 16 drafts 62.5 and 45.1, by tiles 70.5 and 51.8; D = 64 32.2 and 34.3, 36.3 and
//     35.7; at D = 256 8 drafts 65.6 and 82.4 in e4m3, 114.6 and 110.4 in 16 bits.  Long sequences of few heads are the tile kernel's: 27 of 8
//     drafts at 50000, 4 heads over 1, D = 128, 179 us and in e4m3 114, by tiles 133 and 86; of 16 203 and 157, 142 and 102; at D = 64 of 8
//     78 and 43, 73 and 65, of 16 115 and 119, 76 and 71
//   * otherwise the tile kernel, whose waves share a tile of keys, with 32 or 64 rows to a wave.  A wave without rows brings its share
//     of the keys and has nothing else to do, so that a sequence of few rows costs it no more than its stream
template <int D, typename E, bool E4M3>
int launch(TreeParams &p, int max_q, const Workspace &w, hipStream_t st)
{
    const long long rows = (long long)(max_q < p.c.T ? max_q : p.c.T) * p.G;
    const long long tiles16 = (long long)p.c.T * p.G / 16 + (p.c.B < p.c.T ? p.c.B : p.c.T);
    const long long head_bytes = ((long long)p.c.table_width << p.c.page_log2) * D * (E4M3 ? 2 : 4);
    const bool few = rows <= 16 || tiles16 * p.c.H_kv <= kFewBytes / head_bytes;
    if constexpr (D != 256)
        if (few && tiles16 * p.c.H_kv <= kTarget / 2 && head_bytes <= kWholeBytes)
            return launch_rows<D, 1, E, E4M3, true, kWaves>(p, 0x7fffffff, st);
    constexpr int kMid = D != 256 ? 64 : E4M3 ? 32 : 0;
    const bool mid = !few && rows <= kMid, by_rows = few || mid;
    // the kernel has the workspace for itself
    PagedParams::Parts &parts = p.parts[by_rows ? 0 : 1];
    parts.BM = few ? 16 : mid ? 16 * row_tiles(D, rows) : tree_rows(D, rows);
    const long long fit = w.merge / ((long long)parts.BM * (D + 1) * 4);
    parts.slots = (int)(fit < kSlots ? fit : kSlots);
    parts.o = p.parts[0].o;
    parts.lse = parts.o + (long long)parts.slots * parts.BM * D;
    const Merge merge = merge_of<D>(p, !by_rows, by_rows ? kRowsMinRange : kTilesMinRange);
    if (merge.blocks > most_workgroups(256))
        return ATTN_ERR_SHAPE;
    int rc = ATTN_ERR_LAUNCH;
    if (few)
        rc = launch_rows<D, 1, E, E4M3, true>(p, 0x7fffffff, st);
    if constexpr (kMid >= 32)
        if (mid && parts.BM == 32)
            rc = launch_rows<D, 2, E, E4M3, true>(p, 0x7fffffff, st);
    if constexpr (kMid >= 64)
        if (mid && parts.BM == 64)
            rc = launch_rows<D, 4, E, E4M3, true>(p, 0x7fffffff, st);
    if (!by_rows)
        rc = parts.BM == 128 ? launch_tiles<D, E, E4M3, true, 1>(p, 0, st) : launch_tiles<D, E, E4M3, true>(p, 0, st);
    return rc == ATTN_OK ? launch_merge<D, E, true>(p, merge, st) : rc;
}

template <int D, typename E, bool E4M3>
int go(PagedParams &p, int max_q, const Workspace &, hipStream_t st)
{
    return launch<D, E, E4M3>(p, max_q, st);
}
template <int D, typename E, bool E4M3>
int go(TreeParams &p, int max_q, const Workspace &w, hipStream_t st)
{
    return launch<D, E, E4M3>(p, max_q, w, st);
}

// The call of either entry point.  mask: [T][mask_words] words of 64 bits (TREE), otherwise NULL.
template <typename E, bool TREE>
int paged_call(const void *q, const long long *strides, void *o, float *lse, const void *k_pages, const void *v_pages,
              const unsigned char *k_scale, const unsigned char *v_scale, const int *page_table, const int *start,
              const int *kv_len, int kind, void *workspace, long long workspace_bytes, int max_q, int T, int B, int H_q,
              int H_kv, int D, int n_pages, int page_size, int table_width, int causal, const unsigned long long *mask,
              int mask_words, float scale, void *stream)
{
    if (!q || !strides || !o || !lse || !k_pages || !v_pages || !page_table || !start || !kv_len || !workspace ||
        (kind == ATTN_CACHE_E4M3 && (!k_scale || !v_scale)) || (TREE && !mask))
        return ATTN_ERR_NULL;
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || n_pages < 1 || table_width < 1 || max_q < 1 || B > kMostSequences ||
        (TREE && (mask_words < 1 || mask_words > kMostMaskWords)))
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    if ((kind != ATTN_CACHE_16BIT && kind != ATTN_CACHE_E4M3) || page_size < 16 || page_size > 256 ||
        (page_size & (page_size - 1)))
        return ATTN_ERR_UNSUPPORTED;
    if ((long long)T * H_q > 0x3fffffffLL || (long long)n_pages * H_kv > (1LL << 40) / D / page_size || H_kv > (1 << 24) ||
        (long long)table_width * page_size > (1 << 30) || (long long)H_kv * page_size >= (1 << 30) / D)
        return ATTN_ERR_SHAPE;
    for (int i = 0; i < 2; ++i) {
        const long long n = i ? H_q : T;
        if (n > 1 && (strides[i] < 0 || strides[i] % 8 || strides[i] > (1LL << 40) / n))
            return ATTN_ERR_SHAPE;
    }
    if (misaligned(q, 16) || misaligned(o, 16) || misaligned(lse, 4) || misaligned(k_pages, 16) || misaligned(v_pages, 16) ||
        misaligned(workspace, 16) || misaligned(page_table, 4) || misaligned(start, 4) || misaligned(kv_len, 4) ||
        (kind == ATTN_CACHE_E4M3 && (misaligned(k_scale, 16) || misaligned(v_scale, 16))) || (TREE && misaligned(mask, 8)))
        return ATTN_ERR_ALIGN;
    if (!(scale > 0.f) || !(scale < INFINITY))
        return ATTN_ERR_SCALE;
    const Workspace w = TREE ? tree_workspace_of(T, B, H_q / H_kv, D) : workspace_of(T, B, H_q / H_kv, D);
    if (workspace_bytes < w.bytes)
        return ATTN_ERR_WORKSPACE;
    ParamsOf<TREE> p;
    p.c.page_table = page_table, p.c.start = start, p.c.kv_len = kv_len;
    p.c.T = T, p.c.B = B, p.c.H_kv = H_kv, p.c.n_pages = n_pages, p.c.table_width = table_width;
    p.c.page_log2 = __builtin_ctz((unsigned)page_size);
    p.q = q, p.o = o, p.lse = lse, p.k = k_pages, p.v = v_pages, p.k_scale = k_scale, p.v_scale = v_scale;
    p.q_st = strides[0], p.q_sh = strides[1];
    p.H_q = H_q, p.G = H_q / H_kv;
    // see token_of
    int log_g = 0;
    while ((1LL << log_g) < p.G)
        ++log_g;
    p.g_mul = p.G == 1 ? 0 : (uint32_t)(((1ULL << (31 + log_g)) + p.G - 1) / p.G);
    p.g_shift = p.G == 1 ? 0 : log_g - 1;
    p.causal = causal != 0;
    if constexpr (TREE)
        p.mask = reinterpret_cast<const uint32_t *>(mask), p.mask_words = 2 * mask_words;
    p.c_log2 = (float)((double)scale * 1.44269504088896340736);
    unsigned char *const ws = static_cast<unsigned char *>(workspace);
    for (int kernel = 0; kernel < 2; ++kernel) {
        p.parts[kernel].o = reinterpret_cast<float *>(ws + w.part_o[kernel]);
        p.parts[kernel].lse = reinterpret_cast<float *>(ws + w.part_lse[kernel]);
        p.parts[kernel].cut = B > kOwnCut ? reinterpret_cast<int2 *>(ws + w.cut[kernel]) : nullptr;
        p.parts[kernel].slots = w.part_o[kernel] == w.part_lse[kernel] ? 0 : kSlots;
    }
    p.merge = reinterpret_cast<MergeNote *>(ws + w.merge);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool e4m3 = kind == ATTN_CACHE_E4M3;
    switch (D) {
    case 64: return e4m3 ? go<64, E, true>(p, max_q, w, st) : go<64, E, false>(p, max_q, w, st);
    case 128: return e4m3 ? go<128, E, true>(p, max_q, w, st) : go<128, E, false>(p, max_q, w, st);
    default: return e4m3 ? go<256, E, true>(p, max_q, w, st) : go<256, E, false>(p, max_q, w, st);
    }
}

}  // namespace attn
