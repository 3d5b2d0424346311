// attn_paged.hip -- entry points of the attention over the paged cache (include/attn_cache.h).
#include <hip/hip_runtime.h>

#include <math.h>

#include "attn_cache.h"
#include "attn_fwd.h"
#include "attn_launch.h"
#include "attn_paged_asm.h"
#include "attn_paged_tiles.h"

namespace attn {

// Workgroups that the chip holds at once: on each of 256 compute units two of the e4m3 tile kernel, one of the 16-bit one, and of
// the row kernel what its tiling promises the compiler.  (16 sequences of four drafted tokens and 512 .. 4100
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
constexpr int kSlots = 2 * kTarget + 64;

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

}  // namespace attn

namespace {

using attn::PagedParams;

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// The cut of a batch of many sequences, before the kernel that takes its units.
template <int BM>
int launch_cut(PagedParams &p, hipStream_t st)
{
    p.cut = p.parts[p.kernel].cut;
    if (p.cut)
        hipLaunchKernelGGL((attn::attn_paged_plan_kernel<BM>), dim3(1), dim3(1024), 0, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

// Workgroups that a kernel of tiles of BM rows may have units for: a sequence's tiles are at most one more than its rows
// fill; ranges are one for every tile and head, and the target's (twice that where rows are taken to see half).
long long most_units(const PagedParams &p, int BM)
{
    const long long tiles = (long long)p.c.T * p.G / BM + (p.c.B < p.c.T ? p.c.B : p.c.T);
    const long long blocks = (((long long)p.c.table_width << p.c.page_log2) + attn::kPlanBlock - 1) / attn::kPlanBlock;
    const long long most_ranges = (blocks + p.min_range - 1) / p.min_range;
    const long long units = tiles * p.c.H_kv + (long long)p.target * p.rounds * (p.halve ? 2 : 1) + 64;
    return units < tiles * p.c.H_kv * most_ranges ? units : tiles * p.c.H_kv * most_ranges;
}

template <int D, int MT, typename E, bool E4M3, int NW = 4>
int launch_rows(PagedParams p, int upto, hipStream_t st)
{
    p.kernel = 0, p.slots = p.parts[0].slots, p.rows_above = 0, p.rows_upto = upto;
    p.target = attn::row_slots<D, MT>(), p.rounds = attn::kRowsRounds, p.min_range = attn::kRowsMinRange, p.overhead = attn::kRowsOverhead;
    p.merging = attn::kRowsMerging;
    p.halve = 0;
    if (NW > 4)
        p.rounds = 0;                                      // whole sequences
    const long long grid = most_units(p, 16 * MT);
    if (grid > attn::most_workgroups(NW * 64))
        return ATTN_ERR_SHAPE;
    p.most_units = (int)grid;
    if (const int rc = launch_cut<16 * MT>(p, st))
        return rc;
    constexpr int lds = attn::PagedRowsTiling<D, MT, NW>::LDS_BYTES;
    if (!attn::allow_lds(reinterpret_cast<const void *>(attn::attn_paged_rows_kernel<D, MT, E, E4M3, NW>), lds))
        return ATTN_ERR_LAUNCH;
    hipLaunchKernelGGL((attn::attn_paged_rows_kernel<D, MT, E, E4M3, NW>), dim3((unsigned)grid), dim3(NW * 64), lds, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <int D, typename E, bool E4M3>
int launch_rows(const PagedParams &p, int MT, int upto, hipStream_t st)
{
    if (MT == 1)
        return launch_rows<D, 1, E, E4M3>(p, upto, st);
    if constexpr (D != 256)
        if (MT == 4)
            return launch_rows<D, 4, E, E4M3>(p, upto, st);
    return launch_rows<D, 2, E, E4M3>(p, upto, st);
}

template <int D, typename E, bool E4M3>
int launch_tiles(PagedParams p, int above, hipStream_t st)
{
    p.kernel = 1, p.slots = p.parts[1].slots, p.rows_above = above, p.rows_upto = 0x7fffffff;
    p.rounds = attn::kTilesRounds, p.min_range = attn::kTilesMinRange, p.overhead = attn::kTilesOverhead;
    p.merging = attn::kTilesMerging;
    p.halve = p.causal;
    const void *kern;
    int lds, threads;
    if constexpr (E4M3) {
        typedef attn::PagedTilesTiling<D> T;
        p.target = attn::kTarget;                          // two of its workgroups to a compute unit
        kern = reinterpret_cast<const void *>(attn::attn_paged_tiles_kernel<D, E>);
        lds = T::LDS_BYTES, threads = T::THREADS;
    } else {
        typedef attn::PagedAsmTiling<D> T;
        p.target = attn::kTarget / 2;
        kern = reinterpret_cast<const void *>(attn::attn_paged_asm_kernel<D, std::is_same<E, attn::PagedF16>::value>);
        lds = T::LDS_BYTES, threads = T::THREADS;
    }
    const long long units = most_units(p, p.parts[1].BM), grid = units < p.target ? units : p.target;   // (a multiple of 8 if less)
    if (units > 0x7fffffffLL)
        return ATTN_ERR_SHAPE;
    p.most_units = (int)units;
    if (!attn::allow_lds(kern, lds))
        return ATTN_ERR_LAUNCH;
    if (const int rc = launch_cut<E4M3 ? attn::PagedTilesTiling<D>::BM : attn::PagedAsmTiling<D>::BM>(p, st))
        return rc;
    if constexpr (E4M3)
        hipLaunchKernelGGL((attn::attn_paged_tiles_kernel<D, E>), dim3((unsigned)grid), dim3(threads), lds, st, p);
    else
        hipLaunchKernelGGL((attn::attn_paged_asm_kernel<D, std::is_same<E, attn::PagedF16>::value>), dim3((unsigned)grid),
                           dim3(threads), lds, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <int D, typename E, bool E4M3>
int launch(PagedParams &p, int max_q, hipStream_t st)
{
    // Sequences of few rows and of many may be in one batch; each kernel takes its own.  One launch where max_q, or a
    // single sequence, says that there is one kind (and then for whatever the batch holds).
    const int most = attn::rows_kernel_most(D);
    const long long rows = (long long)(max_q < p.c.T ? max_q : p.c.T) * p.G;
    const bool few = rows <= most, many = !few, both = many && p.c.B > 1;
    const int MT = attn::row_tiles(D, rows < most ? rows : most);
    p.parts[0].BM = 16 * MT, p.parts[1].BM = E4M3 ? attn::PagedTilesTiling<D>::BM : attn::PagedAsmTiling<D>::BM;
    int rc = ATTN_OK;
    // Short sequences, and no more of them than compute units.  (The bound is what the page table can hold.)
    if constexpr (D != 256)
        if (few && MT == 1 && ((long long)p.c.T * p.G / 16 + (p.c.B < p.c.T ? p.c.B : p.c.T)) * p.c.H_kv <= attn::kTarget / 2 &&
            ((long long)p.c.table_width << p.c.page_log2) * D * (E4M3 ? 2 : 4) <= attn::kWholeBytes)
            return launch_rows<D, 1, E, E4M3, attn::kWaves>(p, 0x7fffffff, st);
    // no sequence can be longer than one range: nothing to merge
    static_assert(attn::kRowsMinRange <= attn::kTilesMinRange, "the row kernel's ranges are the shorter ones");
    const int shortest = few || both ? attn::kRowsMinRange : attn::kTilesMinRange;
    const bool merged = ((long long)p.c.table_width << p.c.page_log2) > (long long)shortest * attn::kPlanBlock;
    constexpr int kGroups = 256 / (D / 4);
    const long long o_rows = (long long)p.c.T * p.H_q;
    // eight ranges to a walker, of as many as a sequence may be expected to have: a launch has one for each head and row tile,
    // and what the target leaves (twice that, for batches of uneven lengths)
    const long long most_ranges = ((long long)p.c.table_width << p.c.page_log2) / (shortest * attn::kPlanBlock) + 1;
    const long long tiles = (long long)p.c.T * p.G / p.parts[many].BM + 1;
    const long long alone = (p.c.B > tiles ? p.c.B : tiles) * p.c.H_kv;
    const long long expected = 1 + 2 * attn::kTarget / alone;
    int walkers = 1;
    while (walkers < kGroups && 8 * walkers < expected && 8 * walkers < most_ranges)
        walkers *= 2;
    const long long blocks = (o_rows * walkers + kGroups - 1) / kGroups;
    if (merged && blocks > attn::most_workgroups(256))     // (before anything is launched)
        return ATTN_ERR_SHAPE;
    if (few || both)
        rc = launch_rows<D, E, E4M3>(p, MT, both ? most : 0x7fffffff, st);
    if (rc == ATTN_OK && many)
        rc = launch_tiles<D, E, E4M3>(p, both ? most : 0, st);
    if (rc != ATTN_OK || !merged)
        return rc;
    hipLaunchKernelGGL((attn::attn_paged_merge_kernel<D, typename E::t>), dim3((unsigned)blocks), dim3(256), 0, st, p, walkers);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
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
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || n_pages < 1 || table_width < 1 || max_q < 1 || B > attn::kMostSequences)
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
        (kind == ATTN_CACHE_E4M3 && (misaligned(k_scale, 16) || misaligned(v_scale, 16))))
        return ATTN_ERR_ALIGN;
    if (!(scale > 0.f) || !(scale < INFINITY))
        return ATTN_ERR_SCALE;
    const attn::Workspace w = attn::workspace_of(T, B, H_q / H_kv, D);
    if (workspace_bytes < w.bytes)
        return ATTN_ERR_WORKSPACE;
    PagedParams p;
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
    p.c_log2 = (float)((double)scale * 1.44269504088896340736);
    unsigned char *const ws = static_cast<unsigned char *>(workspace);
    for (int kernel = 0; kernel < 2; ++kernel) {
        p.parts[kernel].o = reinterpret_cast<float *>(ws + w.part_o[kernel]);
        p.parts[kernel].lse = reinterpret_cast<float *>(ws + w.part_lse[kernel]);
        p.parts[kernel].cut = B > attn::kOwnCut ? reinterpret_cast<int2 *>(ws + w.cut[kernel]) : nullptr;
        p.parts[kernel].slots = w.part_o[kernel] == w.part_lse[kernel] ? 0 : attn::kSlots;
    }
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
        (long long)T * H_q > 0x3fffffffLL || B > attn::kMostSequences)
        return -1;
    return attn::workspace_of(T, B, H_q / H_kv, D).bytes;
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
