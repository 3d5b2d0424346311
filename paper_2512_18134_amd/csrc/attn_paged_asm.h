// attn_paged_asm.h -- attention over a 16-bit paged cache for many rows, with the hand-scheduled loops of
// gen_attn_paged_loop.py: the schedule of the dense forward kernels (attn_fwd_asm.h), which keeps the matrix pipe and the
// vector unit busy side by side, with tiles that come from pages.
//
// A workgroup owns BM rows of a (sequence, key head) and walks a range of keys.  This file finds the unit, the rows and
// their limits, starts the stream of tiles, takes S(0), and normalises and writes the results; the loop is one
// inline-asm statement.  The tilings are those of the dense kernels for launches that fill the chip:
//   D = 64    8 waves x 32 rows, 64-key tiles, two waves per SIMD
//   D = 128   4 waves x 64 rows, 32-key tiles, O and Q in AGPRs
//   D = 256   4 waves x 32 rows, 32-key tiles, O and Q in AGPRs
// 2048 new tokens at the end of 32768, 32 heads over 8, D = 128: 1065 GFLOP in 795 to 834 us on most cards, 940 on the slowest,
// 1340 to 1130 TFLOP/s (a large matrix product of the library: 1141), the matrix pipe busy in 79 % of the cycles and the
// clock at its power limit; two sequences of 2048 at 16384, D = 64: 500 us; 2048 at 16384, 16 heads over 4, D = 256: 430 us.  K and V of a head come
// from HBM once and are then read from the L2 of the one XCD that walks the head.  A prompt of 4096 from its start, D = 128:
// 135 us.  Before units of a head were kept on an XCD the first took 1567 us.
// Requires H_kv * page_size * D * 2 < 2^31 (the loop multiplies a page's bytes in 32 bits).
#pragma once
#include "attn_fwd_asm.h"      // U32Vec, F32Vec, element types
#include "attn_paged_rows.h"   // PagedBF16, PagedF16

namespace attn {

template <int D>
struct PagedAsmTiling {
    static constexpr int QB = D == 128 ? 2 : 1, SB = D == 64 ? 2 : 1, NW = D == 64 ? 8 : 4;
    static constexpr int BN = 32 * SB, BM = NW * 32 * QB, THREADS = NW * 64;
    static constexpr int LDS_BYTES = 8 * BN * D * 2;          // K ring [4] and V ring [4]
};

// eight rows of zeros: what a tile without a page is made of
__device__ const u32x4 kPagedZeroRows[8 * 512 / 16] = {};

// One unit.
template <int D, bool F16>
__device__ __forceinline__ void attn_paged_asm_unit(const PagedParams &p, const Unit &u, unsigned char *smem)
{
    typedef typename std::conditional<F16, ElemF16, ElemBF16>::type E;
    typedef typename E::t elem_t;
    typedef typename E::x8 ex8;
    typedef PagedAsmTiling<D> T;
    constexpr int QB = T::QB, SB = T::SB, NW = T::NW, BN = T::BN;
    constexpr int CPR = D / 8, KS = D / 16, DB = D / 32, ROWB = D * 2, TB = BN * ROWB;
    constexpr int NLD = TB / (NW * 1024), RPG = 1024 / ROWB;  // direct loads of a wave, tile and tensor; rows of a load
    constexpr int NQP = 4 * QB * KS / 16;
    static_assert(NLD * RPG == 8, "a wave brings eight rows of a tile");
    constexpr uint32_t KRING = 0, VRING = 4 * TB;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, g = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(ATTN_LDS_PTR(unsigned char))smem;

    // ---- rows and limits
    const int tile_row = u.tile * T::BM, first_pos = u.kv - u.n;
    auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    auto scalar64 = [&](uint64_t x) { return (uint64_t)(uint32_t)scalar((int)(x >> 32)) << 32 | (uint32_t)scalar((int)x); };
    auto sees = [&](int row) { return p.causal ? first_pos + p.token_of(min(row, u.n_rows - 1)) : u.kv - 1; };   // last visible key
    const int key1 = scalar(min(u.key1, sees(tile_row + T::BM - 1) + 1));
    const int n_tiles = scalar(key1 > u.key0 ? (key1 - u.key0 + BN - 1) / BN : 0);

    f32x16 o_acc[QB * DB];
#pragma unroll
    for (int i = 0; i < QB * DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o_acc[i][r] = 0.f;
    typename F32Vec<QB>::type m_ref_v = {}, l_run_v = {};

    if (n_tiles > 0) {
        const int *const page_tab = reinterpret_cast<const int *>(scalar64((uintptr_t)(p.c.page_table + (size_t)u.b * p.c.table_width)));
        const int kv_last = scalar(u.kv - 1), end8 = scalar(kv_last & ~7);
        const int page_log2 = scalar(p.c.page_log2), page_mask = scalar((1 << page_log2) - 1), n_pages = scalar(p.c.n_pages);
        // ---- Q: this lane's rows as MFMA B operand (rows behind the last repeat it)
        ex8 bq[QB][KS];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int row = min(tile_row + (wave * QB + qb) * 32 + lq, u.n_rows - 1);
            const int i = p.token_of(row), hq = u.h * p.G + row - i * p.G;
            const elem_t *src = static_cast<const elem_t *>(p.q) + (long long)(u.row0 + i) * p.q_st + (long long)hq * p.q_sh + 8 * g;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                bq[qb][ks] = *reinterpret_cast<const ex8 *>(src + 16 * ks);
        }

        // ---- where the tiles lie: this wave's eight rows of 64 tiles, one tile per lane
        const int key0 = scalar(u.key0), pos_base = scalar(key0 + 8 * wave);
        const int page_bytes = scalar((p.c.H_kv << page_log2) * ROWB);
        const size_t head = ((size_t)u.h << page_log2) * ROWB;
        const uint64_t k_head = scalar64((uintptr_t)p.k + head), v_head = scalar64((uintptr_t)p.v + head);
        const uint64_t zero_rows = scalar64((uintptr_t)kPagedZeroRows);
        const int first_id = page_tab[min(pos_base + BN * lane, end8) >> page_log2];
        // ---- pages missing in the range?  One answer for the workgroup (its loads leave with those above)
        bool miss = false;
#pragma unroll 4
        for (int i = (u.key0 >> page_log2) + tid; i <= (key1 - 1) >> page_log2; i += T::THREADS)
            miss |= (unsigned)page_tab[i] >= (unsigned)n_pages;
        const int missing = scalar(__syncthreads_or(miss));

        u32x4 page_win;
        {
            const int pos = min(pos_base + BN * lane, end8), id = first_id;
            const bool ok = (unsigned)id < (unsigned)n_pages;
            const size_t at = (size_t)(unsigned)id * (unsigned)page_bytes + (size_t)(pos & page_mask) * ROWB;
            const uint64_t k = ok ? k_head + at : zero_rows;
            const uint64_t v = ok ? v_head + at : zero_rows;
            page_win = u32x4{(uint32_t)k, (uint32_t)(k >> 32), (uint32_t)v, (uint32_t)(v >> 32)};
        }

        // ---- direct loads: lane -> (row of the eight, 16-byte chunk); the swizzle of the tile's rows is applied on the global
        // side (attn_fwd_asm.h), load i has the immediate offset i KB
        typename U32Vec<NLD>::type dma_row_v, dma_choff_v, dma_voff_v;
        uint32_t dma_row[NLD], dma_choff[NLD];
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
            dma_row[i] = RPG * i + lane / CPR;
            const int ch = lane % CPR;
            dma_choff[i] = (uint32_t)(((ch & ~15) | ((ch & 15) ^ swz<D>(8 * wave + (int)dma_row[i]))) * 16);
            U32Vec<NLD>::set(dma_row_v, i, dma_row[i]);
            U32Vec<NLD>::set(dma_choff_v, i, dma_choff[i]);
            U32Vec<NLD>::set(dma_voff_v, i, dma_row[i] * ROWB + dma_choff[i] - i * 1024);
        }
        const uint32_t lds_k_wave = scalar(lds0 + KRING + wave * NLD * 1024), lds_v_wave = scalar(lds0 + VRING + wave * NLD * 1024);
        auto bring = [&](int which, int t) {     // tile t (0 .. 3) of K or V into its stage
            const int most = min(kv_last - min(pos_base + BN * t, end8), 7);
            uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)page_win[2 * which + 1], t) << 32 |
                          (uint32_t)__builtin_amdgcn_readlane((int)page_win[2 * which], t);
            asm volatile("s_nop 4" : "+s"(at));      // five wait states between the vector unit's write of a scalar and a load
#pragma unroll
            for (int i = 0; i < NLD; ++i)
                dma16((which ? lds_v_wave : lds_k_wave) + t * TB + i * 1024, reinterpret_cast<const void *>((uintptr_t)at),
                      (uint32_t)min((int)dma_row[i], most) * ROWB + dma_choff[i]);
        };
        bring(0, 0), bring(0, 1), bring(1, 0), bring(0, 2), bring(0, 3), bring(1, 1);

        // ---- operand addressing inside a tile, as in the dense kernels
        uint32_t koff[KS];
        typename U32Vec<KS>::type koff_v;
        {
            const int sw = swz<D>(lq);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int ch = 2 * ks + g;
                koff[ks] = lds0 + KRING + (uint32_t)(lq * ROWB + (((ch & ~15) | ((ch & 15) ^ sw)) * 16));
                koff_v[ks] = koff[ks];
            }
        }
        typename U32Vec<2 * DB>::type voff_v;
        {
            const int i16 = lane & 15, dh = (lane >> 4) & 1, rho = i16 >> 2, pi = i16 & 3;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int hlf = 0; hlf < 2; ++hlf) {
                    const int row = 4 * g + 8 * hlf + rho, ch = 4 * db + 2 * dh + (pi >> 1);
                    voff_v[2 * db + hlf] = lds0 + VRING +
                        (uint32_t)(row * ROWB + (((ch & ~15) | ((ch & 15) ^ swz<D>(row))) * 16) + (pi & 1) * 8);
                }
        }

        // ---- S(0) = K(0) Q^T
        wait_vmcnt<5 * NLD>();                                // K(0) has landed, the five tiles behind it may be in flight
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        f32x16 s_init[QB * SB];
#pragma unroll
        for (int i = 0; i < QB * SB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s_init[i][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int sb = 0; sb < SB; ++sb) {
                const ex8 a = *(ATTN_LDS_PTR(const ex8))(uintptr_t)(koff[ks] + sb * 32 * ROWB);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    s_init[qb * SB + sb] = E::mfma(a, bq[qb][ks], s_init[qb * SB + sb]);
            }
        typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
        u32x16 q_pack[NQP];
#pragma unroll
        for (int i = 0; i < NQP; ++i) {
            struct Four {
                ex8 a[4];
            } f;
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4)
                f.a[k4] = bq[(4 * i + k4) / KS][(4 * i + k4) % KS];
            q_pack[i] = __builtin_bit_cast(u32x16, f);
        }
        // limits of this lane's rows, relative to the range, minus the lane group's part of the accumulator row
        typename U32Vec<QB>::type thr_base_v;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
            U32Vec<QB>::set(thr_base_v, qb, (uint32_t)(sees(tile_row + (wave * QB + qb) * 32 + lq) - key0 - 4 * g));
        const float c_log2e = p.c_log2;
        const int t_full = scalar((u.kv - key0) / BN);                // tiles below this lie inside the sequence
        const int open = min(sees(tile_row) + 1, u.kv) - key0;   // from here on some row does not see a key
        const int j_mask = scalar(missing ? 0 : max(open, 0) / BN);
        // a wave's last tile: the last its last row sees.  A wave without rows takes one tile and then keeps step
        const int row_w = tile_row + wave * QB * 32;
        const int n_tiles_wave =
            scalar(row_w >= u.n_rows ? 1 : max(1, min(n_tiles, (sees(row_w + QB * 32 - 1) - key0 + BN) / BN)));
        const int skv_m1 = 0;                                 // (of the dense loop's operands, not used by this one)

        if constexpr (D == 64 && !F16) {
#include "generated/attn_loop_paged_d64.inc"
        } else if constexpr (D == 64) {
#include "generated/attn_loop_paged_d64_f16.inc"
        } else if constexpr (D == 128 && !F16) {
#include "generated/attn_loop_paged_d128.inc"
        } else if constexpr (D == 128) {
#include "generated/attn_loop_paged_d128_f16.inc"
        } else if constexpr (!F16) {
#include "generated/attn_loop_paged_d256.inc"
        } else {
#include "generated/attn_loop_paged_d256_f16.inc"
        }
    }

    // ---- normalise and write: a lane has 4-element pieces of its rows
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int row = tile_row + (wave * QB + qb) * 32 + lq;
        const float l_lane = F32Vec<QB>::get(l_run_v, qb), sum = l_lane + xor32(l_lane);
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        const float lse = sum > 0.f ? (F32Vec<QB>::get(m_ref_v, qb) * p.c_log2 + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f
                                    : -INFINITY;
        if (row >= u.n_rows)
            continue;
        if (u.n_ranges > 1) {
            const size_t at = (size_t)u.slot * T::BM + row - tile_row;
            if (sum > 0.f)
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const f32x16 &oa = o_acc[qb * DB + db];
                        *reinterpret_cast<f32x4 *>(p.parts[1].o + at * D + 32 * db + 2 * r + 4 * g) =
                            f32x4{oa[r], oa[r + 1], oa[r + 2], oa[r + 3]} * inv;
                    }
            if (g == 0)
                p.parts[1].lse[at] = lse;
        } else {
            const int i = p.token_of(row);
            const size_t at = (size_t)(u.row0 + i) * p.H_q + u.h * p.G + row - i * p.G;
            elem_t *dst = static_cast<elem_t *>(p.o) + at * D;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x16 &oa = o_acc[qb * DB + db];
                    const f32x4 y = f32x4{oa[r], oa[r + 1], oa[r + 2], oa[r + 3]} * inv;
                    *reinterpret_cast<typename E::x4 *>(dst + 32 * db + 2 * r + 4 * g) = __builtin_convertvector(y, typename E::x4);
                }
            if (g == 0)
                p.lse[at] = lse;
        }
    }
}

// A workgroup takes every gridDim.x-th unit: as many workgroups as run at once, and none that only finds out that there is
// nothing for it (2100 of those took 11 us of a call of 64 tokens over 500 positions).
template <int D, bool F16>
__global__ __launch_bounds__(PagedAsmTiling<D>::THREADS, 1) void attn_paged_asm_kernel(const PagedParams p)
{
    typedef PagedAsmTiling<D> T;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    PlanSeq seq;
    const Plan plan = plan_call<T::BM>(p, seq);
    for (int k = 0; k * (int)gridDim.x < plan.total; ++k) {
        const PagedParams again = params_again();
        Unit u;
        if (find_unit<T::BM>(again, plan, seq, unit_of_pass(gridDim.x, k), u)) {
            leave_note<T::BM, T::THREADS>(again, u);
            attn_paged_asm_unit<D, F16>(again, u, smem);
        }
        __syncthreads();                                      // every wave has left the rings
        seq = plan_sequence<T::BM>(params_again(), threadIdx.x & 63);
    }
}

}  // namespace attn
