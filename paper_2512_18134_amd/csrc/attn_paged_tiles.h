// attn_paged_tiles.h -- attention over an e4m3 paged cache for many rows, chunks of prompts, and over both kinds of cache for trees of
// drafted tokens (TREE).
//
// What bounds it is the matrix pipe, and next to it the LDS port and the exponentials.  A workgroup of four waves walks a range
// of keys in tiles of 32, which its waves read from LDS; a wave owns 32 QB rows.  Two workgroups share a compute unit, two
// waves a SIMD: while one takes its softmax the other has products to issue, so that a wave's program can stay in order (S of
// a tile, softmax, O) and its registers hold 64 rows at D = 128 -- an operand read from LDS then feeds two products, with
// one the LDS port would be as busy as the matrix pipe.
//
// Transposed products S^T = K Q^T, O^T = V^T P^T on v_mfma_f32_32x32x16: lane l owns query l % 32 and half g = l / 32 of a
// tile's keys, S^T is the second product's B operand as it stands, V^T comes out of LDS through the transposing read in the
// same order of keys.  The softmax is that of attn_paged_rows.h: a reference that moves only where it lags by more than 8.
//
// A wave brings eight rows of every tile.  They lie in one page, whose number it takes from a register that holds the page
// numbers of 64 tiles.  The rows pass through registers, where they become 16-bit ones once for all waves: e4m3 times a power
// of two is exact in either type.
//
// 2048 new tokens at the end of 32768, 32 heads over 8, D = 128: 1027 to 1146 us by card, 930 to 1040 TFLOP/s, the matrix pipe
// busy in 43 % of the cycles; two sequences of 2048 at the end of 16384, 32 heads over 8, D = 64: 659 us; 2048 at the end of 16384, 16
// heads over 4, D = 256: 611 us.  The scheduled loops of attn_paged_asm.h take 16-bit rows of these in 796, 500 and 429 us on
// the same card as the lower figures: their direct loads cannot convert.
//
// Trees are some tens to some hundreds of rows.  With 32 rows to a wave (QB = 1) three workgroups share a compute unit, and what bounds it is the
// cache again: 32 sequences of up to 8191, up to 96 rows, D = 128, 16 bits, 95 us (4.8 TB/s; the row kernel by 64 rows 130).  16-bit
// tiles come by direct loads, one tile ahead.
#pragma once
#include "attn_dma.h"
#include "attn_paged_rows.h"

namespace attn {

template <typename E>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mfma32<PagedBF16>(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(PagedBF16::x8, a), __builtin_bit_cast(PagedBF16::x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mfma32<PagedF16>(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(PagedF16::x8, a), __builtin_bit_cast(PagedF16::x8, b), c, 0, 0, 0);
}

// QB: 32-row blocks of a wave
template <int D, int QB_ = D == 256 ? 1 : 2>
struct PagedTilesTiling {
    static constexpr int QB = QB_;
    static constexpr int NW = 4, THREADS = NW * 64, BM = NW * QB * 32, BN = 32;
    static constexpr int ROWB = D * 2, TB = BN * ROWB;      // bytes of a tile in LDS
    static constexpr int STAGES = 2;                        // of K and V: tile j is read while j + 1 is written
    // steps of S whose part of Q waits in LDS: 128 registers of O and 64 of Q leave too few for the rest
    static constexpr int QL = D == 64 || (D == 128 && QB == 1) ? 0 : D == 256 ? 4 : 5;
    static constexpr int PER_CU = D < 256 && QB == 1 ? 3 : 2;      // workgroups of a compute unit, for which registers are kept
    static constexpr int Q_BYTES = QL * BM * 32, LDS_BYTES = 2 * STAGES * TB + Q_BYTES;
};

// One unit.  E4M3: the pool's kind.  TREE: the new tokens see each other by the mask.
template <int D, typename E, bool E4M3, bool TREE, int QB>
__device__ __forceinline__ void attn_paged_tiles_unit(const ParamsOf<TREE> &p, const Unit &u, unsigned char *smem)
{
    typedef PagedTilesTiling<D, QB> T;
    constexpr int ROWB = T::ROWB, TB = T::TB, BN = T::BN, ST = T::STAGES;
    constexpr int KS = D / 16, DB = D / 32;
    constexpr int CROWB = D;                                // bytes of a cached row
    // what a lane brings of a wave's eight rows: pieces of 16 bytes of memory (D = 64: 8 bytes)
    constexpr int PB = D == 64 ? 8 : 16;
    constexpr int PPR = CROWB / PB, NP = 8 * PPR / 64;      // pieces of a row, of a lane

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, g = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(ATTN_LDS_PTR(unsigned char))smem;

    // ---- the rows of this lane: last visible key, Q
    const int tile_row = u.tile * T::BM, first_pos = u.kv - u.n;
    int last[QB];
    u32x4 q[QB][KS - T::QL];
    u32x4 *const q_lds = reinterpret_cast<u32x4 *>(smem + 2 * ST * TB) + wave * QB * T::QL * 64 + lane;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = min(tile_row + (wave * QB + b) * 32 + lq, u.n_rows - 1);    // rows behind the last repeat it
        const int i = p.token_of(row), hq = u.h * p.G + row - i * p.G;
        last[b] = p.causal ? first_pos + i : u.kv - 1;
        const typename E::t *src = static_cast<const typename E::t *>(p.q) + (long long)(u.row0 + i) * p.q_st + (long long)hq * p.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(src + 16 * s + 8 * g);
            if (s < KS - T::QL)
                q[b][s] = x;
            else
                q_lds[(b * T::QL + s - (KS - T::QL)) * 64] = x;    // read by this lane alone
        }
    }
    const int low = p.token_of(tile_row), high = p.token_of(min(tile_row + T::BM - 1, u.n_rows - 1));
    const int key1 = __builtin_amdgcn_readfirstlane(p.causal ? min(u.key1, first_pos + high + 1) : u.key1);
    // from here on some row does not see a key
    const int open = __builtin_amdgcn_readfirstlane(TREE ? min(first_pos, u.kv) : p.causal ? min(first_pos + low + 1, u.kv) : u.kv);
    const int n = key1 > u.key0 ? (key1 - u.key0 + BN - 1) / BN : 0;        // tiles

    f32x16 o[QB][DB];
    float mc[QB], l[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        mc[b] = -3.0e38f;                                   // finite: masked scores (-inf) give exactly 0 against it
        l[b] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[b][d][r] = 0.f;
    }

    if (n > 0) {
        // ---- tiles: cache -> LDS.  Rows behind the sequence's last position repeat it (their P is 0, but 0 x NaN is not)
        const int end8 = (u.kv - 1) & ~7;                   // the last eight rows that hold a position
        // Pages of 64 tiles, one tile per lane: of its first and second 16 keys as the table holds them (asked for 64 tiles
        // ahead), then of this wave's eight rows, and which tiles have a page missing (scalar).
        const int *const table = p.c.page_table + (size_t)u.b * p.c.table_width;
        auto ask = [&](int t0, int half) -> int { return table[min(u.key0 + BN * (t0 + lane) + 16 * half, u.kv - 1) >> p.c.page_log2]; };
        constexpr bool AHEAD = D != 256;                    // (D = 256 has no registers for it)
        int next0 = AHEAD ? ask(0, 0) : 0, next1 = AHEAD ? ask(0, 1) : 0, win = 0, win_first = -64;
        unsigned long long missing = 0, missing_before = 0;
        auto advance = [&](int t) {                         // before tile t is located for the first time
            if ((t & 63) == 0 && t < n) {
                if constexpr (!AHEAD)
                    next0 = ask(t, 0), next1 = ask(t, 1);
                win = wave < 2 ? next0 : next1;
                win_first = t;
                missing_before = missing;
                missing = __ballot((unsigned)next0 >= (unsigned)p.c.n_pages || (unsigned)next1 >= (unsigned)p.c.n_pages);
                if constexpr (AHEAD)
                    next0 = ask(t + 64, 0), next1 = ask(t + 64, 1);
            }
        };
        auto any_missing = [&](int t) -> bool { return (t >= win_first ? missing : missing_before) >> (t & 63) & 1; };
        const int page_mask = (1 << p.c.page_log2) - 1;
        // tile t (tiles behind the last repeat it): page of the wave's rows, their first row in the cache, last row of eight
        auto locate = [&](int &t, int &id, size_t &row, int &most) {
            t = min(t, n - 1);
            id = __builtin_amdgcn_readlane(win, t & 63);
            id = (unsigned)id < (unsigned)p.c.n_pages ? id : -1;
            const int pos = min(u.key0 + BN * t + 8 * wave, end8);
            row = p.c.page_row(max(id, 0), u.h) + (pos & page_mask);
            row = (size_t)__builtin_amdgcn_readfirstlane((int)(row >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)row);
            most = min(u.kv - 1 - pos, 7);
        };
        // e4m3: memory -> registers, registers -> LDS
        struct Rows {
            Piece<PB> k[NP], v[NP];
            uint32_t ks[NP], vs[NP];
        };
        Rows x;
        // 16 bits: memory -> LDS, tile t into its stage.  A load takes RPG of the wave's eight rows; lane -> (row, 16-byte chunk), the
        // swizzle of the tile's rows is applied on the global side.  A tile without a page is made of zeros
        constexpr int RPG = 1024 / ROWB;
        auto bring = [&](int t) {
            const uint32_t stage = lds0 + (t % ST) * 2 * TB + 8 * wave * ROWB;
            int id, most;
            size_t row;
            locate(t, id, row, most);
            auto scalar = [](uintptr_t a) {
                return reinterpret_cast<const void *>((uintptr_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 |
                                                      (uint32_t)__builtin_amdgcn_readfirstlane((int)a));
            };
            const void *k = scalar(id < 0 ? (uintptr_t)kPagedZeroRows : (uintptr_t)p.k + row * ROWB);
            const void *v = scalar(id < 0 ? (uintptr_t)kPagedZeroRows : (uintptr_t)p.v + row * ROWB);
            asm volatile("s_nop 4" : "+s"(k), "+s"(v));     // five wait states between the vector unit's write of a scalar and a load
#pragma unroll
            for (int i = 0; i < 8 / RPG; ++i) {
                const int r = i * RPG + lane / (ROWB / 16), ch = lane % (ROWB / 16);
                const uint32_t off = (uint32_t)(min(r, most) * ROWB + ((ch & ~15) | ((ch & 15) ^ swz<D>(8 * wave + r))) * 16);
                dma16(stage + i * 1024, k, off);
                dma16(stage + TB + i * 1024, v, off);
            }
        };
        // (D = 256: places made anew in every tile, as the operands' are below; it has no registers to keep them in)
        auto anew = [](int x) {
            if constexpr (D == 256)
                asm volatile("" : "+v"(x));
            return x;
        };
        auto fetch = [&](int t) {
            const int ln = anew(lane), prow = ln / PPR;     // row of this lane's first piece
            int id, most;
            size_t row;
            locate(t, id, row, most);
            const unsigned char *k = static_cast<const unsigned char *>(p.k) + row * CROWB;
            const unsigned char *v = static_cast<const unsigned char *>(p.v) + row * CROWB;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int r = min(i * (64 / PPR) + prow, most), off = r * CROWB + (ln % PPR) * PB;
                x.k[i].load(k + off);
                x.v[i].load(v + off);
                x.ks[i] = p.k_scale[row + r];
                x.vs[i] = p.v_scale[row + r];
                if (id < 0) {
                    x.vs[i] = 0;
#pragma unroll
                    for (int d = 0; d < PB / 4; ++d)
                        x.v[i].d[d] = 0;
                }
            }
        };
        auto store = [&](int t) {
            const int ln = anew(lane), prow = ln / PPR;
            unsigned char *const k = smem + (t % ST) * 2 * TB, *const v = k + TB;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int r = 8 * wave + i * (64 / PPR) + prow;
                const float ku = unit_of(x.ks[i]), vu = unit_of(x.vs[i]);
#pragma unroll
                for (int e = 0; e < PB / 8; ++e) {
                    const int c = (ln % PPR) * (PB / 8) + e, at = r * ROWB + (((c & ~15) | ((c & 15) ^ swz<D>(r))) * 16);
                    const uint32_t k0 = x.k[i].d[2 * e], k1 = x.k[i].d[2 * e + 1], v0 = x.v[i].d[2 * e], v1 = x.v[i].d[2 * e + 1];
                    *reinterpret_cast<u32x4 *>(k + at) =
                        u32x4{E::template from_e4m3<false>(k0, ku), E::template from_e4m3<true>(k0, ku),
                              E::template from_e4m3<false>(k1, ku), E::template from_e4m3<true>(k1, ku)};
                    *reinterpret_cast<u32x4 *>(v + at) =
                        u32x4{E::template from_e4m3<false>(v0, vu), E::template from_e4m3<true>(v0, vu),
                              E::template from_e4m3<false>(v1, vu), E::template from_e4m3<true>(v1, vu)};
                }
            }
        };
        auto barrier = [] {     // LDS only: loads of later tiles stay in flight
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };

        // ---- operands out of LDS: the chunk index of a step differs from that of step 0 in bits the swizzle leaves to an xor
        uint32_t k0, v0[2];
        k0 = (uint32_t)(lq * ROWB + (((g & ~15) | ((g & 15) ^ swz<D>(lq))) * 16));
        // V^T through ds_read_b64_tr_b16: in a 16-lane block, lane i supplies the 8-byte piece i % 4 of row i / 4 and receives
        // column i of those four rows
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i16 = lane & 15, dh = (lane >> 4) & 1;
            const int row = 4 * g + 8 * h + (i16 >> 2), c = 2 * dh + ((i16 & 3) >> 1);
            v0[h] = (uint32_t)(row * ROWB + ((c ^ swz<D>(row)) * 16) + (i16 & 1) * 8);
        }
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        auto k_operand = [&](int s, uint32_t base) -> u32x4 { return *(ATTN_LDS_PTR(const u32x4))(uintptr_t)((k0 ^ (32 * s)) + base); };
        auto v_operand = [&](int kc, int d, uint32_t base) -> u32x4 {
            struct {
                s16x4 a, b;
            } y = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS_PTR(s16x4))(uintptr_t)((v0[0] ^ (64 * d)) + base + kc * 16 * ROWB)),
                   __builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS_PTR(s16x4))(uintptr_t)((v0[1] ^ (64 * d)) + base + kc * 16 * ROWB))};
            return __builtin_bit_cast(u32x4, y);
        };

        // D = 256: the next rows are asked for once S has left its registers, otherwise first of all
        constexpr bool LATE = D == 256;
        const bool idle = TREE && tile_row + wave * QB * 32 >= u.n_rows;      // (a wave without rows)
        auto tile = [&](int j) {
            if constexpr (TREE)
                if (idle) {
                    if constexpr (E4M3 && LATE)
                        fetch(j + 2);
                    return;
                }
            const uint32_t base = lds0 + (j % ST) * 2 * TB;
            // the offsets of the later steps are made anew in every tile: kept across tiles they take registers from O and Q
            asm volatile("" : "+v"(k0), "+v"(v0[0]), "+v"(v0[1]));
            f32x16 s[QB];
#pragma unroll
            for (int b = 0; b < QB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[b][r] = 0.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const u32x4 a = k_operand(i, base);
#pragma unroll
                for (int b = 0; b < QB; ++b)
                    s[b] = mfma32<E>(a, i < KS - T::QL ? q[b][min(i, KS - T::QL - 1)] : q_lds[(b * T::QL + i - (KS - T::QL)) * 64], s[b]);
            }
            const int j0 = u.key0 + BN * j;
            const bool bad = any_missing(j);
            if (j0 + BN > open || bad) {
                // keys that some row does not see
                int ok = 3;                                 // each 16 keys of the tile: is there a page?
                if (bad)
                    ok = (p.c.page_of(u.b, j0) >= 0) | (p.c.page_of(u.b, min(j0 + 16, u.kv - 1)) >= 0) << 1;
                if constexpr (TREE) {
                    uint32_t there = (ok & 1 ? 0xffffu : 0u) | (ok & 2 ? 0xffff0000u : 0u);
                    if (j0 + BN > u.kv)
                        there &= (1u << (u.kv - j0)) - 1;
#pragma unroll
                    for (int b = 0; b < QB; ++b) {
                        // (the row worked out again: kept across tiles it takes a register that they need)
                        int row = lane;
                        asm volatile("" : "+v"(row));
                        const int i = p.token_of(min(tile_row + (wave * QB + b) * 32 + (row & 31), u.n_rows - 1));
                        const uint32_t seen = (there & seen_in_tree(p.mask + (size_t)(u.row0 + i) * p.mask_words, p.mask_words, first_pos, j0)) >> 4 * (row >> 5);
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (!(seen >> acc_row(r, 0) & 1))
                                s[b][r] = -INFINITY;
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < QB; ++b)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (j0 + acc_row(r, g) > last[b] || !(ok >> (r >> 3) & 1))
                                s[b][r] = -INFINITY;
                }
            }
            u32x4 pt[QB][2];
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                float top = s[b][0];
#pragma unroll
                for (int r = 1; r < 16; ++r)
                    top = fmaxf(top, s[b][r]);
                top *= p.c_log2;
                if (__any(top > mc[b] + 8.f)) {
                    top = fmaxf(fmaxf(top, xor32(top)), mc[b]);
                    const float keep = __builtin_amdgcn_exp2f(mc[b] - top);
                    mc[b] = top;
                    l[b] *= keep;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
                        o[b][d] *= keep;
                }
                float sum = 0.f, sum2 = 0.f;
#pragma unroll
                for (int kc = 0; kc < 2; ++kc)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[b][8 * kc + 2 * i], p.c_log2, -mc[b]));
                        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[b][8 * kc + 2 * i + 1], p.c_log2, -mc[b]));
                        sum += e0, sum2 += e1;
                        pt[b][kc][i] = E::pack(e0, e1);
                    }
                l[b] += sum + sum2;
            }
            if constexpr (E4M3 && LATE)
                fetch(j + 2);
#pragma unroll
            for (int kc = 0; kc < 2; ++kc)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const u32x4 a = v_operand(kc, d, base + TB);
#pragma unroll
                    for (int b = 0; b < QB; ++b)
                        o[b][d] = mfma32<E>(a, pt[b][kc], o[b][d]);
                }
        };

        if constexpr (E4M3) {
            advance(0);
            fetch(0);
            store(0);
            fetch(1);
#pragma clang loop unroll(disable)
            for (int j = 0; j < n; ++j) {
                barrier();                                  // tile j is complete, tile j - 1 has been read
                store(j + 1);
                advance(j + 2);
                if constexpr (!LATE)
                    fetch(j + 2);
                tile(j);
            }
        } else {
            advance(0);
            bring(0);
#pragma clang loop unroll(disable)
            for (int j = 0; j < n; ++j) {
                wait_vmcnt<0>();
                barrier();                                  // tile j is complete, tile j - 1 has been read
                advance(j + 1);
                bring(j + 1);                               // (behind the last tile: that one once more)
                tile(j);
            }
            wait_vmcnt<0>();
        }
    }

    // ---- normalise and write: a lane has 4-element pieces of its row
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int row = tile_row + (wave * QB + b) * 32 + lq;
        const float sum = l[b] + xor32(l[b]);
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        const float lse = sum > 0.f ? (mc[b] + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f : -INFINITY;
        if (row >= u.n_rows)
            continue;
        if (u.n_ranges > 1) {
            const size_t at = (size_t)u.slot * T::BM + row - tile_row;
            if (sum > 0.f)
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<f32x4 *>(p.parts[1].o + at * D + 32 * d + 2 * r + 4 * g) =
                        f32x4{o[b][d][r], o[b][d][r + 1], o[b][d][r + 2], o[b][d][r + 3]} * inv;
            if (g == 0)
                p.parts[1].lse[at] = lse;
        } else {
            const int i = p.token_of(row);
            const size_t at = (size_t)(u.row0 + i) * p.H_q + u.h * p.G + row - i * p.G;
            typename E::t *dst = static_cast<typename E::t *>(p.o) + at * D;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<u32x2 *>(dst + 32 * d + 2 * r + 4 * g) =
                        u32x2{E::pack(o[b][d][r] * inv, o[b][d][r + 1] * inv), E::pack(o[b][d][r + 2] * inv, o[b][d][r + 3] * inv)};
            if (g == 0)
                p.lse[at] = lse;
        }
    }
}

// A workgroup takes every gridDim.x-th unit (attn_paged_asm.h).
template <int D, typename E, bool E4M3, bool TREE, int QB = PagedTilesTiling<D>::QB>
__global__ __launch_bounds__(256, (PagedTilesTiling<D, QB>::PER_CU)) void attn_paged_tiles_kernel(const ParamsOf<TREE> p)
{
    typedef PagedTilesTiling<D, QB> T;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    PlanSeq seq;
    const Plan plan = plan_call<T::BM>(p, seq);
    for (int k = 0; k * (int)gridDim.x < plan.total; ++k) {
        const ParamsOf<TREE> again = params_again<TREE>();
        Unit u;
        if (find_unit<T::BM>(again, plan, seq, unit_of_pass(gridDim.x, k), u)) {
            leave_note<T::BM, T::THREADS>(again, u);
            attn_paged_tiles_unit<D, E, E4M3, TREE, QB>(again, u, smem);
        }
        __syncthreads();                                    // every wave has read its last tile
        seq = plan_sequence<T::BM>(params_again<TREE>(), threadIdx.x & 63);
    }
}

}  // namespace attn
