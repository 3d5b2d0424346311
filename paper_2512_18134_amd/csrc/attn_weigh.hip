// attn_weigh.hip -- attention weights of new tokens, added up for every cached position: kernel and entry points
// (include/attn_evict.h).
//
// S = K Q^T once more, without a second product: exp(S - lse) summed over a position's column of queries.  Every position belongs
// to one wave, which walks the rows that see it (in small batches of many rows to two waves of a workgroup, which add their halves in LDS):
// sums stay in registers, in a fixed order, and nothing is joined in memory.  For few rows the kernel is a stream of keys; for many the
// matrix pipe and the exponentials bound it.
//
// 64 sequences of up to 8191 positions, one token each, 32 heads over 8, D = 128: 455 MB of keys in 98.5 us (4.8 TB/s with the weights).  2048
// tokens at the end of 16384: 258 GFLOP in 259 to 277 us, 930 to 996 TFLOP/s, at the power limit.  The same 64 sequences over e4m3: 244 MB in 72.4
// us (3.4 TB/s); 8 of 131072, 64 heads over 8: 1149 MB in 320 us (3.6 TB/s).  There a compute unit has 16 waves with 4 KB of keys each on their way,
// in 16 bits 20 with 8 KB.
//
// Products of few rows are v_mfma_f32_16x16x32 as in attn_paged_rows.h: lane l has column c = l % 16 (a row of queries) and group g = l / 16,
// K as A operand as it lies in memory, and S leaves lane (c, g) with keys 4g .. 4g+3 of a 16-key block.  A key's weight is the sum of
// its register over the columns, which the 16 lanes of a group exchange once, at the end.
#include <hip/hip_runtime.h>

#include <math.h>

#include "attn_cache.h"
#include "attn_evict.h"
#include "attn_fwd.h"
#include "attn_launch.h"
#include "attn_paged_tiles.h"

namespace attn {

struct WeighParams {
    CacheParams c;
    const void *q, *k;
    const unsigned char *k_scale;
    const float *lse, *weights;
    float *out;
    int *stamps;
    const int *seen;
    long long q_st, q_sh;               // strides of q in elements
    int H_q, G;
    uint32_t g_mul, g_shift;            // row / G (PagedParams::token_of)
    int causal;
    float c_log2, decay;

    __device__ __forceinline__ int token_of(int row) const
    {
        return G == 1 ? row : (int)((uint32_t)(((uint64_t)(uint32_t)row * g_mul) >> 32) >> g_shift);
    }
};

// Units of a batch in the order of its sequences, 2^log2_keys positions of a key head each: block * H_kv + head, the blocks of all
// sequences that have rows counted through.  A wave asks for ascending units; 64 sequences lie in its lanes.
struct WeighUnits {
    long long before;                   // blocks of the sequences before these 64
    int log2_keys;
    int base, n, kv, start, upto, all;  // first of them; this lane's rows, positions, first row, blocks up to it; blocks of all 64

    __device__ __forceinline__ void load(const CacheParams &c)
    {
        const int b = base + (threadIdx.x & 63);
        n = kv = start = 0;
        if (b < c.B)
            start = c.start_of(b), n = max(c.start_of(b + 1) - start, 0), kv = c.length_of(b);
        upto = wave_prefix(n > 0 ? (kv + (1 << log2_keys) - 1) >> log2_keys : 0);
        all = __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ __forceinline__ void begin(const CacheParams &c, int log2)
    {
        before = 0, base = 0, log2_keys = log2;
        load(c);
    }
    // block `g` of the batch: its sequence and the sequence's rows, and its first position; false: there are no more
    __device__ __forceinline__ bool find(const CacheParams &c, long long g, int &b, int &rows, int &row0, int &length, int &key0)
    {
        while (g >= before + all) {
            if (c.B - base <= 64)
                return false;
            before += all, base += 64;
            load(c);
        }
        const int at = (int)(g - before);
        const int l = __ffsll(__ballot(upto > at)) - 1;
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
        b = base + l, rows = of(n), row0 = of(start), length = of(kv);
        key0 = (at - (l ? __builtin_amdgcn_readlane(upto, max(l - 1, 0)) : 0)) << log2_keys;
        return true;
    }
};

// x summed over the 16 lanes of a group, in all of them
__device__ __forceinline__ float sum16(float x)
{
    auto across = [](float v, auto ctrl) {
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x = across(x, std::integral_constant<int, 0xb1>{});                  // quad_perm 1 0 3 2
    x = across(x, std::integral_constant<int, 0x4e>{});                  // quad_perm 2 3 0 1
    x = across(x, std::integral_constant<int, 0x141>{});                 // row_half_mirror
    return across(x, std::integral_constant<int, 0x140>{});              // row_mirror
}

constexpr int kWeighKeys = 32;          // of a wave
constexpr int kWeighGroups = 1024;      // workgroups of a launch where the runtime cannot say how many the chip holds at once

// Few rows: a wave to 32 keys of a head, and no wave waits for another.  The next unit and its pages are looked up while the
// keys of this one are on their way.
template <int D, typename E, bool E4M3>
__global__ __launch_bounds__(256) void attn_weigh_rows_kernel(const WeighParams p)
{
    constexpr int EB = E4M3 ? 1 : 2, ROWB = D * EB, KL = ROWB / 64, KS = D / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int page_mask = (1 << p.c.page_log2) - 1;
    WeighUnits units;
    units.begin(p.c, __builtin_ctz(4 * kWeighKeys));
    struct Next {
        bool exists;
        int b, n, row0, kv, j0, h, page[2];                 // pages as the table has them, in a lane's register
    };
    long long unit = blockIdx.x;
    auto look_up = [&] {
        Next x;
        const long long block = quotient(unit, p.c.H_kv);
        x.h = (int)(unit - block * p.c.H_kv);
        x.exists = units.find(p.c, block, x.b, x.n, x.row0, x.kv, x.j0);
        unit += gridDim.x;
        if (x.exists) {
            x.j0 += wave * kWeighKeys;
#pragma unroll
            for (int t = 0; t < 2; ++t)
                x.page[t] = p.c.page_table[(size_t)x.b * p.c.table_width + (min(x.j0 + 16 * t, x.kv - 1) >> p.c.page_log2)];
        }
        return x;
    };
    for (Next next = look_up(); next.exists;) {
        if (next.j0 >= next.kv) {                           // (none of the unit's last keys)
            next = look_up();
            continue;
        }
        const int b = next.b, n = next.n, row0 = next.row0, kv = next.kv, j0 = next.j0, h = next.h;
        // ---- this wave's keys, on their way
        bool ok[2];
        Piece<16> x[2][KL];
        uint32_t units_k[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int id = __builtin_amdgcn_readfirstlane(next.page[t]);
            ok[t] = (unsigned)id < (unsigned)p.c.n_pages;
            const size_t row = p.c.page_row(ok[t] ? id : 0, h) + (min(j0 + 16 * t, (kv - 1) & ~15) & page_mask);
            const unsigned char *k = static_cast<const unsigned char *>(p.k) + row * ROWB;
#pragma unroll
            for (int i = 0; i < KL; ++i)
                x[t][i].load(k + c * ROWB + g * 16 + i * 64);
            if (E4M3)
                units_k[t] = p.k_scale[row + c];
        }
        // ---- and what they have: four to a group of lanes
        const size_t at0 = ((size_t)b * p.c.H_kv + h) * ((size_t)p.c.table_width << p.c.page_log2) + j0 + 4 * g;
        const int first_pos = kv - n;
        f32x4 old[2] = {};
        if (p.weights && j0 < first_pos) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
                old[t] = *reinterpret_cast<const f32x4 *>(p.weights + at0 + (j0 + 16 * t < kv ? 16 * t : 0));
        }
        next = look_up();
        // ---- as A operands
        u32x4 a[2][KS];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float unit_k = E4M3 ? unit_of(units_k[t]) : 1.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if constexpr (E4M3) {
                    const uint32_t lo = x[t][s >> 1].d[2 * (s & 1)], hi = x[t][s >> 1].d[2 * (s & 1) + 1];
                    a[t][s] = u32x4{E::template from_e4m3<false>(lo, unit_k), E::template from_e4m3<true>(lo, unit_k),
                                    E::template from_e4m3<false>(hi, unit_k), E::template from_e4m3<true>(hi, unit_k)};
                } else {
                    a[t][s] = u32x4{x[t][s].d[0], x[t][s].d[1], x[t][s].d[2], x[t][s].d[3]};
                }
            }
        }
        // ---- the rows that see some of them
        const int n_rows = n * p.G;
        const int from = p.causal ? (int)min((long long)max(j0 - first_pos, 0) * p.G, (long long)n_rows) : 0;
        float w[2][4] = {};
        for (int r0 = from & ~15; r0 < n_rows; r0 += 16) {
            const int row = min(r0 + c, n_rows - 1), i = p.token_of(row), hq = h * p.G + row - i * p.G;
            const typename E::t *src = static_cast<const typename E::t *>(p.q) + (long long)(row0 + i) * p.q_st + (long long)hq * p.q_sh;
            u32x4 q[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s)
                q[s] = *reinterpret_cast<const u32x4 *>(src + (E4M3 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8));
            const float lse = p.lse[(size_t)(row0 + i) * p.H_q + hq];
            // (a row that sees nothing, or is none: exp2(-inf))
            const float shift = r0 + c < n_rows && lse != -INFINITY ? -lse * 1.44269504088896340736f : -INFINITY;
            f32x4 s4[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s4[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    s4[t] = E::mfma16(a[t][s], q[s], s4[t]);
            }
            if (p.causal && __any(first_pos + i < j0 + kWeighKeys - 1)) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (j0 + 16 * t + 4 * g + k > first_pos + i)
                            s4[t][k] = -INFINITY;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[t][k] += __builtin_amdgcn_exp2f(fmaf(s4[t][k], p.c_log2, shift));
        }
        // ---- one sum for every key; lane 0 of a group has four
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = j0 + 16 * t + 4 * g;
            f32x4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                y[k] = ok[t] ? sum16(w[t][k]) : 0.f;
                if (p.weights && j + k < first_pos)
                    y[k] = fmaf(p.decay, old[t][k], y[k]);
            }
            if (c != 0)
                continue;
            if (j + 4 <= kv) {
                *reinterpret_cast<f32x4 *>(p.out + at0 + 16 * t) = y;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j + k < kv)
                        p.out[at0 + 16 * t + k] = y[k];
            }
            if (p.stamps && j + 4 > first_pos) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j + k >= first_pos && j + k < kv)
                        p.stamps[at0 + 16 * t + k] = p.seen[b] - kv + j + k;
            }
        }
    }
}

// Many rows: a workgroup has 256 keys (128 at D = 256), each wave its part of them in registers as A operands of v_mfma_f32_32x32x16,
// and the rows pass through LDS in stages that all waves read.  A batch with few blocks of 256 keys is cut finer: two waves of a workgroup
// then have the same keys, and half of a stage's rows each.  RING stages are there at once, all but one of them on their way: two, and two
// workgroups to a compute unit, or four where the batch has no more units than compute units, whose stages would each wait for memory
// otherwise (2048 rows at 16384 keys, 8 heads over 2, D = 256: two 193 us, four 178).
template <int D>
struct WeighTiling {
    static constexpr int ROWB = D * 2, SUB = D == 256 ? 2 : 4;     // 32-row tiles of a stage
    static constexpr int ROWS = 32 * SUB, STAGE = ROWS * ROWB;
    static constexpr int KB = D == 256 ? 1 : 2;                    // 32-key blocks of a wave
    static constexpr int KEYS = 4 * 32 * KB;                       // of a workgroup
    static constexpr int SHARE = SUB / 2;                          // waves that share keys where the batch has few blocks
    static constexpr int LSE = 4 * 64 * 4;                         // bytes of the rows' lse of a stage: 64 rows of each wave, some of the next one's
    static constexpr int lds_bytes(int ring) { return ring * (STAGE + LSE); }
};
constexpr int kWeighTileGroups = 512;   // workgroups of a launch: two to a compute unit

template <int D, typename E, bool E4M3, int RING>
__global__ __launch_bounds__(256, 2) void attn_weigh_tiles_kernel(const WeighParams p)
{
    typedef WeighTiling<D> T;
    constexpr int ROWB = T::ROWB, SUB = T::SUB, KB = T::KB, KS = D / 16, CROWB = D * (E4M3 ? 1 : 2);
    constexpr int LOADS = T::STAGE / 4096, CPR = ROWB / 16, RPL = 64 / CPR;    // loads of a wave and stage, chunks of a row, rows of a load
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(ATTN_LDS_PTR(unsigned char))smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lq = lane & 31, g = lane >> 5;
    const int page_mask = (1 << p.c.page_log2) - 1;
    WeighUnits units;
    units.begin(p.c, __builtin_ctz(T::KEYS));
    const bool split = T::SHARE > 1 && p.c.B <= 64 && (long long)units.all * p.c.H_kv < kWeighTileGroups;
    if (split)
        units.begin(p.c, __builtin_ctz(T::KEYS / T::SHARE));
    const int my_keys = (split ? wave / T::SHARE : wave) * 32 * KB;
    const int tile0 = split ? wave % T::SHARE * 2 : 0, tile1 = split ? tile0 + 2 : SUB;    // of a stage
    uint32_t k0 = (uint32_t)(lq * ROWB + ((g ^ swz<D>(lq)) * 16));       // chunk g of row lq; chunk 2 s + g: k0 ^ 32 s
    const uint32_t st = (uint32_t)p.q_st * 2, sh = (uint32_t)p.q_sh * 2;       // (the host keeps offsets of a call's rows to 32 bits)

    for (long long unit = blockIdx.x;; unit += gridDim.x) {
        int b, n, row0, kv, key0;
        const long long block = quotient(unit, p.c.H_kv);
        const int h = (int)(unit - block * p.c.H_kv);
        if (!units.find(p.c, block, b, n, row0, kv, key0))
            return;
        const int j0 = key0 + my_keys, n_rows = n * p.G, first_pos = kv - n;
        const int from = p.causal ? (int)min((long long)max(key0 - first_pos, 0) * p.G, (long long)n_rows) : 0;
        const int stages = (n_rows - from + T::ROWS - 1) / T::ROWS;

        // ---- rows and their lse: memory -> LDS, stage i into its part of the ring.  A load takes RPL rows; lane -> (row, 16-byte chunk), the
        // swizzle of a tile's rows is applied on the global side.  Rows behind the last repeat it
        auto scalar = [](const void *at) {
            const uint64_t x = (uint64_t)(uintptr_t)at;
            return reinterpret_cast<const void *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                                                  (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
        };
        const void *rows = scalar(static_cast<const typename E::t *>(p.q) + ((long long)row0 * p.q_st + (long long)h * p.G * p.q_sh));
        const void *lses = scalar(p.lse + ((size_t)row0 * p.H_q + h * p.G));
        asm volatile("s_nop 4" : "+s"(rows), "+s"(lses));   // five wait states between the vector unit's write of a scalar and a load
        uint32_t off[LOADS];
        const uint32_t step = (uint32_t)(T::ROWS / p.G) * st;
        const bool even = T::ROWS % p.G == 0;               // a stage's rows are whole tokens: the next one's lie a step on
        auto bring = [&](int i) {
            if (i >= stages)
                return;
            const int first = from + i * T::ROWS;
            int ln = lane;                                  // (places made anew: kept across stages they take registers)
            asm volatile("" : "+v"(ln));
#pragma unroll
            for (int l = 0; l < LOADS; ++l) {
                const int r = (wave * LOADS + l) * RPL + ln / CPR, ch = ln % CPR;
                if (i == 0 || !even || first + T::ROWS > n_rows) {
                    const int row = min(first + r, n_rows - 1), token = p.token_of(row);
                    off[l] = (uint32_t)token * st + (uint32_t)(row - token * p.G) * sh +
                             (uint32_t)(((ch & ~15) | ((ch & 15) ^ swz<D>(r))) * 16);
                } else {
                    off[l] += step;
                }
                dma16(lds0 + i % RING * T::STAGE + (wave * LOADS + l) * 1024, rows, off[l]);
            }
            const int row = min(first + 64 * wave + ln, n_rows - 1), token = p.token_of(row);
            dma4(lds0 + RING * T::STAGE + i % RING * T::LSE + wave * 256, lses, (uint32_t)(token * p.H_q + row - token * p.G) * 4);
        };
        const float *const raw = reinterpret_cast<const float *>(smem + RING * T::STAGE);
        __syncthreads();                                    // the last unit's rows have been read
#pragma unroll
        for (int i = 0; i < RING - 1; ++i)
            bring(i);

        // ---- keys: lane l has key l % 32 of a block, elements 16 s + 8 g on of step s
        u32x4 a[KB][KS];
#pragma unroll
        for (int t = 0; t < KB; ++t) {
            const int j = min(j0 + 32 * t + lq, kv - 1);
            const size_t row = p.c.page_row(max(p.c.page_of(b, j), 0), h) + (j & page_mask);
            const unsigned char *k = static_cast<const unsigned char *>(p.k) + row * CROWB;
            if constexpr (E4M3) {
                const float unit_k = unit_of(p.k_scale[row]);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    Piece<8> x;
                    x.load(k + 16 * s + 8 * g);
                    a[t][s] = u32x4{E::template from_e4m3<false>(x.d[0], unit_k), E::template from_e4m3<true>(x.d[0], unit_k),
                                    E::template from_e4m3<false>(x.d[1], unit_k), E::template from_e4m3<true>(x.d[1], unit_k)};
                }
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    a[t][s] = *reinterpret_cast<const u32x4 *>(k + 32 * s + 16 * g);
            }
        }
        // (waited for here: at their first use the wait would be part of the loop, and one for the rows on their way as well; D = 64,
        // 2048 rows at 16384 keys, 16 heads over 4: 115 us, 118 without)
#pragma unroll
        for (int t = 0; t < KB; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                asm volatile("" : "+v"(a[t][s]));

        float w[KB][16];
#pragma unroll
        for (int t = 0; t < KB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                w[t][r] = 0.f;
        // Scores of tile t of stage i into `now`; between the products the weights of the tile before are taken, whose scores lie in
        // `then` and are lowered by `down`: the matrix pipe and the vector unit have the same to do, and neither waits for the other.
        float down = -INFINITY;
        auto scores = [&](int i, int t, f32x16 (&now)[KB], f32x16 (&then)[KB]) {
            const uint32_t base = lds0 + i % RING * T::STAGE + t * 32 * ROWB;
            asm volatile("" : "+v"(k0));                    // (its later chunks' offsets made anew: kept they take registers)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    now[kb][r] = 0.f;
            constexpr int AHEAD = 3;                        // operands on their way
            u32x4 q[AHEAD + 1];
            auto operand = [&](int ks) { return *(ATTN_LDS_PTR(const u32x4))(uintptr_t)((k0 ^ (32 * ks)) + base); };
#pragma unroll
            for (int ks = 0; ks < AHEAD; ++ks)
                q[ks] = operand(ks);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + AHEAD < KS)
                    q[(ks + AHEAD) % (AHEAD + 1)] = operand(ks + AHEAD);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    now[kb] = mfma32<E>(a[kb][ks], q[ks % (AHEAD + 1)], now[kb]);
                constexpr int PER = 16 * KB / KS;
                // (side by side, so that no exponential is waited for; and here, not behind the products)
                float e[PER];
#pragma unroll
                for (int x = 0; x < PER; ++x)
                    e[x] = fmaf(then[(ks * PER + x) / 16][(ks * PER + x) % 16], p.c_log2, down);
#pragma unroll
                for (int x = 0; x < PER; ++x)
                    e[x] = __builtin_amdgcn_exp2f(e[x]);
#pragma unroll
                for (int x = 0; x < PER; ++x)
                    w[(ks * PER + x) / 16][(ks * PER + x) % 16] += e[x];
#pragma unroll
                for (int x = 0; x < PER; ++x)
                    asm volatile("" : "+v"(w[(ks * PER + x) / 16][(ks * PER + x) % 16]));
                __builtin_amdgcn_sched_barrier(0);
            }
            // what a row's scores are lowered by (base 2): infinity where it sees nothing or there is no row
            const int first = from + i * T::ROWS + 32 * t;
            const float lse = raw[i % RING * (T::LSE / 4) + 32 * t + lq];
            down = first + lq < n_rows && lse != -INFINITY ? -lse * 1.44269504088896340736f : -INFINITY;
            if (p.causal && first_pos + p.token_of(min(first, n_rows - 1)) < j0 + 32 * KB - 1) {     // some row does not see some key
                // (against constants: positions kept in registers would take 32)
                const int limit = first_pos + p.token_of(min(first + lq, n_rows - 1)) - j0 - 4 * g;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        now[kb][r] = 32 * kb + acc_row(r, 0) > limit ? -INFINITY : now[kb][r];
            }
        };
        f32x16 s0[KB], s1[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s1[kb][r] = 0.f;                            // (lowered by infinity)
#pragma clang loop unroll(disable)
        for (int i = 0; i < stages; ++i) {
            if (RING > 2 && i + RING - 2 < stages)
                wait_vmcnt<(RING - 2) * (LOADS + 1)>();     // of stage i nothing is on its way, of those behind it all may be
            else
                wait_vmcnt<0>();                            // (the last ones: there are fewer behind)
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");     // stage i is complete, stage i - 1 has been read
            bring(i + RING - 1);
#pragma clang loop unroll(disable)
            for (int t = tile0, upto = min(tile1, (n_rows - from - i * T::ROWS + 31) / 32); t < upto; t += 2) {
                scores(i, t, s0, s1);
                scores(i, t + 1, s1, s0);
            }
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                w[kb][r] += __builtin_amdgcn_exp2f(fmaf(s1[kb][r], p.c_log2, down));

        // ---- one sum for every key: over the 32 rows of a tile, and in a split unit over its waves
        float y[KB];                                        // of key acc_row(lq % 16, g)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            y[kb] = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = sum16(w[kb][r]), all = x + __shfl_xor(x, 16, 64);
                y[kb] = (lq & 15) == r ? all : y[kb];
            }
        }
        if (split) {
            float *const part = reinterpret_cast<float *>(smem);
            __syncthreads();                                // the rows have been read
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                part[(wave * KB + kb) * 64 + lane] = y[kb];
            __syncthreads();
            if (tile0 != 0)
                continue;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                y[kb] = 0.f;
                for (int v = wave; v < wave + T::SHARE; ++v)
                    y[kb] += part[(v * KB + kb) * 64 + lane];
            }
        }
        const size_t at0 = ((size_t)b * p.c.H_kv + h) * ((size_t)p.c.table_width << p.c.page_log2);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int j = j0 + 32 * kb + acc_row(lq & 15, g);
            if (lq >= 16 || j >= kv)
                continue;
            float x = p.c.page_of(b, j) >= 0 ? y[kb] : 0.f;
            if (j < first_pos && p.weights)
                x = fmaf(p.decay, p.weights[at0 + j], x);
            p.out[at0 + j] = x;
            if (p.stamps && j >= first_pos)
                p.stamps[at0 + j] = p.seen[b] - kv + j;
        }
    }
}

}  // namespace attn

namespace {

using attn::WeighParams;

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Rows of a sequence up to which the row kernel takes a call: one bound for all head sizes, though they cross at rows of their own.  8 sequences of
// 16384 keys, 4 heads, us by rows and by tiles:
//     rows                     16            32            48            64            80            96           128
//     D = 64,  16 bits     19.1  31.2    22.0  30.3    25.8  30.5    29.2  30.3    33.0  35.8    36.9  35.8    43.9  35.7
//              e4m3        14.3  28.0    18.3  28.5    21.8  28.4    25.7  28.6    29.4  34.2    33.3  33.8    41.3  33.5
//     D = 128, 16 bits     29.6  41.0    36.0  40.7    43.1  41.2    50.1  41.2    57.4  48.3    64.6  48.2    79.5  48.9
//              e4m3        23.1  38.5    30.4  38.3    37.0  38.5    43.5  38.7    50.6  44.3    57.5  44.2    71.7  44.8
//     D = 256, 16 bits     58.4  69.3    70.5  69.3    83.7  71.5    97.4  72.0     112  90.1     125  90.0     154  84.1
//              e4m3        41.0  57.9    55.3  58.9    69.8  59.0    83.9  58.5    98.7  76.3     113  76.3     142  72.8
// One sequence of 4000: 16 to 64 rows by rows 6.0 to 9.5 and by tiles 7.4 to 9.4.
constexpr long long kRowsMost = 64;

template <int D, typename E, bool E4M3>
int launch(const WeighParams &p, int max_q, hipStream_t st)
{
    const long long rows = (long long)(max_q < p.c.T ? max_q : p.c.T) * p.G;
    const long long reach = 2 * ((long long)p.c.T * p.q_st + (long long)p.G * p.q_sh + D);  // bytes of a head's rows
    const bool tiles = rows > kRowsMost && reach < 1LL << 32;
    // no more workgroups than units that the table can hold
    const long long keys = tiles ? attn::WeighTiling<D>::KEYS / attn::WeighTiling<D>::SHARE : 4 * attn::kWeighKeys;
    const long long blocks = (((long long)p.c.table_width << p.c.page_log2) + keys - 1) / keys;
    const long long seqs = p.c.B < p.c.T ? p.c.B : p.c.T;
    const int held = tiles ? attn::kWeighTileGroups : attn::persistent_slots(reinterpret_cast<const void *>(attn::attn_weigh_rows_kernel<D, E, E4M3>), 256, 0, 1);
    const long long most = held > 0 ? held : attn::kWeighGroups, per_seq = blocks < most ? blocks * p.c.H_kv : most;
    const long long grid = per_seq < most / seqs ? per_seq * seqs : most;
    if (!tiles) {
        hipLaunchKernelGGL((attn::attn_weigh_rows_kernel<D, E, E4M3>), dim3((unsigned)grid), dim3(256), 0, st, p);
    } else {
        // (D = 64: four stages leave room for two workgroups)
        const bool deep = D == 64 || grid <= attn::kWeighTileGroups / 2;
        constexpr int two = D == 64 ? 4 : 2;
        auto *const kern = deep ? attn::attn_weigh_tiles_kernel<D, E, E4M3, 4> : attn::attn_weigh_tiles_kernel<D, E, E4M3, two>;
        const int lds = attn::WeighTiling<D>::lds_bytes(deep ? 4 : two);
        if (!attn::allow_lds(reinterpret_cast<const void *>(kern), lds))
            return ATTN_ERR_LAUNCH;
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), lds, st, p);
    }
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

template <typename E>
int weigh(const void *q, const long long *strides, const float *lse, const void *k_pages, const unsigned char *k_scale,
          const int *page_table, const int *start, const int *kv_len, int kind, const float *weights, float *weights_out, int *stamps,
          const int *seen, float decay, int max_q, int T, int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width,
          int causal, float scale, void *stream)
{
    if (!q || !strides || !lse || !k_pages || !page_table || !start || !kv_len || !weights_out || !stamps != !seen ||
        (kind == ATTN_CACHE_E4M3 && !k_scale))
        return ATTN_ERR_NULL;
    if (T < 1 || B < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv || n_pages < 1 || table_width < 1 || max_q < 1 || B > attn::kMostSequences)
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    if ((kind != ATTN_CACHE_16BIT && kind != ATTN_CACHE_E4M3) || page_size < 16 || page_size > 256 ||
        (page_size & (page_size - 1)))
        return ATTN_ERR_UNSUPPORTED;
    const long long width = (long long)table_width * page_size;
    if ((long long)T * H_q > 0x3fffffffLL || (long long)n_pages * H_kv > (1LL << 40) / D / page_size || H_kv > (1 << 24) ||
        width > (1 << 30) || (long long)H_kv * page_size >= (1 << 30) / D || (long long)B * H_kv > (1LL << 40) / width)
        return ATTN_ERR_SHAPE;
    for (int i = 0; i < 2; ++i) {
        const long long n = i ? H_q : T;
        if (n > 1 && (strides[i] < 0 || strides[i] % 8 || strides[i] > (1LL << 40) / n))
            return ATTN_ERR_SHAPE;
    }
    const uintptr_t in = (uintptr_t)weights, out = (uintptr_t)weights_out, bytes = (uintptr_t)B * H_kv * width * 4;
    if (weights && in != out && in < out + bytes && out < in + bytes)
        return ATTN_ERR_SHAPE;
    if (misaligned(q, 16) || misaligned(lse, 4) || misaligned(k_pages, 16) || misaligned(page_table, 4) || misaligned(start, 4) ||
        misaligned(kv_len, 4) || misaligned(weights, 16) || misaligned(weights_out, 16) || misaligned(stamps, 16) ||
        misaligned(seen, 4) || (kind == ATTN_CACHE_E4M3 && misaligned(k_scale, 16)))
        return ATTN_ERR_ALIGN;
    if (!(scale > 0.f) || !(scale < INFINITY) || !(decay >= 0.f) || !(decay < INFINITY))
        return ATTN_ERR_SCALE;
    WeighParams p;
    p.c.page_table = page_table, p.c.start = start, p.c.kv_len = kv_len;
    p.c.T = T, p.c.B = B, p.c.H_kv = H_kv, p.c.n_pages = n_pages, p.c.table_width = table_width;
    p.c.page_log2 = __builtin_ctz((unsigned)page_size);
    p.q = q, p.k = k_pages, p.k_scale = k_scale, p.lse = lse;
    p.weights = decay == 0.f ? nullptr : weights, p.out = weights_out, p.stamps = stamps, p.seen = seen;
    p.q_st = strides[0], p.q_sh = strides[1];
    p.H_q = H_q, p.G = H_q / H_kv;
    int log_g = 0;                                         // (PagedParams::token_of)
    while ((1LL << log_g) < p.G)
        ++log_g;
    p.g_mul = p.G == 1 ? 0 : (uint32_t)(((1ULL << (31 + log_g)) + p.G - 1) / p.G);
    p.g_shift = p.G == 1 ? 0 : log_g - 1;
    p.causal = causal != 0;
    p.c_log2 = (float)((double)scale * 1.44269504088896340736);
    p.decay = decay;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool e4m3 = kind == ATTN_CACHE_E4M3;
    switch (D) {
    case 64: return e4m3 ? launch<64, E, true>(p, max_q, st) : launch<64, E, false>(p, max_q, st);
    case 128: return e4m3 ? launch<128, E, true>(p, max_q, st) : launch<128, E, false>(p, max_q, st);
    default: return e4m3 ? launch<256, E, true>(p, max_q, st) : launch<256, E, false>(p, max_q, st);
    }
}

}  // namespace

#define ATTN_WEIGH_ENTRY(name, E)                                                                                              \
    extern "C" int name(const void *q, const long long *strides, const float *lse, const void *k_pages,                        \
                        const unsigned char *k_scale, const int *page_table, const int *start, const int *kv_len, int kind,    \
                        const float *weights, float *weights_out, int *stamps, const int *seen, float decay, int max_q, int T, \
                        int B, int H_q, int H_kv, int D, int n_pages, int page_size, int table_width, int causal, float scale, \
                        void *stream)                                                                                          \
    {                                                                                                                          \
        return weigh<E>(q, strides, lse, k_pages, k_scale, page_table, start, kv_len, kind, weights, weights_out, stamps,      \
                        seen, decay, max_q, T, B, H_q, H_kv, D, n_pages, page_size, table_width, causal, scale, stream);       \
    }

ATTN_WEIGH_ENTRY(attn_cache_weigh, attn::PagedBF16)
ATTN_WEIGH_ENTRY(attn_cache_weigh_f16, attn::PagedF16)
