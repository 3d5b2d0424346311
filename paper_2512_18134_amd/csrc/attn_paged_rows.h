// attn_paged_rows.h -- attention over the paged cache for few rows: decoding steps and drafted tokens.
//
// What bounds it is the cache: every key and value is read once and used for at most 16 MT rows, so the kernel is a
// stream from memory into registers with the products along the way.  Nothing of the stream passes through LDS and no wave
// waits for another: the waves of a workgroup take the 32-key steps of their unit's range in turn, each
// with a softmax of its own, and meet once at the end.
//
// Transposed products on v_mfma_f32_16x16x32: S^T = K Q^T, O^T = V^T P^T.  Lane l has column c = l % 16 (a row of the tile:
// its query) and group g = l / 16.  The contraction index of a product may run in any order as long as both operands have the
// same one, which is what makes the loads fit the registers:
//   * K as A operand: lane (c, g) holds key c's elements from memory as they lie, 16 bytes a load; Q is read the same way
//   * S^T leaves lane (c, g) with keys 4g .. 4g+3 of two 16-key blocks: those eight are its part of the second contraction
//   * V as A operand: lane (c, g) loads, of each of those eight keys, elements c D/16 .. (c+1) D/16 - 1 (a wave-wide load takes
//     whole rows); product n = 0 .. D/16 - 1 then needs element n of all eight, which v_perm gathers from the eight
//     registers.  Its 16 x 16 result holds elements n, n + D/16, ...: a lane ends up with D/16 neighbouring ones
//
// Measured, with the merge: 64 sequences of up to 8191 keys, 32 heads over 8, D = 128: 909 MB in 175 us, 5.2 TB/s; four of
// 131072 in e4m3, 64 heads over 8: 1082 MB in 189 us, 5.7 TB/s.  (A large sum reads 4.0 TB/s here, a large copy moves 5.1.)
// One sequence of 300 keys: 6.8 us, of which 0.5 go to the cut, 0.6 to the unit, 3 to two steps' chain of page, keys and
// values, 1 to the exchange.
//
// Softmax against a lazily moved reference: a row's reference moves only where a score exceeds it by more than 8 (in the
// base-2 domain), so most steps need no maximum across lanes and no rescaling; sums and accumulators
// are fp32.  P enters the second product in 16 bits (at most half a step, 2^-8 of it in bf16 and 2^-11 in fp16: there
// is no product of fp32 operands at this rate; the row sum keeps its 32), and a P of up to 2^8 is as exact there as one of up to 1.
#pragma once
#include "attn_paged_plan.h"

namespace attn {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// eight rows of zeros: what a tile in LDS without a page is made of
__device__ const u32x4 kPagedZeroRows[8 * 512 / 16] = {};

struct PagedBF16 {
    typedef __bf16 t;
    typedef __attribute__((ext_vector_type(2))) __bf16 x2;
    typedef __attribute__((ext_vector_type(8))) __bf16 x8;
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w, float unit)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit, HI));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, x2));   // to nearest even
    }
};
struct PagedF16 {
    typedef _Float16 t;
    typedef __attribute__((ext_vector_type(2))) _Float16 x2;
    typedef __attribute__((ext_vector_type(8))) _Float16 x8;
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w, float unit)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, unit, HI));
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, x2));
    }
};

// The launch's parameters, read anew from where the launch put them (p is the kernel's only argument): what a loop over units
// keeps of them across a unit takes registers that the unit needs.
template <bool TREE = false>
__device__ __forceinline__ ParamsOf<TREE> params_again()
{
    typedef __attribute__((address_space(4))) const ParamsOf<TREE> Arguments;
    Arguments *args = (Arguments *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    return *(const ParamsOf<TREE> *)args;
}

// 2^(s - 127) of an e4m3 row's exponent byte
__device__ __forceinline__ float unit_of(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

template <int BYTES>
struct Piece {   // BYTES of memory in dwords
    uint32_t d[BYTES / 4];
    __device__ __forceinline__ void load(const unsigned char *p)
    {
        if constexpr (BYTES == 4) {
            d[0] = *reinterpret_cast<const uint32_t *>(p);
        } else if constexpr (BYTES == 8) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(p);
            d[0] = x[0], d[1] = x[1];
        } else {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(p + 16 * i);
                d[4 * i] = x[0], d[4 * i + 1] = x[1], d[4 * i + 2] = x[2], d[4 * i + 3] = x[3];
            }
        }
    }
};

template <int D, int MT, int NW>
struct PagedRowsTiling {
    static constexpr int BM = 16 * MT, THREADS = NW * 64;
    static constexpr int PER_SIMD = NW > 4 ? NW / 4 : (MT == 1 && D <= 128) || (MT == 2 && D == 64) ? 2 : 1;   // waves, at least
    static constexpr int PER_CU = PER_SIMD * 4 / NW;        // workgroups
    static constexpr int XP = D == 256 ? 2 : 1;             // parts in which a row's elements meet (64 KB of LDS hold a part)
    static constexpr int ROWF = D / XP + 4;                 // floats of a row of the exchange, padded
    static constexpr int XCH_FLOATS = NW * 16 * ROWF, ML_FLOATS = NW * 16 * 2;
    static constexpr int LDS_BYTES = (XCH_FLOATS + ML_FLOATS) * 4;
};

// Which of the 32 positions from `from` on a row of a tree sees, bit by bit: `before` is the position of its sequence's first
// new token, and the positions before it are seen by all; mask: the row's words.  A new token behind the mask's last is
// seen by none.
__device__ __forceinline__ uint32_t seen_in_tree(const uint32_t *mask, int words, int before, int from)
{
    const int node = from - before, w = node >> 5;          // (arithmetic: to below)
    auto word = [&](int i) -> uint32_t {
        const uint32_t x = mask[min(max(i, 0), words - 1)];
        return i < 0 ? 0xffffffffu : i < words ? x : 0u;
    };
    return __builtin_amdgcn_alignbit(word(w + 1), word(w), node & 31);
}

// TREE: seen_in_tree of a lane's rows, of the keys of a step.
template <bool TREE, int MT>
struct Seen {};
template <int MT>
struct Seen<true, MT> {
    uint32_t seen[MT];
};

// E4M3: the pool's kind.  MT: 16-row column tiles.  NW: waves; 4, or 8 where a unit is a whole short sequence (kWholeBytes in
// attn_paged_launch.h).  The waves' results meet in one exchange: handed on by four waves at a time, sixteen waves took 3.5 us of
// a launch's 9.  TREE: the sequence's new tokens see each other by the mask instead of by their order.
template <int D, int MT, typename E, bool E4M3, int NW, bool TREE>
__global__ __launch_bounds__(NW * 64, (PagedRowsTiling<D, MT, NW>::PER_CU))
    void attn_paged_rows_kernel(const ParamsOf<TREE> p)
{
    typedef PagedRowsTiling<D, MT, NW> T;
    static_assert(NW == 4 || (MT == 1 && D <= 128), "the exchange holds all waves of 16 rows");
    constexpr int EB = E4M3 ? 1 : 2;                        // bytes of a cached element
    constexpr int ROWB = D * EB;
    constexpr int KL = ROWB / 64;                           // 16-byte loads of a lane's share of a key
    constexpr int KS = D / 32;                              // products of S^T
    constexpr int NV = D / 16;                              // elements of a lane's share of a value row, products of O^T
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *const xch = reinterpret_cast<float *>(lds);
    f32x2 *const ml = reinterpret_cast<f32x2 *>(xch + T::XCH_FLOATS);      // reference and row sum of a wave's rows

    Unit u;
    PlanSeq seq;
    const Plan plan = plan_call<T::BM>(p, seq);
    if (!find_unit<T::BM>(p, plan, seq, blockIdx.x, u))
        return;
    leave_note<T::BM, T::THREADS>(p, u);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;

    // ---- the rows of this lane's columns: last visible key, Q
    int last[MT];
    const uint32_t *sees[MT];                               // TREE: the row's mask
    u32x4 q[MT][KS];
    const int tile_row = u.tile * T::BM;
    const int first_pos = u.kv - u.n;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = min(tile_row + 16 * m + c, u.n_rows - 1);      // rows behind the last repeat it
        const int i = p.token_of(row), hq = u.h * p.G + row - i * p.G;
        last[m] = p.causal ? first_pos + i : u.kv - 1;
        if constexpr (TREE)
            sees[m] = p.mask + (size_t)(u.row0 + i) * p.mask_words;
        const typename E::t *src = static_cast<const typename E::t *>(p.q) + (long long)(u.row0 + i) * p.q_st + (long long)hq * p.q_sh;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            // the elements that a key's A operand holds in product s
            const int e = E4M3 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
            q[m][s] = *reinterpret_cast<const u32x4 *>(src + e);
        }
    }
    // keys that no row of the tile sees are not walked; from `open` on some row does not see a key
    const int low = p.token_of(tile_row), high = p.token_of(min(tile_row + T::BM - 1, u.n_rows - 1));
    const int key1 = p.causal ? min(u.key1, first_pos + high + 1) : u.key1;
    const int open = TREE ? min(first_pos, u.kv) : p.causal ? min(first_pos + low + 1, u.kv) : u.kv;
    const int n_steps = key1 > u.key0 ? (key1 - u.key0 + 31) / 32 : 0;

    f32x4 o[MT][NV];
    float mc[MT], l[MT];                                    // reference (base 2), this lane's part of the row sum
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mc[m] = -3.0e38f;                                   // finite: masked scores (-inf) give exactly 0 against it
        l[m] = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n)
            o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // ---- the stream: registers of one step
    struct Step : Seen<TREE, MT> {
        Piece<16> k[2][KL];
        Piece<NV * EB> v[2][4];
        uint32_t ks[2], vs[2];
        bool bad;                                           // some of its keys have no page
        bool ok[2];
    };
    const int page_mask = (1 << p.c.page_log2) - 1;
    // Pages of the two 16-key blocks (pages hold a multiple of 16 positions) of the wave's next 32 steps, one in a lane: asked
    // for step by step, a page's number would have to arrive before its keys could be asked for.
    int window = 0, turn = 0;
    auto pages_of = [&](int s, int id[2]) {
        if ((turn & 31) == 0)
            window = p.c.page_of(u.b, min(u.key0 + 32 * (s + NW * (lane >> 1)) + 16 * (lane & 1), u.kv - 1));
#pragma unroll
        for (int t = 0; t < 2; ++t)
            id[t] = __builtin_amdgcn_readlane(window, 2 * (turn & 31) + t);
        ++turn;
    };
    // D = 256, two tiles of rows: the accumulators and Q leave registers for the keys or the values, not for both
    constexpr bool LATE_V = D == 256 && MT == 2;
    // The next step's keys are on their way during a step where they are few registers (16): 8 heads of 2000 keys, D = 128, e4m3,
    // 14.6 us without and 13.7 with them, 16 heads of 1000, D = 64, 9.2 and 9.0.  At 32 registers the second copy of the loop
    // gains nothing: 64 sequences of up to 8191 keys, D = 128, 16 bits, 180 and 189 us, of up to 500 keys 19.4 and 20.5.
    constexpr bool AHEAD = KL <= 2 && !LATE_V;
    auto load_k = [&](Step &x, int s, const int id[2]) {
        x.bad = (id[0] | id[1]) < 0;
        if constexpr (TREE) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                x.seen[m] = 0xffffffffu;
            if (u.key0 + 32 * s + 32 > open) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    x.seen[m] = seen_in_tree(sees[m], p.mask_words, first_pos, u.key0 + 32 * s);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            x.ok[t] = id[t] >= 0;
            const int j = min(u.key0 + 32 * s + 16 * t, (u.kv - 1) & ~15);
            const size_t row = p.c.page_row(max(id[t], 0), u.h) + (j & page_mask);
            const unsigned char *k = static_cast<const unsigned char *>(p.k) + row * ROWB;
#pragma unroll
            for (int i = 0; i < KL; ++i)
                x.k[t][i].load(k + c * ROWB + g * 16 + i * 64);
            if (E4M3)
                x.ks[t] = p.k_scale[row + c];
        }
    };
    auto load_v = [&](Step &x, int s, const int id[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int j = min(u.key0 + 32 * s + 16 * t, (u.kv - 1) & ~15);
            const size_t row = p.c.page_row(max(id[t], 0), u.h) + (j & page_mask);
            const unsigned char *v = static_cast<const unsigned char *>(p.v) + row * ROWB;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x.v[t][i].load(v + (4 * g + i) * ROWB + c * NV * EB);
            if (E4M3)
                x.vs[t] = *reinterpret_cast<const uint32_t *>(p.v_scale + row + 4 * g);
        }
    };
    auto mask_v = [&](Step &x, int s) {
        // places that hold no key of this sequence: P is 0 there, but 0 x NaN is not
        const int j0 = u.key0 + 32 * s;
        if (x.bad || j0 + 32 > u.kv) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!x.ok[t] || j0 + 16 * t + 4 * g + i >= u.kv) {
#pragma unroll
                        for (int d = 0; d < NV * EB / 4; ++d)
                            x.v[t][i].d[d] = 0;
                        if (E4M3)
                            x.vs[t] &= ~(0xffu << (8 * i));   // (an exponent byte of 255 would be infinity)
                    }
        }
    };

    auto work = [&](Step &x, int s, const int id[2]) {
        const int j0 = u.key0 + 32 * s;
        if constexpr (!LATE_V)
            mask_v(x, s);
        f32x4 sc[MT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                sc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float unit = E4M3 ? unit_of(x.ks[t]) : 1.f;
#pragma unroll
            for (int n = 0; n < KS; ++n) {
                u32x4 a;
                if constexpr (E4M3) {
                    const uint32_t lo = x.k[t][n >> 1].d[2 * (n & 1)], hi = x.k[t][n >> 1].d[2 * (n & 1) + 1];
                    a = u32x4{E::template from_e4m3<false>(lo, unit), E::template from_e4m3<true>(lo, unit),
                              E::template from_e4m3<false>(hi, unit), E::template from_e4m3<true>(hi, unit)};
                } else {
                    a = u32x4{x.k[t][n].d[0], x.k[t][n].d[1], x.k[t][n].d[2], x.k[t][n].d[3]};
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    sc[m][t] = E::mfma16(a, q[m][n], sc[m][t]);
            }
        }
        if (x.bad || j0 + 32 > open) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        bool hidden = !x.ok[t] || j0 + 16 * t + 4 * g + i > last[m];
                        if constexpr (TREE)
                            hidden |= !(x.seen[m] >> (16 * t + 4 * g + i) & 1);
                        if (hidden)
                            sc[m][t][i] = -INFINITY;
                    }
        }
        if constexpr (LATE_V) {
            load_v(x, s, id);
            mask_v(x, s);
        }
        u32x4 pt[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float top = fmaxf(fmaxf(fmaxf(sc[m][0][0], sc[m][0][1]), fmaxf(sc[m][0][2], sc[m][0][3])),
                              fmaxf(fmaxf(sc[m][1][0], sc[m][1][1]), fmaxf(sc[m][1][2], sc[m][1][3]))) * p.c_log2;
            if (__any(top > mc[m] + 8.f)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), mc[m]);
                const float keep = __builtin_amdgcn_exp2f(mc[m] - top);
                mc[m] = top;
                l[m] *= keep;
#pragma unroll
                for (int n = 0; n < NV; ++n)
                    o[m][n] *= keep;
            }
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(fmaf(sc[m][i >> 2][i & 3], p.c_log2, -mc[m]));
                l[m] += e[i];
            }
            pt[m] = u32x4{E::pack(e[0], e[1]), E::pack(e[2], e[3]), E::pack(e[4], e[5]), E::pack(e[6], e[7])};
        }
        // O^T += V^T P^T: product n takes element n of the lane's share of its eight keys
        if constexpr (E4M3) {
#pragma unroll
            for (int n2 = 0; n2 < NV / 2; ++n2) {
                // two elements at a time: bytes (element, key) -> dwords of two keys, converted with a unit per key first
                u32x4 a[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float unit = unit_of((x.vs[t] >> (8 * i)) & 0xff);
                        const uint32_t d = x.v[t][i].d[n2 / 2];
                        w[i] = n2 & 1 ? E::template from_e4m3<true>(d, unit) : E::template from_e4m3<false>(d, unit);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        a[0][2 * t + i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100);
                        a[1][2 * t + i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302);
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    o[m][2 * n2] = E::mfma16(a[0], pt[m], o[m][2 * n2]);
                    o[m][2 * n2 + 1] = E::mfma16(a[1], pt[m], o[m][2 * n2 + 1]);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const uint32_t sel = n & 1 ? 0x07060302 : 0x05040100;
                u32x4 a;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i] = __builtin_amdgcn_perm(x.v[i >> 1][2 * (i & 1) + 1].d[n / 2], x.v[i >> 1][2 * (i & 1)].d[n / 2], sel);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                    o[m][n] = E::mfma16(a, pt[m], o[m][n]);
            }
        }
    };

    if (wave < n_steps) {
        int id[2];
        Step x;
        pages_of(wave, id);
        load_k(x, wave, id);
        if constexpr (AHEAD) {
            Step y;
            int s = wave;
            auto ahead = [&](Step &now, Step &next) {
                load_v(now, s, id);
                if (s + NW >= n_steps)
                    return false;
                pages_of(s + NW, id);
                load_k(next, s + NW, id);
                work(now, s, id);
                s += NW;
                return true;
            };
            while (ahead(x, y)) {
                if (!ahead(y, x)) {
                    x = y;
                    break;
                }
            }
            work(x, s, id);
        } else {
            for (int s = wave;;) {
                if constexpr (!LATE_V)
                    load_v(x, s, id);
                work(x, s, id);
                s += NW;
                if (s >= n_steps)
                    break;
                pages_of(s, id);
                load_k(x, s, id);
            }
        }
    }

    // ---- the waves' results meet, 16 rows at a time
    constexpr int NX = NV / T::XP;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        l[m] += __shfl_xor(l[m], 16, 64);
        l[m] += __shfl_xor(l[m], 32, 64);
#pragma unroll
        for (int x = 0; x < T::XP; ++x) {
            __syncthreads();                                // what lay there has been read
            const bool exists = tile_row + 16 * m + c < u.n_rows;
            if (g == 0)
                ml[wave * 16 + c] = f32x2{mc[m], l[m]};
#pragma unroll
            for (int i = 0; i < 4 && exists; ++i) {
                float *dst = xch + (wave * 16 + c) * T::ROWF + (4 * g + i) * NX;
#pragma unroll
                for (int n = 0; n < NX; n += 4) {
                    const int k = x * NX + n;
                    *reinterpret_cast<f32x4 *>(dst + n) = f32x4{o[m][k][i], o[m][k + 1][i], o[m][k + 2][i], o[m][k + 3][i]};
                }
            }
            __syncthreads();
            // NW * 4 threads of a row, EPT elements each
            constexpr int TPR = NW * 4, EPT = D / T::XP / TPR;
            typedef float elements __attribute__((ext_vector_type(EPT)));
            const int r = threadIdx.x / TPR, part = threadIdx.x % TPR;
            const int row = tile_row + 16 * m + r;
            if (row >= u.n_rows)
                continue;
            float top = ml[r][0];
#pragma unroll
            for (int w = 1; w < NW; ++w)
                top = fmaxf(top, ml[w * 16 + r][0]);
            float sum = 0.f;
            elements y = {};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const f32x2 stats = ml[w * 16 + r];
                const float weight = __builtin_amdgcn_exp2f(stats[0] - top);
                sum += weight * stats[1];
                y += weight * *reinterpret_cast<const elements *>(xch + (w * 16 + r) * T::ROWF + part * EPT);
            }
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const float lse = sum > 0.f ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f : -INFINITY;
            y *= inv;
            // (NX neighbouring elements of part x belong to one lane's NV)
            const int first = part * EPT / NX * NV + x * NX + part * EPT % NX;
            if (u.n_ranges > 1) {
                const size_t at = (size_t)u.slot * T::BM + 16 * m + r;
                if (sum > 0.f)
                    *reinterpret_cast<elements *>(p.parts[0].o + at * D + first) = y;
                if (part == 0 && x == 0)
                    p.parts[0].lse[at] = lse;
            } else {
                const int i = p.token_of(row);
                const size_t at = (size_t)(u.row0 + i) * p.H_q + u.h * p.G + row - i * p.G;
                typedef typename E::t out __attribute__((ext_vector_type(EPT)));
                *reinterpret_cast<out *>(static_cast<typename E::t *>(p.o) + at * D + first) = __builtin_convertvector(y, out);
                if (part == 0 && x == 0)
                    p.lse[at] = lse;
            }
        }
    }
}

}  // namespace attn
