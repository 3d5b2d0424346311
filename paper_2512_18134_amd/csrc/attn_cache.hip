// attn_cache.hip -- rows of keys and values into the paged cache and back out: kernels and entry points
// (include/attn_cache.h).
//
// Bound by memory (58000 positions written in 16 bits at 6.5 TB/s); for the few rows of a decoding step (64 rows: 2.6 us) by the chain of dependent loads: start -> kv_len -> page table -> row.
// Two kernels.  With few tokens a wave works on one (the chain is uniform and walked once) and on 64 pieces of 8 elements of
// its heads' K and V rows.  With many, a wave takes eight neighbouring tokens and some of their (tensor, head) rows: in the
// pool neighbouring positions of a head are contiguous, so that its accesses there are long, as are the rows'
// in the tensors (eight tokens of all heads are 128-byte pieces of the pool, page_size apart, and a cache line of
// units for every byte of them: 58000 positions of 8 heads, D = 128, read from e4m3 in 107 us that way, in 56 us this way, 6.3 TB/s).
//
// e4m3 with a power of two per row: q = round(x * 2^-e) is an exact product and one rounding, so that the quantised value is
// a function of the numbers alone and not of how a division was carried out; against amplitude / 448 as the
// unit it gives up less than one of the format's seventeen binades at the small end.
#include <hip/hip_runtime.h>

#include <type_traits>

#include <math.h>

#include "attn_cache.h"
#include "attn_cache_rows.h"
#include "attn_common.h"
#include "attn_fwd.h"
#include "attn_launch.h"


namespace attn {

struct RowsParams {
    CacheParams c;
    const void *rows[2];    // k, v (write: read from, read: written to)
    long long st[2], sh[2];   // strides of tokens and heads in elements
    void *pages[2];
    unsigned char *scale[2];
    int slices;             // waves of a group of tokens
};

typedef float f32x8 __attribute__((ext_vector_type(8)));

// the largest magnitude whose multiple of the row's unit the row type can hold: the e4m3 step below 2^16 (fp16), 2^128
template <typename T>
__device__ __forceinline__ constexpr float storable()
{
    return (T)65536.0f == (T)INFINITY ? 61440.f : 0x1.ep+127f;
}

// 8 elements of a row, on their way.  T: row type; E4M3: the pool's kind
template <typename T, bool E4M3>
struct RowPiece {
    typedef T t8 __attribute__((ext_vector_type(8)));
    typedef uint32_t pool_t __attribute__((ext_vector_type(E4M3 ? 2 : 4)));     // in the pool

    // The largest of LPR neighbouring lanes' x, in all of them: exchanges across a pair, a quad, eight and sixteen lanes are part
    // of a vector instruction (through LDS: 58000 positions of 8 heads 89 us, so 86).
    template <int LPR>
    static __device__ __forceinline__ float most(float x)
    {
        auto across = [](float v, auto ctrl) {
            return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true)));
        };
        x = across(x, std::integral_constant<int, 0xb1>{});              // quad_perm 1 0 3 2
        x = across(x, std::integral_constant<int, 0x4e>{});              // quad_perm 2 3 0 1
        x = across(x, std::integral_constant<int, 0x141>{});             // row_half_mirror
        if (LPR > 8)
            x = across(x, std::integral_constant<int, 0x140>{});         // row_mirror
        return LPR > 16 ? fmaxf(x, __shfl_xor(x, 16, 64)) : x;
    }

    // rows -> pool; e4m3: LPR lanes hold the row, its exponent comes back
    template <int LPR>
    static __device__ __forceinline__ pool_t stored(t8 x, int &exponent)
    {
        if constexpr (!E4M3) {
            return __builtin_bit_cast(pool_t, x);
        } else {
            const f32x8 y = __builtin_convertvector(x, f32x8);
            float amp = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                amp = fmaxf(amp, fabsf(y[k]));
            amp = most<LPR>(amp);
            // amp = 1.f * 2^(bits >> 23 - 127), 448 = 1.75 * 2^8
            const int bits = __builtin_bit_cast(int, amp);
            exponent = min(max((bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000), -126), 120);
            const float inv = __builtin_bit_cast(float, (127 - exponent) << 23);
            constexpr float top = storable<T>();
            float z[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                z[k] = fminf(fmaxf(y[k], -top), top) * inv;
            pool_t q;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k], z[4 * k + 1], 0, false);        // to nearest even
                q[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k + 2], z[4 * k + 3], lo, true);
            }
            return q;
        }
    }

    // pool -> rows; scale: the row's exponent byte
    static __device__ __forceinline__ t8 loaded(pool_t q, int scale)
    {
        if constexpr (!E4M3) {
            return __builtin_bit_cast(t8, q);
        } else {
            const float unit = __builtin_amdgcn_ldexpf(1.f, scale - 127);
            f32x8 y;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[k], false), c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[k], true);
                y[4 * k] = a[0] * unit, y[4 * k + 1] = a[1] * unit, y[4 * k + 2] = c[0] * unit, y[4 * k + 3] = c[1] * unit;
            }
            return __builtin_convertvector(y, t8);
        }
    }
};

// Few tokens: a wave has one, and 64 pieces of its rows.  WRITE: rows -> pages, otherwise pages -> rows
template <typename T, int D, bool E4M3, bool WRITE>
__global__ __launch_bounds__(256) void attn_cache_token_kernel(const RowsParams p)
{
    typedef RowPiece<T, E4M3> P;
    typedef typename P::t8 t8;
    typedef typename P::pool_t pool_t;
    constexpr int LPR = D / 8;                          // lanes of a row
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)quotient(wave, p.slices), piece = (int)(wave - (long long)t * p.slices) * 64 + lane;
    if (t >= p.c.T)
        return;
    const int b = p.c.sequence_of(t);
    if (b < 0)
        return;
    const int i = t - p.c.start_of(b), n = p.c.rows_of(b);
    if (i >= n || piece >= 2 * p.c.H_kv * LPR)
        return;
    const int pos = p.c.length_of(b) - n + i;
    const int page = pos < 0 ? -1 : p.c.page_of(b, pos);
    if (WRITE && page < 0)
        return;
    const int r = piece / LPR, column = 8 * (piece % LPR), w = r >= p.c.H_kv, h = r - w * p.c.H_kv;
    t8 *const row = reinterpret_cast<t8 *>(static_cast<T *>(const_cast<void *>(p.rows[w])) + t * p.st[w] + h * p.sh[w] + column);
    const size_t place = p.c.page_row(max(page, 0), h) + (pos & ((1 << p.c.page_log2) - 1));
    pool_t *const at = reinterpret_cast<pool_t *>(static_cast<unsigned char *>(p.pages[w]) + (place * D + column) * (E4M3 ? 1 : 2));
    if (WRITE) {
        int exponent = 0;
        *at = P::template stored<LPR>(*row, exponent);
        if (E4M3 && column == 0)
            p.scale[w][place] = (unsigned char)(exponent + 127);
    } else {
        *row = page < 0 ? t8{} : P::loaded(*at, E4M3 ? p.scale[w][place] : 0);
    }
}

// Many tokens: a wave has eight neighbouring ones and so many of their (tensor, head) rows that they are 8 KB, 128 bytes to a lane.
// (e4m3, written and read: 131000 positions of 8 heads, D = 64, in fours 166 us, in eights 151; 33000 of one, D = 256, in fours
// 31.5, in twos 25.)
constexpr int kRunTokens = 8;
constexpr int run_rows(int D) { return 512 / D; }

template <typename T, int D, bool E4M3, bool WRITE>
__global__ __launch_bounds__(256) void attn_cache_run_kernel(const RowsParams p)
{
    typedef RowPiece<T, E4M3> P;
    typedef typename P::t8 t8;
    typedef typename P::pool_t pool_t;
    constexpr int kRunRows = run_rows(D);
    constexpr int LPR = D / 8, TPI = 64 / LPR, F = kRunTokens / TPI;   // lanes of a row, tokens of an access, accesses of a row
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long run = quotient(wave, p.slices);
    const int t0 = (int)run * kRunTokens, slice = (int)(wave - run * p.slices);
    if (t0 >= p.c.T)
        return;

    // lane k: where token t0 + k lies in the pool (row of head 0), -1: nowhere, -2: it is nobody's
    long long place = -2;
    {
        const int first = p.c.sequence_of(t0);
        int b = -1;
        // the sequences behind the first one start at `next`: one load for 64 of them
        const int next = first >= 0 ? p.c.start_of(min(first + 1 + lane, p.c.B)) : 0;
#pragma unroll
        for (int k = 0; k < kRunTokens; ++k) {
            if (t0 + k >= p.c.T)
                break;
            int of = first;
            if (first >= 0) {
                const unsigned long long begun = __ballot(first + 1 + lane <= p.c.B && next <= t0 + k);
                of = ~begun == 0 ? p.c.sequence_of(t0 + k) : first + __popcll(begun);
                of = of < p.c.B ? of : -1;
            } else {
                of = p.c.sequence_of(t0 + k);
            }
            if (lane == k)
                b = of;
        }
        if (b >= 0) {
            const int i = t0 + lane - p.c.start_of(b), n = p.c.rows_of(b);
            if (i >= 0 && i < n) {
                const int pos = p.c.length_of(b) - n + i;
                const int page = pos < 0 ? -1 : p.c.page_of(b, pos);
                place = page < 0 ? -1 : (long long)p.c.page_row(page, 0) + (pos & ((1 << p.c.page_log2) - 1));
            }
        }
    }
    const int column = 8 * (lane % LPR);
    long long at[F];                                    // of this lane's token in access f
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int from = f * TPI + lane / LPR;
        at[f] = (long long)((uint64_t)(uint32_t)__shfl((int)(place >> 32), from, 64) << 32 | (uint32_t)__shfl((int)place, from, 64));
    }
    auto row_of = [&](int r, int f) {
        const int w = r >= p.c.H_kv, h = r - w * p.c.H_kv;
        const long long t = t0 + f * TPI + lane / LPR;
        return reinterpret_cast<t8 *>(static_cast<T *>(const_cast<void *>(p.rows[w])) + t * p.st[w] + h * p.sh[w] + column);
    };
    auto place_of = [&](int r, int f) -> size_t {
        return (size_t)at[f] + ((size_t)(r - (r >= p.c.H_kv) * p.c.H_kv) << p.c.page_log2);
    };
    auto pool_of = [&](int r, int f) {
        return reinterpret_cast<pool_t *>(static_cast<unsigned char *>(p.pages[r >= p.c.H_kv]) + (place_of(r, f) * D + column) * (E4M3 ? 1 : 2));
    };
    const int r0 = slice * kRunRows, n_rows = 2 * p.c.H_kv;
    t8 x[kRunRows][F];
    pool_t q[kRunRows][F];
    int scale[kRunRows][F];
#pragma unroll
    for (int k = 0; k < kRunRows; ++k)
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int r = min(r0 + k, n_rows - 1);
            if (WRITE && at[f] >= 0) {
                x[k][f] = *row_of(r, f);
            } else if (!WRITE && at[f] >= 0) {
                q[k][f] = *pool_of(r, f);
                if (E4M3)
                    scale[k][f] = p.scale[r >= p.c.H_kv][place_of(r, f)];
            }
        }
    // 16-bit elements are stored past the caches, which so many rows have left before they are read again: 58000 positions of 8
    // heads, D = 128, written in 105 us through them and in 72 past them (6.5 TB/s), read in 109 and 73.  Rows of e4m3 are half as
    // long, and a line of their units is written by several waves: through the caches 87 us, past them 109.
#pragma unroll
    for (int k = 0; k < kRunRows; ++k)
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int r = r0 + k;
            if (r >= n_rows)
                break;
            if (WRITE) {
                int exponent = 0;
                const pool_t y = P::template stored<LPR>(x[k][f], exponent);      // (lanes of a row go the same way)
                if (at[f] >= 0) {
                    if (E4M3)
                        *pool_of(r, f) = y;
                    else
                        __builtin_nontemporal_store(y, pool_of(r, f));
                    if (E4M3 && column == 0)
                        p.scale[r >= p.c.H_kv][place_of(r, f)] = (unsigned char)(exponent + 127);
                }
            } else if (at[f] >= -1) {
                __builtin_nontemporal_store(at[f] < 0 ? t8{} : P::loaded(q[k][f], scale[k][f]), row_of(r, f));
            }
        }
}

}  // namespace attn

namespace {

using attn::RowsParams;

template <typename T, int D, bool E4M3, bool WRITE>
int launch(RowsParams &p, hipStream_t st)
{
    // many tokens, if their runs fill the chip
    const long long runs = ((long long)p.c.T + attn::kRunTokens - 1) / attn::kRunTokens;
    const int row_slices = (2 * p.c.H_kv + attn::run_rows(D) - 1) / attn::run_rows(D);
    const bool many = runs * row_slices >= 1024;
    p.slices = many ? row_slices : (2 * p.c.H_kv * (D / 8) + 63) / 64;
    const long long blocks = ((many ? runs : (long long)p.c.T) * p.slices + 3) / 4;
    if (blocks > attn::most_workgroups(256))
        return ATTN_ERR_SHAPE;
    if (many)
        hipLaunchKernelGGL((attn::attn_cache_run_kernel<T, D, E4M3, WRITE>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((attn::attn_cache_token_kernel<T, D, E4M3, WRITE>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

template <typename T, bool WRITE>
int rows(const void *k, const void *v, const long long *strides, const void *k_pages, const void *v_pages,
         const unsigned char *k_scale, const unsigned char *v_scale, const int *page_table, const int *start,
         const int *kv_len, int kind, int T_rows, int B, int H_kv, int D, int n_pages, int page_size, int table_width,
         void *stream)
{
    if (!k || !v || !strides || !k_pages || !v_pages || !page_table || !start || !kv_len ||
        (kind == ATTN_CACHE_E4M3 && (!k_scale || !v_scale)))
        return ATTN_ERR_NULL;
    if (T_rows < 1 || B < 1 || H_kv < 1 || n_pages < 1 || table_width < 1 || B > attn::kMostSequences)
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    if ((kind != ATTN_CACHE_16BIT && kind != ATTN_CACHE_E4M3) || page_size < 16 || page_size > 256 ||
        (page_size & (page_size - 1)))
        return ATTN_ERR_UNSUPPORTED;
    const long long most = (1LL << 40) / D;
    if ((long long)T_rows * H_kv > most || (long long)n_pages * H_kv > most / page_size || H_kv > (1 << 24) ||
        (long long)table_width * page_size > (1 << 30))
        return ATTN_ERR_SHAPE;
    for (int i = 0; i < 4; ++i) {
        const long long n = i % 2 ? H_kv : T_rows;
        if (n > 1 && (strides[i] < 0 || strides[i] % 8 || strides[i] > (1LL << 40) / n))
            return ATTN_ERR_SHAPE;
    }
    if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) ||
        misaligned(page_table, 4) || misaligned(start, 4) || misaligned(kv_len, 4) ||
        (kind == ATTN_CACHE_E4M3 && (misaligned(k_scale, 16) || misaligned(v_scale, 16))))
        return ATTN_ERR_ALIGN;
    RowsParams p;
    p.c.page_table = page_table, p.c.start = start, p.c.kv_len = kv_len;
    p.c.T = T_rows, p.c.B = B, p.c.H_kv = H_kv, p.c.n_pages = n_pages, p.c.table_width = table_width;
    p.c.page_log2 = __builtin_ctz((unsigned)page_size);
    p.rows[0] = k, p.rows[1] = v;
    for (int w = 0; w < 2; ++w)
        p.st[w] = strides[2 * w], p.sh[w] = strides[2 * w + 1];
    p.pages[0] = const_cast<void *>(k_pages), p.pages[1] = const_cast<void *>(v_pages);
    p.scale[0] = const_cast<unsigned char *>(k_scale), p.scale[1] = const_cast<unsigned char *>(v_scale);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool e4m3 = kind == ATTN_CACHE_E4M3;
    switch (D) {
    case 64: return e4m3 ? launch<T, 64, true, WRITE>(p, st) : launch<T, 64, false, WRITE>(p, st);
    case 128: return e4m3 ? launch<T, 128, true, WRITE>(p, st) : launch<T, 128, false, WRITE>(p, st);
    default: return e4m3 ? launch<T, 256, true, WRITE>(p, st) : launch<T, 256, false, WRITE>(p, st);
    }
}

}  // namespace

#define ATTN_CACHE_ENTRIES(suffix, T)                                                                                        \
    extern "C" int attn_cache_write##suffix(const void *k, const void *v, const long long *strides, void *k_pages,           \
                                            void *v_pages, unsigned char *k_scale, unsigned char *v_scale,                   \
                                            const int *page_table, const int *start, const int *kv_len, int kind,            \
                                            int n_rows, int B, int H_kv, int D, int n_pages, int page_size,                  \
                                            int table_width, void *stream)                                                   \
    {                                                                                                                        \
        return rows<T, true>(k, v, strides, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind, n_rows, B,  \
                             H_kv, D, n_pages, page_size, table_width, stream);                                              \
    }                                                                                                                        \
    extern "C" int attn_cache_read##suffix(void *k, void *v, const long long *strides, const void *k_pages,                  \
                                           const void *v_pages, const unsigned char *k_scale, const unsigned char *v_scale,  \
                                           const int *page_table, const int *start, const int *kv_len, int kind,             \
                                           int n_rows, int B, int H_kv, int D, int n_pages, int page_size, int table_width,  \
                                           void *stream)                                                                     \
    {                                                                                                                        \
        return rows<T, false>(k, v, strides, k_pages, v_pages, k_scale, v_scale, page_table, start, kv_len, kind, n_rows, B, \
                              H_kv, D, n_pages, page_size, table_width, stream);                                             \
    }

ATTN_CACHE_ENTRIES(, __bf16)
ATTN_CACHE_ENTRIES(_f16, _Float16)
