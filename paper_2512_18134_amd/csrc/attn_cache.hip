// attn_cache.hip -- rows of keys and values into the paged cache and back out: kernels and entry points
// (include/attn_cache.h).
//
// Bound by memory, and for the few rows of a decoding step by the chain of dependent loads: start -> kv_len -> page table ->
// row.  A wave works on one token (the chain is uniform and walked once) and on U x 64 sixteen-byte pieces of its heads'
// K and V rows, all in flight together.
//
// e4m3 with a power of two per row: q = round(x * 2^-e) is an exact product and one rounding, so that the quantised value is
// a function of the numbers alone and not of how a division was carried out; against amplitude / 448 as the
// unit it gives up less than one of the format's seventeen binades at the small end.
#include <hip/hip_runtime.h>

#include <math.h>

#include "attn_cache.h"
#include "attn_cache_rows.h"
#include "attn_common.h"
#include "attn_fwd.h"


namespace attn {

struct RowsParams {
    CacheParams c;
    const void *rows[2];    // k, v (write: read from, read: written to)
    long long st[2], sh[2];   // strides of tokens and heads in elements
    void *pages[2];
    unsigned char *scale[2];
    int slices;             // waves of a token
};

template <typename T>
struct Elem8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// the largest magnitude whose multiple of the row's unit the row type can hold: the e4m3 step below 2^16 (fp16), 2^128
template <typename T>
__device__ __forceinline__ constexpr float storable()
{
    return sizeof(T) == 2 && (T)65536.0f == (T)INFINITY ? 61440.f : 0x1.ep+127f;
}

// T: row type; E4M3: the pool's kind; WRITE: rows -> pages, otherwise pages -> rows
template <typename T, int D, bool E4M3, bool WRITE, int U>
__global__ __launch_bounds__(256) void attn_cache_rows_kernel(const RowsParams p)
{
    typedef typename Elem8<T>::type t8;
    constexpr int LPR = D / 8;                     // lanes of a row
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(wave / p.slices), slice = (int)(wave % p.slices);
    if (t >= p.c.T)
        return;
    const int b = p.c.sequence_of(t);
    if (b < 0)
        return;
    const int i = t - p.c.start_of(b), n = p.c.rows_of(b);
    if (i >= n)
        return;
    const int pos = p.c.length_of(b) - n + i;
    const int page = pos < 0 ? -1 : p.c.page_of(b, pos);
    if (WRITE && page < 0)
        return;
    const int place = pos & ((1 << p.c.page_log2) - 1);
    const int pieces = 2 * p.c.H_kv * LPR;
    t8 x[U];
    u32x2 q[U];
    float unit[U];
    const int piece0 = slice * U * 64 + lane;
    auto row_address = [&](int piece) -> T * {
        const int r = piece / LPR, w = r >= p.c.H_kv, h = r - w * p.c.H_kv;
        return static_cast<T *>(const_cast<void *>(p.rows[w])) + t * p.st[w] + h * p.sh[w] + 8 * (piece % LPR);
    };
    auto page_element = [&](int piece, int &w, size_t &row) -> size_t {
        const int r = piece / LPR;
        w = r >= p.c.H_kv;
        row = p.c.page_row(page, r - w * p.c.H_kv) + place;
        return row * D + 8 * (piece % LPR);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int piece = piece0 + 64 * u;
        if (piece >= pieces)
            break;
        if (WRITE) {
            x[u] = *reinterpret_cast<const t8 *>(row_address(piece));
        } else {
            x[u] = t8{};
            q[u] = u32x2{0, 0};
            unit[u] = 1.f;
            if (page >= 0) {
                int w;
                size_t row;
                const size_t e = page_element(piece, w, row);
                if (E4M3) {
                    q[u] = *reinterpret_cast<const u32x2 *>(static_cast<const unsigned char *>(p.pages[w]) + e);
                    // 2^(scale - 127); scale 0 has no normal number and is not written
                    unit[u] = __builtin_amdgcn_ldexpf(1.f, (int)p.scale[w][row] - 127);
                } else {
                    x[u] = *reinterpret_cast<const t8 *>(static_cast<const T *>(p.pages[w]) + e);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int piece = piece0 + 64 * u;
        if (piece >= pieces)
            break;
        if (!WRITE) {
            if (E4M3) {
                f32x8 y;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u][k], false);
                    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[u][k], true);
                    y[4 * k] = a[0] * unit[u], y[4 * k + 1] = a[1] * unit[u];
                    y[4 * k + 2] = c[0] * unit[u], y[4 * k + 3] = c[1] * unit[u];
                }
                x[u] = __builtin_convertvector(y, t8);
            }
            *reinterpret_cast<t8 *>(row_address(piece)) = x[u];
            continue;
        }
        int w;
        size_t row;
        const size_t e = page_element(piece, w, row);
        if (!E4M3) {
            *reinterpret_cast<t8 *>(static_cast<T *>(p.pages[w]) + e) = x[u];
            continue;
        }
        const f32x8 y = __builtin_convertvector(x[u], f32x8);
        float amp = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            amp = fmaxf(amp, fabsf(y[k]));
#pragma unroll
        for (int m = 1; m < LPR; m *= 2)
            amp = fmaxf(amp, __shfl_xor(amp, m, 64));
        // amp = 1.f * 2^(bits >> 23 - 127), 448 = 1.75 * 2^8
        const int bits = __builtin_bit_cast(int, amp);
        const int exponent = min(max((bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000), -126), 120);
        const float inv = __builtin_bit_cast(float, (127 - exponent) << 23);
        constexpr float top = storable<T>();
        float z[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            z[k] = fminf(fmaxf(y[k], -top), top) * inv;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            int d = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k], z[4 * k + 1], 0, false);        // to nearest even
            q[u][k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[4 * k + 2], z[4 * k + 3], d, true);
        }
        *reinterpret_cast<u32x2 *>(static_cast<unsigned char *>(p.pages[w]) + e) = q[u];
        if (piece % LPR == 0)
            p.scale[w][row] = (unsigned char)(exponent + 127);
    }
}

}  // namespace attn

namespace {

using attn::RowsParams;

template <typename T, int D, bool E4M3, bool WRITE>
int launch(RowsParams &p, hipStream_t st)
{
    // pieces of a token, four in flight per lane where there are tokens enough to fill the chip without splitting further
    const int pieces = 2 * p.c.H_kv * (D / 8);
    const bool wide = (long long)p.c.T * ((pieces + 255) / 256) >= 2048;
    p.slices = wide ? (pieces + 255) / 256 : (pieces + 63) / 64;
    const long long blocks = ((long long)p.c.T * p.slices + 3) / 4;
    if (blocks > 0x7fffffffLL)
        return ATTN_ERR_SHAPE;
    if (wide)
        hipLaunchKernelGGL((attn::attn_cache_rows_kernel<T, D, E4M3, WRITE, 4>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((attn::attn_cache_rows_kernel<T, D, E4M3, WRITE, 1>), dim3((unsigned)blocks), dim3(256), 0, st, p);
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
    if (T_rows < 1 || B < 1 || H_kv < 1 || n_pages < 1 || table_width < 1 || B == 0x7fffffff)
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
