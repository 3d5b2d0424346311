// attn_rope.hip -- rotary positions: kernel and entry points (include/attn_rope.h).
//
// Bound by memory: every element is read and written once.  8192 tokens of 40 heads, D = 128: 30.1 us, 5.6 TB/s; 64 tokens: 4.4
// us, one: 4.2, the latency of a launch that loads, turns and stores.  What has to be kept off that path is the sine and cosine of
// a far position's angle, some hundred instructions with the reduction in 64 bits: a lane owns eight pairs of one
// token, forms their sines and cosines once and walks over heads with them.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_cache_rows.h"   // quotient
#include "attn_fwd.h"
#include "attn_launch.h"   // most_workgroups
#include "attn_rope.h"

namespace attn {

struct RopeParams {
    const void *x[2];       // q, k
    void *y[2];
    long long sx[2][3], sy[2][3];   // strides of b, h, s in elements
    const int *pos;
    const double *freq;
    int section_end[4];     // first pair behind each axis' section (the last one: R/2)
    long long tokens;       // B * S
    int S, H_q, H_all;      // H_all: heads of q and k together
    int D, R;
    int lanes_log2;         // lanes of a token: enough for R/2 pairs at eight each, a power of two
    int heads_per_wave, head_groups;
    float sign;             // -1: inverse
};

// element type -> vectors of 8 and the conversions
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8)));
};

// A wave holds 64 >> lanes_log2 neighbouring tokens; of a token's head lane c turns the pairs 8c .. 8c+7 (two 16-byte
// loads) and copies chunks c, c + lanes, ... of the elements behind R.
// PAST: stored past the caches, where the outputs would not stay in them until they are read (see rope below).
template <typename T, bool INTERLEAVED, bool PAST>
__global__ __launch_bounds__(256) void attn_rope_kernel(const RopeParams p)
{
    typedef typename Vec8<T>::type t8;
    typedef float f8 __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long group = quotient(wave, p.head_groups);
    const int head0 = (int)(wave - group * p.head_groups) * p.heads_per_wave;
    // (lanes behind the last token go along with it and store nothing: a wave of eight lanes or fewer took 4 us longer)
    const long long own = (group << (6 - p.lanes_log2)) + (lane >> p.lanes_log2), token = own < p.tokens ? own : p.tokens - 1;
    const bool mine = own < p.tokens;
    const int c = lane & ((1 << p.lanes_log2) - 1);
    if (group << (6 - p.lanes_log2) >= p.tokens)
        return;
    const int half = p.R >> 1;
    const bool turns = 8 * c < half;
    const long long b = p.tokens == p.S ? 0 : quotient(token, p.S), s = token - b * p.S;
    const int head_end = min(head0 + p.heads_per_wave, p.H_all);
    const int first = INTERLEAVED ? 16 * c : 8 * c, second = INTERLEAVED ? 16 * c + 8 : half + 8 * c;
    // U heads at a time, all their loads before their stores (which the compiler must take for aliases); the first ones' before
    // the sines and cosines, since a small call is a chain of latencies (2 x 777 tokens of 20 heads 5.6 us, behind them 5.9),
    // but not in a large one, where other waves fill the wait (4 x 4096 tokens of 32 heads there and back, other tensors every time:
    // 101 us, before them 114)
    constexpr int U = 4;
    t8 lo[U], hi[U];
    T *out[U];
    auto load = [&](int head) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int at = min(head + j, head_end - 1);
            const int w = at >= p.H_q, h = w ? at - p.H_q : at;
            const T *x = static_cast<const T *>(p.x[w]) + b * p.sx[w][0] + h * p.sx[w][1] + s * p.sx[w][2];
            out[j] = static_cast<T *>(p.y[w]) + b * p.sy[w][0] + h * p.sy[w][1] + s * p.sy[w][2];
            if (turns) {
                lo[j] = *reinterpret_cast<const t8 *>(x + first);
                hi[j] = *reinterpret_cast<const t8 *>(x + second);
            }
            if (head + j < head_end && x != out[j] && mine)
                for (int e = p.R + 8 * c; e < p.D; e += 8 << p.lanes_log2)
                    *reinterpret_cast<t8 *>(out[j] + e) = *reinterpret_cast<const t8 *>(x + e);
        }
    };
    if (!PAST)
        load(head0);
    f8 cs, sn;
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = 8 * c + i;
            int axis = 0;
#pragma unroll
            for (int a = 0; a < 3; ++a)
                axis += pair >= p.section_end[a];
            const double turn = (double)p.pos[axis * p.tokens + token] * (p.freq[pair] * 0.15915494309189533577);
            float s1, c1;
            sincospif(2.f * (float)(turn - rint(turn)), &s1, &c1);
            cs[i] = c1;
            sn[i] = p.sign * s1;
        }
    }
    for (int head = head0;;) {
        if (PAST)
            load(head);
#pragma unroll
        for (int j = 0; j < U && turns; ++j) {
            const f8 u = __builtin_convertvector(lo[j], f8), v = __builtin_convertvector(hi[j], f8);
            f8 a, d;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (INTERLEAVED) {   // lo: pairs 0-3, hi: pairs 4-7 of this lane
                    const f8 &z = i < 4 ? u : v;
                    f8 &r = i < 4 ? a : d;
                    const float x1 = z[2 * (i & 3)], x2 = z[2 * (i & 3) + 1];
                    r[2 * (i & 3)] = x1 * cs[i] - x2 * sn[i];
                    r[2 * (i & 3) + 1] = x1 * sn[i] + x2 * cs[i];
                } else {
                    a[i] = u[i] * cs[i] - v[i] * sn[i];
                    d[i] = u[i] * sn[i] + v[i] * cs[i];
                }
            }
            if (head + j < head_end && mine) {
                const t8 ya = __builtin_convertvector(a, t8), yd = __builtin_convertvector(d, t8);      // to nearest even
                if (PAST) {
                    __builtin_nontemporal_store(ya, reinterpret_cast<t8 *>(out[j] + first));
                    __builtin_nontemporal_store(yd, reinterpret_cast<t8 *>(out[j] + second));
                } else {
                    *reinterpret_cast<t8 *>(out[j] + first) = ya;
                    *reinterpret_cast<t8 *>(out[j] + second) = yd;
                }
            }
        }
        head += U;
        if (head >= head_end)
            break;
        if (!PAST)
            load(head);
    }
}

}  // namespace attn

namespace {

bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

template <typename T>
int rope(const void *q, void *q_out, const void *k, void *k_out, const long long *strides, const int *pos,
         const double *freq, const int *sections, int n_axes, int B, int H_q, int H_kv, int S, int D, int interleaved,
         int inverse, void *stream)
{
    if (!q || !q_out || !strides || !pos || !freq || !sections || (H_kv > 0 && (!k || !k_out)))
        return ATTN_ERR_NULL;
    if (B < 1 || H_q < 1 || H_kv < 0 || S < 1 || n_axes < 1 || n_axes > 4)
        return ATTN_ERR_SHAPE;
    if (D != 64 && D != 128 && D != 256)
        return ATTN_ERR_UNSUPPORTED_D;
    attn::RopeParams p;
    long long pairs = 0;
    for (int a = 0; a < 4; ++a) {
        if (a < n_axes) {
            if (sections[a] < 0 || sections[a] > D)
                return ATTN_ERR_SHAPE;
            pairs += sections[a];
        }
        p.section_end[a] = (int)pairs;
    }
    if (pairs < 8 || pairs % 8 || 2 * pairs > D)
        return ATTN_ERR_SHAPE;
    const long long tokens = (long long)B * S, heads = (long long)H_q + H_kv;
    if (tokens > 0x7fffffffLL || heads > 0x7fffffffLL || tokens * heads > (1LL << 40) / D)
        return ATTN_ERR_SHAPE;
    const int extent[3] = {B, 0, S};
    for (int i = 0; i < (H_kv ? 12 : 6); ++i) {
        const long long n = i % 3 == 1 ? (i < 6 ? H_q : H_kv) : extent[i % 3];
        if (n > 1 && (strides[i] < 0 || strides[i] % 8 || strides[i] > (1LL << 40) / n))
            return ATTN_ERR_SHAPE;
    }
    if (misaligned(q, 16) || misaligned(q_out, 16) || (H_kv && (misaligned(k, 16) || misaligned(k_out, 16))) ||
        misaligned(pos, 4) || misaligned(freq, 8))
        return ATTN_ERR_ALIGN;
    p.x[0] = q, p.x[1] = H_kv ? k : q;
    p.y[0] = q_out, p.y[1] = H_kv ? k_out : q_out;
    for (int w = 0; w < 2; ++w)
        for (int i = 0; i < 3; ++i) {
            p.sx[w][i] = w && !H_kv ? 0 : strides[6 * w + i];
            p.sy[w][i] = w && !H_kv ? 0 : strides[6 * w + 3 + i];
        }
    p.pos = pos, p.freq = freq;
    p.tokens = tokens;
    p.S = S, p.H_q = H_q, p.H_all = (int)heads;
    p.D = D, p.R = (int)(2 * pairs);
    p.lanes_log2 = 0;
    while ((8 << p.lanes_log2) < pairs)
        ++p.lanes_log2;
    p.sign = inverse ? -1.f : 1.f;
    // A wave's sines and cosines serve its heads, at the price of fewer waves: as many heads as leave 16 waves to a
    // compute unit, which few tokens never do.
    const long long groups = ((tokens << p.lanes_log2) + 63) / 64;
    p.heads_per_wave = 1;
    while (p.heads_per_wave < 16 && p.heads_per_wave < heads && groups * ((heads + 2 * p.heads_per_wave - 1) / (2 * p.heads_per_wave)) >= 4096)
        p.heads_per_wave *= 2;
    p.head_groups = (int)((heads + p.heads_per_wave - 1) / p.heads_per_wave);
    const long long blocks = (groups * p.head_groups + 3) / 4;
    if (blocks > attn::most_workgroups(256))
        return ATTN_ERR_SHAPE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // Outputs that the 256 MB of the last-level cache do not hold next to the inputs are stored past the caches: forward and back
    // of 4 x 32 heads of 4096 tokens, D = 128, the same tensors again and again, 110 us through them, 93 past them (102 to 106 on
    // tensors that change); 16 heads of 16384, D = 64 (34 MB), 15.0 and 16.0.
    const bool past = tokens * heads * D * 2 > (64LL << 20);
    const dim3 grid((unsigned)blocks), threads(256);
    if (interleaved && past)
        hipLaunchKernelGGL((attn::attn_rope_kernel<T, true, true>), grid, threads, 0, st, p);
    else if (interleaved)
        hipLaunchKernelGGL((attn::attn_rope_kernel<T, true, false>), grid, threads, 0, st, p);
    else if (past)
        hipLaunchKernelGGL((attn::attn_rope_kernel<T, false, true>), grid, threads, 0, st, p);
    else
        hipLaunchKernelGGL((attn::attn_rope_kernel<T, false, false>), grid, threads, 0, st, p);
    return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_ERR_LAUNCH;
}

}  // namespace

extern "C" int attn_rope(const void *q, void *q_out, const void *k, void *k_out, const long long *strides, const int *pos,
                         const double *freq, const int *sections, int n_axes, int B, int H_q, int H_kv, int S, int D,
                         int interleaved, int inverse, void *stream)
{
    return rope<__bf16>(q, q_out, k, k_out, strides, pos, freq, sections, n_axes, B, H_q, H_kv, S, D, interleaved, inverse,
                        stream);
}

extern "C" int attn_rope_f16(const void *q, void *q_out, const void *k, void *k_out, const long long *strides, const int *pos,
                             const double *freq, const int *sections, int n_axes, int B, int H_q, int H_kv, int S, int D,
                             int interleaved, int inverse, void *stream)
{
    return rope<_Float16>(q, q_out, k, k_out, strides, pos, freq, sections, n_axes, B, H_q, H_kv, S, D, interleaved, inverse,
                          stream);
}
