// attn_cache_rows.h -- what the kernels over the paged cache share: who a row belongs to, where a position lies.
//
// The lengths, starts and page numbers are device memory that the host never sees, so every one of them is brought into
// range where it is read: whatever the arrays hold, no access leaves the tensors.
#pragma once
#include <hip/hip_runtime.h>

#include "attn_common.h"

namespace attn {

// a / b for a >= 0, b > 0.  The compiler's division is a chain of some 30 instructions, and the plan of attn_paged_plan.h has a dozen of them
// in a row; below 2^22 a reciprocal's quotient is off by one at most.
__device__ __forceinline__ int quotient(int a, int b)
{
    if (a >= 1 << 22)
        return a / b;
    const int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b)), r = a - q * b;
    return q + (r >= b) - (r < 0);
}
// The same of a count that may pass 32 bits (the compiler's 64-bit division is some 100 instructions).
__device__ __forceinline__ long long quotient(long long a, int b) { return a < 1 << 22 ? quotient((int)a, b) : a / b; }

// Sequences of a call, at most: the kernels count them in steps of up to 1024 lanes, which have to stay below 2^31.
constexpr int kMostSequences = 1 << 30;

struct CacheParams {
    const int *page_table, *start, *kv_len;
    int T, B, H_kv;
    int n_pages, page_log2, table_width;

    __device__ __forceinline__ int start_of(int b) const { return min(max(start[b], 0), T); }
    // new rows and cached positions of sequence b
    __device__ __forceinline__ int rows_of(int b) const { return max(start_of(b + 1) - start_of(b), 0); }
    __device__ __forceinline__ int length_of(int b) const
    {
        const long long most = (long long)table_width << page_log2;
        return (int)min((long long)max(kv_len[b], 0), most);
    }
    // page of position `pos` (0 <= pos < length_of(b)), or -1
    __device__ __forceinline__ int page_of(int b, int pos) const
    {
        const int id = page_table[(size_t)b * table_width + (pos >> page_log2)];
        return (unsigned)id < (unsigned)n_pages ? id : -1;
    }
    // first row of (page, h) in units of rows of D elements
    __device__ __forceinline__ size_t page_row(int page, int h) const { return ((size_t)page * H_kv + h) << page_log2; }

    // The sequence that row t belongs to (the last one that starts at or before t), -1: none.  The whole wave asks for one t:
    // 64 starts are compared at a time, so 63 sequences take one memory latency, 4000 two, instead of the
    // logarithm's six and twelve.  (Starts that decrease: some sequence, with bounds that the caller checks.)
    __device__ __forceinline__ int sequence_of(int t) const
    {
        const int lane = threadIdx.x & 63;
        int lo = 0, n = B + 1;                 // the last start <= t is one of lo .. lo + n - 1, if any is
        while (n > 64) {
            const int step = (n + 63) / 64;
            const int i = lo + min(lane * step, n - 1);
            const int below = __popcll(__ballot(start_of(i) <= t && lane * step < n));
            if (below == 0)
                return -1;
            const int next = (below - 1) * step;
            lo += next;
            n = min(step, n - next);
        }
        const int below = __popcll(__ballot(lane < n && start_of(lo + min(lane, n - 1)) <= t));
        const int b = lo + below - 1;
        return below == 0 || b >= B ? -1 : b;
    }
};

}  // namespace attn
