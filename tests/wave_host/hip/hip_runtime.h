// Device code of the library as host code: a wave is 64 coroutines that take turns at every exchange between lanes.
// Only what the headers under test use.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>

#define __device__
#define __host__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)

struct int2 {
    int x, y;
};
struct int4 {
    int x, y, z, w;
};
struct Dim {
    unsigned x;
};

namespace wave_host {
constexpr int kLanes = 64;
inline ucontext_t scheduler, lanes[kLanes];
inline int current;
inline uint64_t slots[2][kLanes];
inline int turn[kLanes];
inline bool done[kLanes];
inline void *exchange(uint64_t x)      // all lanes' values, once every lane has come here
{
    const int t = turn[current]++ & 1, me = current;
    slots[t][me] = x;
    swapcontext(&lanes[me], &scheduler);
    current = me;
    return slots[t];
}
template <typename T>
T shuffle(T x, int from)
{
    uint64_t bits = 0;
    memcpy(&bits, &x, sizeof x);
    const uint64_t *all = static_cast<uint64_t *>(exchange(bits));
    memcpy(&x, &all[from & (kLanes - 1)], sizeof x);
    return x;
}
typedef void (*Body)(int lane);
inline Body body;
inline void entry(int lane)
{
    body(lane);
    done[lane] = true;
    swapcontext(&lanes[lane], &scheduler);
}
// one wave through `f`; every lane has to reach the same exchanges
inline bool run(Body f)
{
    static char stacks[kLanes][64 * 1024];
    body = f;
    for (int i = 0; i < kLanes; ++i) {
        getcontext(&lanes[i]);
        lanes[i].uc_stack.ss_sp = stacks[i];
        lanes[i].uc_stack.ss_size = sizeof stacks[i];
        lanes[i].uc_link = &scheduler;
        turn[i] = 0, done[i] = false;
        makecontext(&lanes[i], (void (*)())entry, 1, i);
    }
    for (;;) {
        int ended = 0;
        for (int i = 0; i < kLanes; ++i)
            if (!done[i]) {
                current = i;
                swapcontext(&scheduler, &lanes[i]);
            }
        for (int i = 0; i < kLanes; ++i)
            ended += done[i];
        if (ended)
            return ended == kLanes;      // false: the lanes went different ways
    }
}
struct LaneIndex {
    struct X {
        unsigned base;
        operator unsigned() const { return base + current; }
    } x;
};
}  // namespace wave_host

inline wave_host::LaneIndex threadIdx = {{0}};
inline Dim blockIdx = {0}, gridDim = {1};

using std::max;
using std::min;
template <typename T>
T __shfl_xor(T x, int m, int) { return wave_host::shuffle(x, wave_host::current ^ m); }
template <typename T>
T __shfl_up(T x, int m, int) { return wave_host::shuffle(x, wave_host::current >= m ? wave_host::current - m : wave_host::current); }
inline unsigned long long __ballot(bool b)
{
    const uint64_t *all = static_cast<uint64_t *>(wave_host::exchange(b));
    unsigned long long r = 0;
    for (int i = 0; i < 64; ++i)
        r |= (unsigned long long)(all[i] != 0) << i;
    return r;
}
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
inline void __syncthreads() {}
inline int __ffsll(unsigned long long x) { return __builtin_ffsll(x); }
// the lane exchanges that a prefix sum is made of: row_shr 1 .. 8, row_bcast 15 and 31; lanes without a source keep `old`
inline int update_dpp(int old, int x, int ctrl, int rows, int, bool)
{
    const uint64_t *all = static_cast<uint64_t *>(wave_host::exchange((unsigned)x));
    const int lane = wave_host::current, row = lane / 16;
    int from = -1;
    if (ctrl > 0x110 && ctrl < 0x120)
        from = lane % 16 >= ctrl - 0x110 ? lane - (ctrl - 0x110) : -1;
    else if (ctrl == 0x142)
        from = row > 0 ? row * 16 - 1 : -1;
    else if (ctrl == 0x143)
        from = row > 1 ? 31 : -1;
    return from < 0 || !(rows >> row & 1) ? old : (int)all[from];
}
#define __builtin_amdgcn_update_dpp update_dpp
inline float rcpf(float x) { return 1.f / x; }
#define __builtin_amdgcn_rcpf rcpf
#define __builtin_amdgcn_readlane(x, l) wave_host::shuffle(x, l)
#define __builtin_amdgcn_readfirstlane(x) wave_host::shuffle(x, 0)
