// What the kernels over a paged cache share: which sequence a token belongs
// to, and where a position lies.
#pragma once

#include "at_ops.h"

namespace at {

// Division of whole numbers below 2^31 by d (1 <= d < 2^31): with m = ceil(2^(31 + l) / d)
// and l = ceil(log2 d), p / d is the top of p * m, exactly.
struct Divider {
    uint32_t d, m;
    int shift;   // 31 + l
};
inline Divider divider(int64_t d) {
    int l = 0;
    while (((int64_t)1 << l) < d) ++l;
    const unsigned __int128 top = (unsigned __int128)1 << (31 + l);
    return {(uint32_t)d, (uint32_t)((top + (uint64_t)d - 1) / (uint64_t)d), 31 + l};
}
__device__ __forceinline__ uint32_t divided(uint32_t p, const Divider& v) {
    return (uint32_t)(((uint64_t)p * v.m) >> v.shift);
}

// New tokens of a sequence: [first, first + count) of the call's n.
struct Span {
    int first, count;
};
__device__ __forceinline__ Span span_of(const int32_t* starts, int b, int n) {
    const int s = starts[b], e = starts[b + 1];
    const int lo = s < 0 ? 0 : s < n ? s : n, hi = e < 0 ? 0 : e < n ? e : n;
    return {lo, hi > lo ? hi - lo : 0};
}

// The last b of 0 .. batch with of(b) <= i, or -1, where of goes up: 64 places are looked at a step,
// by the lanes of a wave, which all get the answer.
template <class F>
__device__ __forceinline__ int last_upto(int batch, int i, F&& of) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = batch;   // it is in [lo, hi], or none is
    while (true) {
        const int step = (hi - lo) / 64 + 1;
        const int64_t at = lo + (int64_t)lane * step;
        const uint64_t below = __ballot(at <= hi && of((int)(at <= hi ? at : hi)) <= i);
        const int found = below == ~0ull ? 64 : __builtin_ctzll(~below);   // the first `found` places are at most i
        if (found == 0) return lo - 1;                                      // in the first step only: lo is 0
        lo += (found - 1) * step;
        if (step == 1) return lo;
        hi = hi < lo + step - 1 ? hi : lo + step - 1;
    }
}
// The sequence that token i belongs to, if it is in 0 .. batch - 1.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, int i) {
    return last_upto(batch, i, [&](int b) { return starts[b]; });
}

}  // namespace at
