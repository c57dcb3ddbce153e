// The ranges that the attention splits a context into (device and host code).
#pragma once

#include <hip/hip_runtime.h>

namespace tf {

// A context of `ctx` tokens in at most `most` ranges, one for every kSplitLeast
// tokens or fewer, each a multiple of 64 but the last.  Neither a range's end nor the sum
// that finds their number may pass 2^31 for contexts just below it.
constexpr int kSplitLeast = 256, kMostSplits = 64;
struct Split {
    int chunk, count;
    __host__ __device__ int begin(int range) const { return range * chunk; }
    __host__ __device__ int end(int range, int ctx) const {
        const int lo = begin(range);
        return ctx - lo > chunk ? lo + chunk : ctx;
    }
};
__host__ __device__ inline Split split_context(int ctx, int most) {
    if (ctx < 1) return {64, 1};
    int e = (ctx - 1) / kSplitLeast + 1;
    e = e < most ? e : most;
    e = e > 1 ? e : 1;
    const int chunk = ((ctx - 1) / e + 1 + 63) & ~63;
    return {chunk, (ctx - 1) / chunk + 1};
}

}  // namespace tf
