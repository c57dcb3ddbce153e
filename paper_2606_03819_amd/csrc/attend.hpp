// Attention over the paged 8-bit cache: what its kernels share.
#pragma once

#include "attend_split.hpp"
#include "common.hpp"
#include "e4m3.hpp"
#include "launch.hpp"

namespace tf {

constexpr int kAttendThreads = 256;
constexpr int kAttendWaves = kAttendThreads / kWave;
constexpr int kGroupRows = 4;   // most query heads of one position that a workgroup of the row kernel serves

__device__ __forceinline__ int context_of(const AttendArgs& a, int s) {
    return min(max(a.context_len[s], 0), a.max_pages * a.page);
}
__device__ __forceinline__ int new_of(const AttendArgs& a, int s) {
    return a.new_len == nullptr ? a.n : min(max(a.new_len[s], 0), a.n);
}

// The matrix kernel's weights are made 2^kLift as large (at most 2^62, for the
// slack its maximum has; at least 2^-126, which is 2^-182 under the largest), and
// its running maxima are held less kLift.
constexpr int kLift = 56;

// Partials of split contexts: for row r = (s*n + i)*Hq + head and range sp
// the D sums, and behind all of them the running maximum (base 2; of the matrix
// kernel less kLift) and the sum of weights.
__device__ __forceinline__ float* part_sums(const AttendArgs& a, size_t row, int sp, int D) {
    return a.part + ((size_t)sp * a.b * a.n * a.Hq + row) * D;
}
__device__ __forceinline__ float* part_stats(const AttendArgs& a, size_t row, int sp, int D) {
    const size_t rows = (size_t)a.b * a.n * a.Hq;
    return a.part + rows * a.splits * D + ((size_t)sp * rows + row) * 2;
}

__device__ __forceinline__ void store_out(void* out, size_t at, float v, bool bf16) {
    if (bf16) static_cast<uint16_t*>(out)[at] = (uint16_t)f32_to_bf16_bits(v);
    else static_cast<float*>(out)[at] = v;
}

// A finished row: sums over weights (none: zeros and -inf).
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? neg_inf() : (m + __log2f(l)) * kLn2; }

// Blocks of query rows that a key head's positions make, and row tiles a block.
struct TileBlocks {
    int blocks, tiles;
};
TileBlocks tile_blocks(int n, int Hq, int Hkv);
hipError_t launch_attend_tile(const AttendArgs& a, int D, hipStream_t stream);

}  // namespace tf
