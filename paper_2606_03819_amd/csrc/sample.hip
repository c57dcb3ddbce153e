// A token for each row of logits from a given random number (temperature,
// top-k, top-p, min-p).
//
// Tokens rank by (logit desc, id asc); every filter keeps a prefix of that
// order, so the kept set is "keys above a border, and the first few ids of
// those on it".  Weights are integers: w = rint(2^F exp((z - max)/T)) in 64
// bits, F = 62 - bits(V), so that sums are exact in any order of additions
// and a launch's shape cannot change a token.  fp32 sums would not do: a
// draw turns on the borders between up to V running sums, and with V errors
// of 2^-24 one row in a hundred would draw another token.
#include "common.hpp"
#include "launch.hpp"

namespace tf {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / kWave;
constexpr int kSampleTile = 4 * kSampleThreads;   // ids of the draw's first step
constexpr uint32_t kKeyNone = 0x007fffffu;        // -inf's key: that and below is no token
typedef unsigned long long u64;

// A logit's key; NaN (0) ranks with -inf, both zeros are one value.
__device__ __forceinline__ uint32_t logit_key(float z) {
    return z != z ? 0u : f32_key(z == 0.f ? 0.f : z);
}
template <class T>
__device__ __forceinline__ uint32_t key_at(const T* row, int i);
template <>
__device__ __forceinline__ uint32_t key_at<uint16_t>(const uint16_t* row, int i) {
    return logit_key(bf16_bits_to_f32(row[i]));
}
template <>
__device__ __forceinline__ uint32_t key_at<float>(const float* row, int i) { return logit_key(row[i]); }

// One row's scale: weights of keys under its largest.
struct Weigh {
    double top, t;
    double one;   // 2^F
    __device__ double power(uint32_t key) const {
        const double z = (double)key_f32(key);
        const double x = z == top ? 0. : (z - top) / t;
        return x == x ? x : -__builtin_inf();   // from infinite temperatures with infinite logits
    }
    __device__ u64 weight(uint32_t key) const { return key <= kKeyNone ? 0ull : (u64)rint(exp(power(key)) * one); }
};

__device__ __forceinline__ u64 block_max(u64 v, u64* tmp) {
    for (int o = 32; o > 0; o >>= 1) {
        const u64 w = __shfl_xor(v, o);
        v = w > v ? w : v;
    }
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < kSampleWaves; ++w) v = tmp[w] > v ? tmp[w] : v;
    __syncthreads();
    return v;
}
// Exclusive sum over the workgroup's threads.
__device__ __forceinline__ u64 block_before(u64 v, u64* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 sum = v;
    for (int o = 1; o < 64; o <<= 1) {
        const u64 up = __shfl_up(sum, o);
        if (lane >= o) sum += up;
    }
    if (lane == 63) tmp[wave] = sum;
    __syncthreads();
    u64 before = sum - v;
    for (int w = 0; w < wave; ++w) before += tmp[w];
    __syncthreads();
    return before;
}

struct Border {
    uint32_t key;      // kept: keys above it
    uint32_t ties;     // and this many of those on it
    u64 mass;          // weights of the kept
};

// The shortest prefix of the ranking with `target` tokens (BY_MASS false) or
// weights: the row is read once for each byte of the key.
template <class T, bool BY_MASS>
__device__ Border find_border(const T* row, int V, const Weigh& w, u64 target, uint32_t* cnt, u64* mass,
                              u64* s_state) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    u64 above = 0, above_mass = 0;
    for (int level = 0; level < 4; ++level) {
        const int shift = 24 - 8 * level;
        if (tid < 256) cnt[tid] = 0, mass[tid] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kSampleThreads) {
            const uint32_t key = key_at(row, i);
            if (key <= kKeyNone || (level > 0 && (key >> (shift + 8)) != prefix)) continue;
            atomicAdd(&cnt[(key >> shift) & 255], 1u);
            atomicAdd(&mass[(key >> shift) & 255], w.weight(key));
        }
        __syncthreads();
        if (tid == 0) {
            int b = 255;
            for (; b > 0; --b) {
                if ((BY_MASS ? above_mass + mass[b] : above + cnt[b]) >= target) break;
                above += cnt[b];
                above_mass += mass[b];
            }
            s_state[0] = (u64)b;
            s_state[1] = above;
            s_state[2] = above_mass;
            s_state[3] = cnt[b];
        }
        __syncthreads();
        prefix = (prefix << 8) | (uint32_t)s_state[0];
        above = s_state[1];
        above_mass = s_state[2];
        const u64 here = s_state[3];
        __syncthreads();
        if (level == 3) {
            const u64 wk = w.weight(prefix);
            u64 ties = BY_MASS ? (wk > 0 ? (target - above_mass + wk - 1) / wk : here) : target - above;
            ties = ties < here ? ties : here;
            return {prefix, (uint32_t)ties, above_mass + ties * wk};
        }
    }
    return {};
}

// A workgroup a row.
template <class T>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a, int bits) {
    __shared__ uint32_t cnt[256];
    __shared__ u64 mass[256];
    __shared__ u64 tmp[kSampleWaves];
    __shared__ u64 s_state[4];
    __shared__ u64 tile_mass[(1 << 22) / kSampleTile];
    __shared__ uint32_t tile_ties[(1 << 22) / kSampleTile];
    const int tid = threadIdx.x, r = blockIdx.x, s = r / a.n;
    const T* row = static_cast<const T*>(a.logits) + (size_t)r * a.ld;
    const int V = a.V;
    u64 best = 0;
    for (int i = tid; i < V; i += kSampleThreads) {
        const u64 k = (u64)key_at(row, i) << 32 | (uint32_t)~i;
        best = k > best ? k : best;
    }
    best = block_max(best, tmp);
    const uint32_t top = (uint32_t)(best >> 32);
    const float temp = a.temperature != nullptr ? a.temperature[s] : 1.f;
    const float mp = a.min_p != nullptr ? a.min_p[s] : 0.f;
    if (top <= kKeyNone || !(temp > 0.f) || mp > 1.f) {   // no token, or the first one alone
        if (tid == 0) {
            a.token[r] = top <= kKeyNone ? -1 : (int)~(uint32_t)best;
            if (a.logprob != nullptr) a.logprob[r] = top <= kKeyNone ? neg_inf() : 0.f;
        }
        return;
    }
    const Weigh w{(double)key_f32(top), (double)temp, ldexp(1., bits)};
    const int k = a.top_k != nullptr ? a.top_k[s] : 0;
    const float p = a.top_p != nullptr ? a.top_p[s] : 1.f;
    Border kept{0, 0, 0};
    bool whole = true;
    if (k > 0 && k < V) {
        kept = find_border<T, false>(row, V, w, (u64)k, cnt, mass, s_state);
        whole = false;
    }
    if (p < 1.f) {
        if (whole) {
            u64 z = 0;
            for (int i = tid; i < V; i += kSampleThreads) z += w.weight(key_at(row, i));
            const u64 before = block_before(z, tmp);
            if (tid == kSampleThreads - 1) s_state[0] = before + z;
            __syncthreads();
            kept.mass = s_state[0];
            __syncthreads();
        }
        const double want = ceil((double)p * (double)kept.mass);
        kept = find_border<T, true>(row, V, w, want > 1. ? (u64)want : 1ull, cnt, mass, s_state);
        whole = false;
    }
    const u64 tie_w = whole ? 0 : w.weight(kept.key);
    const bool tie_ok = mp <= 0.f || mp != mp || exp(w.power(kept.key)) >= (double)mp;
    // weight of a key that lies above the border
    auto weight = [&](uint32_t key) -> u64 {
        if (key <= kKeyNone || (!whole && key <= kept.key)) return 0;
        if (mp > 0.f && !(exp(w.power(key)) >= (double)mp)) return 0;
        return w.weight(key);
    };
    const int tiles = (V + kSampleTile - 1) / kSampleTile;
    for (int t = tid; t < tiles; t += kSampleThreads) tile_mass[t] = 0, tile_ties[t] = 0;
    __syncthreads();
    for (int i = tid; i < V; i += kSampleThreads) {
        const uint32_t key = key_at(row, i);
        const u64 x = weight(key);
        if (x != 0) atomicAdd(&tile_mass[i / kSampleTile], x);
        else if (!whole && key == kept.key && tie_ok) atomicAdd(&tile_ties[i / kSampleTile], 1u);
    }
    __syncthreads();
    if (tid == 0) {
        u64 total = 0, left = kept.ties;
        for (int t = 0; t < tiles; ++t) {
            const u64 take = tile_ties[t] < left ? tile_ties[t] : left;
            left -= take;
            total += tile_mass[t] + take * tie_w;
        }
        float u = a.uniform[r];
        u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
        const u64 target = (u64)((double)u * (double)total);
        u64 sum = 0;
        left = kept.ties;
        int t = 0;
        for (; t < tiles - 1; ++t) {
            const u64 take = tile_ties[t] < left ? tile_ties[t] : left;
            const u64 here = tile_mass[t] + take * tie_w;
            if (sum + here > target) break;
            sum += here;
            left -= take;
        }
        s_state[0] = (u64)t;
        s_state[1] = target - sum;
        s_state[2] = left;
        s_state[3] = total;
    }
    __syncthreads();
    const u64 target = s_state[1], left = s_state[2], total = s_state[3];
    const int i0 = (int)s_state[0] * kSampleTile + tid * 4;
    uint32_t key[4];
    u64 x[4], ties = 0, sum = 0;
    for (int j = 0; j < 4; ++j) {
        key[j] = i0 + j < V ? key_at(row, i0 + j) : 0u;
        x[j] = weight(key[j]);
        ties += x[j] == 0 && !whole && key[j] == kept.key && key[j] > kKeyNone && tie_ok ? 1 : 0;
    }
    u64 tie_at = block_before(ties, tmp);
    for (int j = 0; j < 4; ++j) {
        if (x[j] == 0 && !whole && key[j] == kept.key && key[j] > kKeyNone && tie_ok && tie_at++ < left) x[j] = tie_w;
        sum += x[j];
    }
    u64 at = block_before(sum, tmp);
    for (int j = 0; j < 4; ++j) {
        if (at <= target && target < at + x[j]) {
            a.token[r] = i0 + j;
            if (a.logprob != nullptr) a.logprob[r] = (float)(w.power(key[j]) - log((double)total / w.one));
        }
        at += x[j];
    }
}

size_t sample_ws_bytes(long long rows, int V) { return 0; }

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t stream) {
    int bits = 62;
    for (int v = a.V; v > 0; v >>= 1) --bits;
    if (bf16) hipLaunchKernelGGL(sample_row_kernel<uint16_t>, dim3(a.rows), dim3(kSampleThreads), 0, stream, a, bits);
    else hipLaunchKernelGGL(sample_row_kernel<float>, dim3(a.rows), dim3(kSampleThreads), 0, stream, a, bits);
    return hipGetLastError();
}

}  // namespace tf
