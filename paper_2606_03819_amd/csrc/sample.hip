// A token for each row of logits from a given random number (temperature,
// top-k, top-p, min-p).
//
// Tokens rank by (logit desc, id asc); every filter keeps a prefix of that
// order, so the kept set is "keys above a border, and the first few ids of
// those on it".  Sums are exact far beyond fp32, as integers or in 64 bits: a
// draw turns on the borders between up to V running sums, and with V errors
// of 2^-24 one row in a hundred would draw another token.  A weight's own error
// is at most 2^-46 of the largest, or half a unit of the integers, 2^(bits of V
// - 63), if that is more.  Whatever is added by atomics is an integer, so that
// the order of additions changes nothing.
//
// Two launches.  scan_kernel reads the logits once, a slice of 8192 at a
// time, and leaves what the row's settings need:
//   few   (top-k of at most 64, or the largest alone) -- of each 2048 logits
//         the ones that can be among the row's best k;
//   whole (else) -- masses of the slice by the value's distance from its
//         largest, in steps of 1/16.
// pick_kernel joins a row's slices.  `few` rows are ranked by waves, 64 entries
// at a time.  For `whole` rows the steps' masses give each filter's border to
// one step; the tokens of that step alone are looked up again and selected
// among, and once the border is known the slices' masses give the slice that
// the draw falls into, which is walked token by token.  Rows that this cannot
// serve are read once for each byte of their keys instead (hard_row): `whole`
// rows whose largest 16 |z| / T is 2^20 or more (an infinite logit; T below 3e-4
// at a logit of 20), or with more than 6144 tokens in a border's step; `few`
// rows whose lists leave more than 8064 entries (thousands of ties in 64 lists
// or more).
//
// Measured: 528 rows of 151936 bf16 with settings of all kinds 76 us of scan
// (2.1 TB/s; bound by 64-bit arithmetic, vector instructions issue in 65% of its
// cycles, and LDS atomics) and 80 of pick (each row's chain of filters, and the
// second read: its waves wait 62% of the time); one row with top-k 20: 5.5 and
// 9.7.  A pick is one workgroup a row, so that few rows with a filter but no
// small top-k take nearly what many do: one row with top-p 56 us a call, 64 rows
// 69.
#include "common.hpp"
#include "launch.hpp"

namespace tf {

constexpr int kSampleThreads = 512;
constexpr int kSampleWaves = kSampleThreads / kWave;
constexpr int kSampleTile = 4096;   // ids of the draw's first step
constexpr int kTileEach = kSampleTile / kSampleThreads;
constexpr int kSlice = 8192;                      // logits a workgroup of the scan reads
constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / kWave;
constexpr int kChunk = kSlice / kScanWaves;       // of a wave
constexpr int kFew = 64;                          // tokens that one wave ranks
constexpr int kList = 128;                        // of a chunk, entries kept
constexpr int kSteps = 512;                       // of 1/16: e^-32 of the largest (2^-46) counts as no weight
constexpr int kPerUnit = 16;
// Entries of a row's lists that are ranked in LDS: all of them where the row has
// no more than 63 lists, which cannot be bounded for top-k 64 by their largest
// alone (with 2048, top-k 50 of 50257 logits went to hard_row: four rows 211
// us, 23 now).
constexpr int kSurvivors = (kFew - 1) * kList;
// Tokens of a border's step that LDS holds beside a second workgroup of its CU
// (which registers allow): all of a step wherever the logits over T spread by
// 0.6 or more in 150 thousand.  A list of 2048 sent rows of spread 1 to
// hard_row: one row 714 us, 72 now; 528 rows 1824, 226 now.
constexpr int kBorderList = 6144;
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

// What one sequence asks for.
struct RowSettings {
    float t, p, mp;
    int k;
    // most tokens a row of them keeps, when that is few (0: it is not)
    __device__ int few(int V) const {
        if (!(t > 0.f) || mp > 1.f) return 1;
        const int n = k > 0 ? min(k, V) : V;
        return n <= kFew ? n : 0;
    }
};
__device__ __forceinline__ RowSettings settings_of(const SampleArgs& a, int r) {
    const int s = r / a.n;
    const float t = a.temperature != nullptr ? a.temperature[s] : 1.f;
    // beyond 1e30 the weights are flat already, and z / T must not become 0 * inf
    return {t > 0.f ? fminf(t, 1e30f) : 0.f, a.top_p != nullptr ? a.top_p[s] : 1.f,
            a.min_p != nullptr ? a.min_p[s] : 0.f, a.top_k != nullptr ? a.top_k[s] : 0};
}
// A random number as the draw takes it: within [0, 1 - 2^-24].
__device__ __forceinline__ double unit(float u) { return u > 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.; }

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

struct HardShared {
    uint32_t cnt[256];
    u64 mass[256];
    u64 tile_mass[(1 << 22) / kSampleTile];
    uint32_t tile_ties[(1 << 22) / kSampleTile];
};

// A row whose weights are w = rint(2^bits exp((z - max)/T)) in 64 bits; it has
// a token, and more than the largest may be kept.
template <class T>
__device__ __noinline__ void hard_row(const SampleArgs& a, const RowSettings& set, uint32_t top, int bits,
                                      HardShared& sh, u64* tmp, u64* s_state) {
    uint32_t* cnt = sh.cnt;
    u64* mass = sh.mass;
    u64* tile_mass = sh.tile_mass;
    uint32_t* tile_ties = sh.tile_ties;
    const int tid = threadIdx.x, r = blockIdx.x;
    const T* row = static_cast<const T*>(a.logits) + (size_t)r * a.ld;
    const int V = a.V;
    const Weigh w{(double)key_f32(top), (double)set.t, ldexp(1., bits)};
    const int k = set.k;
    const float p = set.p, mp = set.mp;
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
        const u64 target = (u64)(unit(a.uniform[r]) * (double)total);
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
    const int i0 = (int)s_state[0] * kSampleTile + tid * kTileEach;
    uint32_t key[kTileEach];
    u64 x[kTileEach], ties = 0, sum = 0;
#pragma unroll
    for (int j = 0; j < kTileEach; ++j) {
        key[j] = i0 + j < V ? key_at(row, i0 + j) : 0u;
        x[j] = weight(key[j]);
        ties += x[j] == 0 && !whole && key[j] == kept.key && key[j] > kKeyNone && tie_ok ? 1 : 0;
    }
    u64 tie_at = block_before(ties, tmp);
#pragma unroll
    for (int j = 0; j < kTileEach; ++j) {
        if (x[j] == 0 && !whole && key[j] == kept.key && key[j] > kKeyNone && tie_ok && tie_at++ < left) x[j] = tie_w;
        sum += x[j];
    }
    u64 at = block_before(sum, tmp);
#pragma unroll
    for (int j = 0; j < kTileEach; ++j) {
        if (at <= target && target < at + x[j]) {
            a.token[r] = i0 + j;
            if (a.logprob != nullptr) a.logprob[r] = (float)(w.power(key[j]) - log((double)total / w.one));
        }
        at += x[j];
    }
}

// ------------------------------------------------------------------ the scan

// What the scan leaves of a slice (workspace, one for each row and slice).
struct SliceHead {
    int top;       // whole: step of the slice's largest
    int used;      // whole: steps that hold anything
    float largest; // -inf: no token
    int unused;
};
struct ChunkList {
    float largest;
    int count;
    u64 entry[kList];   // key << 32 | ~id
};
struct SliceData {
    SliceHead head;
    union {
        struct {
            u64 mass[kSteps];
            uint32_t count[kSteps];
        };
        ChunkList few[kScanWaves];
    };
};

// Logit e of a 16-byte vector.
template <class T>
__device__ __forceinline__ float vector_at(const u32x4& x, int e) {
    if (sizeof(T) == 4) return __uint_as_float(x[e & 3]);
    return __uint_as_float(e & 1 ? x[(e >> 1) & 3] & 0xffff0000u : x[(e >> 1) & 3] << 16);
}

// Vectors of 16 bytes that a lane holds of a chunk; the row is read from the
// 16-byte boundary at or before its first logit, `skip` logits earlier.
template <class T>
struct Chunk {
    static constexpr int kPer = 16 / sizeof(T);
    static constexpr int kVecs = kChunk / (kWave * kPer);
    u32x4 raw[kVecs];
    __device__ static int skip_of(const T* row) { return (int)(reinterpret_cast<uintptr_t>(row) / sizeof(T) % kPer); }
    // logits [first, first + kChunk) counted from the boundary; what is no
    // logit of the row becomes NaN
    __device__ void load(const T* row, int skip, int V, int first) {
        const int lane = threadIdx.x & 63, end = V + skip;
        const u32x4* p = reinterpret_cast<const u32x4*>(row - skip);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = first + (i * kWave + lane) * kPer;
            raw[i] = u32x4{~0u, ~0u, ~0u, ~0u};
            if (at < end) raw[i] = p[at / kPer];
        }
        if (first >= skip && first + kChunk <= end) return;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const int at = first + (i * kWave + lane) * kPer + e;
                if (at >= skip && at < end) continue;
                if (sizeof(T) == 4) raw[i][e & 3] = ~0u;
                else raw[i][(e >> 1) & 3] |= e & 1 ? 0xffff0000u : 0xffffu;
            }
    }
    __device__ float at(int i, int e) const { return vector_at<T>(raw[i], e); }
};

__device__ __forceinline__ int lanes_below(unsigned long long m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// The largest t that at least n of the wave's values reach (0: fewer have one).
__device__ __forceinline__ uint32_t reached_by(uint32_t key, int n) {
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t up = t | 1u << bit;
        if (__popcll(__ballot(key >= up)) >= n) t = up;
    }
    return t;
}

// A wave's chunk: the logits among which its n best are.  The n-th largest of
// the lanes' own largest is a bound that at least n logits reach, and in a
// chunk without order few more do; a chunk in which too many do is searched
// for its n-th largest itself.
template <class T>
__device__ void scan_few(const Chunk<T>& c, int first, int skip, int n, ChunkList* out) {
    constexpr int kPer = Chunk<T>::kPer, kVecs = Chunk<T>::kVecs;
    const int lane = threadIdx.x & 63;
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) mx = fmaxf(mx, c.at(i, e));   // NaN is passed over
    const uint32_t bound = reached_by(logit_key(mx), n);
    const float least = bound > kKeyNone ? key_f32(bound) : -__FLT_MAX__;   // -inf is no token
    int count = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) count += __popcll(__ballot(c.at(i, e) >= least));
    mx = wave_max(mx);
    if (count <= kList) {
        int at = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const float z = c.at(i, e);
                const unsigned long long m = __ballot(z >= least);
                if (m == 0) continue;
                if (z >= least)
                    out->entry[at + lanes_below(m)] = (u64)logit_key(z) << 32 | (uint32_t)~(first - skip + (i * kWave + lane) * kPer + e);
                at += __popcll(m);
            }
    } else {
        uint32_t t = 0;   // the n-th largest key
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t up = t | 1u << bit;
            int reach = 0;
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int e = 0; e < kPer; ++e) reach += __popcll(__ballot(logit_key(c.at(i, e)) >= up));
            if (reach >= n) t = up;
        }
        int at = 0;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const uint32_t key = logit_key(c.at(i, e));
                const unsigned long long m = __ballot(key > t);
                if (key > t) out->entry[at + lanes_below(m)] = (u64)key << 32 | (uint32_t)~(first - skip + (i * kWave + lane) * kPer + e);
                at += __popcll(m);
            }
        // of those equal to it the first by id: a vector's lanes hold ids in order
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            int mine = 0;
#pragma unroll
            for (int e = 0; e < kPer; ++e) mine += logit_key(c.at(i, e)) == t ? 1 : 0;
            int before = mine;
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(before, o);
                if (lane >= o) before += up;
            }
            const int all = __shfl(before, 63);
            int slot = at + before - mine;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (logit_key(c.at(i, e)) == t) {
                    if (slot < n) out->entry[slot] = (u64)t << 32 | (uint32_t)~(first - skip + (i * kWave + lane) * kPer + e);
                    ++slot;
                }
            at = min(n, at + all);
        }
        count = at;
    }
    if (lane == 0) {
        out->largest = mx;
        out->count = count;
    }
}

// Where a logit lies: y = 16 z / T, its step b (the nearest integer) and exp
// of what is left, |rest| <= 1/32, by its series to the 6th power (error 2^-47).
// Adding 1.5 * 2^52 rounds to an integer and leaves it in the sum's low bits,
// which takes three operations for step and rest.  Rows whose largest y is
// not within kFar are left to hard_row: there a step is no longer far above the
// logits' own rounding.  The scan leaves out slices by the same test of their
// own largest, so a row's has to be farther inside at the lower end than
// any slice that matters to it can be below it.
constexpr double kRound = 0x1.8p52;
constexpr double kFar = 0x1p20;
struct Step {
    int step;
    double rest;   // of y
};
__device__ __forceinline__ Step step_of(float z, double per) {
    const double t = fma((double)z, per, kRound), b = t - kRound;
    return {(int)(uint32_t)__double_as_longlong(t), fma((double)z, per, -b)};
}
// exp(rest / 16) as an integer, 2^bits the one (bits <= 48): the coefficients
// carry that factor, and a constant term 2^52 more rounds the sum and leaves
// the integer in its low bits.
struct Series {
    double c[7];
    __device__ explicit Series(double one) {
        double f = one;
#pragma unroll
        for (int n = 0; n < 7; ++n) {
            c[n] = f;
            f *= 1. / kPerUnit / (n + 1);
        }
        c[0] += 0x1p52;
    }
    __device__ u64 operator()(double r) const {
        double s = c[6];
#pragma unroll
        for (int n = 5; n >= 0; --n) s = fma(s, r, c[n]);
        return (u64)__double_as_longlong(s) & ((1ull << 52) - 1);
    }
};

struct ScanShared {
    u64 mass[kSteps];
    uint32_t count[kSteps];
    float top[kScanWaves];
    int used;
};

// A slice's masses by step.  What it costs is fp64 arithmetic (a dozen
// operations a logit, at fp32's rate here) and one LDS atomic.
template <class T>
__device__ void scan_whole(const Chunk<T>& c, const RowSettings& set, double one, ScanShared& sh, SliceData* out) {
    constexpr int kPer = Chunk<T>::kPer, kVecs = Chunk<T>::kVecs;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int j = tid; j < kSteps; j += kScanThreads) sh.mass[j] = 0, sh.count[j] = 0;
    if (tid == 0) sh.used = 0;
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) mx = fmaxf(mx, c.at(i, e));
    mx = wave_max(mx);
    if (lane == 0) sh.top[wave] = mx;
    __syncthreads();
    for (int w = 0; w < kScanWaves; ++w) mx = fmaxf(mx, sh.top[w]);
    const double per = kPerUnit / (double)set.t;
    const bool counted = set.k > 0;
    int last = -1, top = 0;
    if (mx > neg_inf() && fabs((double)mx * per) < kFar) {
        top = step_of(mx, per).step;
        // what lies further down, -inf and NaN stop just outside the steps
        const float least = (float)((top - (kSteps + 8)) / per);
        const Series weight(one);
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const Step s = step_of(fmaxf(c.at(i, e), least), per);
                const int j = top - s.step;
                if (j < kSteps) {
                    last = max(last, j);
                    atomicAdd(&sh.mass[j], weight(s.rest));
                    if (counted) atomicAdd(&sh.count[j], 1u);
                }
            }
    }
    atomicMax(&sh.used, last + 1);
    __syncthreads();
    const int used = sh.used;
    for (int j = tid; j < used; j += kScanThreads) {
        out->mass[j] = sh.mass[j];
        if (counted) out->count[j] = sh.count[j];
    }
    if (tid == 0) out->head = {top, used, mx, 0};
}

// Workgroup (slice, row).
template <class T>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(SampleArgs a, int bits) {
    __shared__ ScanShared sh;
    const int r = blockIdx.y * 32768 + blockIdx.z, wave = threadIdx.x >> 6;
    if (r >= a.rows) return;
    const T* row = static_cast<const T*>(a.logits) + (size_t)r * a.ld;
    const int skip = Chunk<T>::skip_of(row);
    const int first = blockIdx.x * kSlice + wave * kChunk;
    SliceData* out = reinterpret_cast<SliceData*>(a.ws) + (size_t)r * gridDim.x + blockIdx.x;
    const RowSettings set = settings_of(a, r);
    Chunk<T> c;
    c.load(row, skip, a.V, first);
    const int n = set.few(a.V);
    if (n > 0) {
        scan_few(c, first, skip, n, &out->few[wave]);
    } else {
        scan_whole(c, set, ldexp(1., bits), sh, out);
    }
}

// ------------------------------------------------------------------ the pick

__device__ __forceinline__ u64 lane_xor64(u64 v, int j) {
    return (u64)(uint32_t)lane_xor_n((int)(v >> 32), j) << 32 | (uint32_t)lane_xor_n((int)v, j);
}
// The value of one lane, the same for the whole wave.
__device__ __forceinline__ u64 lane_value(u64 v, int lane) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// 64 values, a lane each, sorted with the largest in lane 0.
__device__ __forceinline__ u64 wave_sort(u64 v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
        for (int j = size >> 1; j > 0; j >>= 1) {
            const u64 w = lane_xor64(v, j);
            const bool low = (lane & j) == 0, down = (lane & size) == 0;   // this lane takes the larger
            v = (low == down) == (v > w) ? v : w;
        }
    return v;
}
// The 64 largest of two such lists, sorted.
__device__ __forceinline__ u64 wave_merge(u64 a, u64 b) {
    const int lane = threadIdx.x & 63;
    const u64 r = __shfl(b, 63 - lane);
    u64 v = a > r ? a : r;
#pragma unroll
    for (int j = 32; j > 0; j >>= 1) {
        const u64 w = lane_xor64(v, j);
        v = ((lane & j) == 0) == (v > w) ? v : w;
    }
    return v;
}

// A row's list entries, dealt out over the workgroup: a wave a list, with the
// loads of several lists in flight (what lies behind a list's end is read, but
// not used).
template <class F>
__device__ __forceinline__ void each_entry(const SliceData* data, int lists, F f) {
    constexpr int kDeep = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i0 = wave; i0 < lists; i0 += kDeep * kSampleWaves) {
        u64 x[kDeep][kList / kWave];
        int count[kDeep];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int i = min(i0 + d * kSampleWaves, lists - 1);
            const ChunkList& l = data[i / kScanWaves].few[i % kScanWaves];
            count[d] = i0 + d * kSampleWaves < lists ? l.count : 0;
#pragma unroll
            for (int h = 0; h < kList / kWave; ++h) x[d][h] = l.entry[h * kWave + lane];
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d)
#pragma unroll
            for (int h = 0; h < kList / kWave; ++h)
                if (h * kWave + lane < count[d]) f(x[d][h]);
    }
}

struct FewShared {
    u64 list[kSurvivors];
    u64 rank[kSampleWaves][kWave];
    int count;
};

// The draw from at most 64 ranked tokens, in one wave.
__device__ void draw_few(const SampleArgs& a, const RowSettings& set, u64 best, int n, int bits) {
    const int lane = threadIdx.x & 63, r = blockIdx.x;
    const uint32_t key = (uint32_t)(best >> 32);
    const int id = (int)~(uint32_t)best;
    const u64 real = __ballot(lane < n && key > kKeyNone);
    n = __popcll(real);
    if (n == 0) {
        if (lane == 0) {
            a.token[r] = -1;
            if (a.logprob != nullptr) a.logprob[r] = neg_inf();
        }
        return;
    }
    const bool first = !(set.t > 0.f) || set.mp > 1.f;
    const Weigh w{(double)key_f32((uint32_t)__builtin_amdgcn_readfirstlane((int)key)), (double)set.t, ldexp(1., bits)};
    u64 x = first ? (u64)(lane == 0) << bits : lane < n ? w.weight(key) : 0ull;
    if (first) n = 1;
    u64 c = x;
    for (int o = 1; o < 64; o <<= 1) {
        const u64 up = __shfl_up(c, o);
        if (lane >= o) c += up;
    }
    if (set.p < 1.f && !first) {
        const double want = ceil((double)set.p * (double)lane_value(c, 63));
        n = min(n, __popcll(__ballot(lane < n && (double)c < want)) + 1);
    }
    if (set.mp > 0.f && !first) n = max(1, min(n, __popcll(__ballot(lane < n && exp(w.power(key)) >= (double)set.mp))));
    const u64 total = lane_value(c, n - 1);
    const u64 target = (u64)(unit(a.uniform[r]) * (double)total);
    u64 before = 0;   // of the kept with a lower id
    for (int o = 0; o < n; ++o)
        before += __builtin_amdgcn_readlane(id, o) < id ? lane_value(x, o) : 0ull;
    if (lane < n && before <= target && target < before + x) {
        a.token[r] = id;
        if (a.logprob != nullptr) a.logprob[r] = first ? 0.f : (float)(w.power(key) - log((double)total / w.one));
    }
}

// Joins a row's lists.  The n-th largest of the lanes' largest list heads
// bounds what can be among the best n (fewer lists than n: everything can);
// the waves rank these survivors 64 at a time, each its share, and one joins
// them.  Returns false where too many survive.
__device__ bool pick_few(const SampleArgs& a, const RowSettings& set, const SliceData* data, int slices, int n,
                         int bits, FewShared& sh, u64* tmp) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lists = slices * kScanWaves;
    if (n == 1) {
        u64 best = 0;
        each_entry(data, lists, [&](u64 x) { best = x > best ? x : best; });
        best = block_max(best, tmp);
        if (wave == 0) draw_few(a, set, lane == 0 ? best : 0ull, 1, bits);
        return true;
    }
    float mx = neg_inf();
    for (int i = lane; i < lists; i += kWave) mx = fmaxf(mx, data[i / kScanWaves].few[i % kScanWaves].largest);
    const uint32_t bound = reached_by(logit_key(mx), n);
    if (tid == 0) sh.count = 0;
    __syncthreads();
    each_entry(data, lists, [&](u64 x) {
        if ((uint32_t)(x >> 32) < bound) return;
        const int at = atomicAdd(&sh.count, 1);
        if (at < kSurvivors) sh.list[at] = x;
    });
    __syncthreads();
    const int count = sh.count;
    if (count > kSurvivors) return false;
    auto ranked = [&](int i) { return wave_sort(i + lane < count ? sh.list[i + lane] : 0ull); };
    u64 best = 0;
    if (wave * kWave < count) {
        best = ranked(wave * kWave);
        for (int i = wave * kWave + kSampleThreads; i < count; i += kSampleThreads) best = wave_merge(best, ranked(i));
        sh.rank[wave][lane] = best;
    }
    __syncthreads();
    if (wave == 0) {
        for (int w = 1; w < min(kSampleWaves, (count + kWave - 1) / kWave); ++w) best = wave_merge(best, sh.rank[w][lane]);
        draw_few(a, set, best, n, bits);
    }
    return true;
}

constexpr int kMaxSlices = ((1 << 22) + kSlice - 1) / kSlice + 1;

struct WholeShared {
    u64 mass[kSteps];
    uint32_t count[kSteps];
    double upto[kSteps];      // mass of steps 0..j, the largest logit's weight being 1
    double unit[kSteps];      // weight of a step's middle
    u64 list[kBorderList];    // the border's step: key << 32 | ~id
    u64 ends[2][kSampleWaves];
    u64 border[kMaxSlices];   // kept mass of that step, by slice
    double slice[kMaxSlices];
    unsigned short holds[kMaxSlices];
    int listed, cut, pick, last;
};

// Inclusive sum of one double a thread, in a fixed order.
__device__ __forceinline__ double block_upto(double v, double* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const double up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    double before = 0.;
    for (int w = 0; w < wave; ++w) before += tmp[w];
    __syncthreads();
    return before + v;
}

// Smallest value over the workgroup.
__device__ __forceinline__ int block_min(int v, int* cell) {
    if (threadIdx.x == 0) *cell = 0x7fffffff;
    __syncthreads();
    if (v != 0x7fffffff) atomicMin(cell, v);
    __syncthreads();
    v = *cell;
    __syncthreads();
    return v;
}

template <class T>
struct Whole {
    const SampleArgs& a;
    const RowSettings& set;
    const SliceData* data;
    WholeShared& sh;
    u64* tmp;
    const T* row;
    int slices, skip, r;
    double per, ytop, one;
    int top;
    float largest;
    Series weight;

    // steps from the row's top to the slice's
    __device__ int step_below(const SliceHead& h) const {
        return h.largest > neg_inf() ? min(top - h.top, kSteps) : kSteps;
    }
    // A logit's step below the top; kSteps or more: of no weight.
    __device__ Step place(float z) const {
        const Step s = step_of(fmaxf(z, (float)((top - (kSteps + 8)) / per)), per);
        return {top - s.step, s.rest};
    }
    // The lowest (UP false) or highest logit of step j.
    template <bool UP>
    __device__ float step_end(int j) const {
        const double edge = UP ? (top - j + 0.5) / per : (top - j - 0.5) / per;
        const float z = (float)edge;
        // the nearest fp32 values around the edge, the outermost that is in the step
        const uint32_t key = f32_key(z);
        float found = key_f32(key);
#pragma unroll 1
        for (int d = 2; d >= -2; --d) {
            const float c = key_f32(UP ? key - d : key + d);   // from inside the step outwards
            if (place(c).step == j) found = c;
        }
        return found;
    }
    // Lists the tokens of step j; false where they are too many.
    __device__ bool list_step(int j) {
        const int tid = threadIdx.x;
        constexpr int kPer = Chunk<T>::kPer;
        if (tid == 0) sh.listed = 0, sh.pick = 0;
        __syncthreads();
        // the slices that hold any
        for (int s = tid; s < slices; s += kSampleThreads) {
            const SliceHead h = data[s].head;
            const int at = j - step_below(h);
            if (at >= 0 && at < h.used && data[s].mass[at] != 0) sh.holds[atomicAdd(&sh.pick, 1)] = (unsigned short)s;
        }
        __syncthreads();
        // a step is a range of logits: its ends, exactly
        const float lo = step_end<false>(j), hi = step_end<true>(j);
        const u32x4* p = reinterpret_cast<const u32x4*>(row - skip);
        const int vecs = sh.pick * (kSlice / kPer), end = a.V + skip;
        constexpr int kDeep = 32 / kPer;   // loads in flight a thread, 32 logits
        for (int i0 = tid; i0 < vecs; i0 += kDeep * kSampleThreads) {
            u32x4 raw[kDeep];
            int first[kDeep];
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                const int i = i0 + d * kSampleThreads;
                first[d] = i < vecs ? sh.holds[i / (kSlice / kPer)] * kSlice + i % (kSlice / kPer) * kPer : end;
                raw[d] = u32x4{~0u, ~0u, ~0u, ~0u};
                if (first[d] < end) raw[d] = p[first[d] / kPer];
            }
            uint32_t hit = 0;   // of the lane's logits
#pragma unroll
            for (int d = 0; d < kDeep; ++d)
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const float z = vector_at<T>(raw[d], e);
                    hit |= __builtin_amdgcn_fmed3f(z, lo, hi) == z ? 1u << (d * kPer + e) : 0u;
                }
#pragma unroll
            for (int d = 0; d < kDeep; ++d)   // at the row's ends, what is no logit of it
                if (first[d] < skip || first[d] + kPer > end)
#pragma unroll
                    for (int e = 0; e < kPer; ++e)
                        if (first[d] + e < skip || first[d] + e >= end) hit &= ~(1u << (d * kPer + e));
            // a wave's hits are counted a bit of the lanes' counts at a time
            const int mine = __popc(hit);
            int before = 0, all = 0;
#pragma unroll
            for (int b = 0; b < 6; ++b) {
                const unsigned long long m = __ballot(mine >> b & 1);
                before += lanes_below(m) << b;
                all += __popcll(m) << b;
            }
            if (all == 0) continue;
            int base = 0;
            if ((tid & 63) == 0) base = atomicAdd(&sh.listed, all);
            int at = __builtin_amdgcn_readfirstlane(base) + before;
            for (; hit != 0; hit &= hit - 1, ++at) {
                const int bit = __builtin_ctz(hit), i = i0 + bit / kPer * kSampleThreads;
                if (at < kBorderList) sh.list[at] = sh.holds[i / (kSlice / kPer)] * kSlice + i % (kSlice / kPer) * kPer + bit % kPer - skip;
            }
        }
        __syncthreads();
        const int n = sh.listed;
        if (n > kBorderList) return false;
        // ids so far: now their logits, several loads in flight
        constexpr int kKeys = 4;
        for (int i0 = tid; i0 < n; i0 += kKeys * kSampleThreads) {
            int id[kKeys];
            uint32_t key[kKeys];
#pragma unroll
            for (int d = 0; d < kKeys; ++d) {
                id[d] = (int)sh.list[min(i0 + d * kSampleThreads, n - 1)];
                key[d] = i0 + d * kSampleThreads < n ? key_at(row, id[d]) : 0u;
            }
#pragma unroll
            for (int d = 0; d < kKeys; ++d)
                if (i0 + d * kSampleThreads < n) sh.list[i0 + d * kSampleThreads] = (u64)key[d] << 32 | (uint32_t)~id[d];
        }
        __syncthreads();
        return true;
    }
    __device__ u64 weight_of(u64 entry) const { return weight(place(key_f32((uint32_t)(entry >> 32))).rest); }

    // Entries of the listed step, a thread's share of them.
    template <class F>
    __device__ void each_listed(F f) const {
        for (int i = threadIdx.x; i < sh.listed; i += kSampleThreads) f(sh.list[i]);
    }
    // Smallest and largest of a value a thread.
    __device__ void block_extremes(u64& mn, u64& mx) {
#pragma unroll
        for (int j = 32; j > 0; j >>= 1) {
            const u64 a = lane_xor64(mn, j), b = lane_xor64(mx, j);
            mn = a < mn ? a : mn;
            mx = b > mx ? b : mx;
        }
        if ((threadIdx.x & 63) == 0) sh.ends[0][threadIdx.x >> 6] = mn, sh.ends[1][threadIdx.x >> 6] = mx;
        __syncthreads();
        for (int w = 0; w < kSampleWaves; ++w) {
            mn = sh.ends[0][w] < mn ? sh.ends[0][w] : mn;
            mx = sh.ends[1][w] > mx ? sh.ends[1][w] : mx;
        }
        __syncthreads();
    }
    // The first of kSteps values whose running sum, on top of `from`, reaches
    // `target`, and the sum before it; 0x7fffffff: none.
    template <class N>
    __device__ int first_reaching(const N* v, u64 from, double target, u64* before) {
        constexpr int kEach = kSteps / kSampleThreads;
        const int j0 = threadIdx.x * kEach;
        u64 sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += v[j0 + i];
        u64 at = from + block_before(sum, tmp);
        int found = 0x7fffffff;
        u64 found_at = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const u64 next = at + v[j0 + i];
            if (found == 0x7fffffff && (double)next >= target) found = j0 + i, found_at = at;
            at = next;
        }
        const int first = block_min(found, &sh.cut);
        if (first != 0x7fffffff && found == first) tmp[0] = found_at;
        __syncthreads();
        *before = tmp[0];
        __syncthreads();
        return first;
    }
    // The listed entry, at least `from`, at which those from the largest down
    // reach `target` weights (BY_MASS) or entries, found nine bits at a time
    // among the bits in which what is left differs; the last one if all
    // together do not.  The first always counts: a target of nothing (top_p
    // 0), which a bin without entries would reach, is one unit of weight.
    template <bool BY_MASS>
    __device__ u64 reach(double target, u64 from) {
        const int tid = threadIdx.x;
        target = fmax(target, 1.);
        u64 lo = from, hi = ~0ull, above = 0;
        for (;;) {
            u64 mn = ~0ull, mx = 0;
            each_listed([&](u64 x) {
                if (x < lo || x > hi) return;
                mn = x < mn ? x : mn;
                mx = x > mx ? x : mx;
            });
            block_extremes(mn, mx);
            if (mn >= mx) return mn;   // entries differ: one is left
            const int bits = 64 - __builtin_clzll(mn ^ mx), shift = bits > 9 ? bits - 9 : 0;
            for (int j = tid; j < kSteps; j += kSampleThreads) sh.mass[j] = 0;
            __syncthreads();
            each_listed([&](u64 x) {
                if (x >= lo && x <= hi) atomicAdd(&sh.mass[kSteps - 1 - (int)((x >> shift) & (kSteps - 1))], BY_MASS ? weight_of(x) : 1ull);
            });
            __syncthreads();
            u64 bin_above;
            const int bin = first_reaching(sh.mass, above, target, &bin_above);
            if (bin == 0x7fffffff) return mn;
            above = bin_above;
            lo = (mn >> shift & ~(u64)(kSteps - 1) | (u64)(kSteps - 1 - bin)) << shift;
            hi = lo | ((1ull << shift) - 1);
            if (shift == 0) return lo;
        }
    }
    // Weights of the listed entries from `from` up.
    __device__ double mass_from(u64 from) {
        u64 sum = 0;
        each_listed([&](u64 x) { sum += x >= from ? weight_of(x) : 0ull; });
        return (double)block_sum(sum);
    }
    __device__ u64 block_sum(u64 v) {
        const u64 before = block_before(v, tmp);
        if (threadIdx.x == kSampleThreads - 1) tmp[0] = before + v;
        __syncthreads();
        const u64 all = tmp[0];
        __syncthreads();
        return all;
    }

    // Every slice's steps, a slice a wave and a step a lane, all loads of a
    // slice in flight at once (steps that it does not use hold anything); then
    // `done`.
    template <class F, class G>
    __device__ void for_slices(F f, G done) const {
        constexpr int kLoads = kSteps / kWave;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const bool counted = set.k > 0;
        for (int s = wave; s < slices; s += kSampleWaves) {
            const SliceHead h = data[s].head;
            u64 m[kLoads];
            uint32_t n[kLoads] = {};
#pragma unroll
            for (int i = 0; i < kLoads; ++i) m[i] = data[s].mass[i * kWave + lane];
            if (counted)
#pragma unroll
                for (int i = 0; i < kLoads; ++i) n[i] = data[s].count[i * kWave + lane];
            const int below = step_below(h);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) f(s, h, below, i * kWave + lane, m[i], n[i]);
            done(s);
        }
    }

    // Draws the row's token; false where the row is to be read byte by byte.
    __device__ bool draw() {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        for (int j = tid; j < kSteps; j += kSampleThreads) {
            sh.mass[j] = 0;
            sh.count[j] = 0;
        }
        for (int s = tid; s < slices; s += kSampleThreads) sh.border[s] = 0;
        __syncthreads();
        const bool counted = set.k > 0;
        for_slices([&](int s, const SliceHead& h, int below, int j, u64 m, uint32_t n) {
            if (j >= min(h.used, kSteps - below)) return;
            if (m != 0) atomicAdd(&sh.mass[j + below], m);
            if (counted && n != 0) atomicAdd(&sh.count[j + below], n);
        }, [](int) {});
        __syncthreads();
        constexpr int kStepsEach = kSteps / kSampleThreads;   // a thread's, side by side
        const int j0 = tid * kStepsEach;
        double m[kStepsEach], sum = 0.;
        double each = exp((((double)top - ytop) - (double)j0) * (1. / kPerUnit)) / one;
#pragma unroll
        for (int i = 0; i < kStepsEach; ++i) {
            sh.unit[j0 + i] = each;
            sum += (double)sh.mass[j0 + i] * each;
            m[i] = sum;
            each *= 0.93941306281347581;   // exp(-1/16)
        }
        const double before_mine = block_upto(sum, reinterpret_cast<double*>(tmp)) - sum;
#pragma unroll
        for (int i = 0; i < kStepsEach; ++i) sh.upto[j0 + i] = before_mine + m[i];
        __syncthreads();
        // the kept: steps above `edge` whole, of that one the entries from `least` up
        int edge = kSteps, listed = -1;
        u64 least = 0;
        double total = sh.upto[kSteps - 1];
        auto above = [&](int j) { return j > 0 ? sh.upto[j - 1] : 0.; };
        if (counted && set.k < a.V) {
            u64 n;
            const int j = first_reaching(sh.count, 0, (double)set.k, &n);
            if (j < kSteps) {
                if (!list_step(j)) return false;
                edge = listed = j;
                least = reach<false>((double)(set.k - (int)n), 0);
                total = above(j) + mass_from(least) * sh.unit[j];
            }
        }
        if (set.p < 1.f) {
            const double target = (double)set.p * total;
            int j = 0x7fffffff;
#pragma unroll
            for (int i = kStepsEach - 1; i >= 0; --i)
                if (j0 + i <= edge && sh.upto[j0 + i] >= target) j = j0 + i;
            j = block_min(j, &sh.cut);
            if (j == 0x7fffffff && edge < kSteps) j = edge;   // the border's own rounding
            if (j < kSteps) {
                if (j != listed && !list_step(j)) return false;
                if (j != edge) least = 0;
                edge = listed = j;
                least = reach<true>((target - above(j)) / sh.unit[j], least);
                total = above(j) + mass_from(least) * sh.unit[j];
            }
        }
        if (set.mp > 0.f) {
            const double floor = (double)set.mp;
            // ytop is rounded where `top` is not: at an end of the largest
            // logit's step, and min_p 1, this would be the step above it
            const double d = fmax((double)top - rint(ytop + kPerUnit * log(floor)), 0.);
            const int j = d < (double)kSteps ? (int)d : kSteps;
            if (j <= edge && j < kSteps) {
                if (j != listed && !list_step(j)) return false;
                if (j != edge) least = 0;
                edge = listed = j;
                u64 first = ~0ull;   // none: the steps above alone
                each_listed([&](u64 x) {
                    const double z = ((double)key_f32((uint32_t)(x >> 32)) - (double)largest) / (double)set.t;
                    if (x >= least && x < first && exp(z) >= floor) first = x;
                });
                u64 any = 0;
                block_extremes(first, any);
                least = first;
                total = above(j) + mass_from(least) * sh.unit[j];
            }
        }
        if (edge < kSteps)
            each_listed([&](u64 x) {
                if (x >= least) atomicAdd(&sh.border[((int)~(uint32_t)x + skip) / kSlice], weight_of(x));
            });
        if (tid == 0) sh.last = -1;
        __syncthreads();
        double part = 0.;
        for_slices([&](int s, const SliceHead& h, int below, int j, u64 m, uint32_t) {
            if (j < h.used && j + below < edge) part += (double)m * sh.unit[j + below];
        }, [&](int s) {
            for (int o = 32; o > 0; o >>= 1) part += __shfl_xor(part, o);
            if (lane == 0) sh.slice[s] = part + (edge < kSteps ? (double)sh.border[s] * sh.unit[edge] : 0.);
            part = 0.;
        });
        __syncthreads();
        // every thread finds the slice: the first whose running sum exceeds
        // the target, or by rounding the last that holds anything
        const double target = unit(a.uniform[r]) * total;
        double before = 0.;
        int at = 0;
        sum = 0.;
        for (int s = 0; s < slices; ++s) {
            const double m = sh.slice[s];
            if (m > 0.) {
                at = s;
                before = sum;
            }
            sum += m;
            if (m > 0. && sum > target) break;
        }
        constexpr int kEach = kSlice / kSampleThreads;
        const int v0 = at * kSlice + tid * kEach;
        constexpr int kPer = Chunk<T>::kPer;
        u32x4 raw[kEach / kPer];
#pragma unroll
        for (int i = 0; i < kEach / kPer; ++i) {
            raw[i] = u32x4{~0u, ~0u, ~0u, ~0u};
            if (v0 + i * kPer < a.V + skip) raw[i] = *reinterpret_cast<const u32x4*>(row - skip + v0 + i * kPer);
        }
        auto kept_weight = [&](int e) -> double {
            const int v = v0 + e;
            const float z = vector_at<T>(raw[e / kPer], e % kPer);
            const Step st = place(z);   // NaN and -inf: beyond the steps
            if (v < skip || v >= a.V + skip || st.step >= kSteps || st.step > edge) return 0.;
            if (st.step == edge && ((u64)logit_key(z) << 32 | (uint32_t)~(v - skip)) < least) return 0.;
            return (double)weight(st.rest) * sh.unit[st.step];
        };
        double mine = 0.;
#pragma unroll
        for (int e = 0; e < kEach; ++e) mine += kept_weight(e);
        const double run = before + block_upto(mine, reinterpret_cast<double*>(tmp));
        // the first thread whose running sum exceeds the target, or by rounding the last that holds anything
        const int found = block_min(mine > 0. && run > target ? tid : 0x7fffffff, &sh.cut);
        if (mine > 0.) atomicMax(&sh.last, tid);
        __syncthreads();
        const int who = found != 0x7fffffff ? found : sh.last;
        if (tid == who) tmp[0] = (u64)__double_as_longlong(run - mine);
        __syncthreads();
        if (wave != 0) return true;
        // its logits, one a lane
        static_assert(kEach <= kWave, "a logit a lane");
        const int v = at * kSlice + who * kEach + min(lane, kEach - 1);
        const bool real = lane < kEach && v >= skip && v < a.V + skip;
        const uint32_t key = real ? key_at(row, v - skip) : 0u;
        const Step st = place(key_f32(max(key, kKeyNone)));
        const bool keep = real && st.step < kSteps && (st.step < edge || (st.step == edge && ((u64)key << 32 | (uint32_t)~(v - skip)) >= least));
        const double w = keep ? (double)weight(st.rest) * sh.unit[min(st.step, kSteps - 1)] : 0.;
        double upto = w;
        for (int o = 1; o < kWave; o <<= 1) {
            const double up = __shfl_up(upto, o);
            if (lane >= o) upto += up;
        }
        upto += __longlong_as_double((long long)tmp[0]);
        const u64 some = __ballot(w > 0.), over = __ballot(w > 0. && upto > target);
        if (lane == (over != 0 ? __builtin_ctzll(over) : 63 - __builtin_clzll(some))) {
            a.token[r] = v - skip;
            if (a.logprob != nullptr)
                a.logprob[r] = (float)(((double)key_f32(key) - (double)largest) / (double)set.t - log(total));
        }
        return true;
    }
};

// A workgroup a row.
template <class T>
__global__ __launch_bounds__(kSampleThreads, 4) void pick_kernel(SampleArgs a, int slices, int bits) {
    __shared__ union {
        FewShared few;
        WholeShared whole;
        HardShared hard;
    } sh;
    __shared__ u64 tmp[kSampleWaves];
    __shared__ u64 s_state[4];
    const int r = blockIdx.x, lane = threadIdx.x & 63;
    const SliceData* data = reinterpret_cast<const SliceData*>(a.ws) + (size_t)r * slices;
    const RowSettings set = settings_of(a, r);
    const int n = set.few(a.V);
    float largest = neg_inf();
    if (n > 0) {
        if (pick_few(a, set, data, slices, n, bits, sh.few, tmp)) return;
        for (int i = lane; i < slices * kScanWaves; i += kWave)
            largest = fmaxf(largest, data[i / kScanWaves].few[i % kScanWaves].largest);
    } else {
        for (int i = lane; i < slices; i += kWave) largest = fmaxf(largest, data[i].head.largest);
    }
    largest = wave_max(largest);
    if (n == 0) {
        if (largest == neg_inf()) {
            if (threadIdx.x == 0) {
                a.token[r] = -1;
                if (a.logprob != nullptr) a.logprob[r] = neg_inf();
            }
            return;
        }
        const double per = kPerUnit / (double)set.t, ytop = (double)largest * per;
        if (ytop < kFar && ytop > 2 * kSteps - kFar) {
            const T* row = static_cast<const T*>(a.logits) + (size_t)r * a.ld;
            const double one = ldexp(1., bits);
            Whole<T> w{a, set, data, sh.whole, tmp, row, slices, Chunk<T>::skip_of(row), r, per, ytop, one,
                       step_of(largest, per).step, largest, Series(one)};
            if (w.draw()) return;
        }
    }
    __syncthreads();
    hard_row<T>(a, set, logit_key(largest), bits, sh.hard, tmp, s_state);
}

namespace {
int slices_of(int V) { return (V + 7 + kSlice - 1) / kSlice; }   // a row may begin up to 7 logits behind a boundary
}

size_t sample_ws_bytes(long long rows, int V) { return (size_t)rows * slices_of(V) * sizeof(SliceData); }

hipError_t launch_sample(const SampleArgs& a, bool bf16, hipStream_t stream) {
    int bits = 62;   // sums of V weights of at most 1.07 * 2^bits stay below 2^63
    for (int v = a.V; v > 0; v >>= 1) --bits;
    bits = bits < 48 ? bits : 48;
    const int slices = slices_of(a.V);
    const dim3 grid(slices, (a.rows - 1) / 32768 + 1, a.rows < 32768 ? a.rows : 32768);
    if (bf16) hipLaunchKernelGGL(scan_kernel<uint16_t>, grid, dim3(kScanThreads), 0, stream, a, bits);
    else hipLaunchKernelGGL(scan_kernel<float>, grid, dim3(kScanThreads), 0, stream, a, bits);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (bf16) hipLaunchKernelGGL(pick_kernel<uint16_t>, dim3(a.rows), dim3(kSampleThreads), 0, stream, a, slices, bits);
    else hipLaunchKernelGGL(pick_kernel<float>, dim3(a.rows), dim3(kSampleThreads), 0, stream, a, slices, bits);
    return hipGetLastError();
}

}  // namespace tf
