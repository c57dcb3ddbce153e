// The paged 8-bit cache: pages and slots from lengths (cache_plan_kernel,
// cache_fill_kernel, cache_release_kernel), keys and values into it
// (cache_append_kernel).
#include "common.hpp"
#include "e4m3.hpp"
#include "launch.hpp"

namespace tf {

constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;
constexpr int kFillPer = 4;            // tokens a thread of the fill places
constexpr int kFillSeqs = 2048;        // sequences whose offsets it keeps in LDS
// Tokens up to which the planning workgroup fills the lists itself, which
// saves the second launch.
constexpr int kFillAlone = 1 << 14;

__device__ __forceinline__ int pages_of(int len, int page) { return (len + page - 1) / page; }

// Inclusive sum over the workgroup's threads (all call); `tmp` holds one
// value a wave and is free again on return.
__device__ __forceinline__ long long block_scan(long long v, long long* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const long long up = __shfl_up(v, o);
        if (lane >= o) v += up;
    }
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    long long before = 0;
    for (int w = 0; w < waves; ++w) before += w < wave ? tmp[w] : 0;
    __syncthreads();
    return v + before;
}

// Places tokens [i0, i1) of the lists.  `start` and `page_start` are whole
// and new_len, new_free_count written: the old length of a sequence is its
// new one less its tokens, and its pages sit below the old top of the stack.
__device__ __forceinline__ void fill_slots(const SlotsArgs& a, const int32_t* start, const int32_t* page_start, int i0,
                                           int i1, int step) {
    const int total = start[a.b];
    const int top = a.new_free_count[0] + page_start[a.b];   // pages on the stack before the call
    for (int i = i0; i < i1; i += step) {
        int sl = -1, ps = -1, src = -1;
        if (i < total) {
            int lo = 0, hi = a.b;   // start[lo] <= i < start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (start[mid] <= i) lo = mid;
                else hi = mid;
            }
            const int s = lo, j = i - start[s];
            const int ctx = a.new_len[s] - (start[s + 1] - start[s]);
            ps = ctx + j;
            const int col = ps / a.page, off = ps - col * a.page;
            const int had = pages_of(ctx, a.page);
            const size_t at = (size_t)s * a.max_pages + col;
            int id;
            if (col < had) {
                id = a.block_table[at];
            } else {
                id = a.free_pages[top - 1 - (page_start[s] + col - had)];
                if (off == 0) a.block_table[at] = id;   // a new page's first token is a new token
            }
            const long long slot = (long long)id * a.page + off;
            sl = id >= 0 && slot <= 0x7fffffffll ? (int)slot : -1;
            const long long row = a.n == 0 ? i
                                           : (long long)s * a.n +
                                                 (a.accepted == nullptr ? j : (j == 0 ? 0 : 1 + a.accepted[(size_t)s * a.gamma + j - 1]));
            src = (int)row;
        }
        a.slot[i] = sl;
        if (a.position != nullptr) a.position[i] = ps;
        if (a.source != nullptr) a.source[i] = src;
    }
}

// One workgroup: sums of tokens and pages over the sequences, whether all of
// them fit, then lengths and list offsets; `alone`: the lists as well.  What
// bounds it is a chain of loads and scans, so a batch of up to kPlanThreads
// sequences is read and scanned once and its offsets are kept in LDS for the
// lists.  All reads of lengths and count end before the first write (new_len
// and new_free_count may be the same arrays).
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(SlotsArgs a, int alone) {
    __shared__ long long tmp[kPlanThreads / 64];
    __shared__ long long carry_tok, carry_page;
    __shared__ int bad;
    __shared__ int32_t s_start[kPlanThreads + 1], s_page[kPlanThreads + 1];
    const int tid = threadIdx.x;
    const int extra = a.accepted != nullptr ? 1 : 0;
    const bool once = a.b <= kPlanThreads;
    if (tid == 0) bad = 0;
    const int left = a.free_count[0];
    long long tok = 0, pg = 0;
    int wrong = left < 0 || left > a.max_free ? 1 : 0, wide = 0;
    int ctx = 0, add = 0, need = 0;
    for (int s = tid; s < a.b; s += kPlanThreads) {
        ctx = a.context_len[s];
        add = a.add_len[s];
        need = 0;
        if (ctx < 0 || add < -extra || (extra && add > a.gamma) || (a.n > 0 && (long long)add + extra > a.n)) {
            wrong = 1;
            continue;
        }
        add += extra;   // below 2^31: a.gamma bounds it where extra is 1
        const long long after = (long long)ctx + add;
        tok += add;
        if (after > (long long)a.max_pages * a.page) {
            wide = 1;
            continue;
        }
        need = pages_of((int)after, a.page) - pages_of(ctx, a.page);
        pg += need;
    }
    __syncthreads();
    if (wrong) atomicOr(&bad, 1);
    if (wide) atomicOr(&bad, 2);
    const long long upto_tok = block_scan(tok, tmp), upto_page = block_scan(pg, tmp);
    if (tid == kPlanThreads - 1) carry_tok = upto_tok, carry_page = upto_page;
    __syncthreads();
    const long long all_tok = carry_tok, all_page = carry_page;
    const int status = (bad & 1) ? 1 : all_tok > a.max_tokens ? 2 : (bad & 2) ? 3 : all_page > left ? 4 : 0;
    if (tid == 0) {
        a.status[0] = status;
        a.start[0] = s_start[0] = 0;
        a.page_start[0] = s_page[0] = 0;
        a.new_free_count[0] = status == 0 ? left - (int)all_page : left;
    }
    if (once) {
        if (tid < a.b) {
            a.start[tid + 1] = s_start[tid + 1] = status == 0 ? (int)upto_tok : 0;
            a.page_start[tid + 1] = s_page[tid + 1] = status == 0 ? (int)upto_page : 0;
            a.new_len[tid] = status == 0 ? ctx + add : ctx;
        }
    } else {
        __syncthreads();
        if (tid == 0) carry_tok = carry_page = 0;
        for (int s0 = 0; s0 < a.b; s0 += kPlanThreads) {
            const int s = s0 + tid;
            ctx = add = need = 0;
            if (s < a.b) {
                ctx = a.context_len[s];
                if (status == 0) {
                    add = a.add_len[s] + extra;
                    need = pages_of(ctx + add, a.page) - pages_of(ctx, a.page);
                }
            }
            const long long t = block_scan(add, tmp), p = block_scan(need, tmp);
            const long long bt = carry_tok, bp = carry_page;   // written before the scans' barriers
            if (s < a.b) {
                a.start[s + 1] = (int)(bt + t);
                a.page_start[s + 1] = (int)(bp + p);
                a.new_len[s] = ctx + add;
            }
            __syncthreads();
            if (tid == kPlanThreads - 1) carry_tok = bt + t, carry_page = bp + p;
            __syncthreads();
        }
    }
    if (alone) {
        __threadfence_block();
        __syncthreads();
        if (once) fill_slots(a, s_start, s_page, tid, a.max_tokens, kPlanThreads);
        else fill_slots(a, a.start, a.page_start, tid, a.max_tokens, kPlanThreads);
    }
}

// The search for a token's sequence goes through LDS where the offsets fit.
__global__ __launch_bounds__(kFillThreads) void cache_fill_kernel(SlotsArgs a) {
    __shared__ int32_t start[kFillSeqs + 1], page_start[kFillSeqs + 1];
    const int i0 = blockIdx.x * (kFillThreads * kFillPer);
    const int i1 = min(i0 + kFillThreads * kFillPer, a.max_tokens);
    if (a.b <= kFillSeqs) {
        for (int s = threadIdx.x; s <= a.b; s += kFillThreads) start[s] = a.start[s], page_start[s] = a.page_start[s];
        __syncthreads();
        fill_slots(a, start, page_start, i0 + threadIdx.x, i1, kFillThreads);
    } else {
        fill_slots(a, a.start, a.page_start, i0 + threadIdx.x, i1, kFillThreads);
    }
}

// One workgroup: the finished sequences' pages go onto the stack in order, a
// sequence a wave.
__global__ __launch_bounds__(kPlanThreads) void cache_release_kernel(ReleaseArgs a) {
    __shared__ long long tmp[kPlanThreads / 64];
    __shared__ long long carry;
    __shared__ int s_at[kPlanThreads], s_give[kPlanThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int count = min(max(a.free_count[0], 0), a.max_free);
    if (tid == 0) carry = count;
    __syncthreads();
    for (int s0 = 0; s0 < a.b; s0 += kPlanThreads) {
        const int s = s0 + tid;
        int len = 0, give = 0;
        bool done = false;
        if (s < a.b) {
            len = a.context_len[s];
            done = a.done[s] != 0;
            if (done && len > 0) give = (int)min((long long)len + a.page - 1, (long long)a.max_pages * a.page) / a.page;
        }
        const long long t = block_scan(give, tmp);
        const long long at = carry + t - give;
        s_at[tid] = (int)min(at, (long long)a.max_free);
        s_give[tid] = (int)min((long long)give, (long long)a.max_free - s_at[tid]);
        if (s < a.b) a.new_len[s] = done ? 0 : len;
        __syncthreads();
        if (tid == kPlanThreads - 1) carry += t;
        for (int q = wave; q < min(kPlanThreads, a.b - s0); q += kPlanThreads / kWave)
            for (int p = lane; p < s_give[q]; p += kWave)
                a.free_pages[s_at[q] + p] = a.block_table[(size_t)(s0 + q) * a.max_pages + p];
        __syncthreads();
    }
    if (tid == 0) a.new_free_count[0] = (int)min(carry, (long long)a.max_free);
}

// ------------------------------------------------------------------ append

constexpr int kAppendThreads = 256;

__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.f;   // neither infinities nor NaN enter the scale
}

// Four tokens' eight dimensions that a thread turns into codes.
template <class T>
struct TokenQuad {
    static constexpr int kWords = sizeof(T) * 8 / 16;
    u32x4 raw[4][kWords];
    __device__ void load(const T* rows, long long ld, const int (&row)[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                raw[t][w] = u32x4{};
                if (row[t] >= 0) raw[t][w] = reinterpret_cast<const u32x4*>(rows + (size_t)row[t] * ld)[w];
            }
    }
    __device__ float at(int t, int e) const {
        if (sizeof(T) == 4) return __uint_as_float(raw[t][(e >> 2) & (kWords - 1)][e & 3]);
        const uint32_t w = raw[t][0][e >> 1];
        return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ float largest() const {
        float m = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(at(t, e)));
        return m;
    }
};

// Workgroup (`per` tokens of the list, head, keys or values): for each run that
// begins among its tokens, the run's largest value, the scale, what the page
// held rounded again where the scale rose, the new codes.  The page's first
// token of the list leads its run, so every page and head has one writer and
// no atomics.  A thread takes four tokens' eight dimensions (tokens 4q..4q+3 of
// the page), all loads in flight at once: four conversions then give a dword
// along the dimensions for the keys, or along the tokens for the values' [D,
// page] side, which goes through LDS so that a store holds 16 tokens.  What
// bounds it is a chain of three loads (slot, source, row), so how many
// workgroups a CU holds: keys and values apart and at most 64 registers give
// eight (27 thousand tokens of 8 heads in pages of 64: 70 us together at four a
// CU, 44 so).
template <class T, int D>
__global__ __launch_bounds__(kAppendThreads, sizeof(T) == 2 ? 8 : 6) void cache_append_kernel(AppendArgs a, int per) {
    constexpr int kChunks = D / 8;                        // threads across a row
    constexpr int kQuads = kAppendThreads / kChunks;      // quads of tokens a pass
    constexpr int kPitch = 128 / 4 + 1;
    __shared__ float s_max[kAppendThreads / 64];
    __shared__ uint32_t turned[D * kPitch];               // values: four tokens' codes a dword
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // keys and values and the heads of the same tokens follow one another on an
    // XCD: their pieces of a row and of the lists come from its L2
    const int y = blockIdx.x / 8, unit = y % (2 * a.Hkv);
    const int block = y / (2 * a.Hkv) * 8 + blockIdx.x % 8, h = unit / 2;
    const bool values = (unit & 1) != 0;                  // uniform
    const int end = (int)min((long long)a.N, (long long)(block + 1) * per);
    const long long limit = (long long)a.num_pages * a.page;
    const int c8 = (tid % kChunks) * 8;
    const T* rows = static_cast<const T*>(values ? a.v_new : a.k_new) + (size_t)h * D + c8;
    float* scale = values ? a.v_scale : a.k_scale;
    // the tokens that lead a run, all looked at at once (per <= 64)
    const int mine = block * per + lane;
    bool leads = false;
    if (lane < per && mine < end) {
        const int sl = a.slot[mine], before = mine > 0 ? a.slot[mine - 1] : -1;
        leads = sl >= 0 && sl < limit && ((sl & (a.page - 1)) == 0 || before != sl - 1);
    }
    for (unsigned long long todo = __ballot(leads); todo != 0; todo &= todo - 1) {   // uniform over the workgroup
        const int i = block * per + __builtin_ctzll(todo);
        const int sl = a.slot[i];
        const int off = sl & (a.page - 1), id = sl / a.page;
        const int most = min(a.page - off, a.N - i);
        const unsigned long long b0 = __ballot(lane < most && a.slot[i + min(lane, most - 1)] == sl + lane);
        const unsigned long long b1 = __ballot(lane + 64 < most && a.slot[i + min(lane + 64, most - 1)] == sl + lane + 64);
        const int run = ~b0 != 0 ? __builtin_ctzll(~b0) : (~b1 != 0 ? 64 + __builtin_ctzll(~b1) : 128);

        const int q0 = off / 4, passes = ((off + run + 3) / 4 - q0 + kQuads - 1) / kQuads;
        TokenQuad<T> x;
        auto load = [&](int pass) {
            const int o = 4 * (q0 + pass * kQuads + tid / kChunks) - off;   // the quad's first token, in the run
            int row[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                row[t] = -1;
                if (o + t >= 0 && o + t < run) row[t] = a.source != nullptr ? a.source[i + o + t] : i + o + t;
                if (row[t] >= a.rows) row[t] = -1;
            }
            x.load(rows, a.ld_new, row);
        };
        float most_abs = 0.f;
        for (int pass = 0; pass < passes; ++pass) {
            load(pass);
            most_abs = fmaxf(most_abs, x.largest());
        }
        most_abs = wave_max(most_abs);
        if (lane == 0) s_max[wave] = most_abs;
        __syncthreads();
        for (int w = 0; w < kAppendThreads / 64; ++w) most_abs = fmaxf(most_abs, s_max[w]);
        const size_t head = (size_t)id * a.Hkv + h;
        const float old = off > 0 ? scale[head] : 0.f;
        const float now = fmaxf(pow2_scale(most_abs), old);
        uint8_t* cache = static_cast<uint8_t*>(values ? a.v_cache : a.k_cache) + head * a.page * D;
        if (off > 0 && now != old) {
            if (!values) {
                uint32_t* p = reinterpret_cast<uint32_t*>(cache);
                for (int e = tid; e < off * (D / 4); e += kAppendThreads) p[e] = e4m3_rescale(p[e], old / now);
            } else {
                const int quads = (off + 3) / 4;
                for (int e = tid; e < D * quads; e += kAppendThreads) {
                    const int d = e / quads, t = (e - d * quads) * 4;
                    uint8_t* p = cache + (size_t)d * a.page + t;
                    const uint32_t w = e4m3_rescale(*reinterpret_cast<const uint32_t*>(p), old / now);
                    if (t + 4 <= off) *reinterpret_cast<uint32_t*>(p) = w;
                    else   // the dword that the run goes on in
                        for (int q = 0; t + q < off; ++q) p[q] = (uint8_t)(w >> (8 * q));
                }
            }
        }
        __syncthreads();   // that dword is read before the new codes are written; s_max is free again
        const float f = 1.f / now;   // a power of two: exact
        for (int pass = 0; pass < passes; ++pass) {
            if (passes > 1) load(pass);   // one pass's are still there
            const int o = 4 * (q0 + pass * kQuads + tid / kChunks);
            const int lo = max(off - o, 0), hi = min(off + run - o, 4);   // the quad's tokens of the run
            if (lo >= hi) continue;
            if (!values) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (t >= lo && t < hi) {
                        uint2 w;
                        w.x = e4m3_quad(x.at(t, 0) * f, x.at(t, 1) * f, x.at(t, 2) * f, x.at(t, 3) * f);
                        w.y = e4m3_quad(x.at(t, 4) * f, x.at(t, 5) * f, x.at(t, 6) * f, x.at(t, 7) * f);
                        *reinterpret_cast<uint2*>(cache + (size_t)(o + t) * D + c8) = w;
                    }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    turned[(c8 + e) * kPitch + o / 4] = e4m3_quad(x.at(0, e) * f, x.at(1, e) * f, x.at(2, e) * f, x.at(3, e) * f);
            }
        }
        if (values) {   // a dimension's tokens lie together: 16 of them a store
            __syncthreads();
            const int g0 = off / 16, groups = (off + run + 15) / 16 - g0;
            for (int e = tid; e < D * groups; e += kAppendThreads) {
                const int d = e / groups, o = (g0 + e - d * groups) * 16;
                const uint32_t* from = turned + d * kPitch + o / 4;
                uint8_t* p = cache + (size_t)d * a.page + o;
                if (o >= off && o + 16 <= off + run) {
                    *reinterpret_cast<u32x4*>(p) = u32x4{from[0], from[1], from[2], from[3]};
                } else {
                    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(from);
                    for (int t = max(off - o, 0); t < min(off + run - o, 16); ++t) p[t] = bytes[t];
                }
            }
            __syncthreads();   // `turned` is free again
        }
        if (tid == 0) scale[head] = now;
    }
}

hipError_t launch_cache_slots(const SlotsArgs& a, hipStream_t stream) {
    const int alone = a.max_tokens <= kFillAlone ? 1 : 0;
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, alone);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || alone) return e;
    const int per = kFillThreads * kFillPer;
    hipLaunchKernelGGL(cache_fill_kernel, dim3((a.max_tokens - 1) / per + 1), dim3(kFillThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_cache_release(const ReleaseArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(cache_release_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_cache_append(const AppendArgs& a, int D, bool bf16, hipStream_t stream) {
    // single tokens get a workgroup each while there are few, long lists one for
    // up to 64 tokens (27 thousand tokens of 8 heads: 58 us by 32, 44 by 64,
    // where fewer workgroups find no run of their own)
    int per = 1;
    while (per < 64 && (long long)a.N * a.Hkv > 4096ll * per) per *= 2;
    const long long blocks = (((long long)a.N - 1) / per / 8 + 1) * 8;
    const dim3 grid((unsigned)(blocks * a.Hkv * 2));
    if (bf16 && D == 128)
        hipLaunchKernelGGL((cache_append_kernel<uint16_t, 128>), grid, dim3(kAppendThreads), 0, stream, a, per);
    else if (bf16)
        hipLaunchKernelGGL((cache_append_kernel<uint16_t, 64>), grid, dim3(kAppendThreads), 0, stream, a, per);
    else if (D == 128)
        hipLaunchKernelGGL((cache_append_kernel<float, 128>), grid, dim3(kAppendThreads), 0, stream, a, per);
    else
        hipLaunchKernelGGL((cache_append_kernel<float, 64>), grid, dim3(kAppendThreads), 0, stream, a, per);
    return hipGetLastError();
}

}  // namespace tf
