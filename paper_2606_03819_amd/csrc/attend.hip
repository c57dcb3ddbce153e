// Attention of a tree's positions over the paged 8-bit cache and the tree.
//
// A row is one query head at one position.  With t running over the cached
// tokens and the new positions that the mask admits,
//   out = sum_t w_t v_t / sum_t w_t,   w_t = 2^(x_t - m),
//   x_t = log2(e) * scale * q.k_t,
// in one pass: m is the running maximum, and sums made under an older one are
// scaled by 2^(old - new).  Ranges of a long context are worked on side by
// side and joined by merge_kernel in the same way.
#include "attend.hpp"

namespace tf {

// fp32.  Workgroup (position, up to G heads of one key head, range): its
// waves take 64 tokens in turn.  For the products q.k a lane is a token, for
// the sums over values a dimension, so both read 16 contiguous codes a lane
// and the weights change places through LDS.  New positions are few and their
// rows wide: four lanes share one, sixteen go to a wave, and a wave's loads of
// them are all in flight at once.  What bounds it: the latency of these loads
// while there are few positions (2 trees of 100 over 500 tokens, 4 heads a key
// head: 29 us, 57 with the queries in registers), then fp32 arithmetic.
template <int D, int G>
__global__ __launch_bounds__(kAttendThreads) void attend_rows_kernel(AttendArgs a) {
    constexpr int kDims = D / kWave;
    constexpr int kNew = kWave / 4;   // new positions a wave takes at once, four lanes each
    __shared__ float qs[G][D];
    __shared__ float ps[kAttendWaves][G][kWave];
    __shared__ float sm[kAttendWaves][G], sl[kAttendWaves][G];
    __shared__ float so[kAttendWaves][G][D];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = blockIdx.x / a.n, i = blockIdx.x % a.n;
    const int nl = new_of(a, s);
    const int ctx = context_of(a, s);
    const Split sp = split_context(ctx, a.splits);
    if (i >= nl || (int)blockIdx.z >= sp.count) return;   // uniform
    const int group = a.Hq / a.Hkv, blocks = (group + G - 1) / G;
    const int hk = blockIdx.y / blocks, g0 = (blockIdx.y % blocks) * G;
    const int ng = min(G, group - g0);
    const int head0 = hk * group + g0;
    const float* q = static_cast<const float*>(a.q) + (size_t)blockIdx.x * a.ld_q + (size_t)head0 * D;
    for (int e = tid; e < G * D; e += kAttendThreads)
        qs[e / D][e % D] = e / D < ng ? q[e] * (a.scale * kLog2e) : 0.f;
    __syncthreads();

    float m[G], l[G], o[G][kDims];
    for (int g = 0; g < G; ++g) {
        m[g] = neg_inf();
        l[g] = 0.f;
        for (int c = 0; c < kDims; ++c) o[g][c] = 0.f;
    }
    // the lane's products x become weights: LDS gets them, m, l and o follow
    auto weigh = [&](const float* x) {
        for (int g = 0; g < G; ++g) {
            const float mn = fmaxf(m[g], wave_max(x[g]));
            const float back = mn == neg_inf() ? 1.f : exp2f(m[g] - mn);   // 0 from an empty start
            const float p = exp2f(x[g] - (mn == neg_inf() ? 0.f : mn));   // a NaN stays one
            m[g] = mn;
            l[g] = l[g] * back + p;
            for (int c = 0; c < kDims; ++c) o[g][c] *= back;
            ps[wave][g][lane] = p;
        }
    };

    const int32_t* table = a.block_table + (size_t)s * a.max_pages;
    const int lo = sp.begin(blockIdx.z), hi = sp.end(blockIdx.z, ctx);
    for (int t0 = lo + wave * kWave; t0 < hi; t0 += kAttendThreads) {
        // The queries are read from LDS for every 64 tokens.  Without this the
        // compiler keeps all G * D of them in registers (330 for four heads of
        // 64), and one wave a SIMD waits out every load.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int t = t0 + lane;
        int id = t < hi ? table[t / a.page] : -1;
        if (id >= a.num_pages) id = -1;
        float x[G] = {};
        if (id >= 0) {
            const size_t head = (size_t)id * a.Hkv + hk;
            const u32x4* k = reinterpret_cast<const u32x4*>(a.k_cache + head * a.page * D + (size_t)(t & (a.page - 1)) * D);
            for (int c = 0; c < D / 16; ++c) {
                const u32x4 w = k[c];
                for (int e = 0; e < 4; ++e) {
                    const f32pair u = e4m3_pair<false>(w[e]), v = e4m3_pair<true>(w[e]);
                    for (int g = 0; g < G; ++g) {
                        const float* qq = &qs[g][c * 16 + e * 4];
                        x[g] += qq[0] * u[0] + qq[1] * u[1] + qq[2] * v[0] + qq[3] * v[1];
                    }
                }
            }
            const float ks = a.k_scale[head];
            for (int g = 0; g < G; ++g) x[g] *= ks;
        } else {
            for (int g = 0; g < G; ++g) x[g] = neg_inf();
        }
        weigh(x);
        for (int part = 0; part < kWave / 16; ++part) {   // 16 tokens lie in one page
            const int first = t0 + part * 16;
            if (first >= hi) break;
            const int page = __shfl(id, part * 16);
            if (page < 0) continue;
            const size_t head = (size_t)page * a.Hkv + hk;
            const float vs = a.v_scale[head];
            for (int c = 0; c < kDims; ++c) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(
                    a.v_cache + head * a.page * D + (size_t)(c * kWave + lane) * a.page + (first & (a.page - 1)));
                for (int e = 0; e < 4; ++e) {
                    const f32pair u = e4m3_pair<false>(w[e]), v = e4m3_pair<true>(w[e]);
                    const float y[4] = {u[0], u[1], v[0], v[1]};
                    for (int j = 0; j < 4; ++j) {
                        const int tt = e * 4 + j;
                        const float val = first + tt < hi ? y[j] * vs : 0.f;   // what lies behind may be NaN
                        for (int g = 0; g < G; ++g) o[g][c] += ps[wave][g][part * 16 + tt] * val;
                    }
                }
            }
        }
    }
    if ((int)blockIdx.z == sp.count - 1) {   // the new positions go with the last range
        const uint8_t* mask = a.mask != nullptr ? a.mask + (size_t)blockIdx.x * a.n : nullptr;
        for (int j0 = wave * kNew; j0 < nl; j0 += kNew * kAttendWaves) {
            const int j = j0 + lane / 4, part = lane % 4;
            const bool sees = j < nl && (mask != nullptr ? mask[j] != 0 : j <= i);
            unsigned long long todo = __ballot(sees && part == 0);
            if (todo == 0) continue;
            float x[G] = {};
            if (sees) {
                const f32x4* k = reinterpret_cast<const f32x4*>(
                    static_cast<const float*>(a.k_new) + ((size_t)s * a.n + j) * a.ld_new + (size_t)hk * D);
                f32x4 kv[D / 16];
#pragma unroll
                for (int c = 0; c < D / 16; ++c) kv[c] = k[c * 4 + part];
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
                    for (int g = 0; g < G; ++g) {
                        const float* qq = &qs[g][c * 16 + part * 4];
                        x[g] += qq[0] * kv[c][0] + qq[1] * kv[c][1] + qq[2] * kv[c][2] + qq[3] * kv[c][3];
                    }
            }
            for (int g = 0; g < G; ++g) {
                x[g] += __shfl_xor(x[g], 1);
                x[g] += __shfl_xor(x[g], 2);
                if (!sees || part != 0) x[g] = neg_inf();   // one lane of the four has the weight
            }
            weigh(x);
            while (todo != 0) {   // the rows attended to, four in flight
                float val[4][kDims];
                int at[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    at[r] = todo != 0 ? __builtin_ctzll(todo) : -1;
                    todo &= todo - 1;
                    const float* v = static_cast<const float*>(a.v_new) + ((size_t)s * a.n + j0 + max(at[r], 0) / 4) * a.ld_new + (size_t)hk * D;
#pragma unroll
                    for (int c = 0; c < kDims; ++c) val[r][c] = at[r] >= 0 ? v[c * kWave + lane] : 0.f;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at[r] >= 0)
#pragma unroll
                        for (int c = 0; c < kDims; ++c)
                            for (int g = 0; g < G; ++g) o[g][c] += ps[wave][g][at[r]] * val[r][c];
            }
        }
    }
    for (int g = 0; g < G; ++g) {
        const float sum = wave_sum(l[g]);
        if (lane == 0) sm[wave][g] = m[g], sl[wave][g] = sum;
        for (int c = 0; c < kDims; ++c) so[wave][g][c * kWave + lane] = o[g][c];
    }
    __syncthreads();
    for (int e = tid; e < ng * D; e += kAttendThreads) {
        const int g = e / D, d = e % D;
        float mt = neg_inf();
        for (int w = 0; w < kAttendWaves; ++w) mt = fmaxf(mt, sm[w][g]);
        float lt = 0.f, ot = 0.f;
        for (int w = 0; w < kAttendWaves; ++w) {
            const float f = sm[w][g] == neg_inf() ? 1.f : exp2f(sm[w][g] - mt);
            lt += sl[w][g] * f;
            ot += so[w][g][d] * f;
        }
        const size_t row = (size_t)blockIdx.x * a.Hq + head0 + g;
        if (sp.count == 1) {
            static_cast<float*>(a.out)[row * D + d] = lt == 0.f ? 0.f : ot / lt;
            if (d == 0 && a.lse != nullptr) a.lse[row] = lse_of(mt, lt);
        } else {
            part_sums(a, row, blockIdx.z, D)[d] = ot;
            if (d == 0) {
                float* ml = part_stats(a, row, blockIdx.z, D);
                ml[0] = mt;
                ml[1] = lt;
            }
        }
    }
}

// One wave a row: the ranges of a split context joined.
template <class T, int D>
__global__ __launch_bounds__(kAttendThreads) void merge_kernel(AttendArgs a) {
    const int lane = threadIdx.x & 63;
    const size_t row = (size_t)blockIdx.x * kAttendWaves + (threadIdx.x >> 6);
    if (row >= (size_t)a.b * a.n * a.Hq) return;
    const int s = (int)(row / ((size_t)a.n * a.Hq)), i = (int)(row / a.Hq % a.n);
    const int count = split_context(context_of(a, s), a.splits).count;
    if (count == 1 || i >= new_of(a, s)) return;
    // every range's factor first, a range a lane
    static_assert(kMostSplits <= kWave, "a range a lane");
    float mp = neg_inf(), lp = 0.f;
    if (lane < count) {
        const float* ml = part_stats(a, row, lane, D);
        mp = ml[0];
        lp = ml[1];
    }
    const float m = wave_max(mp);
    // a sum that is no number stays one; in halves, since 2^(mp - m) alone may be nothing where lp is 2^64
    const float h = mp == neg_inf() ? (lp == 0.f ? 0.f : lp) : exp2f(0.5f * (mp - m)), f = h * h;
    const float l = wave_sum(lp * h * h);
    float o[D / kWave] = {};
    constexpr int kDeep = 8;
    for (int s0 = 0; s0 < count; s0 += kDeep) {
        float x[kDeep][D / kWave];
#pragma unroll
        for (int i = 0; i < kDeep; ++i)
#pragma unroll
            for (int c = 0; c < D / kWave; ++c)
                x[i][c] = s0 + i < count ? part_sums(a, row, s0 + i, D)[c * kWave + lane] : 0.f;
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), s0 + i));
#pragma unroll
            for (int c = 0; c < D / kWave; ++c)
                if (s0 + i < count && g != 0.f) o[c] += x[i][c] * g;
        }
    }
    for (int c = 0; c < D / kWave; ++c) store_out(a.out, row * D + c * kWave + lane, l == 0.f ? 0.f : o[c] / l, sizeof(T) == 2);
    if (lane == 0 && a.lse != nullptr) a.lse[row] = lse_of(sizeof(T) == 2 ? m + kLift : m, l);
}

namespace {

// Ranges a context is split into at most.  `groups` workgroups serve one range
// and `slots` of them run at once.  Few groups are split to fill the slots
// once (a second round of mostly idle units costs what the first does: 24
// groups over 8192 tokens 32 us against 37); many are split so that uneven
// contexts spread over two rounds or more (384 groups over up to 16384 tokens:
// 239 us in two ranges, 218 in three, 227 in four, and the partial sums grow).
int most_splits(long long groups, int slots, int max_pages, int page) {
    const long long longest = ((long long)max_pages * page + kSplitLeast - 1) / kSplitLeast;
    long long want = groups * 2 <= slots ? slots / groups : (2 * slots + groups - 1) / groups;
    want = want < longest ? want : longest;
    return (int)(want < 1 ? 1 : want > kMostSplits ? kMostSplits : want);
}

int row_blocks(int Hq, int Hkv) { return (Hq / Hkv + kGroupRows - 1) / kGroupRows; }

int splits_of(int b, int n, int Hq, int Hkv, int page, int max_pages, bool bf16) {
    // workgroups on 256 CUs: two by the matrix kernel's registers, four of the row kernel
    if (bf16) return most_splits((long long)b * Hkv * tile_blocks(n, Hq, Hkv).blocks, 512, max_pages, page);
    return most_splits((long long)b * n * Hkv * row_blocks(Hq, Hkv), 1024, max_pages, page);
}

// A key head's G is the smallest that holds its group, since every product,
// maximum and exponent is made for all G heads (11 sequences of 25 positions, 2
// heads a key head: 24 us, 37 by four; 4 of 33 over 2000 tokens, single heads of
// 64: 40 us, 70 by four).
template <int D>
void launch_rows(const AttendArgs& a, hipStream_t stream) {
    const int group = a.Hq / a.Hkv;
    const dim3 grid(a.b * a.n, a.Hkv * row_blocks(a.Hq, a.Hkv), a.splits), w(kAttendThreads);
    if (group == 1) hipLaunchKernelGGL((attend_rows_kernel<D, 1>), grid, w, 0, stream, a);
    else if (group == 2) hipLaunchKernelGGL((attend_rows_kernel<D, 2>), grid, w, 0, stream, a);
    else hipLaunchKernelGGL((attend_rows_kernel<D, kGroupRows>), grid, w, 0, stream, a);
}

template <class T>
hipError_t launch_merge(const AttendArgs& a, int D, hipStream_t stream) {
    const dim3 grid((unsigned)(((long long)a.b * a.n * a.Hq + kAttendWaves - 1) / kAttendWaves));
    if (D == 128) hipLaunchKernelGGL((merge_kernel<T, 128>), grid, dim3(kAttendThreads), 0, stream, a);
    else hipLaunchKernelGGL((merge_kernel<T, 64>), grid, dim3(kAttendThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

size_t attend_part_bytes(int b, int n, int Hq, int Hkv, int D, int page, int max_pages, bool bf16) {
    const int splits = splits_of(b, n, Hq, Hkv, page, max_pages, bf16);
    return splits == 1 ? 0 : (size_t)splits * b * n * Hq * (D + 2) * 4;
}

hipError_t launch_tree_attention(AttendArgs a, int D, bool bf16, hipStream_t stream) {
    a.splits = splits_of(a.b, a.n, a.Hq, a.Hkv, a.page, a.max_pages, bf16);
    hipError_t e;
    if (bf16) {
        e = launch_attend_tile(a, D, stream);
    } else {
        if (D == 128) launch_rows<128>(a, stream);
        else launch_rows<64>(a, stream);
        e = hipGetLastError();
    }
    if (e != hipSuccess || a.splits == 1) return e;
    return bf16 ? launch_merge<uint16_t>(a, D, stream) : launch_merge<float>(a, D, stream);
}

}  // namespace tf
