// Attention of bf16 queries on the matrix cores.
//
// A wave holds NQ * 16 query rows (one position's heads of a key head,
// position after position) against 32 tokens at a time, all of it in
// registers, with 16x16x32 products:
//   S^T [16 tokens, 16 rows] = K Q^T        (bf16: stored codes are exact in it)
//   O^T [16 dims, 16 rows] += V^T W         (fp16: codes are exact in it, the
//                                            weights rounded to 11 bits)
// The tokens of a tile may come in any order as long as both products use the
// same one, so row r of S^T tile s is token 8*(r>>2) + 4*s + (r&3): then the
// accumulators of a lane's quarter hold 8 consecutive tokens, which is what
// the second product's operand wants -- the weights never leave their lane --
// and what one 8-byte load of the transposed values gives.  The keys'
// dimensions are dealt out the same way, 16 contiguous ones a quarter.
//
// The page's value scale 2^e enters the exponent: with u = x + e and m the
// running maximum of u, weights 2^(u - m) stay within fp16's range whatever
// the scales, the products take the bare codes, and the denominator adds
// 2^(u - m) * 2^-e in fp32.  m is only raised when it is passed by more than
// kSlack, since raising it means scaling all of O^T and a maximum over the
// lanes that share a row.  Beside pages of scale 2^64 the weights of pages of
// 2^-64 (those of zeros) are 2^-128 and less: nothing to the products, but not to
// the denominator.  So weights are made 2^kLift as large, and the products' are
// brought back as they are rounded to fp16.
//
// What bounds it: with few rows the reads (64 sequences' single tokens over up
// to 8192: 153 us, 5.2 TB/s of cache); with many the latency of a tile's chain --
// products, the codes' conversion, which the NQ row tiles share, 8 exponents a row
// tile, products -- at the one or two waves a SIMD that registers allow: 16
// sequences, 33 positions of 4 heads a key head, up to 16384 tokens take 205 us
// (0.53 PFLOP/s), vector instructions issue in 46% of the cycles, the matrix units
// are busy in 24%, a wave waits a third of its time for data and a third for its
// turn, and 18% of the CUs' time is the uneven contexts' end.
#include "attend.hpp"

namespace tf {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr int kTileRows = 16, kMostTiles = 3;
constexpr float kSlack = 6.f;   // weights up to 2^6: far inside fp16

// Eight codes (two dwords) as bf16 or fp16, exact.
__device__ __forceinline__ u32x4 codes_bf16(uint32_t a, uint32_t b) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true));
    return r;
}
__device__ __forceinline__ u32x4 codes_f16(uint32_t a, uint32_t b) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true));
    return r;
}
__device__ __forceinline__ f32x4 mfma_bf16(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// two floats to fp16, round to nearest even
__device__ __forceinline__ uint32_t f16_pair(float a, float b) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32pair){a, b}, h2));
}

// Pages of a wave's next 64 tiles, a tile a lane, so that a tile's loads do
// not wait for its table entry.  Pages of 16 tokens: one for each of the
// tile's halves.  A page that is none becomes -1.
template <int PAGE>
struct TilePages {
    int id[PAGE == 16 ? 2 : 1];
    __device__ void load(const AttendArgs& a, const int32_t* table, int t0, int kStep) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int h = 0; h < (PAGE == 16 ? 2 : 1); ++h) {
            const long long t = (long long)t0 + (long long)lane * kStep + 16 * h;
            const int p = table[min((int)(t / PAGE), a.max_pages - 1)];
            id[h] = p >= 0 && p < a.num_pages ? p : -1;
        }
    }
};

// One tile's place in the cache: pages (no page: page 0, which is there, and
// its tokens count for nothing) and the tokens that are real.
template <int PAGE>
struct TilePlace {
    size_t head[PAGE == 16 ? 2 : 1];   // page and head, of the tile's halves
    int off;                           // of the tile's first token in its page
    int ends[PAGE == 16 ? 2 : 1];      // tokens from the tile's first on that are real
    __device__ void set(const AttendArgs& a, const TilePages<PAGE>& pages, int nth, int hk, int t0, int hi) {
#pragma unroll
        for (int h = 0; h < (PAGE == 16 ? 2 : 1); ++h) {
            const int p = __builtin_amdgcn_readlane(pages.id[h], nth);
            head[h] = (size_t)max(p, 0) * a.Hkv + hk;
            ends[h] = p >= 0 ? hi - t0 : 0;
        }
        off = t0 & (PAGE - 1);
    }
    __device__ bool whole() const { return ends[0] >= 32 && (PAGE != 16 || ends[PAGE == 16 ? 1 : 0] >= 32); }
    // of the lane's quarter, 8 or less
    __device__ int left(int quarter) const {
        const int e = PAGE == 16 && quarter >= 2 ? ends[PAGE == 16 ? 1 : 0] : ends[0];
        return min(max(e - 8 * quarter, 0), 8);
    }
};

// What a wave reads of a tile; `lane_k`, `lane_v`: the lane's place in a page and head.
template <int D, int PAGE>
__device__ __forceinline__ void load_keys(u32x4 (&k)[2][D / 64], const AttendArgs& a, const TilePlace<PAGE>& at, int lane_k) {
    const uint8_t* p;
    if constexpr (PAGE == 16) p = a.k_cache + ((threadIdx.x & 8) != 0 ? at.head[1] : at.head[0]) * (16 * D) + lane_k;
    else p = a.k_cache + (at.head[0] * PAGE + at.off) * D + (unsigned)lane_k;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) k[s][c] = *reinterpret_cast<const u32x4*>(p + 4 * s * D + 64 * c);
}
template <int D, int PAGE>
__device__ __forceinline__ void load_values(uint2 (&v)[D / 16], const AttendArgs& a, const TilePlace<PAGE>& at, int lane_v) {
    const uint8_t* p;
    if constexpr (PAGE == 16) p = a.v_cache + ((threadIdx.x & 32) != 0 ? at.head[1] : at.head[0]) * (16 * D) + lane_v;
    else p = a.v_cache + at.head[0] * (PAGE * D) + at.off + (unsigned)lane_v;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) v[c] = *reinterpret_cast<const uint2*>(p + 16 * c * PAGE);
}
// of the lane's quarter
template <int PAGE>
__device__ __forceinline__ float scale_of(const float* scale, const TilePlace<PAGE>& at) {
    if constexpr (PAGE == 16) return scale[(threadIdx.x & 32) != 0 ? at.head[1] : at.head[0]];
    else return scale[at.head[0]];
}

// The running softmax of a lane's query row (the four lanes of a row hold the
// same m, which stands here less kLift).
struct Running {
    float m, l;
};

// x[8] become weights 2^(x ks + e - m + LIFT); O^T and l follow a raised m.  ks
// is not negative, so the largest x has the largest weight; -inf is not there
// (ks is 1 then).  `inv`: what the denominator's weights carry, 2^-(e + LIFT).
template <int D, int LIFT>
__device__ __forceinline__ void weigh(float (&x)[8], float ks, float e, float inv, Running& s, f32x4 (&o)[D / 16]) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
    top = fmaf(top, ks, e);
    if (__any(top > s.m + (kSlack + kLift))) {   // also from an empty start (-inf)
        top = fmaxf(top, lane_xor<16>(top));
        top = fmaxf(top, lane_xor<32>(top));
        const bool raise = top > s.m + (kSlack + kLift);
        top -= kLift;
        // in halves: l is 2^64 after quiet pages alone, and that under a loud one's m
        const float h = raise ? __builtin_amdgcn_exp2f(0.5f * (s.m - top)) : 1.f, f = h * h;
        s.m = raise ? top : s.m;
        s.l = s.l * h * h;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[c][j] *= f;
    }
    const float off = (s.m == neg_inf() ? 0.f : e - s.m) - (kLift - LIFT);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = __builtin_amdgcn_exp2f(fmaf(x[j], ks, off));
        sum += x[j];
    }
    s.l = fmaf(sum, inv, s.l);
}

// Workgroup (block of NQ * 16 query rows of a key head, range of the context):
// its four waves take 32 tokens in turn, all for the same rows, and are joined
// through LDS.  Blocks of the same tokens follow one another on an XCD, whose
// L2 then serves all but the first.
template <int D, int NQ, int PAGE>
__global__ __launch_bounds__(kAttendThreads, 2) void attend_tile_kernel(AttendArgs a, int blocks) {
    constexpr int kC = D / 64, kT = D / 16;
    constexpr int kPitch = D + 4;
    constexpr int kValuePitch = D + 8;
    union WaveShared {
        float sums[kTileRows][kPitch];          // at the end
        uint16_t values[32][kValuePitch];       // of new positions
        float weights[32][kTileRows];
    };
    __shared__ __align__(16) WaveShared shared[kAttendWaves];
    __shared__ float sm[kAttendWaves][kTileRows], sl[kAttendWaves][kTileRows];
    const int tid = threadIdx.x, lane = tid & 63, quarter = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // so that a tile's addresses are scalars
    const int y = blockIdx.x / 8, block = y % blocks;
    const long long unit = (long long)(y / blocks) * 8 + blockIdx.x % 8;
    if (unit >= (long long)a.b * a.Hkv * a.splits) return;
    const int range = (int)(unit % a.splits), sh = (int)(unit / a.splits);
    const int hk = sh % a.Hkv, s = sh / a.Hkv;
    const int nl = new_of(a, s), ctx = context_of(a, s);
    const int group = a.Hq / a.Hkv, rows = nl * group;
    const Split sp = split_context(ctx, a.splits);
    const int row0 = block * (NQ * kTileRows);
    if (row0 >= rows || range >= sp.count) return;   // uniform

    u32x4 q[NQ][kC][2];
    int pos[NQ];
    Running st[NQ];
    f32x4 o[NQ][kT];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = min(row0 + n * kTileRows + col, rows - 1);
        pos[n] = row / group;
        const uint16_t* p = static_cast<const uint16_t*>(a.q) + ((size_t)s * a.n + pos[n]) * a.ld_q +
                            (size_t)(hk * group + row % group) * D + 16 * quarter;
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                q[n][c][h] = *reinterpret_cast<const u32x4*>(p + 64 * c + 8 * h);
                if (a.scale < 0.f)   // the sign goes to the queries
#pragma unroll
                    for (int w = 0; w < 4; ++w) q[n][c][h][w] ^= 0x80008000u;
            }
#pragma unroll
        for (int c = 0; c < kT; ++c) o[n][c] = f32x4{};
        st[n] = {neg_inf(), 0.f};
    }
    const float qscale = fabsf(a.scale) * kLog2e;
    const int32_t* table = a.block_table + (size_t)s * a.max_pages;
    const int lo = sp.begin(range), hi = sp.end(range, ctx);
    constexpr int kStep = kAttendWaves * 32;
    const int kt = 8 * (col >> 2) + (col & 3);   // token of the lane's key row (s = 0)
    const int lane_k = (kt & (PAGE - 1)) * D + 16 * quarter;
    const int lane_v = col * PAGE + (8 * quarter & (PAGE - 1));
    int t0 = lo + wave * 32;
    // The next tile's keys and values are in flight through the work on this one;
    // with three row tiles there are registers for one set alone, and each is
    // read again as soon as it has been used.
    constexpr bool kOneSet = NQ == kMostTiles;
    struct Tile {
        u32x4 k[2][kC];
        uint2 v[kT];
        float ks, vs;
        TilePlace<PAGE> place;
    } even, odd;
    TilePages<PAGE> pages, later;   // of tiles 64i.. and 64(i+1)..
    int nth = 0;
    auto work = [&](Tile& t, Tile& next) {
        const TilePlace<PAGE> place = t.place;
        const float k_scale = t.ks, v_scale = t.vs;
        const bool more = t0 + kStep < hi;
        TilePlace<PAGE> to = place;
        if (more) {
            if ((nth & 63) == 0) later.load(a, table, (int)min((long long)t0 + 64 * kStep, (long long)hi - 1), kStep);   // used 63 tiles on
            if ((nth & 63) == 63) pages = later;
            ++nth;
            to.set(a, pages, nth & 63, hk, t0 + kStep, hi);
            if (!kOneSet) {
                load_keys<D, PAGE>(next.k, a, to, lane_k);
                load_values<D, PAGE>(next.v, a, to, lane_v);
            }
            next.ks = scale_of<PAGE>(a.k_scale, to);
            next.vs = scale_of<PAGE>(a.v_scale, to);
        }
        f32x4 acc[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) acc[n][0] = acc[n][1] = f32x4{};
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const u32x4 k0 = codes_bf16(t.k[0][c][2 * d], t.k[0][c][2 * d + 1]);
                const u32x4 k1 = codes_bf16(t.k[1][c][2 * d], t.k[1][c][2 * d + 1]);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    acc[n][0] = mfma_bf16(k0, q[n][c][d], acc[n][0]);
                    acc[n][1] = mfma_bf16(k1, q[n][c][d], acc[n][1]);
                }
            }
        if (kOneSet && more) load_keys<D, PAGE>(next.k, a, to, lane_k);
        __builtin_amdgcn_sched_barrier(0);   // the values' operands are made after the weights: else they spill
        const int e = (int)(__float_as_uint(v_scale) >> 23) - 127;
        const bool part = !place.whole();   // uniform
        const int left = place.left(quarter);
        // where a quarter has no token, the scale is a page's that may never have been written
        const float ks = k_scale * qscale, inv = left == 0 ? 1.f : __uint_as_float((uint32_t)(127 - kLift - e) << 23);
        constexpr float kDrop = 1.f / (1ull << kLift);
        u32x4 p[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = acc[n][j >> 2][j & 3];
            float k1 = ks, e1 = (float)e;
            if (part) {
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = j < left ? fmaf(u[j], ks, e1) : neg_inf();
                k1 = 1.f;
                e1 = 0.f;
            }
            weigh<D, kLift>(u, k1, e1, inv, st[n], o[n]);
#pragma unroll
            for (int j = 0; j < 4; ++j) p[n][j] = f16_pair(u[2 * j] * kDrop, u[2 * j + 1] * kDrop);
        }
        if (part) {   // what lies behind the tokens may be NaN
            const int l0 = min(left, 4), l1 = max(left - 4, 0);
            const uint32_t m0 = l0 == 4 ? ~0u : (1u << (8 * l0)) - 1u, m1 = l1 == 4 ? ~0u : (1u << (8 * l1)) - 1u;
#pragma unroll
            for (int c = 0; c < kT; ++c) t.v[c].x &= m0, t.v[c].y &= m1;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < kT; ++c) {
            const u32x4 x = codes_f16(t.v[c].x, t.v[c].y);
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[n][c] = mfma_f16(x, p[n], o[n][c]);
        }
        if (kOneSet && more) load_values<D, PAGE>(next.v, a, to, lane_v);
        next.place = to;
        t0 += kStep;
    };
    if (t0 < hi) {
        pages.load(a, table, t0, kStep);
        later = pages;
        even.place.set(a, pages, 0, hk, t0, hi);
        load_keys<D, PAGE>(even.k, a, even.place, lane_k);
        load_values<D, PAGE>(even.v, a, even.place, lane_v);
        even.ks = scale_of<PAGE>(a.k_scale, even.place);
        even.vs = scale_of<PAGE>(a.v_scale, even.place);
    }
    while (t0 < hi) {
        if constexpr (kOneSet) {
            work(even, even);
        } else {
            work(even, odd);
            if (t0 >= hi) break;
            work(odd, even);
        }
    }

    if (range == sp.count - 1) {
        // The new positions go with the last range.  Their values are bf16, so
        // the weights enter as a bf16 hi/lo pair (16 bits).  A value that is no
        // number must not reach the rows that do not attend to it, through
        // 0 * NaN: it is taken out of the product and added row by row.
        const int jend = a.mask != nullptr ? nl : min(nl, (row0 + NQ * kTileRows - 1) / group + 1);   // a chain's last row ends it
        // a bit for each of 8 positions from j that row n attends to
        auto seen = [&](int n, int j) {
            unsigned bits = 0;
            if (a.mask != nullptr) {   // every byte's load in flight before the first is looked at
                const uint8_t* mask = a.mask + ((size_t)s * a.n + pos[n]) * a.n;
                uint8_t m[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) m[e] = mask[min(j + e, nl - 1)];
#pragma unroll
                for (int e = 0; e < 8; ++e) bits |= (m[e] != 0 ? 1u : 0u) << e;
            } else {
                bits = (1u << min(max(pos[n] - j + 1, 0), 8)) - 1u;
            }
            return bits & ((1u << min(max(nl - j, 0), 8)) - 1u);
        };
        for (int j0 = wave * 32; j0 < jend; j0 += kStep) {
            const int jv = j0 + 8 * quarter;   // first of the lane's 8 positions
            // Where a wave has several turns, one of which no row sees anything
            // is left out (4 trees of 513 positions: 164 us, 190 with all turns);
            // a single turn reads its keys without waiting for the mask.
            if (a.mask != nullptr && nl > kStep) {
                unsigned some = 0;
#pragma unroll
                for (int n = 0; n < NQ; ++n) some |= seen(n, jv);
                if (!__any(some != 0)) continue;
            }
            f32x4 acc[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) acc[n][0] = acc[n][1] = f32x4{};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* k = static_cast<const uint16_t*>(a.k_new) +
                                    ((size_t)s * a.n + min(j0 + kt + 4 * h, nl - 1)) * a.ld_new + (size_t)hk * D + 16 * quarter;
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    const u32x4 k0 = *reinterpret_cast<const u32x4*>(k + 64 * c);
                    const u32x4 k1 = *reinterpret_cast<const u32x4*>(k + 64 * c + 8);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        acc[n][h] = mfma_bf16(k0, q[n][c][0], acc[n][h]);
                        acc[n][h] = mfma_bf16(k1, q[n][c][1], acc[n][h]);
                    }
                }
            }
            u32x4 ph[NQ], pl[NQ];
            float w[NQ][8];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const unsigned sees = seen(n, jv);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[n][j] = sees >> j & 1 ? acc[n][j >> 2][j & 3] * qscale : neg_inf();
                weigh<D, 0>(w[n], 1.f, 0.f, 1.f, st[n], o[n]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t h = f32x2_to_bf16x2_bits(w[n][2 * j], w[n][2 * j + 1]);
                    ph[n][j] = h;
                    pl[n][j] = f32x2_to_bf16x2_bits(w[n][2 * j] - __uint_as_float(h << 16),
                                                    w[n][2 * j + 1] - __uint_as_float(h & 0xffff0000u));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)   // for the row-by-row sums: 0 where the row does not attend
                    w[n][j] = sees >> j & 1 ? fmaxf(w[n][j], 1e-30f) : 0.f;
            }
            const uint16_t* vn = static_cast<const uint16_t*>(a.v_new) + (size_t)s * a.n * a.ld_new + (size_t)hk * D;
            // whole rows into LDS, columns out of it: a lane's operand is 8
            // positions of one dimension (single loads from memory took 4-17 us
            // of the workgroup)
            uint16_t (&turn)[32][kValuePitch] = shared[wave].values;
            constexpr int kRowLanes = D / 8;
#pragma unroll
            for (int i = 0; i < 32 * kRowLanes / kWave; ++i) {
                const int r = i * (kWave / kRowLanes) + lane / kRowLanes, d = lane % kRowLanes * 8;
                *reinterpret_cast<u32x4*>(&turn[r][d]) =
                    *reinterpret_cast<const u32x4*>(vn + (size_t)min(j0 + r, nl - 1) * a.ld_new + d);
            }
            __builtin_amdgcn_wave_barrier();
            bool strange = false;
#pragma unroll
            for (int c = 0; c < kT; ++c) {
                u32x4 v;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t x = turn[8 * quarter + j][16 * c + col];
                    const bool bad = (x & 0x7f80u) == 0x7f80u;
                    strange |= bad;
                    x = bad ? 0u : x;
                    if (j & 1) v[j >> 1] |= x << 16;
                    else v[j >> 1] = x;
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][c] = mfma_bf16(v, ph[n], o[n][c]);
                    o[n][c] = mfma_bf16(v, pl[n], o[n][c]);
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (__any(strange)) {
                float (&lw)[32][kTileRows] = shared[wave].weights;
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) lw[8 * quarter + j][col] = w[n][j];
                    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                    for (int j = 0; j < min(32, nl - j0); ++j) {
                        const float f = lw[j][col];
                        const uint16_t* row = vn + (size_t)(j0 + j) * a.ld_new;
                        if (f == 0.f) continue;
#pragma unroll
                        for (int c = 0; c < kT; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t x = row[16 * c + 4 * quarter + i];
                                if ((x & 0x7f80u) == 0x7f80u) o[n][c][i] += f * bf16_bits_to_f32(x);
                            }
                    }
                    __builtin_amdgcn_wave_barrier();
                }
            }
        }
    }

    // the four waves joined, a row tile at a time
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float l = st[n].l + lane_xor<16>(st[n].l);
        l += lane_xor<32>(l);
        if (quarter == 0) sm[wave][col] = st[n].m, sl[wave][col] = l;
        __syncthreads();   // sm, sl written; the waves' parts are free
        float mt = neg_inf();
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) mt = fmaxf(mt, sm[w][col]);
        const float f = st[n].m == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(st[n].m - mt);
#pragma unroll
        for (int c = 0; c < kT; ++c)
            *reinterpret_cast<f32x4*>(&shared[wave].sums[col][16 * c + 4 * quarter]) =
                f32x4{o[n][c][0] * f, o[n][c][1] * f, o[n][c][2] * f, o[n][c][3] * f};
        __syncthreads();
        for (int i = tid; i < kTileRows * (D / 4); i += kAttendThreads) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            const int row = row0 + n * kTileRows + r;
            if (row >= rows) continue;
            float m = neg_inf(), lt = 0.f;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, sm[w][r]);
            for (int w = 0; w < kAttendWaves; ++w) {
                const float h = sm[w][r] == neg_inf() ? 1.f : __builtin_amdgcn_exp2f(0.5f * (sm[w][r] - m));
                lt += sl[w][r] * h * h;
                const f32x4 v = *reinterpret_cast<const f32x4*>(&shared[w].sums[r][d]);
                for (int k = 0; k < 4; ++k) x[k] += v[k];
            }
            const size_t to = ((size_t)s * a.n + row / group) * a.Hq + hk * group + row % group;
            if (sp.count == 1) {
                const bool none = lt == 0.f;   // a NaN sum stays one
                const float g = none ? 0.f : 1.f / lt;
                uint2 v;
                v.x = f32x2_to_bf16x2_bits(none ? 0.f : x[0] * g, none ? 0.f : x[1] * g);
                v.y = f32x2_to_bf16x2_bits(none ? 0.f : x[2] * g, none ? 0.f : x[3] * g);
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to * D + d) = v;
                if (d == 0 && a.lse != nullptr) a.lse[to] = lse_of(m + kLift, lt);
            } else {
                *reinterpret_cast<f32x4*>(part_sums(a, to, range, D) + d) = x;
                if (d == 0) {
                    float* ml = part_stats(a, to, range, D);
                    ml[0] = m;
                    ml[1] = lt;
                }
            }
        }
        __syncthreads();   // all of it is free again
    }
}

// Row tiles spread evenly over the fewest blocks of up to three.
TileBlocks tile_blocks(int n, int Hq, int Hkv) {
    const long long tiles = ((long long)n * (Hq / Hkv) + kTileRows - 1) / kTileRows;
    const long long blocks = (tiles + kMostTiles - 1) / kMostTiles;
    return {(int)blocks, (int)((tiles + blocks - 1) / blocks)};
}

namespace {
template <int D, int NQ>
void launch_blocks(const AttendArgs& a, int blocks, unsigned grid, hipStream_t stream) {
    const dim3 g(grid), w(kAttendThreads);
    if (a.page == 16) hipLaunchKernelGGL((attend_tile_kernel<D, NQ, 16>), g, w, 0, stream, a, blocks);
    else if (a.page == 32) hipLaunchKernelGGL((attend_tile_kernel<D, NQ, 32>), g, w, 0, stream, a, blocks);
    else if (a.page == 64) hipLaunchKernelGGL((attend_tile_kernel<D, NQ, 64>), g, w, 0, stream, a, blocks);
    else hipLaunchKernelGGL((attend_tile_kernel<D, NQ, 128>), g, w, 0, stream, a, blocks);
}
}  // namespace

hipError_t launch_attend_tile(const AttendArgs& a, int D, hipStream_t stream) {
    const TileBlocks tb = tile_blocks(a.n, a.Hq, a.Hkv);
    const long long units = (long long)a.b * a.Hkv * a.splits;
    const long long grid = (units + 7) / 8 * 8 * tb.blocks;
    const unsigned g = (unsigned)grid;
    if (D == 128) {
        if (tb.tiles == 1) launch_blocks<128, 1>(a, tb.blocks, g, stream);
        else if (tb.tiles == 2) launch_blocks<128, 2>(a, tb.blocks, g, stream);
        else launch_blocks<128, 3>(a, tb.blocks, g, stream);
    } else {
        if (tb.tiles == 1) launch_blocks<64, 1>(a, tb.blocks, g, stream);
        else if (tb.tiles == 2) launch_blocks<64, 2>(a, tb.blocks, g, stream);
        else launch_blocks<64, 3>(a, tb.blocks, g, stream);
    }
    return hipGetLastError();
}

}  // namespace tf
