// Attention of bf16 queries on the matrix cores.
//
// A wave holds 32 query rows (one position's heads of a key head, position
// after position) against 32 tokens at a time, all of it in registers:
//   S^T [32 tokens, 32 rows] = K Q^T      (bf16: stored codes are exact in it)
//   O^T [D, 32 rows] += V^T W             (fp16: codes are exact in it, the
//                                          weights rounded to 11 bits)
// The tokens of a tile may come in any order as long as both products use the
// same one, so row r of S^T is token 16*((r>>2)&1) + 4*(r>>3) + (r&3): then the
// accumulator of a lane's half holds 16 consecutive tokens, which is what the
// second product's operand wants -- the weights never leave their lane -- and
// what one 16-byte load of the transposed values gives.  The keys' dimensions
// are dealt out the same way, 16 contiguous ones a half.
//
// The page's value scale 2^e enters the exponent: with u = x + e and m the
// running maximum of u, weights 2^(u - m) stay within fp16's range whatever
// the scales, the products take the bare codes, and the denominator adds
// 2^(u - m) * 2^-e in fp32.  m is only raised when it is passed by more than
// kSlack, since raising it means scaling all of O^T.
#include "attend.hpp"

namespace tf {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr int kTileRows = 32;
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
__device__ __forceinline__ f32x16 mfma_32x32x16_f16(const u32x4& a, const u32x4& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// two floats to fp16, round to nearest even
__device__ __forceinline__ uint32_t f16_pair(float a, float b) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32pair){a, b}, h2));
}

// 32 tokens as a wave reads them, with what they are scaled by.
template <int D>
struct TokenTile {
    u32x4 k[D / 32], v[D / 32];
    float ks, vs;   // of the lane's half: key scale, value scale
    int left;       // tokens of the lane's half that are real, 16 or less
};

// Pages of a wave's next 64 tiles, a tile a lane and each of the tile's halves
// apart, so that a tile's loads do not wait for its table entry.  A page that
// is none becomes -1.
struct TilePages {
    int id[2];
    __device__ void load(const AttendArgs& a, const int32_t* table, int t0, int step) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long t = (long long)t0 + (long long)lane * step + 16 * h;
            const int p = table[min((int)(t / a.page), a.max_pages - 1)];
            id[h] = p >= 0 && p < a.num_pages ? p : -1;
        }
    }
};

template <int D>
__device__ __forceinline__ void load_tile(TokenTile<D>& t, const AttendArgs& a, const TilePages& pages, int nth, int hk,
                                          int t0, int hi) {
    const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
    const int kb = (r >> 2) & 1;
    const int p0 = __builtin_amdgcn_readlane(pages.id[0], nth), p1 = __builtin_amdgcn_readlane(pages.id[1], nth);
    const int id0 = max(p0, 0), id1 = max(p1, 0);   // no page: its tokens count for nothing, and page 0 is there
    const int idk = kb ? id1 : id0, idv = half ? id1 : id0;
    const int tk = (t0 + 16 * kb + 4 * (r >> 3) + (r & 3)) & (a.page - 1);
    const int tv = (t0 + 16 * half) & (a.page - 1);
    const size_t headk = (size_t)idk * a.Hkv + hk, headv = (size_t)idv * a.Hkv + hk;
    const uint8_t* k = a.k_cache + (headk * a.page + tk) * D + 16 * half;
    const uint8_t* v = a.v_cache + (headv * D + r) * a.page + tv;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        t.k[c] = *reinterpret_cast<const u32x4*>(k + 32 * c);
        t.v[c] = *reinterpret_cast<const u32x4*>(v + (size_t)(32 * c) * a.page);
    }
    t.ks = a.k_scale[headv];
    t.vs = a.v_scale[headv];
    t.left = (half ? p1 : p0) >= 0 ? min(max(hi - t0 - 16 * half, 0), 16) : 0;
}

// The running softmax of a lane's query row (both halves hold the same m).
struct Running {
    float m, l;
};

// x[16] become weights 2^(x ks + e - m); O^T and l follow a raised m.  ks is
// not negative, so the largest x has the largest weight; -inf is not there
// (ks is 1 then).  `inv`: what the denominator's weights carry, 2^-e.
template <int D>
__device__ __forceinline__ void weigh(float (&x)[16], float ks, float e, float inv, Running& s, f32x16 (&o)[D / 32]) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, x[j]);
    top = fmaf(top, ks, e);
    top = fmaxf(top, lane_xor<32>(top));
    const bool raise = top > s.m + kSlack;   // also from an empty start (-inf)
    if (__any(raise)) {
        const float f = raise ? __builtin_amdgcn_exp2f(s.m - top) : 1.f;
        s.m = raise ? top : s.m;
        s.l *= f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[c][j] *= f;
    }
    const float off = s.m == neg_inf() ? 0.f : e - s.m;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        x[j] = __builtin_amdgcn_exp2f(fmaf(x[j], ks, off));
        sum += x[j];
    }
    s.l = fmaf(sum, inv, s.l);
}

// Workgroup (block of NQ * 32 query rows of a key head, range of the context):
// its four waves take 32 tokens in turn, all for the same rows, and are joined
// through LDS.  Blocks of the same tokens follow one another on an XCD, whose
// L2 then serves all but the first.
template <int D, int NQ>
__global__ __launch_bounds__(kAttendThreads, 2) void attend_tile_kernel(AttendArgs a, int blocks) {
    constexpr int kC = D / 32;
    constexpr int kPitch = D / 2 + 4;
    __shared__ __align__(16) float so[kAttendWaves][kTileRows][kPitch];
    __shared__ float sm[kAttendWaves][kTileRows], sl[kAttendWaves][kTileRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
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
    f32x16 o[NQ][kC];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = min(row0 + n * kTileRows + col, rows - 1);
        pos[n] = row / group;
        const uint16_t* p = static_cast<const uint16_t*>(a.q) + ((size_t)s * a.n + pos[n]) * a.ld_q +
                            (size_t)(hk * group + row % group) * D + 16 * half;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            q[n][c][0] = *reinterpret_cast<const u32x4*>(p + 32 * c);
            q[n][c][1] = *reinterpret_cast<const u32x4*>(p + 32 * c + 8);
            o[n][c] = f32x16{};
            if (a.scale < 0.f)   // the sign goes to the queries
#pragma unroll
                for (int w = 0; w < 4; ++w) q[n][c][0][w] ^= 0x80008000u, q[n][c][1][w] ^= 0x80008000u;
        }
        st[n] = {neg_inf(), 0.f};
    }
    const float qscale = fabsf(a.scale) * kLog2e;
    const int32_t* table = a.block_table + (size_t)s * a.max_pages;
    const int lo = range * sp.chunk, hi = min(ctx, lo + sp.chunk);
    constexpr int kStep = kAttendWaves * 32;
    int t0 = lo + wave * 32;
    TokenTile<D> next;
    TilePages pages, later;   // of tiles 64i.. and 64(i+1)..
    if (t0 < hi) {
        pages.load(a, table, t0, kStep);
        later = pages;
        load_tile<D>(next, a, pages, 0, hk, t0, hi);
    }
    for (int nth = 0; t0 < hi; t0 += kStep, ++nth) {
        TokenTile<D> t = next;
        if (t0 + kStep < hi) {
            if ((nth & 63) == 0) later.load(a, table, (int)min((long long)t0 + 64 * kStep, (long long)hi - 1), kStep);   // used 63 tiles on
            if ((nth & 63) == 63) pages = later;
            load_tile<D>(next, a, pages, (nth + 1) & 63, hk, t0 + kStep, hi);
        }
        f32x16 acc[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) acc[n] = f32x16{};
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const u32x4 k0 = codes_bf16(t.k[c][0], t.k[c][1]), k1 = codes_bf16(t.k[c][2], t.k[c][3]);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                acc[n] = mfma_32x32x16_bf16(k0, q[n][c][0], acc[n]);
                acc[n] = mfma_32x32x16_bf16(k1, q[n][c][1], acc[n]);
            }
        }
        const bool part = __any(t.left < 16);
        if (part) {   // what lies behind the tokens may be NaN
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int keep = min(max(t.left - 4 * w, 0), 4);
                    t.v[c][w] &= keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
                }
        }
        const int e = (int)(__float_as_uint(t.vs) >> 23) - 127;
        const float ks = t.ks * qscale, inv = __uint_as_float((uint32_t)(127 - e) << 23);
        u32x4 p[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float u[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] = acc[n][j];
            float k1 = ks, e1 = (float)e;
            if (part) {
#pragma unroll
                for (int j = 0; j < 16; ++j) u[j] = j < t.left ? fmaf(u[j], ks, e1) : neg_inf();
                k1 = 1.f;
                e1 = 0.f;
            }
            weigh<D>(u, k1, e1, inv, st[n], o[n]);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[n][j >> 2][j & 3] = f16_pair(u[2 * j], u[2 * j + 1]);
        }
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const u32x4 v0 = codes_f16(t.v[c][0], t.v[c][1]), v1 = codes_f16(t.v[c][2], t.v[c][3]);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                o[n][c] = mfma_32x32x16_f16(v0, p[n][0], o[n][c]);
                o[n][c] = mfma_32x32x16_f16(v1, p[n][1], o[n][c]);
            }
        }
    }

    if (range == sp.count - 1) {
        // The new positions go with the last range.  Their values are bf16, so
        // the weights enter as a bf16 hi/lo pair (16 bits).  A value that is no
        // number must not reach the rows that do not attend to it, through
        // 0 * NaN: it is taken out of the product and added row by row.
        for (int j0 = wave * 32; j0 < nl; j0 += kStep) {
            const int jk = min(j0 + 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3), nl - 1);
            const uint16_t* k = static_cast<const uint16_t*>(a.k_new) + ((size_t)s * a.n + jk) * a.ld_new +
                                (size_t)hk * D + 16 * half;
            f32x16 acc[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) acc[n] = f32x16{};
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                const u32x4 k0 = *reinterpret_cast<const u32x4*>(k + 32 * c);
                const u32x4 k1 = *reinterpret_cast<const u32x4*>(k + 32 * c + 8);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    acc[n] = mfma_32x32x16_bf16(k0, q[n][c][0], acc[n]);
                    acc[n] = mfma_32x32x16_bf16(k1, q[n][c][1], acc[n]);
                }
            }
            const int jv = j0 + 16 * half;   // first of the lane's 16 positions
            u32x4 ph[NQ][2], pl[NQ][2];
            float w[NQ][16];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const uint8_t* mask = a.mask != nullptr ? a.mask + ((size_t)s * a.n + pos[n]) * a.n : nullptr;
                unsigned sees = 0;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int jj = jv + j;
                    const bool see = jj < nl && (mask != nullptr ? mask[jj < nl ? jj : 0] != 0 : jj <= pos[n]);
                    sees |= see ? 1u << j : 0u;
                    w[n][j] = see ? acc[n][j] * qscale : neg_inf();
                }
                weigh<D>(w[n], 1.f, 0.f, 1.f, st[n], o[n]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t h = f32x2_to_bf16x2_bits(w[n][2 * j], w[n][2 * j + 1]);
                    ph[n][j >> 2][j & 3] = h;
                    pl[n][j >> 2][j & 3] = f32x2_to_bf16x2_bits(w[n][2 * j] - __uint_as_float(h << 16),
                                                                w[n][2 * j + 1] - __uint_as_float(h & 0xffff0000u));
                }
#pragma unroll
                for (int j = 0; j < 16; ++j)   // for the row-by-row sums: 0 where the row does not attend
                    w[n][j] = sees >> j & 1 ? fmaxf(w[n][j], 1e-30f) : 0.f;
            }
            const uint16_t* vn = static_cast<const uint16_t*>(a.v_new) + (size_t)s * a.n * a.ld_new + (size_t)hk * D;
            bool odd = false;
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                u32x4 v[2];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    uint32_t x = vn[(size_t)min(jv + j, nl - 1) * a.ld_new + 32 * c + col];
                    const bool bad = (x & 0x7f80u) == 0x7f80u;
                    odd |= bad;
                    x = bad ? 0u : x;
                    if (j & 1) v[j >> 3][(j >> 1) & 3] |= x << 16;
                    else v[j >> 3][(j >> 1) & 3] = x;
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][c] = mfma_32x32x16_bf16(v[0], ph[n][0], o[n][c]);
                    o[n][c] = mfma_32x32x16_bf16(v[1], ph[n][1], o[n][c]);
                    o[n][c] = mfma_32x32x16_bf16(v[0], pl[n][0], o[n][c]);
                    o[n][c] = mfma_32x32x16_bf16(v[1], pl[n][1], o[n][c]);
                }
            }
            if (__any(odd)) {
                float* lw = &so[wave][0][0];   // the wave's own part, free until the end
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) lw[(16 * half + j) * kTileRows + col] = w[n][j];
                    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                    for (int j = 0; j < min(32, nl - j0); ++j) {
                        const float f = lw[j * kTileRows + col];
                        const uint16_t* row = vn + (size_t)(j0 + j) * a.ld_new;
                        if (f == 0.f) continue;
#pragma unroll
                        for (int c = 0; c < kC; ++c)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const uint32_t x = row[32 * c + acc_row(e, lane)];
                                if ((x & 0x7f80u) == 0x7f80u) o[n][c][e] += f * bf16_bits_to_f32(x);
                            }
                    }
                    __builtin_amdgcn_wave_barrier();
                }
            }
        }
    }

    // the four waves joined, half of the dimensions at a time
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l = st[n].l + lane_xor<32>(st[n].l);
        if (half == 0) sm[wave][col] = st[n].m, sl[wave][col] = l;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            __syncthreads();   // sm, sl written; so free again
            float mt = neg_inf();
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) mt = fmaxf(mt, sm[w][col]);
            const float f = st[n].m == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(st[n].m - mt);
#pragma unroll
            for (int c = 0; c < kC / 2; ++c)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& x = o[n][part * (kC / 2) + c];
                    *reinterpret_cast<f32x4*>(&so[wave][col][32 * c + 8 * g + 4 * half]) =
                        f32x4{x[4 * g] * f, x[4 * g + 1] * f, x[4 * g + 2] * f, x[4 * g + 3] * f};
                }
            __syncthreads();
            for (int e = tid; e < kTileRows * (D / 8); e += kAttendThreads) {
                const int r = e / (D / 8), d = e % (D / 8) * 4;
                const int row = row0 + n * kTileRows + r;
                if (row >= rows) continue;
                float m = neg_inf(), lt = 0.f;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, sm[w][r]);
                for (int w = 0; w < kAttendWaves; ++w) {
                    lt += sm[w][r] == neg_inf() ? sl[w][r] : sl[w][r] * __builtin_amdgcn_exp2f(sm[w][r] - m);
                    const f32x4 y = *reinterpret_cast<const f32x4*>(&so[w][r][d]);
                    for (int i = 0; i < 4; ++i) x[i] += y[i];
                }
                const size_t at = ((size_t)s * a.n + row / group) * a.Hq + hk * group + row % group;
                const int dd = part * (D / 2) + d;
                if (sp.count == 1) {
                    const bool none = lt == 0.f;   // a NaN sum stays one
                    const float g = none ? 0.f : 1.f / lt;
                    uint2 y;
                    y.x = f32x2_to_bf16x2_bits(none ? 0.f : x[0] * g, none ? 0.f : x[1] * g);
                    y.y = f32x2_to_bf16x2_bits(none ? 0.f : x[2] * g, none ? 0.f : x[3] * g);
                    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * D + dd) = y;
                    if (dd == 0 && a.lse != nullptr) a.lse[at] = lse_of(m, lt);
                } else {
                    *reinterpret_cast<f32x4*>(part_sums(a, at, range, D) + dd) = x;
                    if (dd == 0) {
                        float* ml = part_stats(a, at, range, D);
                        ml[0] = m;
                        ml[1] = lt;
                    }
                }
            }
        }
        __syncthreads();   // sm and sl are free again
    }
}

int tile_blocks(int n, int Hq, int Hkv) {
    return (int)(((long long)n * (Hq / Hkv) + kTileRows - 1) / kTileRows);
}

hipError_t launch_attend_tile(const AttendArgs& a, int D, hipStream_t stream) {
    const int blocks = tile_blocks(a.n, a.Hq, a.Hkv);
    const long long units = (long long)a.b * a.Hkv * a.splits;
    const long long grid = (units + 7) / 8 * 8 * blocks;
    if (grid > 0x7fffffffll) return hipErrorInvalidValue;
    if (D == 128)
        hipLaunchKernelGGL((attend_tile_kernel<128, 1>), dim3((unsigned)grid), dim3(kAttendThreads), 0, stream, a, blocks);
    else
        hipLaunchKernelGGL((attend_tile_kernel<64, 1>), dim3((unsigned)grid), dim3(kAttendThreads), 0, stream, a, blocks);
    return hipGetLastError();
}

}  // namespace tf
