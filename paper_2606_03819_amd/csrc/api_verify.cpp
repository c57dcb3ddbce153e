// C ABI of the verification step beside the tree: sampling, the paged 8-bit
// cache, attention over it.  Every argument is checked before the first HIP call.
#include <math.h>
#include <stdint.h>

#include "treeflash.h"
#include "checks.hpp"
#include "launch.hpp"

namespace {

using namespace tf;

constexpr long long kMaxPositions = 1 << 20;   // b * n
constexpr int kMaxVocab = 1 << 22;
constexpr long long kMaxQueryRows = 1 << 23;   // b * n * Hq: a launch's threads stay below 2^32
constexpr long long kMaxHeadTokens = 1 << 28;  // N * Hkv of an append, likewise

bool opt4(const void* p) { return p == nullptr || aligned4(p); }

// Shape of a cache's pages: sizes the kernels are built for.
tf_status_t page_status(int page_size, int max_pages) {
    if (page_size < 1 || max_pages < 1 || (long long)page_size * max_pages > 0x7fffff00ll) return TF_ERR_INVALID_ARG;
    return page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128 ? TF_OK : TF_ERR_UNSUPPORTED;
}
tf_status_t head_status(int Hkv, int D) {
    if (Hkv < 1 || Hkv > 1024 || D < 1) return TF_ERR_INVALID_ARG;
    return D == 64 || D == 128 ? TF_OK : TF_ERR_UNSUPPORTED;
}
// rows of `width` elements at a distance of ld, read 16 bytes at a time
tf_status_t row_status(long long ld, long long width, tf_dtype_t dt) {
    if (ld < width || ld > (1ll << 32)) return TF_ERR_INVALID_ARG;
    return ld * (long long)elem_bytes(dt) % 16 == 0 ? TF_OK : TF_ERR_UNSUPPORTED;
}

bool sample_shapes(int b, int n, int V) {
    return b >= 1 && n >= 1 && V >= 1 && V <= kMaxVocab && (long long)b * n <= kMaxPositions;
}

tf_status_t attend_shapes(int b, int n, int Hq, int Hkv, int D, int page_size, int max_pages, tf_dtype_t dt) {
    if (!dtype_ok(dt) || b < 1 || n < 1 || n > 4096 || (long long)b * n > kMaxPositions) return TF_ERR_INVALID_ARG;
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq > 4096) return TF_ERR_INVALID_ARG;
    tf_status_t st = head_status(Hkv, D);
    if (st == TF_OK) st = page_status(page_size, max_pages);
    if (st == TF_OK && (long long)b * n * Hq > kMaxQueryRows) st = TF_ERR_UNSUPPORTED;
    return st;
}

}  // namespace

extern "C" {

size_t treeflash_sample_workspace_bytes(int b, int n, int V) {
    return sample_shapes(b, n, V) ? 256 + sample_ws_bytes((long long)b * n, V) : 0;
}

tf_status_t treeflash_sample(const void* logits, long long ld, int b, int n, int V, tf_dtype_t dt,
                             const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                             const float* uniform, int32_t* token, float* logprob, void* workspace,
                             size_t workspace_bytes, hipStream_t stream) {
    if (logits == nullptr || uniform == nullptr || token == nullptr || !dtype_ok(dt)) return TF_ERR_INVALID_ARG;
    if (!sample_shapes(b, n, V) || ld < V || ld > (1ll << 32)) return TF_ERR_INVALID_ARG;
    if (!elem_aligned(logits, dt) || !aligned4(uniform) || !aligned4(token) || !opt4(temperature) || !opt4(top_k) ||
        !opt4(top_p) || !opt4(min_p) || !opt4(logprob))
        return TF_ERR_INVALID_ARG;
    if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < treeflash_sample_workspace_bytes(b, n, V))
        return TF_ERR_WORKSPACE;
    SampleArgs a{logits, ld, n, b * n, V, temperature, top_k, top_p, min_p, uniform, token, logprob,
                 static_cast<unsigned char*>(workspace)};
    return launch_sample(a, dt == TF_BF16, stream) == hipSuccess ? TF_OK : TF_ERR_HIP;
}

tf_status_t treeflash_cache_slots(const int32_t* context_len, const int32_t* add_len, const int32_t* accepted,
                                  const int32_t* free_pages, const int32_t* free_count, int b, int gamma, int n,
                                  int page_size, int max_pages, int max_free, int max_tokens, int32_t* block_table,
                                  int32_t* new_len, int32_t* new_free_count, int32_t* start, int32_t* page_start,
                                  int32_t* slot, int32_t* position, int32_t* source, int32_t* status,
                                  hipStream_t stream) {
    const void* need[] = {context_len, add_len, free_pages, free_count, block_table, new_len, new_free_count, start,
                          page_start, slot, status};
    for (const void* p : need)
        if (p == nullptr || !aligned4(p)) return TF_ERR_INVALID_ARG;
    if (!opt4(accepted) || !opt4(position) || !opt4(source)) return TF_ERR_INVALID_ARG;
    if (b < 1 || b > kMaxPositions || n < 0 || max_free < 1 || max_tokens < 1 || max_tokens > 1 << 30)
        return TF_ERR_INVALID_ARG;
    if (accepted != nullptr && (gamma < 1 || gamma > 255 || n < 1)) return TF_ERR_INVALID_ARG;
    if ((long long)b * n > 0x7fffffffll) return TF_ERR_INVALID_ARG;
    const tf_status_t st = page_status(page_size, max_pages);
    if (st != TF_OK) return st;
    const SlotsArgs a{context_len, add_len, accepted, free_pages, free_count, b, gamma, n, page_size, max_pages,
                      max_free, max_tokens, block_table, new_len, new_free_count, start, page_start, slot, position,
                      source, status};
    return launch_cache_slots(a, stream) == hipSuccess ? TF_OK : TF_ERR_HIP;
}

tf_status_t treeflash_cache_release(const uint8_t* done, const int32_t* context_len, const int32_t* block_table,
                                    const int32_t* free_count, int b, int page_size, int max_pages, int max_free,
                                    int32_t* free_pages, int32_t* new_len, int32_t* new_free_count,
                                    hipStream_t stream) {
    const void* need[] = {context_len, block_table, free_count, free_pages, new_len, new_free_count};
    for (const void* p : need)
        if (p == nullptr || !aligned4(p)) return TF_ERR_INVALID_ARG;
    if (done == nullptr || b < 1 || b > kMaxPositions || max_free < 1) return TF_ERR_INVALID_ARG;
    const tf_status_t st = page_status(page_size, max_pages);
    if (st != TF_OK) return st;
    const ReleaseArgs a{done, context_len, block_table, free_count, b, page_size, max_pages, max_free, free_pages,
                        new_len, new_free_count};
    return launch_cache_release(a, stream) == hipSuccess ? TF_OK : TF_ERR_HIP;
}

tf_status_t treeflash_cache_append(const void* k_new, const void* v_new, long long ld_new, int rows,
                                   const int32_t* slot, const int32_t* source, int N, int Hkv, int D, int page_size,
                                   int num_pages, tf_dtype_t dt, void* k_cache, void* v_cache, float* k_scale,
                                   float* v_scale, hipStream_t stream) {
    if (k_new == nullptr || v_new == nullptr || slot == nullptr || k_cache == nullptr || v_cache == nullptr ||
        k_scale == nullptr || v_scale == nullptr || !dtype_ok(dt))
        return TF_ERR_INVALID_ARG;
    if (N < 1 || rows < 1 || !aligned4(slot) || !opt4(source) || !aligned4(k_scale) || !aligned4(v_scale))
        return TF_ERR_INVALID_ARG;
    tf_status_t st = head_status(Hkv, D);
    if (st != TF_OK) return st;
    if ((st = page_status(page_size, num_pages)) != TF_OK) return st;
    if ((long long)N * Hkv > kMaxHeadTokens) return TF_ERR_UNSUPPORTED;
    if ((st = row_status(ld_new, (long long)Hkv * D, dt)) != TF_OK) return st;
    if ((st = vec_status_all({k_new, v_new}, dt)) != TF_OK) return st;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return TF_ERR_UNSUPPORTED;
    const AppendArgs a{k_new, v_new, ld_new, rows, slot, source, N, Hkv, page_size, num_pages, k_cache, v_cache,
                       k_scale, v_scale};
    return launch_cache_append(a, D, dt == TF_BF16, stream) == hipSuccess ? TF_OK : TF_ERR_HIP;
}

size_t treeflash_tree_attention_workspace_bytes(int b, int n, int Hq, int Hkv, int D, int page_size, int max_pages,
                                                tf_dtype_t dt) {
    if (attend_shapes(b, n, Hq, Hkv, D, page_size, max_pages, dt) != TF_OK) return 0;
    return 256 + attend_part_bytes(b, n, Hq, Hkv, D, page_size, max_pages, dt == TF_BF16);
}

tf_status_t treeflash_tree_attention(const void* q, long long ld_q, const void* k_new, const void* v_new,
                                     long long ld_new, const uint8_t* mask, const int32_t* new_len,
                                     const int32_t* context_len, const int32_t* block_table, const void* k_cache,
                                     const void* v_cache, const float* k_scale, const float* v_scale, int b, int n,
                                     int Hq, int Hkv, int D, int page_size, int max_pages, int num_pages, float scale,
                                     tf_dtype_t dt, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
    if (q == nullptr || k_new == nullptr || v_new == nullptr || context_len == nullptr || block_table == nullptr ||
        k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr || out == nullptr)
        return TF_ERR_INVALID_ARG;
    tf_status_t st = attend_shapes(b, n, Hq, Hkv, D, page_size, max_pages, dt);
    if (st != TF_OK) return st;
    if (num_pages < 1 || (long long)num_pages * page_size > 0x7fffff00ll || !isfinite(scale)) return TF_ERR_INVALID_ARG;
    if (!aligned4(context_len) || !aligned4(block_table) || !aligned4(k_scale) || !aligned4(v_scale) ||
        !opt4(new_len) || !opt4(lse))
        return TF_ERR_INVALID_ARG;
    if ((st = row_status(ld_q, (long long)Hq * D, dt)) != TF_OK) return st;
    if ((st = row_status(ld_new, (long long)Hkv * D, dt)) != TF_OK) return st;
    if ((st = vec_status_all({q, k_new, v_new, out}, dt)) != TF_OK) return st;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return TF_ERR_UNSUPPORTED;
    const size_t bytes = treeflash_tree_attention_workspace_bytes(b, n, Hq, Hkv, D, page_size, max_pages, dt);
    if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < bytes) return TF_ERR_WORKSPACE;
    const AttendArgs a{q, ld_q, k_new, v_new, ld_new, mask, new_len, context_len, block_table,
                       static_cast<const uint8_t*>(k_cache), static_cast<const uint8_t*>(v_cache), k_scale, v_scale,
                       b, n, Hq, Hkv, page_size, max_pages, num_pages, scale, out, lse,
                       static_cast<float*>(workspace), 1};
    return launch_tree_attention(a, D, dt == TF_BF16, stream) == hipSuccess ? TF_OK : TF_ERR_HIP;
}

}  // extern "C"
