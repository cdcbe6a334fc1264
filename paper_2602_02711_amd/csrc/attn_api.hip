// C entry points of the attention block (dmr_kv_*, dmr_attn_*): argument checks, all before the first HIP call, and the plan of a call.
#include <cmath>

#include "attn.hpp"

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 22, kMaxRequests = int64_t(1) << 20;
constexpr int32_t kMaxHeads = 4096;
constexpr int64_t kMaxGroups = UINT32_MAX / 256;      // workgroups of 256 threads in a launch

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P>
bool all_there(P... p) { return ((p != nullptr) && ...); }
template <typename... P>
bool all_aligned(P... p) { return (aligned16(p) && ...); }
// Arrays of int32 are read word by word, so that a part of a batch can be passed from any request on.
template <typename... P>
bool words_aligned(P... p) { return (((reinterpret_cast<uintptr_t>(p) & 3u) == 0) && ...); }

dmr_status_t hip_status(hipError_t e) { return e == hipSuccess ? DMR_OK : DMR_ERR_HIP; }

int page_shift_of(int32_t page_tokens) {
    for (int s = 4; s <= 8; ++s)
        if (page_tokens == 1 << s) return s;
    return -1;
}

// Shape of a cache: DMR_OK, or what is wrong with it.
dmr_status_t check_layout(int32_t page_tokens, int32_t kv_heads, int32_t head_dim, dmr_kv_type_t type) {
    if (page_tokens <= 0 || kv_heads <= 0 || kv_heads > kMaxHeads || head_dim <= 0) return DMR_ERR_SHAPE;
    if (page_shift_of(page_tokens) < 0 || (head_dim != 64 && head_dim != 128)) return DMR_ERR_UNSUPPORTED;
    return type == DMR_KV_BF16 || type == DMR_KV_E4M3 ? DMR_OK : DMR_ERR_UNSUPPORTED;
}

dmr_status_t check_cache(const dmr_kv_cache_t *c, int32_t q_heads, dmr::CacheView *view) {
    if (!c) return DMR_ERR_NULL;
    const dmr_status_t layout = check_layout(c->page_tokens, c->kv_heads, c->head_dim, c->type);
    if (layout != DMR_OK) return layout;
    if (c->pages <= 0 || c->pages > INT32_MAX / c->page_tokens) return DMR_ERR_SHAPE;
    if (q_heads <= 0 || q_heads > kMaxHeads || q_heads % c->kv_heads != 0) return DMR_ERR_SHAPE;
    auto good = [](float s) { return s > 0.f && std::isfinite(s) && std::isfinite(1.0f / s); };
    if (!good(c->k_scale) || !good(c->v_scale)) return DMR_ERR_UNSUPPORTED;
    if (c->type == DMR_KV_BF16 && (c->k_scale != 1.0f || c->v_scale != 1.0f)) return DMR_ERR_UNSUPPORTED;
    *view = dmr::CacheView{static_cast<uint8_t *>(c->d_k), static_cast<uint8_t *>(c->d_v), c->pages, page_shift_of(c->page_tokens),
                           c->kv_heads, c->head_dim, c->type == DMR_KV_E4M3, c->k_scale, c->v_scale};
    return DMR_OK;
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

// Partial outputs, their (reference, sum), and what a request's items are.
struct Workspace {
    size_t ml, split, bytes;
};
Workspace workspace_of(const dmr::AttnPlan &p, int64_t requests, int kv_heads, int D) {
    if (!p.split) return Workspace{0, 0, 0};
    const size_t rows = (size_t)p.items * (size_t)kv_heads * (size_t)p.tile_rows;
    Workspace w;
    w.ml = align256(rows * (size_t)D * sizeof(float));
    w.split = w.ml + align256(rows * sizeof(float2));
    w.bytes = w.split + (p.few ? (size_t)requests * sizeof(int2) : 0);
    return w;
}

}  // namespace

extern "C" {

size_t dmr_kv_page_bytes(int32_t page_tokens, int32_t kv_heads, int32_t head_dim, dmr_kv_type_t type) {
    if (check_layout(page_tokens, kv_heads, head_dim, type) != DMR_OK) return 0;
    return (size_t)page_tokens * (size_t)kv_heads * (size_t)head_dim * (type == DMR_KV_BF16 ? 2 : 1);
}

dmr_status_t dmr_kv_assign(int64_t requests, int64_t rows, int64_t table_width, int32_t page_tokens, int64_t free_capacity,
                           const int32_t *d_new_tokens, const int32_t *d_lens, const int32_t *d_free_pages,
                           const int32_t *d_free_count, int32_t *d_block_table, int32_t *d_query_start, int32_t *d_kv_lens,
                           int32_t *d_positions, int32_t *d_slots, int32_t *d_left, void *stream) {
    if (requests < 0 || requests > kMaxRequests || rows < 0 || rows > kMaxRows || table_width < 0 || free_capacity < 0 ||
        free_capacity > INT32_MAX || page_tokens <= 0)
        return DMR_ERR_SHAPE;
    const int shift = page_shift_of(page_tokens);
    if (shift < 0) return DMR_ERR_UNSUPPORTED;
    if (table_width > INT32_MAX / page_tokens) return DMR_ERR_SHAPE;
    // arrays of no elements may be NULL
    if (!all_there(d_free_count, d_query_start, d_left) || (requests && !all_there(d_new_tokens, d_lens, d_kv_lens)) ||
        (requests && table_width && !d_block_table) || (free_capacity && !d_free_pages) || (rows && !all_there(d_positions, d_slots)))
        return DMR_ERR_NULL;
    if (!words_aligned(d_new_tokens, d_lens, d_free_pages, d_free_count, d_block_table, d_query_start, d_kv_lens, d_positions, d_slots, d_left))
        return DMR_ERR_ALIGN;
    return hip_status(dmr::launch_kv_assign(requests, rows, table_width, shift, free_capacity, d_new_tokens, d_lens, d_free_pages, d_free_count,
                                            d_block_table, d_query_start, d_kv_lens, d_positions, d_slots, d_left,
                                            static_cast<hipStream_t>(stream)));
}

dmr_status_t dmr_kv_append(const dmr_kv_cache_t *cache, const uint16_t *d_qkv, int64_t rows, int32_t q_heads, const uint16_t *d_gamma_q,
                           const uint16_t *d_gamma_k, float eps, const float *d_inv_freq, dmr_rope_t pairs, const int32_t *d_positions,
                           const int32_t *d_slots, uint16_t *d_q, void *stream) {
    dmr::CacheView view;
    const dmr_status_t st = check_cache(cache, q_heads, &view);
    if (st != DMR_OK) return st;
    if (rows < 0 || rows > kMaxRows) return DMR_ERR_SHAPE;
    if (((d_gamma_q || d_gamma_k) && !(eps >= 0.f)) || (pairs != DMR_ROPE_HALVES && pairs != DMR_ROPE_ADJACENT)) return DMR_ERR_UNSUPPORTED;
    if (rows == 0) return DMR_OK;
    if (!all_there(cache->d_k, cache->d_v, d_qkv, d_slots, d_q) || (d_inv_freq && !d_positions)) return DMR_ERR_NULL;
    if (!all_aligned(cache->d_k, cache->d_v, d_qkv, d_gamma_q, d_gamma_k, d_inv_freq, d_q) || !words_aligned(d_positions, d_slots))
        return DMR_ERR_ALIGN;
    return hip_status(dmr::launch_kv_append(view, d_qkv, rows, q_heads, d_gamma_q, d_gamma_k, eps, d_inv_freq, pairs == DMR_ROPE_ADJACENT,
                                            d_positions, d_slots, d_q, static_cast<hipStream_t>(stream)));
}

size_t dmr_attn_paged_workspace_bytes(int64_t rows, int64_t requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                      int64_t max_query) {
    if (rows <= 0 || rows > kMaxRows || requests <= 0 || requests > kMaxRequests || q_heads <= 0 || kv_heads <= 0 || q_heads > kMaxHeads ||
        q_heads % kv_heads != 0 || (head_dim != 64 && head_dim != 128) || max_query <= 0)
        return 0;
    const dmr::AttnPlan plan = dmr::plan_attn(rows, requests, q_heads, kv_heads, head_dim, false, max_query, INT64_MAX);
    return workspace_of(plan, requests, kv_heads, head_dim).bytes;
}

dmr_status_t dmr_attn_paged(const dmr_kv_cache_t *cache, const uint16_t *d_q, int64_t rows, int32_t q_heads, int64_t requests,
                            const int32_t *d_query_start, const int32_t *d_kv_lens, const int32_t *d_block_table, int64_t table_width,
                            int64_t max_query, float scale, uint16_t *d_out, void *d_ws, size_t ws_bytes, void *stream) {
    dmr::CacheView view;
    const dmr_status_t st = check_cache(cache, q_heads, &view);
    if (st != DMR_OK) return st;
    if (rows < 0 || rows > kMaxRows || requests < 0 || requests > kMaxRequests || table_width <= 0 ||
        table_width > INT32_MAX / cache->page_tokens || max_query < 0 || rows * (int64_t)(q_heads / cache->kv_heads) > INT32_MAX)
        return DMR_ERR_SHAPE;
    const float scale_log2 = scale * view.k_scale * 1.44269504088896340736f;
    if (!(scale > 0.f) || !std::isnormal(scale_log2)) return DMR_ERR_UNSUPPORTED;
    if (rows == 0 || requests == 0 || max_query == 0) return DMR_OK;
    if (!all_there(cache->d_k, cache->d_v, d_q, d_query_start, d_kv_lens, d_block_table, d_out)) return DMR_ERR_NULL;
    if (!all_aligned(cache->d_k, cache->d_v, d_q, d_out, d_ws) || !words_aligned(d_query_start, d_kv_lens, d_block_table)) return DMR_ERR_ALIGN;
    const dmr::AttnPlan plan = dmr::plan_attn(rows, requests, q_heads, cache->kv_heads, view.D, view.e4m3, max_query,
                                               table_width * cache->page_tokens);
    const Workspace need = workspace_of(plan, requests, cache->kv_heads, cache->head_dim);
    if (need.bytes > 0 && (!d_ws || ws_bytes < need.bytes)) return DMR_ERR_WORKSPACE;
    if (plan.items * cache->kv_heads > kMaxGroups) return DMR_ERR_SHAPE;
    uint8_t *ws = plan.split ? static_cast<uint8_t *>(d_ws) : nullptr;
    const dmr::AttnArgs a{d_q, d_out, view.k, view.v, d_query_start, d_kv_lens, d_block_table,
                          reinterpret_cast<float *>(ws), reinterpret_cast<float2 *>(ws ? ws + need.ml : nullptr),
                          reinterpret_cast<int2 *>(ws ? ws + need.split : nullptr),
                          (int32_t)rows, (int32_t)requests, (int32_t)table_width, q_heads, cache->kv_heads, q_heads / cache->kv_heads,
                          (int32_t)cache->pages, view.page_shift, scale_log2, view.v_scale,
                          (int32_t)plan.items, plan.max_tiles, plan.parts};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = plan.few ? dmr::launch_attn_few(a, plan, view.D, view.e4m3, s) : dmr::launch_attn_tiles(a, view.D, view.e4m3, s);
    if (e != hipSuccess || !plan.split) return hip_status(e);
    return hip_status(dmr::launch_attn_join(a, plan, (int)std::min<int64_t>(std::min(max_query, rows) * a.G, plan.tile_rows), view.D, s));
}

}  // extern "C"
