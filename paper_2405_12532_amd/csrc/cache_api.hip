// C ABI of the cache held in 4 bits: argument checks on the host, then the launchers.  See include/pyr.h for the contract of every entry point.
#include <math.h>

#include "cache_device.h"

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
constexpr int64_t kMost = (int64_t)1 << 31;
constexpr int64_t kMostGroups = (int64_t)1 << 24;                // workgroups of 256 threads: a launch has fewer than 2^32 threads
int64_t head_groups(const pyr_cache* c) { return (c->n_kv_heads + 3) / 4; }      // (workgroups of a tile, at most)

int check_layout(const pyr_cache* c) {
    if (c == nullptr) return PYR_ERR_NULL;
    if (c->n_kv_heads < 1 || c->page_tokens < 1) return PYR_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return PYR_ERR_UNSUPPORTED;
    if (c->page_tokens < 32 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)) != 0) return PYR_ERR_UNSUPPORTED;
    if (c->n_kv_heads > 32767) return PYR_ERR_UNSUPPORTED;      // (as the packed calls)
    return PYR_OK;
}

int check_sizes(const pyr_cache* c) {
    const int rc = check_layout(c);
    if (rc != PYR_OK) return rc;
    if (c->n_pages < 1 || c->n_slots < 1 || c->max_pages < 1 || c->n_slots > PYR_CACHE_MAX_SLOTS) return PYR_ERR_SHAPE;
    if ((int64_t)c->n_slots * c->max_pages >= kMost || (int64_t)c->n_pages * c->page_tokens >= kMost || (int64_t)c->max_pages * c->page_tokens >= kMost) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int check_cache(const pyr_cache* c) {
    const int rc = check_sizes(c);
    if (rc != PYR_OK) return rc;
    if (!c->pages || !c->refs || !c->table || !c->lens) return PYR_ERR_NULL;
    if ((uintptr_t)c->pages % kAlign != 0) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int32_t within_row(const pyr_cache* c, int32_t tokens) {         // a limit on tokens of a slot, no larger than a row of the table needs (it may be INT32_MAX)
    const int64_t capacity = (int64_t)c->max_pages * c->page_tokens;
    return tokens < capacity ? tokens : (int32_t)capacity;
}

int check_rows(const pyr_cache* c, int32_t n) {                  // of a call that hands out or shares pages
    if (n < 0 || n > PYR_CACHE_MAX_ROWS) return PYR_ERR_SHAPE;
    return (int64_t)n * (1 + (int64_t)c->max_pages) >= kMost ? PYR_ERR_UNSUPPORTED : PYR_OK;
}

pyr::PoolView view(const pyr_cache* c) {
    int shift = 5;
    while ((1 << shift) < c->page_tokens) ++shift;
    return pyr::PoolView{{(uint8_t*)c->pages, c->table, c->lens, c->n_pages, c->n_slots, c->max_pages, shift, c->n_kv_heads}, c->refs};
}

int check_attention(const pyr_cache* c, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, pyr::CacheAttention* plan) {
    if (n < 0 || n_tokens < 1 || n_q_heads < 1 || max_len < 0) return PYR_ERR_SHAPE;
    if (n_q_heads % c->n_kv_heads != 0 || n_q_heads > 32767) return PYR_ERR_UNSUPPORTED;
    if ((int64_t)n * n_tokens >= kMost || (int64_t)(n > 1 ? n : 1) * n_tokens * n_q_heads >= kMost) return PYR_ERR_UNSUPPORTED;
    *plan = pyr::plan_cache_attention(n, n_tokens, n_q_heads, c->n_kv_heads, c->head_dim, within_row(c, max_len));
    if ((int64_t)n * plan->col_groups * c->n_kv_heads * plan->waves >= 4 * kMostGroups) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

size_t attention_bytes(const pyr::CacheAttention& plan) { return align_up(plan.part_bytes) + align_up(plan.stat_bytes); }

bool workspace_ok(const void* ws, size_t have, size_t need) { return need == 0 || (ws != nullptr && (uintptr_t)ws % kAlign == 0 && have >= need); }

}  // namespace

extern "C" {

int pyr_cache_page_bytes(const pyr_cache* cache, size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    const int rc = check_layout(cache);
    if (rc != PYR_OK) return rc;
    *bytes_out = (size_t)cache->n_kv_heads * (cache->page_tokens / 32) * 34 * cache->head_dim;
    return PYR_OK;
}

int pyr_cache_reserve(const pyr_cache* cache, const int32_t* slots, const int32_t* n_new, int32_t n, int32_t* start, int32_t* status, void* stream) {
    int rc = check_cache(cache);
    if (rc == PYR_OK) rc = check_rows(cache, n);
    if (rc != PYR_OK) return rc;
    if (!status || (n > 0 && (!slots || !n_new || !start))) return PYR_ERR_NULL;
    return pyr::launch_cache_reserve(view(cache), slots, n_new, n, start, status, (hipStream_t)stream);
}

int pyr_cache_fork(const pyr_cache* cache, const int32_t* parents, const int32_t* children, int32_t n, int32_t* status, void* stream) {
    int rc = check_cache(cache);
    if (rc == PYR_OK) rc = check_rows(cache, n);
    if (rc != PYR_OK) return rc;
    if (!status || (n > 0 && (!parents || !children))) return PYR_ERR_NULL;
    return pyr::launch_cache_fork(view(cache), 34 * cache->head_dim, parents, children, n, status, (hipStream_t)stream);
}

int pyr_cache_release(const pyr_cache* cache, const int32_t* slots, int32_t n, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    if (n < 0) return PYR_ERR_SHAPE;
    if (n == 0) return PYR_OK;
    if (!slots) return PYR_ERR_NULL;
    if (n >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    return pyr::launch_cache_release(view(cache), slots, n, (hipStream_t)stream);
}

int pyr_cache_compact_workspace_bytes(const pyr_cache* cache, int32_t n, size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc == PYR_OK) rc = check_rows(cache, n);
    if (rc != PYR_OK) return rc;
    *bytes_out = align_up((size_t)n * (1 + (size_t)cache->max_pages) * sizeof(int32_t));
    return PYR_OK;
}

int pyr_cache_compact(const pyr_cache* cache, const int32_t* slots, int32_t n, const int32_t* kept_idx, int32_t n_kept, const int32_t* seq_offsets,
                      const int32_t* out_offsets, int32_t max_keep, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc == PYR_OK) rc = check_rows(cache, n);
    if (rc != PYR_OK) return rc;
    if (n_kept < 0 || max_keep < 0) return PYR_ERR_SHAPE;
    if (!status || (n > 0 && (!slots || !seq_offsets || !out_offsets || (n_kept > 0 && !kept_idx)))) return PYR_ERR_NULL;
    size_t need = 0;
    pyr_cache_compact_workspace_bytes(cache, n, &need);
    if (!workspace_ok(workspace, workspace_bytes, need)) return PYR_ERR_WORKSPACE;
    max_keep = within_row(cache, max_keep < n_kept ? max_keep : n_kept);      // (more are refused on the device)
    if ((int64_t)n * (((int64_t)max_keep + 31) / 32) >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    const pyr::PoolView c = view(cache);
    rc = pyr::launch_cache_cut(c, slots, out_offsets, n, n_kept, max_keep, (int32_t*)workspace, status, (hipStream_t)stream);
    if (rc != PYR_OK) return rc;
    return pyr::launch_cache_move(c, cache->head_dim, slots, kept_idx, n_kept, seq_offsets, out_offsets, (const int32_t*)workspace, status, n, max_keep,
                                  (hipStream_t)stream);
}

int pyr_cache_store(const pyr_cache* cache, const void* k, const void* v, int32_t n_rows, const int32_t* row_idx, int32_t n_list, const int32_t* offsets,
                    const int32_t* slots, const int32_t* start, int32_t n, int32_t max_new, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    if (n < 0 || n_rows < 0 || n_list < 0 || max_new < 0 || (row_idx == nullptr && n_list != n_rows)) return PYR_ERR_SHAPE;
    if (n == 0 || n_rows == 0 || n_list == 0 || max_new == 0) return PYR_OK;
    if (!k || !v || !offsets || !slots || !start) return PYR_ERR_NULL;
    if (!aligned16(k) || !aligned16(v)) return PYR_ERR_UNSUPPORTED;
    max_new = within_row(cache, max_new < n_list ? max_new : n_list);
    if ((int64_t)n * (((int64_t)max_new + 30) / 32 + 1) * head_groups(cache) >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    return pyr::launch_cache_store(view(cache), cache->head_dim, k, v, n_rows, row_idx, n_list, offsets, slots, start, n, max_new, (hipStream_t)stream);
}

int pyr_cache_load(const pyr_cache* cache, const int32_t* slots, const int32_t* offsets, int32_t n, int32_t max_len, void* k_out, void* v_out,
                   int32_t n_rows, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    if (n < 0 || n_rows < 0 || max_len < 0) return PYR_ERR_SHAPE;
    if (n == 0 || n_rows == 0 || max_len == 0) return PYR_OK;
    if ((!k_out && !v_out) || !slots || !offsets) return PYR_ERR_NULL;
    if (!aligned16(k_out) || !aligned16(v_out)) return PYR_ERR_UNSUPPORTED;
    max_len = within_row(cache, max_len < n_rows ? max_len : n_rows);
    if ((int64_t)n * (((int64_t)max_len + 31) / 32) * head_groups(cache) >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    return pyr::launch_cache_load(view(cache), cache->head_dim, slots, offsets, n, max_len, k_out, v_out, n_rows, (hipStream_t)stream);
}

int pyr_cache_attention_workspace_bytes(const pyr_cache* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, &plan);
    if (rc != PYR_OK) return rc;
    *bytes_out = attention_bytes(plan);
    return PYR_OK;
}

int pyr_cache_attention(const pyr_cache* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                        float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, &plan);
    if (rc != PYR_OK) return rc;
    if (n == 0) return PYR_OK;
    if (!q || !slots || !out) return PYR_ERR_NULL;
    if (!aligned16(q) || !aligned16(out)) return PYR_ERR_UNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, attention_bytes(plan))) return PYR_ERR_WORKSPACE;
    const float scale = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * pyr::kLog2e;
    return pyr::launch_cache_attention(plan, view(cache), cache->head_dim, q, slots, n, n_tokens, n_q_heads, scale, out, lse, workspace,
                                       (float*)((char*)workspace + align_up(plan.part_bytes)), (hipStream_t)stream);
}

int pyr_diag_cache_attention(const pyr_cache* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, pyr_cache_route* route_out) {
    if (route_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, &plan);
    if (rc != PYR_OK) return rc;
    *route_out = pyr_cache_route{plan.col_tiles, plan.repeats, plan.waves, plan.col_groups, plan.chunk, plan.splits};
    return PYR_OK;
}

}  // extern "C"
