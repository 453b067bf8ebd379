// C ABI of the cache held in 8 bits: argument checks on the host, then the launchers.  See include/pyr.h for the contract of every entry point.
#include <math.h>

#include "cache8_device.h"

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
constexpr int64_t kMost = (int64_t)1 << 31;
constexpr int64_t kMostGroups = (int64_t)1 << 24;                // workgroups of four wavefronts: a launch has fewer than 2^32 threads

constexpr int64_t kMostBlocks = (int64_t)1 << 26;               // of a list: no pool has more

int check_layout(const pyr_cache8* cache) {
    if (cache == nullptr) return PYR_ERR_NULL;
    const pyr_cache* c = &cache->pool;
    if (c->n_kv_heads < 1 || c->page_tokens < 1) return PYR_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return PYR_ERR_UNSUPPORTED;
    if (c->page_tokens < 32 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1)) != 0) return PYR_ERR_UNSUPPORTED;
    if (c->n_kv_heads > 32767 || pyr::cache8_page_bytes(c->head_dim, c->n_kv_heads, c->page_tokens / 32) >= kMost) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int check_sizes(const pyr_cache8* cache) {
    const int rc = check_layout(cache);
    if (rc != PYR_OK) return rc;
    const pyr_cache* c = &cache->pool;
    if (c->n_pages < 1 || c->n_slots < 1 || c->max_pages < 1 || c->n_slots > PYR_CACHE_MAX_SLOTS) return PYR_ERR_SHAPE;
    if ((int64_t)c->n_slots * c->max_pages >= kMost || (int64_t)c->n_pages * c->page_tokens >= kMost || (int64_t)c->max_pages * c->page_tokens >= kMost) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int check_cache(const pyr_cache8* cache) {
    const int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    const pyr_cache* c = &cache->pool;
    if (!c->pages || !c->refs || !c->table || !c->lens) return PYR_ERR_NULL;
    if ((uintptr_t)c->pages % kAlign != 0) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int32_t within_row(const pyr_cache8* cache, int32_t tokens) {    // a limit on tokens of a slot, no larger than a row of the table needs (it may be INT32_MAX)
    const int64_t capacity = (int64_t)cache->pool.max_pages * cache->pool.page_tokens;
    return tokens < capacity ? tokens : (int32_t)capacity;
}

pyr::PoolView view(const pyr_cache8* cache) {
    const pyr_cache* c = &cache->pool;
    int shift = 5;
    while ((1 << shift) < c->page_tokens) ++shift;
    return pyr::PoolView{{(uint8_t*)c->pages, c->table, c->lens, c->n_pages, c->n_slots, c->max_pages, shift, c->n_kv_heads}, c->refs};
}

// rows of an operand: the stride in 16 bytes, or -1
int32_t stride_of(int64_t stride, int64_t heads, int32_t d) {
    if (stride == 0) stride = heads * d;
    return stride < heads * d || stride % 8 != 0 || stride / 8 >= kMost ? -1 : (int32_t)(stride / 8);
}

int check_rows(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len) {
    if (n < 0 || n_tokens < 1 || n_q_heads < 1 || max_len < 0) return PYR_ERR_SHAPE;
    if (n_q_heads % cache->pool.n_kv_heads != 0 || n_q_heads > 32767) return PYR_ERR_UNSUPPORTED;
    if ((int64_t)n * n_tokens >= kMost || (int64_t)(n > 1 ? n : 1) * n_tokens * n_q_heads >= kMost) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

int check_attention(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, int32_t n_blocks, pyr::CacheAttention* plan) {
    const int rc = check_rows(cache, n, n_tokens, n_q_heads, max_len);
    if (rc != PYR_OK) return rc;
    if (n_blocks < 0) return PYR_ERR_SHAPE;
    if (n_blocks > kMostBlocks) return PYR_ERR_UNSUPPORTED;
    const pyr_cache* c = &cache->pool;
    *plan = pyr::plan_cache8_attention(n, n_tokens, n_q_heads, c->n_kv_heads, c->head_dim, within_row(cache, max_len), n_blocks);
    if ((int64_t)n * (n_blocks > 0 ? n_tokens : 1) * plan->col_groups * c->n_kv_heads * plan->waves >= 4 * kMostGroups) return PYR_ERR_UNSUPPORTED;
    return PYR_OK;
}

size_t attention_bytes(const pyr::CacheAttention& plan) { return align_up(plan.part_bytes) + align_up(plan.stat_bytes); }

int check_select(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, pyr::CacheSelect* plan) {
    const int rc = check_rows(cache, n, n_tokens, n_q_heads, max_len);
    if (rc != PYR_OK) return rc;
    if ((int64_t)n * n_tokens * cache->pool.n_kv_heads >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    *plan = pyr::plan_cache8_select(n, n_tokens, cache->pool.n_kv_heads, within_row(cache, max_len));
    const int64_t units = (int64_t)n * n_tokens * cache->pool.n_kv_heads;
    return units * plan->chunks >= kMostGroups || units * plan->waves >= 4 * kMostGroups ? PYR_ERR_UNSUPPORTED : PYR_OK;
}

bool workspace_ok(const void* ws, size_t have, size_t need) { return need == 0 || (ws != nullptr && (uintptr_t)ws % kAlign == 0 && have >= need); }

}  // namespace

extern "C" {

int pyr_cache8_page_bytes(const pyr_cache8* cache, size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    const int rc = check_layout(cache);
    if (rc != PYR_OK) return rc;
    *bytes_out = (size_t)pyr::cache8_page_bytes(cache->pool.head_dim, cache->pool.n_kv_heads, cache->pool.page_tokens / 32);
    return PYR_OK;
}

int pyr_cache8_fork(const pyr_cache8* cache, const int32_t* parents, const int32_t* children, int32_t n, int32_t* status, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    if (n < 0 || n > PYR_CACHE_MAX_ROWS) return PYR_ERR_SHAPE;
    if ((int64_t)n * (1 + (int64_t)cache->pool.max_pages) >= kMost) return PYR_ERR_UNSUPPORTED;
    if (!status || (n > 0 && (!parents || !children))) return PYR_ERR_NULL;
    const pyr::PoolView c = view(cache);
    const int launched = pyr::launch_cache_fork(c, 0, parents, children, n, status, (hipStream_t)stream);
    if (launched != PYR_OK) return launched;
    return pyr::launch_cache8_fork_copy(c, cache->pool.head_dim, parents, children, n, status, (hipStream_t)stream);
}

int pyr_cache8_append(const pyr_cache8* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride, int32_t n_rows, const int32_t* row_idx,
                      int32_t n_list, const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n, int32_t max_new,
                      const pyr_rotation* rotation, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    const pyr_cache* c = &cache->pool;
    const int32_t d = c->head_dim;
    if (n < 0 || n_rows < 0 || n_list < 0 || max_new < 0 || (row_idx == nullptr && n_list != n_rows)) return PYR_ERR_SHAPE;
    if (q == nullptr) n_q_heads = 0;
    else if (n_q_heads < 1) return PYR_ERR_SHAPE;
    if (n_q_heads % c->n_kv_heads != 0 || n_q_heads > 32767) return PYR_ERR_UNSUPPORTED;
    pyr::Cache8Rows rows{k, v, q, q_out, row_idx, nullptr, nullptr, stride_of(k_stride, c->n_kv_heads, d), stride_of(v_stride, c->n_kv_heads, d),
                         stride_of(q_stride, n_q_heads, d), n_rows, n_list, n_q_heads, 0, 0};
    if (rows.k_stride < 0 || rows.v_stride < 0 || rows.q_stride < 0) return PYR_ERR_UNSUPPORTED;
    if (rotation != nullptr) {
        if (rotation->dims < 0 || rotation->dims > d) return PYR_ERR_SHAPE;
        if (rotation->dims % 16 != 0) return PYR_ERR_UNSUPPORTED;
        rows.positions = rotation->positions;
        rows.freqs = rotation->freqs;
        rows.dims = rotation->dims;
        rows.interleaved = rotation->interleaved != 0;
    }
    if (n == 0 || n_rows == 0 || n_list == 0 || max_new == 0) return PYR_OK;
    if (!k || !v || !offsets || !slots || !start || (q != nullptr && q_out == nullptr)) return PYR_ERR_NULL;
    if (rows.dims > 0 && (!rows.positions || !rows.freqs)) return PYR_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out)) return PYR_ERR_UNSUPPORTED;
    max_new = within_row(cache, max_new);
    if ((int64_t)n * (((int64_t)max_new + 30) / 32 + 1) * ((2 * c->n_kv_heads + (int64_t)n_q_heads + 3) / 4) >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    return pyr::launch_cache8_append(view(cache), d, rows, offsets, slots, start, n, max_new, (hipStream_t)stream);
}

int pyr_cache8_load(const pyr_cache8* cache, const int32_t* slots, const int32_t* first, const int32_t* offsets, int32_t n, int32_t max_len, void* k_out,
                    void* v_out, int32_t n_rows, void* stream) {
    const int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    if (n < 0 || n_rows < 0 || max_len < 0) return PYR_ERR_SHAPE;
    if (n == 0 || n_rows == 0 || max_len == 0) return PYR_OK;
    if ((!k_out && !v_out) || !slots || !offsets) return PYR_ERR_NULL;
    if (!aligned16(k_out) || !aligned16(v_out)) return PYR_ERR_UNSUPPORTED;
    max_len = within_row(cache, max_len < n_rows ? max_len : n_rows);
    if ((int64_t)n * (((int64_t)max_len + 62) / 32) * ((cache->pool.n_kv_heads + 3) / 4) >= kMostGroups) return PYR_ERR_UNSUPPORTED;
    return pyr::launch_cache8_load(view(cache), cache->pool.head_dim, slots, first, offsets, n, max_len, k_out, v_out, n_rows, (hipStream_t)stream);
}

int pyr_cache8_select_workspace_bytes(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheSelect plan;
    rc = check_select(cache, n, n_tokens, n_q_heads, max_len, &plan);
    if (rc != PYR_OK) return rc;
    *bytes_out = align_up(plan.key_bytes);
    return PYR_OK;
}

int pyr_cache8_select(const pyr_cache8* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                      int32_t n_first, int32_t n_recent, int32_t n_best, int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheSelect plan;
    rc = check_select(cache, n, n_tokens, n_q_heads, max_len, &plan);
    if (rc != PYR_OK) return rc;
    if (n_first < 0 || n_recent < 1 || n_best < 0) return PYR_ERR_SHAPE;
    if ((int64_t)n_first + n_recent + n_best > kMostBlocks) return PYR_ERR_UNSUPPORTED;
    if (n == 0) return PYR_OK;
    if (!q || !slots || !blocks) return PYR_ERR_NULL;
    if (!aligned16(q)) return PYR_ERR_UNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, align_up(plan.key_bytes))) return PYR_ERR_WORKSPACE;
    return pyr::launch_cache8_select(plan, view(cache), cache->pool.head_dim, q, slots, n, n_tokens, n_q_heads, n_first, n_recent, n_best, blocks, workspace,
                                     (hipStream_t)stream);
}

int pyr_cache8_attention_workspace_bytes(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, int32_t n_blocks,
                                         size_t* bytes_out) {
    if (bytes_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, n_blocks, &plan);
    if (rc != PYR_OK) return rc;
    *bytes_out = attention_bytes(plan);
    return PYR_OK;
}

int pyr_cache8_attention(const pyr_cache8* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                         float softmax_scale, const int32_t* blocks, int32_t n_blocks, void* out, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream) {
    int rc = check_cache(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, n_blocks, &plan);
    if (rc != PYR_OK) return rc;
    if ((blocks == nullptr) != (n_blocks == 0)) return PYR_ERR_SHAPE;
    if (n == 0) return PYR_OK;
    if (!q || !slots || !out) return PYR_ERR_NULL;
    if (!aligned16(q) || !aligned16(out)) return PYR_ERR_UNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, attention_bytes(plan))) return PYR_ERR_WORKSPACE;
    const float scale = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)cache->pool.head_dim)) * pyr::kLog2e;
    return pyr::launch_cache8_attention(plan, view(cache), cache->pool.head_dim, q, slots, n, n_tokens, n_q_heads, blocks, n_blocks, scale, out, lse, workspace,
                                        (float*)((char*)workspace + align_up(plan.part_bytes)), (hipStream_t)stream);
}

int pyr_diag_cache8_attention(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, int32_t n_blocks,
                              pyr_cache_route* route_out) {
    if (route_out == nullptr) return PYR_ERR_NULL;
    int rc = check_sizes(cache);
    if (rc != PYR_OK) return rc;
    pyr::CacheAttention plan;
    rc = check_attention(cache, n, n_tokens, n_q_heads, max_len, n_blocks, &plan);
    if (rc != PYR_OK) return rc;
    *route_out = pyr_cache_route{plan.col_tiles, plan.repeats, plan.waves, plan.col_groups, plan.chunk, plan.splits};
    return PYR_OK;
}

}  // extern "C"
