// C ABI of the paged-cache calls: host-side validation and launches (kernels in duo_page.h and duo_page_attn.h).
#include "../../include/duo_verify.h"

#include <math.h>

#include "duo_internal.h"
#include "duo_page.h"
#include "duo_page_attn.h"

namespace {

int page_shift_of(int slots) {
    for (int s = 5; s <= 10; ++s)
        if (slots == 1 << s) return s;
    return -1;
}
bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// The sizes that every call is given: model, pages and batch maxima.
int check_sizes(const duo_model_config* cfg, const duo_page_cache* cache, const duo_page_batch* b) {
    if (const int rc = duo_internal_check_config(cfg)) return rc;
    if (!cache || !b) return DUO_ERR_NULL;
    if (cache->n_pages < 1 || page_shift_of(cache->page_slots) < 0 || cache->max_pages < 1) return DUO_ERR_SHAPE;
    if ((int64_t)cache->n_pages * cache->page_slots > 0x7fffffff || (int64_t)cache->max_pages * cache->page_slots > DUO_PAGE_MAX_SLOTS) return DUO_ERR_SHAPE;
    if (b->n_requests < 1 || b->n_requests > DUO_PAGE_MAX_REQUESTS || b->max_rows < 1 || b->max_rows > DUO_PAGE_MAX_ROWS || b->max_new < 1 ||
        b->max_new > b->max_rows)
        return DUO_ERR_SHAPE;
    return DUO_OK;
}

PageLayout layout_of(const duo_model_config* cfg, const duo_page_cache* cache, const duo_page_batch* b) {
    return page_layout(b->n_requests, b->max_rows, b->max_new, cache->max_pages * cache->page_slots / 32, cfg->n_q_heads, cfg->n_kv_heads, cfg->head_dim);
}

int check_workspace(const PageLayout& lay, const void* ws, size_t bytes) {
    if (!ws) return DUO_ERR_NULL;
    if (off16(ws)) return DUO_ERR_ALIGN;
    return bytes < lay.total ? DUO_ERR_WORKSPACE : DUO_OK;
}

int check_tables(const duo_page_tables* t) {
    if (!t || !t->block_table || !t->held || !t->free_pages || !t->free_count) return DUO_ERR_NULL;
    return off4(t->block_table) || off4(t->held) || off4(t->free_pages) || off4(t->free_count) ? DUO_ERR_ALIGN : DUO_OK;
}

int check_rows(const void* p, int64_t stride, int64_t width) {
    if (!p) return DUO_ERR_NULL;
    if (off16(p) || stride % 8) return DUO_ERR_ALIGN;
    return stride < width ? DUO_ERR_SHAPE : DUO_OK;
}

// Whether two matrices of `rows` rows (start, elements from row to row, elements a row) have an element in common.  Column ranges of one matrix
// are told apart row by row; matrices with other distances between their rows are taken to meet where their address ranges do.
bool rows_meet(const uint16_t* a, int64_t a_stride, int64_t a_width, const uint16_t* b, int64_t b_stride, int64_t b_width, int rows) {
    const __int128 last = rows - 1, delta = ((__int128)(intptr_t)b - (intptr_t)a) / 2;  // both 16-byte aligned
    if (a_stride != b_stride || rows == 1) return delta < last * a_stride + a_width && delta + last * b_stride + b_width > 0;
    // row i of b starts delta + d * stride behind row i - d of a: no row is wider than the distance, so two values of d can meet
    const __int128 d0 = -delta / a_stride;
    for (__int128 d = d0 - 1; d <= d0 + 1; ++d) {
        const __int128 at = delta + d * a_stride;
        if (d >= -last && d <= last && at < a_width && at + b_width > 0) return true;
    }
    return false;
}

size_t layer_elems(const duo_model_config* cfg, const duo_page_cache* c) { return (size_t)c->n_pages * cfg->n_kv_heads * c->page_slots * cfg->head_dim; }

template <int D>
void launch_page_attention(const PageAttnArgs& a, const PageLayout& lay, hipStream_t s) {
    constexpr int TEAMS = D == 64 ? 2 : 1;
    // Nothing can be cut and every workgroup has a compute unit to itself: eight waves (9 rows of 32 heads behind 512 keys: 7.9 us, 11.4 with four).
    const bool alone = lay.merges == 0 && a.requests * a.hkv <= 256;
    const unsigned few = (lay.merges == 0 ? a.requests : lay.stream_items) * a.hkv;  // more workgroups than the plan has items end at once
    duo_internal_prof(DUO_PROF_ATTN);
    if (lay.tile_items > 0) DUO_LAUNCH((page_mixed_kernel<D>), dim3(lay.tile_items * a.hkv + few), dim3(256), s, a);
    else if (lay.stream_rows <= 16 && alone) DUO_LAUNCH((page_stream_kernel<D, 8>), dim3(few), dim3(512), s, a);
    else if (lay.stream_rows <= 16) DUO_LAUNCH((page_stream_kernel<D, 4>), dim3(few), dim3(256), s, a);
    else if (lay.stream_rows <= 32) DUO_LAUNCH((page_team_kernel<D, 1, TEAMS>), dim3(few), dim3(64 * TEAMS), s, a);
    else DUO_LAUNCH((page_team_kernel<D, 2, TEAMS>), dim3(few), dim3(128 * TEAMS), s, a);
    if (lay.merges > 0) {
        const long long units = (long long)lay.merges * a.hkv;
        duo_internal_prof(DUO_PROF_ATTN_COMB);
        DUO_LAUNCH((page_merge_kernel<D>), dim3(units < 1024 ? (int)units : 1024), dim3(256), s, a);
    }
}

}  // namespace

extern "C" int duo_page_workspace_bytes(const duo_model_config* cfg, const duo_page_cache* cache, const duo_page_batch* batch, size_t* bytes) {
    if (!bytes) return DUO_ERR_NULL;
    if (const int rc = check_sizes(cfg, cache, batch)) return rc;
    *bytes = layout_of(cfg, cache, batch).total;
    return DUO_OK;
}

extern "C" int duo_page_plan(const duo_model_config* cfg, const duo_page_cache* cache, const duo_page_tables* from, const duo_page_tables* to,
                             const duo_page_batch* b, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int rc = check_sizes(cfg, cache, b)) return rc;
    if (const int rc = check_tables(from)) return rc;
    if (const int rc = check_tables(to)) return rc;
    // all four in place, or none
    const int same = (from->block_table == to->block_table) + (from->held == to->held) + (from->free_pages == to->free_pages) + (from->free_count == to->free_count);
    if (same != 0 && same != 4) return DUO_ERR_ARG;
    if (!b->cached || !b->trunk || !b->n || !b->k || !b->row_start || !b->position || !b->slot || !b->status) return DUO_ERR_NULL;
    if (off4(b->cached) || off4(b->trunk) || off4(b->n) || off4(b->k) || off4(b->row_start) || off4(b->position) || off4(b->slot) || off4(b->status))
        return DUO_ERR_ALIGN;
    const PageLayout lay = layout_of(cfg, cache, b);
    if (const int rc = check_workspace(lay, workspace, workspace_bytes)) return rc;
    PagePlanArgs a{};
    a.cached = b->cached, a.trunk = b->trunk, a.n = b->n, a.k = b->k;
    a.table_in = from->block_table, a.held_in = from->held, a.free_in = from->free_pages, a.count_in = from->free_count;
    a.table_out = to->block_table, a.held_out = to->held, a.free_out = to->free_pages, a.count_out = to->free_count;
    a.row_start = b->row_start, a.position = b->position, a.slot = b->slot, a.status = b->status;
    a.requests = b->n_requests, a.max_rows = b->max_rows, a.max_new = b->max_new;
    a.n_pages = cache->n_pages, a.page_shift = page_shift_of(cache->page_slots), a.max_pages = cache->max_pages;
    a.hq = cfg->n_q_heads, a.hkv = cfg->n_kv_heads, a.head_dim = cfg->head_dim;
    a.ws = static_cast<char*>(workspace);
    a.lay = lay;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    if (b->n_requests <= PAGE_SMALL_REQUESTS && b->max_rows <= PAGE_SMALL_ROWS && cache->n_pages <= PAGE_SMALL_PAGES) {
        const int waves = b->n_requests < 4 ? 4 : b->n_requests;
        duo_internal_prof(DUO_PROF_SETUP);
        DUO_LAUNCH(page_plan_kernel, dim3(1), dim3(64 * waves), s, a);
        return duo_internal_hip_ok(hipGetLastError(), "duo_page_plan");
    }
    static_assert(4 * PAGE_PLAN_THREADS == PAGE_MAX_REQUESTS && PAGE_MAX_REQUESTS == DUO_PAGE_MAX_REQUESTS, "four requests a thread");
    duo_internal_prof(DUO_PROF_SETUP);
    if (b->n_requests <= PAGE_PLAN_THREADS) DUO_LAUNCH((page_sum_kernel<1>), dim3(1), dim3((b->n_requests + 63) / 64 * 64), s, a);
    else DUO_LAUNCH((page_sum_kernel<4>), dim3(1), dim3(PAGE_PLAN_THREADS), s, a);
    const int longest = b->max_new > cache->max_pages ? b->max_new : cache->max_pages;
    const int spread = longest > 8192 ? 16 : (longest + 511) / 512;
    const int beyond = (cache->n_pages + 4095) / 4096 / spread + 1;
    duo_internal_prof(DUO_PROF_SETUP);
    DUO_LAUNCH(page_fill_kernel, dim3(b->n_requests + beyond, spread), dim3(256), s, a);
    return duo_internal_hip_ok(hipGetLastError(), "duo_page_plan");
}

extern "C" int duo_page_append(const duo_model_config* cfg, const duo_page_cache* cache, const duo_page_batch* b, int layer, const uint16_t* q,
                               int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride, uint16_t* q_out,
                               int64_t q_out_stride, void* hip_stream) {
    if (const int rc = check_sizes(cfg, cache, b)) return rc;
    if (layer < 0 || layer >= cfg->n_layers) return DUO_ERR_ARG;
    if (!cache->k || !cache->v || !b->position || !b->slot || !b->status) return DUO_ERR_NULL;
    if (off16(cache->k) || off16(cache->v) || off4(b->position) || off4(b->slot) || off4(b->status)) return DUO_ERR_ALIGN;
    const int D = cfg->head_dim, qd = cfg->n_q_heads * D, kd = cfg->n_kv_heads * D;
    if (const int rc = check_rows(q, q_stride, qd)) return rc;
    if (const int rc = check_rows(k, k_stride, kd)) return rc;
    if (const int rc = check_rows(v, v_stride, kd)) return rc;
    if (const int rc = check_rows(q_out, q_out_stride, qd)) return rc;
    // q_out is q or apart from it, and apart from k and v, which other workgroups read while it is written
    if (q_out == q ? q_out_stride != q_stride : rows_meet(q_out, q_out_stride, qd, q, q_stride, qd, b->max_rows)) return DUO_ERR_ARG;
    if (rows_meet(q_out, q_out_stride, qd, k, k_stride, kd, b->max_rows) || rows_meet(q_out, q_out_stride, qd, v, v_stride, kd, b->max_rows)) return DUO_ERR_ARG;
    PageAppendArgs a{};
    a.q = q, a.k = k, a.v = v, a.q_out = q_out;
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
    const size_t at = layer_elems(cfg, cache) * layer;
    a.kc = cache->k + at, a.vc = cache->v + at;
    a.position = b->position, a.slot = b->slot, a.status = b->status;
    a.rows = b->max_rows, a.hq = cfg->n_q_heads, a.hkv = cfg->n_kv_heads, a.page_shift = page_shift_of(cache->page_slots), a.n_pages = cache->n_pages;
    // theta^(-2d/D) as a product of at most six powers, one for each bit of d: within 2^-50, and 0.8 us less than a power for every channel
    a.turns[0] = 1.0 / (2.0 * M_PI);
    for (int n = 1; n < D / 2; n *= 2) {
        const double factor = pow((double)cfg->rope_theta, -2.0 * n / D);
        for (int d = 0; d < n; ++d) a.turns[n + d] = a.turns[d] * factor;
    }
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    // Heads that share a row's angles: as many as leave 1024 workgroups, at most eight.
    const int windows = (b->max_rows + PAGE_APPEND_ROWS - 1) / PAGE_APPEND_ROWS, heads = cfg->n_q_heads + cfg->n_kv_heads;
    const long long each = (long long)windows * heads / 1024;
    a.heads_each = each < 1 ? 1 : each > 8 ? 8 : (int)each;
    a.rope_groups = (heads + a.heads_each - 1) / a.heads_each;
    const dim3 grid(windows, a.rope_groups + cfg->n_kv_heads);
    duo_internal_prof(DUO_PROF_QKV_FINISH);
    if (D == 64) DUO_LAUNCH((page_append_kernel<64>), grid, dim3(256), s, a);
    else DUO_LAUNCH((page_append_kernel<128>), grid, dim3(256), s, a);
    return duo_internal_hip_ok(hipGetLastError(), "duo_page_append");
}

extern "C" int duo_page_attention(const duo_model_config* cfg, const duo_page_cache* cache, const int32_t* block_table, const duo_page_batch* b, int layer,
                                  const uint16_t* q, int64_t q_stride, uint16_t* out, int64_t out_stride, float scale, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
    if (const int rc = check_sizes(cfg, cache, b)) return rc;
    if (layer < 0 || layer >= cfg->n_layers || !(scale >= 0.f) || isinf(scale)) return DUO_ERR_ARG;
    if (!cache->k || !cache->v || !block_table || !b->status) return DUO_ERR_NULL;
    if (off16(cache->k) || off16(cache->v) || off4(block_table) || off4(b->status)) return DUO_ERR_ALIGN;
    const int D = cfg->head_dim, qd = cfg->n_q_heads * D;
    if (const int rc = check_rows(q, q_stride, qd)) return rc;
    if (const int rc = check_rows(out, out_stride, qd)) return rc;
    if (rows_meet(out, out_stride, qd, q, q_stride, qd, b->max_rows)) return DUO_ERR_ARG;
    const PageLayout lay = layout_of(cfg, cache, b);
    if (const int rc = check_workspace(lay, workspace, workspace_bytes)) return rc;
    PageAttnArgs a{};
    a.q = q, a.out = out, a.q_stride = q_stride, a.out_stride = out_stride;
    const size_t at = layer_elems(cfg, cache) * layer;
    a.kc = cache->k + at, a.vc = cache->v + at;
    a.table = block_table, a.status = b->status;
    char* const ws = static_cast<char*>(workspace);
    a.ws = ws, a.stream = lay.stream, a.tile = lay.tile, a.merge = lay.merge;
    a.part_stream = reinterpret_cast<float*>(ws + lay.part_stream), a.part_tile = reinterpret_cast<float*>(ws + lay.part_tile);
    a.stream_rows = lay.stream_rows, a.tile_items = lay.tile_items;
    a.requests = b->n_requests, a.hq = cfg->n_q_heads, a.hkv = cfg->n_kv_heads, a.page_shift = page_shift_of(cache->page_slots);
    a.n_pages = cache->n_pages, a.max_pages = cache->max_pages, a.max_rows = b->max_rows, a.max_new = b->max_new;
    a.scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    if (D == 64) launch_page_attention<64>(a, lay, s);
    else launch_page_attention<128>(a, lay, s);
    return duo_internal_hip_ok(hipGetLastError(), "duo_page_attention");
}

extern "C" int duo_page_commit(const duo_model_config* cfg, const duo_page_cache* cache, const int32_t* block_table, const duo_page_batch* b,
                               const int32_t* records, int32_t* cached_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int rc = check_sizes(cfg, cache, b)) return rc;
    if (!cache->k || !cache->v || !block_table || !b->status || !b->cached || !records || !cached_out) return DUO_ERR_NULL;
    if (off16(cache->k) || off16(cache->v) || off4(block_table) || off4(b->status) || off4(b->cached) || off4(records) || off4(cached_out)) return DUO_ERR_ALIGN;
    const PageLayout lay = layout_of(cfg, cache, b);
    if (const int rc = check_workspace(lay, workspace, workspace_bytes)) return rc;
    PageCommitArgs a{};
    a.kc = cache->k, a.vc = cache->v, a.cached = b->cached, a.table = block_table, a.records = records, a.cached_out = cached_out, a.status = b->status;
    a.requests = b->n_requests, a.layers = cfg->n_layers, a.hkv = cfg->n_kv_heads, a.page_shift = page_shift_of(cache->page_slots), a.n_pages = cache->n_pages;
    a.max_pages = cache->max_pages, a.max_new = b->max_new, a.hq = cfg->n_q_heads, a.head_dim = cfg->head_dim, a.max_rows = b->max_rows;
    a.ws = static_cast<const char*>(workspace), a.info = lay.info;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    const dim3 grid(b->n_requests, cfg->n_layers, cfg->n_kv_heads);
    duo_internal_prof(DUO_PROF_COMMIT);
    if (cfg->head_dim == 64) DUO_LAUNCH((page_commit_kernel<64>), grid, dim3(128), s, a);
    else DUO_LAUNCH((page_commit_kernel<128>), grid, dim3(128), s, a);
    return duo_internal_hip_ok(hipGetLastError(), "duo_page_commit");
}
