// C ABI of the paged cache of text tokens (sali.h): argument checks and launches.
#include <math.h>
#include <algorithm>
#include <new>

#include "pages.h"

struct sali_pages {
    sali_pages_config cfg;
    uint8_t* pool;
    uint8_t* scratch;
    sali::PagesScratch layout;
    uint64_t layer_bytes;
};

namespace sali {

namespace {

bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }

int check_pages_config(const sali_pages_config* c) {
    if (c == nullptr) return SALI_ERR_NULL;
    if (c->n_layers < 1 || c->n_layers > 65535 || c->n_kv_heads < 1 || c->n_heads < 1 || c->n_heads > 65535) return SALI_ERR_CONFIG;
    if (c->n_heads % c->n_kv_heads != 0) return SALI_ERR_CONFIG;
    if (c->head_dim != 64 && c->head_dim != 128) return SALI_ERR_CONFIG;
    if (c->page_tokens < kBlockTokens || c->page_tokens > 256 || !power_of_two(c->page_tokens)) return SALI_ERR_CONFIG;
    if (c->n_pages < 1 || c->n_pages > (1 << 24)) return SALI_ERR_CONFIG;
    if (c->dtype != SALI_DTYPE_FP16 && c->dtype != SALI_DTYPE_BF16) return SALI_ERR_CONFIG;
    if (c->store != SALI_STORE_16 && c->store != SALI_STORE_INT8 && c->store != SALI_STORE_INT4) return SALI_ERR_CONFIG;
    return SALI_OK;
}

uint64_t head_bytes_of(const sali_pages_config& c) {
    return (uint64_t)(c.page_tokens / kBlockTokens) * block_layout(c.store, c.head_dim).bytes;
}
uint64_t layer_bytes_of(const sali_pages_config& c) { return head_bytes_of(c) * c.n_kv_heads * c.n_pages; }

// what an append, a read or an attention of `layer` needs of its batch
int check_batch(const sali_pages* p, int32_t layer, const sali_page_batch* b) {
    if (p == nullptr || b == nullptr) return SALI_ERR_NULL;
    if (layer < 0 || layer >= p->cfg.n_layers) return SALI_ERR_SHAPE;
    if (b->n_seqs < 0 || b->n_tokens < 0 || b->table_width < 0 || b->max_q < 0 || b->max_kv < 0) return SALI_ERR_SHAPE;
    // positions, and those of the tiles asked for behind a sequence's last, are counted in 31 bits
    if (std::min((int64_t)b->max_kv, (int64_t)b->table_width * p->cfg.page_tokens) > kMostPositions) return SALI_ERR_SHAPE;
    if (b->n_seqs > p->cfg.n_pages || b->n_tokens > (int64_t)p->cfg.n_pages * p->cfg.page_tokens) return SALI_ERR_SHAPE;
    if (b->n_seqs > 0 && (b->d_start == nullptr || b->d_length == nullptr || (b->d_table == nullptr && b->table_width > 0))) return SALI_ERR_NULL;
    if (((uintptr_t)b->d_start | (uintptr_t)b->d_length | (uintptr_t)b->d_table) % 4 != 0) return SALI_ERR_ALIGN;
    return SALI_OK;
}
bool nothing_to_do(const sali_page_batch& b) { return b.n_seqs == 0 || b.n_tokens == 0 || b.max_q == 0 || b.max_kv == 0; }

int check_rows(const sali_rows* r, bool needed) {
    if (r == nullptr || (needed && r->d == nullptr)) return SALI_ERR_NULL;
    if ((uintptr_t)r->d % 16 != 0 || r->token_stride % 8 != 0 || r->head_stride % 8 != 0) return SALI_ERR_ALIGN;
    return SALI_OK;
}

PageGeom geom_of(const sali_pages* p, int32_t layer) {
    PageGeom g;
    g.pool = reinterpret_cast<char*>(p->pool + p->layer_bytes * (uint64_t)layer);
    g.head_bytes = (uint32_t)head_bytes_of(p->cfg);
    g.page_bytes = (uint64_t)g.head_bytes * p->cfg.n_kv_heads;
    g.n_pages = p->cfg.n_pages;
    g.n_kv = p->cfg.n_kv_heads;
    g.blocks_log2 = 0;
    while ((kBlockTokens << g.blocks_log2) < p->cfg.page_tokens) ++g.blocks_log2;
    return g;
}
PageSeqs seqs_of(const sali_pages* p, const sali_page_batch& b) {
    return {b.d_start, b.d_length, b.d_table, reinterpret_cast<uint32_t*>(p->scratch), b.n_seqs, b.table_width, b.n_tokens, b.max_q, b.max_kv};
}

template <typename R>
R rows_of(const sali_rows& r) {
    return {static_cast<decltype(R::d)>(r.d), r.token_stride * 2, r.head_stride * 2};
}

// what both forms of attention need besides their masks
int check_attend(const sali_pages* p, int32_t layer, const sali_page_batch* batch, const sali_rows* q, const float* prior, const float* prior_lse,
                 const sali_rows* out, const float* lse) {
    int rc = check_batch(p, layer, batch);
    if (rc == SALI_OK) rc = check_rows(q, batch->n_tokens > 0);
    if (rc == SALI_OK) rc = check_rows(out, batch->n_tokens > 0);
    if (rc != SALI_OK) return rc;
    if ((prior == nullptr) != (prior_lse == nullptr)) return SALI_ERR_NULL;
    if ((uintptr_t)prior % 16 != 0 || ((uintptr_t)prior_lse | (uintptr_t)lse) % 4 != 0) return SALI_ERR_ALIGN;
    return SALI_OK;
}
int check_window(int32_t window, int32_t sinks) { return window < 0 || sinks < 0 || window > (1 << 30) || sinks > (1 << 30) ? SALI_ERR_SHAPE : SALI_OK; }
int check_scale(float softmax_scale) { return isfinite(softmax_scale * 1.44269504088896340736f) ? SALI_OK : SALI_ERR_CONFIG; }
// rows and tiles are counted in 31 bits
int check_sizes(const sali_pages* p, const sali_page_batch& b) {
    if ((int64_t)b.n_tokens * (p->cfg.n_heads / p->cfg.n_kv_heads) >= 0x7FFFFFFF - 1024) return SALI_ERR_SHAPE;
    if (((int64_t)b.max_kv / kTileTokens + 2) * p->cfg.n_kv_heads > 0x7FFFFFFFll / b.n_seqs) return SALI_ERR_SHAPE;
    return SALI_OK;
}

float scale2_of(float softmax_scale) { return softmax_scale == 0.0f ? 1.0f : fabsf(softmax_scale) * 1.44269504088896340736f; }
uint32_t keep_of(float softmax_scale) { return softmax_scale == 0.0f ? 0u : ~0u; }
uint32_t flip_of(float softmax_scale) { return softmax_scale < 0.0f ? 0x80008000u : 0u; }
PagesAttend attend_of(sali_pages* p, int32_t layer, const sali_page_batch& batch, const sali_rows& q, float softmax_scale, const float* prior,
                      const float* prior_lse, const sali_rows& out, float* lse) {
    PagesAttend a = {};
    a.geom = geom_of(p, layer);
    a.seqs = seqs_of(p, batch);
    a.q = rows_of<RowsIn>(q);
    a.out = rows_of<RowsOut>(out);
    a.lse = lse;
    a.prior = prior;
    a.prior_lse = prior_lse;
    a.scale2 = scale2_of(softmax_scale);
    a.q_keep = keep_of(softmax_scale);
    a.q_flip = flip_of(softmax_scale);
    a.heads = p->cfg.n_heads;
    a.group = p->cfg.n_heads / p->cfg.n_kv_heads;
    a.partial = reinterpret_cast<float*>(p->scratch + p->layout.partial);
    a.records = reinterpret_cast<int32_t*>(p->scratch + p->layout.records);
    return a;
}

}  // namespace

}  // namespace sali

using namespace sali;

extern "C" {

int sali_pages_bytes(const sali_pages_config* cfg, size_t* pool_bytes, size_t* scratch_bytes) {
    const int rc = check_pages_config(cfg);
    if (rc != SALI_OK) return rc;
    if (pool_bytes != nullptr) *pool_bytes = (size_t)(layer_bytes_of(*cfg) * cfg->n_layers);
    if (scratch_bytes != nullptr)
        *scratch_bytes = pages_scratch(cfg->n_pages, cfg->page_tokens, cfg->n_kv_heads, cfg->n_heads / cfg->n_kv_heads, cfg->head_dim).bytes;
    return SALI_OK;
}

int sali_pages_create(const sali_pages_config* cfg, void* d_pool, void* d_scratch, sali_pages** out) {
    if (out == nullptr) return SALI_ERR_NULL;
    *out = nullptr;
    const int rc = check_pages_config(cfg);
    if (rc != SALI_OK) return rc;
    if (d_pool == nullptr || d_scratch == nullptr) return SALI_ERR_NULL;
    if ((uintptr_t)d_pool % 256 != 0 || (uintptr_t)d_scratch % 256 != 0) return SALI_ERR_ALIGN;
    sali_pages* p = new (std::nothrow) sali_pages();
    if (p == nullptr) return SALI_ERR_STATE;
    p->cfg = *cfg;
    p->pool = static_cast<uint8_t*>(d_pool);
    p->scratch = static_cast<uint8_t*>(d_scratch);
    p->layout = pages_scratch(cfg->n_pages, cfg->page_tokens, cfg->n_kv_heads, cfg->n_heads / cfg->n_kv_heads, cfg->head_dim);
    p->layer_bytes = layer_bytes_of(*cfg);
    if (hipMemset(p->scratch, 0, kPagesStatusBytes) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        delete p;
        return SALI_ERR_HIP;
    }
    *out = p;
    return SALI_OK;
}

void sali_pages_destroy(sali_pages* p) { delete p; }

int sali_pages_append(sali_pages* p, int32_t layer, const sali_page_batch* batch, const sali_rows* k, const sali_rows* v, void* stream) {
    int rc = check_batch(p, layer, batch);
    if (rc == SALI_OK) rc = check_rows(k, batch->n_tokens > 0);
    if (rc == SALI_OK) rc = check_rows(v, batch->n_tokens > 0);
    if (rc != SALI_OK) return rc;
    if (nothing_to_do(*batch)) return SALI_OK;
    const hipError_t e = launch_pages_append(p->cfg.dtype, p->cfg.store, p->cfg.head_dim, geom_of(p, layer), seqs_of(p, *batch), rows_of<RowsIn>(*k),
                                             rows_of<RowsIn>(*v), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_read(sali_pages* p, int32_t layer, const sali_page_batch* batch, const sali_rows* k_out, const sali_rows* v_out, void* stream) {
    int rc = check_batch(p, layer, batch);
    if (rc == SALI_OK) rc = check_rows(k_out, batch->n_tokens > 0);
    if (rc == SALI_OK) rc = check_rows(v_out, batch->n_tokens > 0);
    if (rc != SALI_OK) return rc;
    if (nothing_to_do(*batch)) return SALI_OK;
    const hipError_t e = launch_pages_read(p->cfg.dtype, p->cfg.store, p->cfg.head_dim, geom_of(p, layer), seqs_of(p, *batch), rows_of<RowsOut>(*k_out),
                                           rows_of<RowsOut>(*v_out), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_attend(sali_pages* p, int32_t layer, const sali_page_batch* batch, const sali_rows* q, float softmax_scale, int32_t window, int32_t sinks,
                      const float* d_prior_or_null, const float* d_prior_lse_or_null, const sali_rows* out, float* d_lse_or_null, void* stream) {
    int rc = check_attend(p, layer, batch, q, d_prior_or_null, d_prior_lse_or_null, out, d_lse_or_null);
    if (rc == SALI_OK) rc = check_window(window, sinks);
    if (rc == SALI_OK) rc = check_scale(softmax_scale);
    if (rc != SALI_OK) return rc;
    if (nothing_to_do(*batch)) return SALI_OK;
    rc = check_sizes(p, *batch);
    if (rc != SALI_OK) return rc;
    PagesAttend a = attend_of(p, layer, *batch, *q, softmax_scale, d_prior_or_null, d_prior_lse_or_null, *out, d_lse_or_null);
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = p->cfg.dtype == SALI_DTYPE_BF16 ? launch_pages_attend_bf16(p->cfg.store, p->cfg.head_dim, a, s)
                                                         : launch_pages_attend_fp16(p->cfg.store, p->cfg.head_dim, a, s);
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_attend_tree(sali_pages* p, int32_t layer, const sali_page_batch* batch, const uint64_t* d_seen, const sali_rows* q, float softmax_scale,
                           const float* d_prior_or_null, const float* d_prior_lse_or_null, const sali_rows* out, float* d_lse_or_null, void* stream) {
    int rc = check_attend(p, layer, batch, q, d_prior_or_null, d_prior_lse_or_null, out, d_lse_or_null);
    if (rc == SALI_OK) rc = check_scale(softmax_scale);
    if (rc != SALI_OK) return rc;
    if (batch->max_q > kMostDrafted) return SALI_ERR_SHAPE;
    if (d_seen == nullptr && batch->n_tokens > 0) return SALI_ERR_NULL;
    if ((uintptr_t)d_seen % 8 != 0) return SALI_ERR_ALIGN;
    if (nothing_to_do(*batch)) return SALI_OK;
    rc = check_sizes(p, *batch);
    if (rc != SALI_OK) return rc;
    PagesAttend a = attend_of(p, layer, *batch, *q, softmax_scale, d_prior_or_null, d_prior_lse_or_null, *out, d_lse_or_null);
    a.seen = d_seen;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = p->cfg.dtype == SALI_DTYPE_BF16 ? launch_pages_attend_tree_bf16(p->cfg.store, p->cfg.head_dim, a, s)
                                                         : launch_pages_attend_tree_fp16(p->cfg.store, p->cfg.head_dim, a, s);
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_rotate(sali_pages* p, const sali_rotary* rotary, const int32_t* d_position, int32_t n_tokens, int32_t inverse, const sali_rows* q_or_null,
                      const sali_rows* k_or_null, const sali_rows* q_out_or_null, const sali_rows* k_out_or_null, void* stream) {
    if (p == nullptr || rotary == nullptr) return SALI_ERR_NULL;
    if ((q_or_null == nullptr) != (q_out_or_null == nullptr) || (k_or_null == nullptr) != (k_out_or_null == nullptr)) return SALI_ERR_NULL;
    if (rotary->pairs < 1 || rotary->pairs > p->cfg.head_dim / 2 || rotary->axes < 1 || rotary->axes > 4) return SALI_ERR_CONFIG;
    int64_t pairs = 0;
    for (int i = 0; i < rotary->axes; ++i) {
        if (rotary->section[i] < 0) return SALI_ERR_CONFIG;
        pairs += rotary->section[i];
    }
    if (pairs != rotary->pairs) return SALI_ERR_CONFIG;
    if (n_tokens < 0 || n_tokens > kMostBlocks) return SALI_ERR_SHAPE;
    if (n_tokens > 0 && (d_position == nullptr || rotary->d_frequency == nullptr)) return SALI_ERR_NULL;
    if ((uintptr_t)d_position % 4 != 0 || (uintptr_t)rotary->d_frequency % 8 != 0) return SALI_ERR_ALIGN;
    for (const sali_rows* r : {q_or_null, k_or_null, q_out_or_null, k_out_or_null}) {
        const int rc = r == nullptr ? SALI_OK : check_rows(r, n_tokens > 0);
        if (rc != SALI_OK) return rc;
    }
    if (n_tokens == 0 || (q_or_null == nullptr && k_or_null == nullptr)) return SALI_OK;
    Rotate r = {};
    if (q_or_null != nullptr) {
        r.q = rows_of<RowsIn>(*q_or_null);
        r.q_out = rows_of<RowsOut>(*q_out_or_null);
        r.q_heads = p->cfg.n_heads;
    }
    if (k_or_null != nullptr) {
        r.k = rows_of<RowsIn>(*k_or_null);
        r.k_out = rows_of<RowsOut>(*k_out_or_null);
        r.k_heads = p->cfg.n_kv_heads;
    }
    r.frequency = rotary->d_frequency;
    r.position = d_position;
    r.axis_stride = n_tokens;
    r.dim = p->cfg.head_dim;
    r.pairs = rotary->pairs;
    r.adjacent = rotary->adjacent != 0;
    r.inverse = inverse != 0;
    r.n_tokens = n_tokens;
    for (int i = 0, upto = 0; i < 3; ++i) {
        upto += i < rotary->axes ? rotary->section[i] : 0;
        r.until[i] = i + 1 < rotary->axes ? upto : 0x7FFFFFFF;
    }
    return launch_rotate(p->cfg.dtype, r, static_cast<hipStream_t>(stream)) == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_weigh(sali_pages* p, int32_t layer, const sali_page_batch* batch, const sali_rows* q, float softmax_scale, int32_t window, int32_t sinks,
                     const float* d_lse, int32_t add, float* d_weights, void* stream) {
    int rc = check_batch(p, layer, batch);
    if (rc == SALI_OK) rc = check_rows(q, batch->n_tokens > 0);
    if (rc == SALI_OK) rc = check_window(window, sinks);
    if (rc == SALI_OK) rc = check_scale(softmax_scale);
    if (rc != SALI_OK) return rc;
    if (batch->n_tokens > 0 && (d_lse == nullptr || d_weights == nullptr)) return SALI_ERR_NULL;
    if (((uintptr_t)d_lse | (uintptr_t)d_weights) % 4 != 0) return SALI_ERR_ALIGN;
    if (nothing_to_do(*batch)) return SALI_OK;
    rc = check_sizes(p, *batch);
    if (rc != SALI_OK) return rc;
    PagesWeigh a = {};
    a.geom = geom_of(p, layer);
    a.seqs = seqs_of(p, *batch);
    if (weigh_blocks(a.seqs) * p->cfg.n_kv_heads > kMostBlocks / 2 / batch->n_seqs) return SALI_ERR_SHAPE;        // half as many of 512 threads
    // (a scale of zero makes queries zero, as in attention: 0 times a product that is no fp32 number would be a NaN)
    a.q = softmax_scale == 0.0f ? RowsIn{reinterpret_cast<const char*>(p->scratch + kPagesZeros), 0, 0} : rows_of<RowsIn>(*q);
    a.lse = d_lse;
    a.weights = d_weights;
    a.scale2 = softmax_scale * 1.44269504088896340736f;
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    a.heads = p->cfg.n_heads;
    a.group = p->cfg.n_heads / p->cfg.n_kv_heads;
    a.add = add != 0;
    a.partial = reinterpret_cast<float*>(p->scratch + p->layout.partial);
    a.partial_bytes = p->layout.records - p->layout.partial;
    const hipError_t e = launch_pages_weigh(p->cfg.dtype, p->cfg.store, p->cfg.head_dim, a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_select(sali_pages* p, const sali_page_batch* batch, const float* d_weights, int32_t budget, int32_t sinks, int32_t recent, int32_t* d_keep,
                      void* stream) {
    const int rc = check_batch(p, 0, batch);
    if (rc != SALI_OK) return rc;
    if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget) return SALI_ERR_SHAPE;
    if (batch->n_tokens > 0 && (d_weights == nullptr || d_keep == nullptr)) return SALI_ERR_NULL;
    if (((uintptr_t)d_weights | (uintptr_t)d_keep) % 4 != 0) return SALI_ERR_ALIGN;
    if (nothing_to_do(*batch)) return SALI_OK;
    if (4ll * p->cfg.n_kv_heads > kMostBlocks / batch->n_seqs) return SALI_ERR_SHAPE;        // of 1024 threads
    const PagesSelect a = {geom_of(p, 0), seqs_of(p, *batch), d_weights, d_keep, budget, sinks, recent};
    return launch_pages_select(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_keep(sali_pages* p, int32_t layer, const sali_page_batch* batch, const int32_t* d_keep, int32_t keep_heads, int32_t keep_width,
                    const int32_t* d_to_or_null, int32_t to_width, float* d_weights_or_null, void* stream) {
    const int rc = check_batch(p, layer, batch);
    if (rc != SALI_OK) return rc;
    if ((keep_heads != 1 && keep_heads != p->cfg.n_kv_heads) || keep_width < 0 || to_width < 0) return SALI_ERR_SHAPE;
    if (batch->n_tokens > 0 && keep_width > 0 && d_keep == nullptr) return SALI_ERR_NULL;
    if (((uintptr_t)d_keep | (uintptr_t)d_to_or_null | (uintptr_t)d_weights_or_null) % 4 != 0) return SALI_ERR_ALIGN;
    if (nothing_to_do(*batch) || keep_width == 0) return SALI_OK;
    PagesKeep a = {};
    a.geom = geom_of(p, layer);
    a.seqs = seqs_of(p, *batch);
    a.keep = d_keep;
    a.in_place = d_to_or_null == nullptr;
    a.to = a.in_place ? batch->d_table : d_to_or_null;
    a.weights = d_weights_or_null;
    a.width = keep_width;
    a.keep_heads = keep_heads;
    a.to_width = a.in_place ? batch->table_width : to_width;
    if (keep_chunks(a.seqs, a.width, a.in_place != 0) * p->cfg.n_kv_heads * keep_strips(p->cfg.head_dim, true) > kMostBlocks / batch->n_seqs) return SALI_ERR_SHAPE;
    return launch_pages_keep(p->cfg.store, p->cfg.head_dim, a, static_cast<hipStream_t>(stream)) == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_get_status(sali_pages* p, uint32_t* h_status, void* stream) {
    if (p == nullptr || h_status == nullptr) return SALI_ERR_NULL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (hipMemcpyAsync(h_status, p->scratch, sizeof(*h_status), hipMemcpyDeviceToHost, s) != hipSuccess) return SALI_ERR_HIP;
    return hipStreamSynchronize(s) == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

}  // extern "C"
