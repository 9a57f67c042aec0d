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
    int rc = check_batch(p, layer, batch);
    if (rc == SALI_OK) rc = check_rows(q, batch->n_tokens > 0);
    if (rc == SALI_OK) rc = check_rows(out, batch->n_tokens > 0);
    if (rc != SALI_OK) return rc;
    if ((d_prior_or_null == nullptr) != (d_prior_lse_or_null == nullptr)) return SALI_ERR_NULL;
    if ((uintptr_t)d_prior_or_null % 16 != 0 || ((uintptr_t)d_prior_lse_or_null | (uintptr_t)d_lse_or_null) % 4 != 0) return SALI_ERR_ALIGN;
    if (window < 0 || sinks < 0 || window > (1 << 30) || sinks > (1 << 30)) return SALI_ERR_SHAPE;
    if (!isfinite(softmax_scale * 1.44269504088896340736f)) return SALI_ERR_CONFIG;
    if (nothing_to_do(*batch)) return SALI_OK;
    // rows and tiles are counted in 31 bits
    if ((int64_t)batch->n_tokens * (p->cfg.n_heads / p->cfg.n_kv_heads) >= 0x7FFFFFFF - 1024) return SALI_ERR_SHAPE;
    if (((int64_t)batch->max_kv / kTileTokens + 2) * p->cfg.n_kv_heads > 0x7FFFFFFFll / batch->n_seqs) return SALI_ERR_SHAPE;
    PagesAttend a = {};
    a.geom = geom_of(p, layer);
    a.seqs = seqs_of(p, *batch);
    a.q = rows_of<RowsIn>(*q);
    a.out = rows_of<RowsOut>(*out);
    a.lse = d_lse_or_null;
    a.prior = d_prior_or_null;
    a.prior_lse = d_prior_lse_or_null;
    a.scale2 = softmax_scale == 0.0f ? 1.0f : fabsf(softmax_scale) * 1.44269504088896340736f;
    a.q_keep = softmax_scale == 0.0f ? 0u : ~0u;
    a.q_flip = softmax_scale < 0.0f ? 0x80008000u : 0u;
    a.window = window;
    a.sinks = window > 0 ? sinks : 0;
    a.heads = p->cfg.n_heads;
    a.group = p->cfg.n_heads / p->cfg.n_kv_heads;
    a.partial = reinterpret_cast<float*>(p->scratch + p->layout.partial);
    a.records = reinterpret_cast<int32_t*>(p->scratch + p->layout.records);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = p->cfg.dtype == SALI_DTYPE_BF16 ? launch_pages_attend_bf16(p->cfg.store, p->cfg.head_dim, a, s)
                                                         : launch_pages_attend_fp16(p->cfg.store, p->cfg.head_dim, a, s);
    return e == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

int sali_pages_get_status(sali_pages* p, uint32_t* h_status, void* stream) {
    if (p == nullptr || h_status == nullptr) return SALI_ERR_NULL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (hipMemcpyAsync(h_status, p->scratch, sizeof(*h_status), hipMemcpyDeviceToHost, s) != hipSuccess) return SALI_ERR_HIP;
    return hipStreamSynchronize(s) == hipSuccess ? SALI_OK : SALI_ERR_HIP;
}

}  // extern "C"
