// C ABI of the serving-layer operators: argument validation on the host, then kernel launches.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/vitq.h"
#include "attention_paged.h"
#include "gemm_e4m3.h"
#include "quantize_e4m3.h"
#include "rotate.h"

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p) % 16 == 0; }
bool is16bit(int32_t t) { return t == VQ_BF16 || t == VQ_F16; }
bool is_float(int32_t t) { return t == VQ_F32 || is16bit(t); }
int64_t size_of(int32_t t) { return t == VQ_F32 ? 4 : (t == VQ_E4M3 ? 1 : 2); }

vq_status check_fmat(const vq_fmat *m) {
    if (!m) return VQ_ERR_NULL;
    if (m->block_rows != 1 && m->block_rows != 128) return VQ_ERR_UNSUPPORTED;
    if (m->rows < 0 || m->cols <= 0 || m->rows > (1 << 27) || m->cols > (1 << 22)) return VQ_ERR_SHAPE;
    if (m->row_stride <= 0 || m->row_stride % 16 != 0 || m->row_stride < m->cols) return VQ_ERR_STRIDE;
    if (m->scale_stride < (m->rows + m->block_rows - 1) / m->block_rows) return VQ_ERR_STRIDE;
    if (m->rows > 0 && (!m->data || !m->scales)) return VQ_ERR_NULL;
    if (!aligned16(m->data) || ((uintptr_t)m->scales) % 4 != 0) return VQ_ERR_STRIDE;
    return VQ_OK;
}

vq_status check_cache(const vq_kv_cache *c) {
    if (!c || !c->k || !c->v) return VQ_ERR_NULL;
    if (!is16bit(c->dtype) && c->dtype != VQ_E4M3) return VQ_ERR_BITS;
    if (c->heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || c->pages <= 0) return VQ_ERR_SHAPE;
    if (c->heads > 4096 || c->head_dim > 256 || c->pages > INT32_MAX) return VQ_ERR_SHAPE;
    if (c->pages * (int64_t)c->page_size > INT32_MAX) return VQ_ERR_SHAPE;
    const int64_t size = size_of(c->dtype), unit = 16 / size;       // elements of 16 bytes
    const int64_t limit = (int64_t(1) << 36) / size;
    const int64_t s[3] = {c->page_stride, c->head_stride, c->token_stride};
    const int64_t n[3] = {c->pages, c->heads, c->page_size};
    int64_t last = c->head_dim;
    for (int i = 0; i < 3; ++i) {
        if (n[i] > 1 && s[i] < c->head_dim) return VQ_ERR_STRIDE;   // (a stride of an extent of one is never used)
        if (s[i] < 0 || s[i] % unit != 0 || s[i] > limit) return VQ_ERR_STRIDE;
        if (n[i] > 1 && s[i] > limit / (n[i] - 1)) return VQ_ERR_SHAPE;
        last += (n[i] - 1) * s[i];
    }
    if (last > limit) return VQ_ERR_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v)) return VQ_ERR_STRIDE;
    if (!isfinite(c->k_scale) || !isfinite(c->v_scale) || c->k_scale <= 0.0f || c->v_scale <= 0.0f) return VQ_ERR_STEP;
    if (c->dtype != VQ_E4M3 && (c->k_scale != 1.0f || c->v_scale != 1.0f)) return VQ_ERR_STEP;
    return VQ_OK;
}

// Rows of `cols` elements: 16-byte aligned, far enough apart.
vq_status check_rows(const void *p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype) {
    if (rows > 0 && !p) return VQ_ERR_NULL;
    if (ld < cols || (ld * size_of(dtype)) % 16 != 0 || !aligned16(p)) return VQ_ERR_STRIDE;
    if (ld > (int64_t(1) << 40)) return VQ_ERR_STRIDE;
    return VQ_OK;
}

vq_status check_attention_sizes(int64_t tokens, int32_t seqs, int32_t q_heads, const vq_kv_cache *cache, int64_t max_kv) {
    vq_status st = check_cache(cache);
    if (st != VQ_OK) return st;
    if (tokens < 0 || seqs < 0 || q_heads <= 0 || max_kv < 0) return VQ_ERR_SHAPE;
    if (q_heads % cache->heads != 0) return VQ_ERR_SHAPE;
    // rows are counted, and workgroups launched, in 32 bits
    if (tokens > (1 << 22) || seqs > (1 << 20) || q_heads > 4096 || tokens * q_heads > (1 << 26)) return VQ_ERR_SHAPE;
    if ((int64_t)seqs * cache->heads > (1 << 21)) return VQ_ERR_SHAPE;
    if (cache->head_dim != 64 && cache->head_dim != 128) return VQ_ERR_UNSUPPORTED;
    return VQ_OK;
}

size_t split_bytes(int splits, int64_t tokens, int32_t q_heads, int32_t head_dim) {
    return splits > 1 ? (size_t)splits * tokens * q_heads * (head_dim + 1) * 4 : 0;
}

}  // namespace

extern "C" {

vq_status vq_quantize_e4m3(const void *x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ld, const vq_fmat *out,
                           void *stream) {
    vq_status st = check_fmat(out);
    if (st != VQ_OK) return st;
    if (!is_float(x_dtype)) return VQ_ERR_BITS;
    if (rows != out->rows || cols != out->cols) return VQ_ERR_SHAPE;
    if (ld < cols) return VQ_ERR_SHAPE;
    if (rows == 0) return VQ_OK;
    if (!x) return VQ_ERR_NULL;
    const int64_t size = size_of(x_dtype);
    if (((uintptr_t)x) % size != 0) return VQ_ERR_STRIDE;
    vitq::QuantE4M3Params p{};
    p.x = x; p.rows = rows; p.cols = cols; p.ld = ld;
    p.aligned = aligned16(x) && (ld * size) % 16 == 0;
    p.codes = (uint8_t *)out->data; p.code_stride = out->row_stride;
    p.scales = out->scales; p.scale_stride = out->scale_stride;
    return vitq::quantize_e4m3_launch(p, x_dtype, out->block_rows, (hipStream_t)stream) == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

vq_status vq_linear_e4m3(const vq_fmat *x, const vq_fmat *w, const float *bias, int32_t act, void *y, int32_t y_dtype,
                         int64_t ld, void *stream) {
    vq_status st;
    if ((st = check_fmat(x)) != VQ_OK) return st;
    if ((st = check_fmat(w)) != VQ_OK) return st;
    if (x->block_rows != 1 || w->block_rows != 128) return VQ_ERR_UNSUPPORTED;
    if (x->cols != w->cols || x->cols > 65536) return VQ_ERR_SHAPE;
    if (x->row_stride >= (1 << 24) || w->row_stride >= (1 << 24)) return VQ_ERR_STRIDE;
    if (!is_float(y_dtype)) return VQ_ERR_BITS;
    if (act != 0 && act != 1) return VQ_ERR_UNSUPPORTED;
    if (ld < w->rows) return VQ_ERR_STRIDE;
    if (x->rows == 0 || w->rows == 0) return VQ_OK;
    if (!y) return VQ_ERR_NULL;
    const int64_t size = size_of(y_dtype);
    if (((uintptr_t)y) % size != 0 || ((uintptr_t)bias) % 4 != 0) return VQ_ERR_STRIDE;
    vitq::GemmE4M3Params p{};
    p.x = (const uint8_t *)x->data; p.x_stride = x->row_stride; p.xs = x->scales; p.xs_stride = x->scale_stride; p.M = (int)x->rows;
    p.w = (const uint8_t *)w->data; p.w_stride = w->row_stride; p.ws = w->scales; p.ws_stride = w->scale_stride; p.Nout = (int)w->rows;
    p.K = (int)x->cols; p.kbytes16 = (int)((x->cols + 15) / 16 * 16);
    p.bias = bias; p.act = act; p.y = y; p.y_dtype = y_dtype; p.ld = ld;
    p.vec_ok = aligned16(y) && (ld * size) % 16 == 0;
    return vitq::gemm_e4m3_launch(p, (hipStream_t)stream) == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

vq_status vq_qkv_norm_rotate(const vq_rotate_desc *d, const void *qkv, int32_t dtype, int64_t tokens, int64_t ld,
                             const int32_t *positions, void *q_out, int32_t q_dtype, int64_t q_ld,
                             const vq_kv_cache *cache, const int64_t *slots, void *stream) {
    if (!d) return VQ_ERR_NULL;
    if (d->q_heads <= 0 || d->kv_heads <= 0 || d->q_heads > 4096 || d->kv_heads > 4096) return VQ_ERR_SHAPE;
    if (d->head_dim <= 0 || d->head_dim > 256 || d->head_dim % 8 != 0) return VQ_ERR_SHAPE;
    if (tokens < 0 || tokens > (1 << 23)) return VQ_ERR_SHAPE;
    if (d->norm < 0 || d->norm > 2) return VQ_ERR_UNSUPPORTED;
    if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 16 != 0) return VQ_ERR_SHAPE;
    if (!is_float(dtype)) return VQ_ERR_BITS;
    vq_status st;
    if ((st = check_rows(qkv, tokens, (int64_t)(d->q_heads + 2 * d->kv_heads) * d->head_dim, ld, dtype)) != VQ_OK) return st;
    if ((cache != nullptr) != (slots != nullptr)) return VQ_ERR_NULL;
    if (!q_out && !cache) return VQ_ERR_NULL;
    if (q_out) {
        if (!is16bit(q_dtype)) return VQ_ERR_BITS;
        if ((st = check_rows(q_out, tokens, (int64_t)d->q_heads * d->head_dim, q_ld, q_dtype)) != VQ_OK) return st;
    }
    if (cache) {
        if ((st = check_cache(cache)) != VQ_OK) return st;
        if (cache->heads != d->kv_heads || cache->head_dim != d->head_dim) return VQ_ERR_SHAPE;
        if (cache->dtype == VQ_E4M3 && d->head_dim % 16 != 0) return VQ_ERR_SHAPE;
        if (!isfinite(1.0f / cache->k_scale) || !isfinite(1.0f / cache->v_scale)) return VQ_ERR_STEP;
        if (((uintptr_t)slots) % 8 != 0) return VQ_ERR_STRIDE;
    }
    if (d->norm != 0) {
        if ((q_out && !d->q_gamma) || (cache && !d->k_gamma)) return VQ_ERR_NULL;
        if (!isfinite(d->eps) || d->eps < 0.0f) return VQ_ERR_STEP;
        if (d->gamma_head_stride != 0 && (d->gamma_head_stride < d->head_dim || d->gamma_head_stride % 4 != 0)) return VQ_ERR_STRIDE;
        if (!aligned16(d->q_gamma) || !aligned16(d->k_gamma) || !aligned16(d->q_beta) || !aligned16(d->k_beta)) return VQ_ERR_STRIDE;
    }
    if (d->rot_dim > 0) {
        if (!d->cos_table || !d->sin_table || (tokens > 0 && !positions)) return VQ_ERR_NULL;
        if (d->table_rows <= 0) return VQ_ERR_SHAPE;
        if (!aligned16(d->cos_table) || !aligned16(d->sin_table) || ((uintptr_t)positions) % 4 != 0) return VQ_ERR_STRIDE;
    }
    if (tokens == 0) return VQ_OK;
    vitq::RotateParams p{};
    p.qkv = qkv; p.ld = ld; p.tokens = tokens;
    p.q_heads = d->q_heads; p.kv_heads = d->kv_heads; p.head_dim = d->head_dim;
    p.head_begin = q_out ? 0 : d->q_heads;
    p.head_end = cache ? d->q_heads + 2 * d->kv_heads : d->q_heads;
    p.norm = d->norm; p.rot_dim = d->rot_dim; p.interleaved = d->interleaved ? 1 : 0;
    p.q_gamma = d->q_gamma; p.q_beta = d->q_beta; p.k_gamma = d->k_gamma; p.k_beta = d->k_beta;
    p.gamma_stride = d->gamma_head_stride;
    p.cos_table = d->cos_table; p.sin_table = d->sin_table; p.table_rows = d->table_rows;
    p.eps = d->eps; p.inv_dim = 1.0f / (float)d->head_dim;
    p.positions = positions; p.q_out = q_out; p.q_dtype = q_dtype; p.q_ld = q_ld;
    if (cache) {
        p.k = (uint8_t *)cache->k; p.v = (uint8_t *)cache->v; p.cache_dtype = cache->dtype;
        p.page_stride = cache->page_stride; p.head_stride = cache->head_stride; p.token_stride = cache->token_stride;
        p.page_size = (uint32_t)cache->page_size; p.page_div = vitq::fast_div(p.page_size); p.slots_end = cache->pages * cache->page_size;
        p.k_inv = 1.0f / cache->k_scale; p.v_inv = 1.0f / cache->v_scale;
        p.slots = slots;
    }
    return vitq::rotate_launch(p, dtype, (hipStream_t)stream) == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

vq_status vq_attention_paged_workspace(int64_t tokens, int32_t seqs, int32_t q_heads, const vq_kv_cache *cache,
                                       int64_t max_kv, size_t *bytes) {
    if (!bytes) return VQ_ERR_NULL;
    vq_status st = check_attention_sizes(tokens, seqs, q_heads, cache, max_kv);
    if (st != VQ_OK) return st;
    if (tokens == 0 || seqs == 0) { *bytes = 0; return VQ_OK; }
    if (max_kv == 0) max_kv = INT32_MAX;
    *bytes = split_bytes(vitq::paged_splits(tokens, seqs, q_heads, cache->heads, cache->head_dim, max_kv), tokens, q_heads,
                         cache->head_dim);
    return VQ_OK;
}

vq_status vq_attention_paged(const void *q, int32_t dtype, int64_t tokens, int64_t q_ld, int32_t q_heads,
                             const int32_t *q_offsets, const int32_t *kv_lens, int32_t seqs, const int32_t *page_table,
                             int64_t table_stride, int32_t table_cols, const vq_kv_cache *cache, float scale,
                             int32_t causal, int32_t window, int64_t max_kv, void *out, int64_t out_ld, float *lse,
                             void *workspace, size_t workspace_bytes, void *stream) {
    vq_status st = check_attention_sizes(tokens, seqs, q_heads, cache, max_kv);
    if (st != VQ_OK) return st;
    if (!is16bit(dtype) || (cache->dtype != VQ_E4M3 && cache->dtype != dtype)) return VQ_ERR_BITS;
    const int64_t cols = (int64_t)q_heads * cache->head_dim;
    if ((st = check_rows(q, tokens, cols, q_ld, dtype)) != VQ_OK) return st;
    if ((st = check_rows(out, tokens, cols, out_ld, dtype)) != VQ_OK) return st;
    if (table_cols < 0 || window < 0 || (int64_t)table_cols * cache->page_size > (1 << 30)) return VQ_ERR_SHAPE;
    if (table_stride < table_cols) return VQ_ERR_STRIDE;
    if (!isfinite(scale)) return VQ_ERR_STEP;
    if (tokens == 0 || seqs == 0) return VQ_OK;
    if (!q_offsets || !kv_lens || (table_cols > 0 && !page_table)) return VQ_ERR_NULL;
    if (((uintptr_t)q_offsets | (uintptr_t)kv_lens | (uintptr_t)page_table | (uintptr_t)lse) % 4 != 0) return VQ_ERR_STRIDE;
    // an `out` that overlaps q must be q: the rows are read and written by the same workgroup
    if (q == out && q_ld != out_ld) return VQ_ERR_STRIDE;
    const int64_t most = (int64_t)table_cols * cache->page_size;
    if (max_kv == 0 || max_kv > most) max_kv = most;
    if (window > (1 << 30)) window = 0;                       // reaches past every first key
    // A window shortens what a tile of rows sees, to itself and the tile's tokens (up to 256) under the causal mask, and without it, when
    // rows see up to the last key, to itself and the sequence's new tokens, of which the host knows the mean.  (The workspace, which
    // knows of no window, is then more than enough.)
    const int64_t mean = tokens / seqs, reach = window + (causal || mean < 256 ? 256 : mean);
    const int64_t longest = window > 0 && reach < max_kv ? reach : max_kv;
    vitq::PagedParams p{};
    p.splits = vitq::paged_splits(tokens, seqs, q_heads, cache->heads, cache->head_dim, longest);
    const size_t need = split_bytes(p.splits, tokens, q_heads, cache->head_dim);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return VQ_ERR_WORKSPACE;
        if (!aligned16(workspace)) return VQ_ERR_STRIDE;
        p.part = (float *)workspace;
        p.part_lse = p.part + (int64_t)p.splits * tokens * cols;
    }
    p.q = (const uint8_t *)q; p.q_ld = q_ld; p.tokens = tokens;
    p.q_heads = q_heads; p.kv_heads = cache->heads; p.group = q_heads / cache->heads;
    p.q_offsets = q_offsets; p.kv_lens = kv_lens; p.seqs = seqs;
    p.page_table = page_table; p.table_stride = table_stride; p.table_cols = table_cols;
    p.k = (const uint8_t *)cache->k; p.v = (const uint8_t *)cache->v;
    p.pages = (uint32_t)cache->pages; p.page_size = (uint32_t)cache->page_size;
    const int64_t size = size_of(cache->dtype);
    p.page_units = (uint32_t)(cache->page_stride * size / 16);
    p.head_units = (uint32_t)(cache->head_stride * size / 16);
    p.token_units = (uint32_t)(cache->token_stride * size / 16);
    p.whole_rows = p.page_size % 16 == 0 && p.token_units < (1u << 23);
    p.page_div = vitq::fast_div(p.page_size); p.group_div = vitq::fast_div((uint32_t)p.group);
    // The kernels take maxima before scaling and mask with -infinity, so they get a positive factor: the sign goes to the
    // queries, and zero becomes a number that leaves every finite score at zero.
    p.negative = scale < 0.0f ? 1 : 0;
    p.scale_log2 = (float)(fabs((double)scale) * (double)cache->k_scale * 1.4426950408889634);
    if (!isfinite(p.scale_log2)) return VQ_ERR_STEP;
    if (p.scale_log2 < 0x1p-126f) p.scale_log2 = 0x1p-126f;
    p.v_scale = cache->v_scale;
    p.causal = causal ? 1 : 0; p.window = window;
    p.out = (uint8_t *)out; p.out_ld = out_ld; p.lse = lse;
    return vitq::paged_launch(p, dtype, cache->dtype, cache->head_dim, longest, (hipStream_t)stream) == hipSuccess ? VQ_OK : VQ_ERR_HIP;
}

}  // extern "C"
