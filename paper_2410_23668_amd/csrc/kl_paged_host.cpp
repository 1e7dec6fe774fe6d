// Host entry points of the paged KV cache: argument checks and launches.

#include <hip/hip_runtime.h>

#include <cmath>

#include "kl_error.h"
#include "kl_paged.h"

using namespace kl;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

size_t element_bytes(int dtype) { return dtype == KL_DTYPE_FP32 ? 4 : 2; }

kl_status check_cache(const kl_paged_cache *c, const char *who) {
    if (!c) return fail(KL_ERR_INVALID_ARGUMENT, "%s: cache is NULL", who);
    if (c->dtype != KL_DTYPE_BF16 && c->dtype != KL_DTYPE_E4M3)
        return fail(KL_ERR_UNSUPPORTED, "%s: cache dtype %d (KL_DTYPE_BF16 or KL_DTYPE_E4M3)", who,
                    c->dtype);
    if (c->head_dim != 64 && c->head_dim != 128)
        return fail(KL_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (64 or 128)", who, c->head_dim);
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: n_layers, n_pages and n_kv_heads must be >= 1", who);
    if (c->page_size < 8 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(KL_ERR_UNSUPPORTED, "%s: page_size %d is not a power of two in [8, 4096]", who,
                    c->page_size);
    return KL_OK;
}

}  // namespace

namespace kl {

kl_status check_paged_pool(const kl_paged_cache *c, int32_t layer, const kl_page_table *t,
                           const char *who) {
    const kl_status st = check_cache(c, who);
    if (st != KL_OK) return st;
    if (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: cache k and v must be 16-byte aligned pointers", who);
    if (c->dtype == KL_DTYPE_E4M3 &&
        (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 8) || !aligned(c->v_scale, 8)))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: an e4m3 cache needs k_scale and v_scale, 8-byte "
                                             "aligned", who);
    if (layer < 0 || layer >= c->n_layers)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: layer %d outside [0, %d)", who, layer, c->n_layers);
    if (!t || !t->pages || !aligned(t->pages, 4))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: the page table must be a 4-byte aligned pointer", who);
    if (t->batch < 1 || t->max_pages < 1 || t->stride < t->max_pages)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: page table batch %d, max_pages %d, stride %d", who,
                    t->batch, t->max_pages, t->stride);
    if ((int64_t)t->max_pages * c->page_size > (1 << 30))
        return fail(KL_ERR_UNSUPPORTED, "%s: max_pages * page_size above 2^30", who);
    return KL_OK;
}

PagedLayer paged_layer(const kl_paged_cache &c, int32_t layer) {
    PagedLayer p{};
    p.e4m3 = c.dtype == KL_DTYPE_E4M3;
    p.n_pages = c.n_pages; p.nkv = c.n_kv_heads; p.page_log2 = log2_of(c.page_size); p.d = c.head_dim;
    const size_t rows = (size_t)c.n_pages * c.n_kv_heads * c.page_size;
    const size_t off = (size_t)layer * rows * c.head_dim * (p.e4m3 ? 1 : 2);
    p.k = reinterpret_cast<uint8_t *>(c.k) + off;
    p.v = reinterpret_cast<uint8_t *>(c.v) + off;
    if (p.e4m3) {
        p.ks = c.k_scale + layer * rows;
        p.vs = c.v_scale + layer * rows;
    }
    return p;
}

}  // namespace kl

namespace {

kl_status check_device(const kl_paged_cache *c, const char *who) {
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev != c->device)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: current device %d is not the cache's device %d", who,
                    dev, c->device);
    return KL_OK;
}

kl_status check_rows(const kl_rows *r, int64_t rows, int heads, int d, bool output,
                     const char *what, const char *who) {
    if (!r || !r->data) return fail(KL_ERR_INVALID_ARGUMENT, "%s: %s is NULL", who, what);
    if (r->dtype != KL_DTYPE_BF16 && r->dtype != KL_DTYPE_FP16 && r->dtype != KL_DTYPE_FP32)
        return fail(KL_ERR_UNSUPPORTED, "%s: %s dtype %d (KL_DTYPE_BF16, _FP16 or _FP32)", who, what,
                    r->dtype);
    if (!aligned(r->data, element_bytes(r->dtype)))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: %s is not aligned to its elements", who, what);
    const int64_t least = output ? d : 0;
    if ((rows > 1 && r->row_stride < least) || (heads > 1 && r->head_stride < least))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: %s strides %lld, %lld", who, what,
                    (long long)r->row_stride, (long long)r->head_stride);
    return KL_OK;
}

// Whether 8 elements from any multiple of 8 of any head may be moved as 16-byte words.
bool vector_rows(const kl_rows &r, int64_t rows, int heads) {
    const int64_t el = (int64_t)element_bytes(r.dtype);
    return aligned(r.data, 16) && (rows == 1 || r.row_stride * el % 16 == 0) &&
           (heads == 1 || r.head_stride * el % 16 == 0);
}

PagedTable table_of(const kl_page_table &t) {
    return PagedTable{t.pages, t.batch, t.max_pages, t.stride};
}

// kl_paged_append and kl_paged_read: the checks and the kernel's arguments.
kl_status row_params(const kl_paged_cache *cache, int32_t layer, const kl_page_table *table,
                     const int32_t *seq, const int32_t *positions, int64_t rows, const kl_rows *k,
                     const kl_rows *v, int32_t *error, bool output, const char *who, RowParams *p) {
    kl_status st = check_paged_pool(cache, layer, table, who);
    if (st != KL_OK) return st;
    if (rows < 0 || rows > INT32_MAX)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: rows %lld outside [0, 2^31)", who, (long long)rows);
    if (!aligned(seq, 4) || !aligned(positions, 4) || !aligned(error, 4))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: int32 buffers must be 4-byte aligned", who);
    if (!seq && rows > table->batch)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: %lld rows without seq, %d sequences", who,
                    (long long)rows, table->batch);
    if (rows > 0) {
        if (!positions) return fail(KL_ERR_INVALID_ARGUMENT, "%s: positions is NULL", who);
        st = check_rows(k, rows, cache->n_kv_heads, cache->head_dim, output, "k", who);
        if (st != KL_OK) return st;
        st = check_rows(v, rows, cache->n_kv_heads, cache->head_dim, output, "v", who);
        if (st != KL_OK) return st;
        *p = RowParams{paged_layer(*cache, layer), table_of(*table), seq, positions, rows, k->data,
                       v->data, k->dtype, v->dtype, k->row_stride, k->head_stride, v->row_stride,
                       v->head_stride, vector_rows(*k, rows, cache->n_kv_heads),
                       vector_rows(*v, rows, cache->n_kv_heads), error};
    }
    return check_device(cache, who);
}

}  // namespace

extern "C" {

kl_status kl_paged_append(const kl_paged_cache *cache, int32_t layer, const kl_page_table *table,
                          const int32_t *seq, const int32_t *positions, int64_t rows,
                          const kl_rows *k, const kl_rows *v, int32_t *error, void *stream) {
    g_last_error.clear();
    RowParams p;
    const kl_status st = row_params(cache, layer, table, seq, positions, rows, k, v, error, false,
                                    "kl_paged_append", &p);
    if (st != KL_OK || rows == 0) return st;
    HIP_TRY(launch_paged_append(p, reinterpret_cast<hipStream_t>(stream)));
    return KL_OK;
}

kl_status kl_paged_read(const kl_paged_cache *cache, int32_t layer, const kl_page_table *table,
                        const int32_t *seq, const int32_t *positions, int64_t rows,
                        const kl_rows *k, const kl_rows *v, int32_t *error, void *stream) {
    g_last_error.clear();
    RowParams p;
    const kl_status st = row_params(cache, layer, table, seq, positions, rows, k, v, error, true,
                                    "kl_paged_read", &p);
    if (st != KL_OK || rows == 0) return st;
    HIP_TRY(launch_paged_read(p, reinterpret_cast<hipStream_t>(stream)));
    return KL_OK;
}

size_t kl_paged_attention_workspace(const kl_paged_cache *cache, int32_t batch) {
    if (check_cache(cache, "kl_paged_attention_workspace") != KL_OK) return 0;
    if (batch < 1 || batch > kMaxPagedBatch) {
        fail(KL_ERR_INVALID_ARGUMENT, "kl_paged_attention_workspace: batch %d outside [1, %d]",
             batch, kMaxPagedBatch);
        return 0;
    }
    return kPagedPartBytes + (size_t)batch * cache->n_kv_heads * sizeof(unsigned);
}

kl_status kl_paged_attention(const kl_paged_cache *cache, int32_t layer,
                             const kl_page_table *table, const int32_t *lengths, const kl_rows *q,
                             int32_t n_heads, float scale, int32_t window, const kl_rows *out,
                             float *lse, void *workspace, size_t workspace_bytes, int32_t *error,
                             void *stream) {
    const char *const who = "kl_paged_attention";
    g_last_error.clear();
    kl_status st = check_paged_pool(cache, layer, table, who);
    if (st != KL_OK) return st;
    const kl_paged_cache &c = *cache;
    const int B = table->batch;
    if (B > kMaxPagedBatch)
        return fail(KL_ERR_UNSUPPORTED, "%s: batch %d above %d", who, B, kMaxPagedBatch);
    if (n_heads < 1 || n_heads % c.n_kv_heads != 0)
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: n_heads %d is not a multiple of n_kv_heads %d", who,
                    n_heads, c.n_kv_heads);
    if (n_heads / c.n_kv_heads > kMaxGroup)
        return fail(KL_ERR_UNSUPPORTED, "%s: %d query heads per KV head (at most %d)", who,
                    n_heads / c.n_kv_heads, kMaxGroup);
    if (!lengths || !aligned(lengths, 4) || !aligned(lse, 4) || !aligned(error, 4))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: lengths must not be NULL, and int32/fp32 buffers "
                                             "4-byte aligned", who);
    // (tiles, of 32 positions at least, are counted in 32 bits)
    if ((int64_t)B * c.n_kv_heads * (((int64_t)table->max_pages * c.page_size + 31) / 32) > (1 << 30))
        return fail(KL_ERR_UNSUPPORTED, "%s: batch * n_kv_heads * max_pages * page_size above 2^35",
                    who);
    st = check_rows(q, B, n_heads, c.head_dim, false, "q", who);
    if (st != KL_OK) return st;
    st = check_rows(out, B, n_heads, c.head_dim, true, "out", who);
    if (st != KL_OK) return st;
    // (times log2 e it has to be finite)
    if (!(std::fabs(scale) <= 0x1p127f))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: scale is not at most 2^127 in magnitude", who);
    if (window < 0) return fail(KL_ERR_INVALID_ARGUMENT, "%s: window %d < 0", who, window);
    if (!workspace || !aligned(workspace, 16) ||
        workspace_bytes < kl_paged_attention_workspace(cache, B))
        return fail(KL_ERR_INVALID_ARGUMENT, "%s: the workspace must be 16-byte aligned and hold %zu "
                                             "bytes", who, kl_paged_attention_workspace(cache, B));
    st = check_device(cache, who);
    if (st != KL_OK) return st;
    AttnParams p{};
    p.c = paged_layer(c, layer); p.t = table_of(*table);
    p.lengths = lengths;
    p.q = q->data; p.q_type = q->dtype; p.q_row = q->row_stride; p.q_head = q->head_stride;
    p.q_vec = vector_rows(*q, B, n_heads);
    p.out_vec = vector_rows(*out, B, n_heads);
    p.out = out->data; p.out_type = out->dtype;
    p.out_row = out->row_stride; p.out_head = out->head_stride;
    p.nq = n_heads; p.group = n_heads / c.n_kv_heads;
    p.scale = scale; p.window = window; p.lse = lse; p.error = error;
    p.parts = reinterpret_cast<float *>(workspace);
    p.arrived = reinterpret_cast<unsigned *>(reinterpret_cast<uint8_t *>(workspace) +
                                             kPagedPartBytes);
    HIP_TRY(launch_paged_attention(p, reinterpret_cast<hipStream_t>(stream)));
    return KL_OK;
}

}  // extern "C"
