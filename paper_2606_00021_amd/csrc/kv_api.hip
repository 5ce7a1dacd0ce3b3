// Host layer of the 4-bit paged key/value cache (the sense_kv_* entry points
// of include/sense.h): argument validation, workspace sizes, launches.
#include <initializer_list>

#include "host.h"
#include "internal.h"
#include "kv.h"
#include "sense.h"

#define SENSE_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using sense::aligned;
using sense::fail;
using sense::KvBatch;
using sense::KvCache;
using sense::ok;

sense_status_t launched(hipError_t e, const char* where) {
    if (e == hipSuccess) return ok();
    return fail(SENSE_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
}

// One dispatch holds fewer than 2^32 work-items per dimension; workgroups here
// have up to 256.
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 8;

sense_status_t check_shape(const sense_kv_cache_t* c) {
    if (!c) return fail(SENSE_ERR_INVALID_ARGUMENT, "cache is NULL");
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "page_size = %d is none of 16, 32, 64, 128",
                    c->page_size);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "head_dim = %d is none of 64, 128, 256",
                    c->head_dim);
    if (c->n_layers < 1 || c->n_layers > 4096)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n_layers = %d outside [1, 4096]", c->n_layers);
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n_kv_heads = %d outside [1, 1024]",
                    c->n_kv_heads);
    if (c->n_pages < 1 || c->n_pages > (1 << 26))
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n_pages = %d outside [1, 2^26]", c->n_pages);
    if (c->n_seqs < 1 || c->n_seqs > (1 << 26))
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n_seqs = %d outside [1, 2^26]", c->n_seqs);
    if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > ((int64_t)1 << 30))
        return fail(SENSE_ERR_INVALID_ARGUMENT,
                    "max_pages = %d: at least 1, and at most 2^30 positions", c->max_pages);
    return SENSE_OK;
}

sense_status_t check_cache(const sense_kv_cache_t* c, KvCache* out) {
    sense_status_t s = check_shape(c);
    if (s != SENSE_OK) return s;
    if (!c->codes || !c->scales || !c->page_table || !c->seq_len || !c->page_refs)
        return fail(SENSE_ERR_INVALID_ARGUMENT,
                    "codes, scales, page_table, seq_len and page_refs must be non-NULL");
    if (!aligned(c->codes, 16) || !aligned(c->scales, 16))
        return fail(SENSE_ERR_MISALIGNED, "codes and scales must be 16-byte aligned");
    if (!aligned(c->page_table, 4) || !aligned(c->seq_len, 4) || !aligned(c->page_refs, 4))
        return fail(SENSE_ERR_MISALIGNED, "page_table, seq_len and page_refs are int32 arrays");
    out->codes = (uint8_t*)c->codes;
    out->scales = (uint8_t*)c->scales;
    out->page_table = c->page_table;
    out->seq_len = c->seq_len;
    out->page_refs = c->page_refs;
    out->n_layers = c->n_layers;
    out->n_pages = c->n_pages;
    out->lg_page = __builtin_ctz((unsigned)c->page_size);
    out->heads = c->n_kv_heads;
    out->d = c->head_dim;
    out->n_seqs = c->n_seqs;
    out->max_pages = c->max_pages;
    return SENSE_OK;
}

sense_status_t check_batch(const KvCache& c, const sense_kv_batch_t* b, KvBatch* out) {
    if (!b) return fail(SENSE_ERR_INVALID_ARGUMENT, "batch is NULL");
    if (b->n < 0 || b->n > 65536)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d outside [0, 65536]", b->n);
    if (b->max_rows < 1 || b->max_rows > sense::kKvMaxRows)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "max_rows = %d outside [1, %d]", b->max_rows,
                    sense::kKvMaxRows);
    if (!b->seqs && b->n > c.n_seqs)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d entries of %d sequences without seqs",
                    b->n, c.n_seqs);
    if (b->n_rows < 0) return fail(SENSE_ERR_INVALID_ARGUMENT, "n_rows < 0");
    if (!aligned(b->seqs, 4) || !aligned(b->row_start, 4) || !aligned(b->row_len, 4))
        return fail(SENSE_ERR_MISALIGNED, "seqs, row_start and row_len are int32 arrays");
    *out = KvBatch{b->seqs, b->row_start, b->row_len, b->n, b->max_rows, b->n_rows};
    return SENSE_OK;
}

sense_status_t check_rows(const void* p, int elem, int64_t stride, int64_t least,
                          const char* name) {
    if (stride < least)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "%s: row stride %lld below %lld elements", name,
                    (long long)stride, (long long)least);
    if (!aligned(p, 16) || stride * elem % 16)
        return fail(SENSE_ERR_MISALIGNED, "%s: base and row stride must be multiples of 16 bytes",
                    name);
    return SENSE_OK;
}

sense_status_t rows_call(bool write, const sense_kv_cache_t* cache, int32_t layer,
                         int32_t n_layers, const void* k, const void* v, sense_dtype_t dtype,
                         int64_t row_stride, int64_t layer_stride, const sense_kv_batch_t* batch,
                         void* stream) {
    KvCache c;
    KvBatch b;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK || (s = check_batch(c, batch, &b)) != SENSE_OK) return s;
    if (n_layers < 1 || layer < 0 || layer > c.n_layers - n_layers)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "layers [%d, %d) of %d", layer, layer + n_layers,
                    c.n_layers);
    if (dtype != SENSE_F32 && dtype != SENSE_F16 && dtype != SENSE_BF16)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "unknown dtype %d", (int)dtype);
    if (b.n == 0) return ok();
    if (!k || !v) return fail(SENSE_ERR_INVALID_ARGUMENT, "k and v must be non-NULL");
    const int elem = dtype == SENSE_F32 ? 4 : 2;
    const int64_t least = (int64_t)c.heads * c.d;
    if ((s = check_rows(k, elem, row_stride, least, "k")) != SENSE_OK) return s;
    if ((s = check_rows(v, elem, row_stride, least, "v")) != SENSE_OK) return s;
    if (n_layers > 1 && (layer_stride < 0 || layer_stride * elem % 16))
        return fail(SENSE_ERR_MISALIGNED, "layer_stride must be a multiple of 16 bytes");
    if (sense::kv_rows_blocks(c, b) > kMaxBlocks)
        return fail(SENSE_ERR_UNSUPPORTED, "%d entries of up to %d rows: too many for one call",
                    b.n, b.max_rows);
    const sense::KvRows r = {(void*)k, (void*)v, (int)dtype, row_stride, layer_stride, layer,
                             n_layers};
    const hipStream_t st = (hipStream_t)stream;
    return launched(write ? sense::launch_kv_write(c, b, r, st) : sense::launch_kv_read(c, b, r, st),
                    write ? "cache write" : "cache read");
}

sense_status_t check_entries(const KvCache& c, const int32_t* seqs, int32_t n) {
    if (n < 0 || n > sense::kKvMaxEntries)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d outside [0, %d]", n,
                    sense::kKvMaxEntries);
    if (!seqs && n > c.n_seqs)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d entries of %d sequences without seqs", n,
                    c.n_seqs);
    return SENSE_OK;
}

// int32 arrays of a page operation (NULL where one is not given).
sense_status_t check_ints(const char* names, std::initializer_list<const void*> arrays) {
    for (const void* p : arrays)
        if (!aligned(p, 4))
            return fail(SENSE_ERR_MISALIGNED, "%s are int32 arrays", names);
    return SENSE_OK;
}

sense_status_t check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return SENSE_OK;
    if (!ws || have < need)
        return fail(SENSE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : (size_t)0,
                    need);
    if (!aligned(ws, 256)) return fail(SENSE_ERR_MISALIGNED, "workspace must be 256-byte aligned");
    return SENSE_OK;
}

sense_status_t check_heads(int n_heads, int kv_heads) {
    if (n_heads < kv_heads || n_heads % kv_heads || n_heads > 4096)
        return fail(SENSE_ERR_INVALID_ARGUMENT,
                    "n_heads = %d: a multiple of %d key heads, at most 4096", n_heads, kv_heads);
    return SENSE_OK;
}

// A bound on the lengths: the caller's, or the capacity.
int bound_of(const sense_kv_cache_t* c, int32_t max_kv) {
    const int cap = c->max_pages * c->page_size;
    return max_kv > 0 && max_kv < cap ? max_kv : cap;
}

}  // namespace

SENSE_EXPORT sense_status_t sense_kv_write(const sense_kv_cache_t* cache, int32_t layer,
                                           int32_t n_layers, const void* k, const void* v,
                                           sense_dtype_t dtype, int64_t row_stride,
                                           int64_t layer_stride, const sense_kv_batch_t* batch,
                                           void* stream) {
    return rows_call(true, cache, layer, n_layers, k, v, dtype, row_stride, layer_stride, batch,
                     stream);
}

SENSE_EXPORT sense_status_t sense_kv_read(const sense_kv_cache_t* cache, int32_t layer,
                                          int32_t n_layers, void* out_k, void* out_v,
                                          sense_dtype_t dtype, int64_t row_stride,
                                          int64_t layer_stride, const sense_kv_batch_t* batch,
                                          void* stream) {
    return rows_call(false, cache, layer, n_layers, out_k, out_v, dtype, row_stride, layer_stride,
                     batch, stream);
}

SENSE_EXPORT sense_status_t sense_kv_attention_workspace_size(const sense_kv_cache_t* cache,
                                                              int32_t n, int32_t max_rows,
                                                              int32_t n_heads, int32_t max_kv,
                                                              size_t* bytes) {
    if (!bytes) return fail(SENSE_ERR_INVALID_ARGUMENT, "bytes is NULL");
    sense_status_t s = check_shape(cache);
    if (s != SENSE_OK || (s = check_heads(n_heads, cache->n_kv_heads)) != SENSE_OK) return s;
    if (n < 0 || n > 65536 || max_rows < 1 || max_rows > sense::kKvMaxRows || max_kv < 0)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d, max_rows = %d, max_kv = %d", n, max_rows,
                    max_kv);
    if (n > 0 && sense::kv_attention_blocks(n, max_rows, n_heads, cache->n_kv_heads,
                                            cache->head_dim) > kMaxBlocks)
        return fail(SENSE_ERR_UNSUPPORTED, "%d entries of up to %d rows: too many for one call", n,
                    max_rows);
    *bytes = n == 0 ? 0
                    : sense::kv_attention_workspace_bytes(n, max_rows, n_heads, cache->n_kv_heads,
                                                          cache->head_dim, bound_of(cache, max_kv));
    return ok();
}

SENSE_EXPORT sense_status_t sense_kv_attention(
    const sense_kv_cache_t* cache, int32_t layer, const void* q, sense_dtype_t q_dtype,
    int32_t n_heads, int64_t q_stride, const sense_kv_batch_t* batch, const uint8_t* mask,
    int64_t mask_ld, int64_t mask_stride, float softmax_scale, int32_t max_kv, void* out,
    int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
    KvCache c;
    KvBatch b;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK || (s = check_batch(c, batch, &b)) != SENSE_OK) return s;
    if (layer < 0 || layer >= c.n_layers)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "layer %d of %d", layer, c.n_layers);
    if (q_dtype != SENSE_F16 && q_dtype != SENSE_BF16)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "q_dtype = %d is neither F16 nor BF16",
                    (int)q_dtype);
    if ((s = check_heads(n_heads, c.heads)) != SENSE_OK) return s;
    if (!(softmax_scale > 0.f) || !(softmax_scale <= 0x1p127f))
        return fail(SENSE_ERR_INVALID_ARGUMENT, "softmax_scale = %g outside (0, 2^127]",
                    (double)softmax_scale);
    if (max_kv < 0) return fail(SENSE_ERR_INVALID_ARGUMENT, "max_kv = %d < 0", max_kv);
    if (mask && (mask_ld < b.max_rows || mask_stride < 0))
        return fail(SENSE_ERR_INVALID_ARGUMENT, "mask_ld = %lld below %d rows, or mask_stride < 0",
                    (long long)mask_ld, b.max_rows);
    if (b.n == 0) return ok();
    if (!q || !out) return fail(SENSE_ERR_INVALID_ARGUMENT, "q and out must be non-NULL");
    const int64_t least = (int64_t)n_heads * c.d;
    if ((s = check_rows(q, 2, q_stride, least, "q")) != SENSE_OK) return s;
    if ((s = check_rows(out, 2, out_stride, least, "out")) != SENSE_OK) return s;
    if (sense::kv_attention_blocks(b.n, b.max_rows, n_heads, c.heads, c.d) > kMaxBlocks)
        return fail(SENSE_ERR_UNSUPPORTED, "%d entries of up to %d rows: too many for one call",
                    b.n, b.max_rows);
    sense::KvAttention a;
    a.q = q;
    a.out = out;
    a.dtype = (int)q_dtype;
    a.layer = layer;
    a.n_heads = n_heads;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.mask = mask;
    a.mask_ld = mask_ld;
    a.mask_stride = mask_stride;
    a.scale = softmax_scale;
    a.max_kv = bound_of(cache, max_kv);
    if ((s = check_workspace(workspace, workspace_bytes,
                             sense::kv_attention_workspace_bytes(b.n, b.max_rows, n_heads, c.heads,
                                                                 c.d, a.max_kv))) != SENSE_OK)
        return s;
    return launched(sense::launch_kv_attention(c, b, a, workspace, (hipStream_t)stream),
                    "cache attention");
}

SENSE_EXPORT sense_status_t sense_kv_truncate(const sense_kv_cache_t* cache, const int32_t* seqs,
                                              const int32_t* lens, int32_t n, int32_t* out_status,
                                              void* stream) {
    KvCache c;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK || (s = check_entries(c, seqs, n)) != SENSE_OK) return s;
    if (n == 0) return ok();
    if ((s = check_ints("seqs, lens and out_status", {seqs, lens, out_status})) != SENSE_OK)
        return s;
    return launched(sense::launch_kv_truncate(c, seqs, lens, n, out_status, (hipStream_t)stream),
                    "cache truncate");
}

SENSE_EXPORT sense_status_t sense_kv_fork(const sense_kv_cache_t* cache, const int32_t* src,
                                          const int32_t* dst, int32_t n, int32_t* out_status,
                                          void* stream) {
    KvCache c;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK) return s;
    if (n < 0 || n > sense::kKvMaxEntries)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d outside [0, %d]", n,
                    sense::kKvMaxEntries);
    if (n == 0) return ok();
    if (!src || !dst) return fail(SENSE_ERR_INVALID_ARGUMENT, "src and dst must be non-NULL");
    if ((s = check_ints("src, dst and out_status", {src, dst, out_status})) != SENSE_OK) return s;
    return launched(sense::launch_kv_fork(c, src, dst, n, out_status, (hipStream_t)stream),
                    "cache fork");
}

SENSE_EXPORT sense_status_t sense_kv_reserve_workspace_size(const sense_kv_cache_t* cache,
                                                            int32_t n, size_t* bytes) {
    if (!bytes) return fail(SENSE_ERR_INVALID_ARGUMENT, "bytes is NULL");
    sense_status_t s = check_shape(cache);
    if (s != SENSE_OK) return s;
    if (n < 0 || n > sense::kKvMaxEntries)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d outside [0, %d]", n,
                    sense::kKvMaxEntries);
    *bytes = n == 0 ? 0 : sense::kv_reserve_workspace_bytes(n, cache->n_pages);
    return ok();
}

SENSE_EXPORT sense_status_t sense_kv_reserve(const sense_kv_cache_t* cache, const int32_t* seqs,
                                             const int32_t* counts, int32_t n,
                                             int32_t* out_status, void* workspace,
                                             size_t workspace_bytes, void* stream) {
    KvCache c;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK || (s = check_entries(c, seqs, n)) != SENSE_OK) return s;
    if (n == 0) return ok();
    if (!counts) return fail(SENSE_ERR_INVALID_ARGUMENT, "counts is NULL");
    if ((s = check_ints("seqs, counts and out_status", {seqs, counts, out_status})) != SENSE_OK)
        return s;
    if ((s = check_workspace(workspace, workspace_bytes,
                             sense::kv_reserve_workspace_bytes(n, c.n_pages))) != SENSE_OK)
        return s;
    return launched(sense::launch_kv_reserve(c, seqs, counts, n, out_status, workspace,
                                             (hipStream_t)stream),
                    "cache reserve");
}

SENSE_EXPORT sense_status_t sense_kv_compact_workspace_size(int32_t n, int32_t keep_ld,
                                                            size_t* bytes) {
    if (!bytes) return fail(SENSE_ERR_INVALID_ARGUMENT, "bytes is NULL");
    if (n < 0 || n > sense::kKvMaxEntries || keep_ld < 1 || keep_ld > 4096)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "n = %d outside [0, %d] or keep_ld = %d outside "
                    "[1, 4096]", n, sense::kKvMaxEntries, keep_ld);
    *bytes = n == 0 ? 0 : sense::kv_compact_workspace_bytes(n, keep_ld);
    return ok();
}

SENSE_EXPORT sense_status_t sense_kv_compact(const sense_kv_cache_t* cache, const int32_t* seqs,
                                             const int32_t* tails, const int32_t* keep,
                                             const int32_t* keep_len, const int32_t* pick,
                                             int32_t keep_rows, int32_t keep_ld, int32_t n,
                                             int32_t* out_status, void* workspace,
                                             size_t workspace_bytes, void* stream) {
    KvCache c;
    sense_status_t s = check_cache(cache, &c);
    if (s != SENSE_OK || (s = check_entries(c, seqs, n)) != SENSE_OK) return s;
    if (keep_ld < 1 || keep_ld > 4096)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "keep_ld = %d outside [1, 4096]", keep_ld);
    if (keep_rows < 1 || (keep_rows > 1 && !pick))
        return fail(SENSE_ERR_INVALID_ARGUMENT, "keep_rows = %d without pick", keep_rows);
    if (n == 0) return ok();
    if (!tails || !keep || !keep_len)
        return fail(SENSE_ERR_INVALID_ARGUMENT, "tails, keep and keep_len must be non-NULL");
    if ((s = check_ints("seqs, tails, keep, keep_len, pick and out_status",
                        {seqs, tails, keep, keep_len, pick, out_status})) != SENSE_OK)
        return s;
    if ((int64_t)n * (1 + (int64_t)c.n_layers * 2 * c.heads) / 4 > kMaxBlocks)
        return fail(SENSE_ERR_UNSUPPORTED, "%d entries of %d layers: too many for one call", n,
                    c.n_layers);
    if ((s = check_workspace(workspace, workspace_bytes,
                             sense::kv_compact_workspace_bytes(n, keep_ld))) != SENSE_OK)
        return s;
    const sense::KvKeep k = {tails, keep, keep_len, pick, keep_rows, keep_ld};
    return launched(sense::launch_kv_compact(c, seqs, k, n, out_status, workspace,
                                             (hipStream_t)stream),
                    "cache compact");
}
