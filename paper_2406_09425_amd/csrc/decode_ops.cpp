// Entry points of the decoding step's operators: argument validation, then enqueue on the partition's stream.  A call
// that fails validation enqueues nothing.
#include <algorithm>
#include <cmath>

#include "decode_ops.h"

namespace sgprs {

int check_rms_norm(const sgprs_rms_norm_desc_t* d, sgprs_rms_norm_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, SGPRS_ACT_NONE);
    if (rc) return rc;
    if (d->out_dtype != d->dtype && d->out_dtype != SGPRS_I8)
        return fail(SGPRS_ERR_UNSUPPORTED, "out_dtype %d: supported are the dtype, %d, and SGPRS_I8", d->out_dtype, d->dtype);
    if (d->m < 0 || d->c <= 0) return fail(SGPRS_ERR_INVALID_ARG, "m %d, c %d: need m >= 0, c > 0", d->m, d->c);
    if (!(d->eps >= 0.f) || d->eps > 3e38f) return fail(SGPRS_ERR_INVALID_ARG, "eps %g is not a finite number >= 0", (double)d->eps);
    *full = *d;
    if ((rc = fill_stride("ldx", &full->ldx, d->c)) || (rc = fill_stride("ldr", &full->ldr, d->c)) || (rc = fill_stride("ldh", &full->ldh, d->c)) ||
        (rc = fill_stride("ldy", &full->ldy, d->c)))
        return rc;
    return SGPRS_OK;
}

int check_quantize(const sgprs_quantize_desc_t* d, sgprs_quantize_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, SGPRS_ACT_NONE);
    if (rc) return rc;
    if (d->m < 0 || d->c <= 0) return fail(SGPRS_ERR_INVALID_ARG, "m %d, c %d: need m >= 0, c > 0", d->m, d->c);
    *full = *d;
    if ((rc = fill_stride("ldx", &full->ldx, d->c)) || (rc = fill_stride("ldy", &full->ldy, d->c))) return rc;
    return SGPRS_OK;
}

int check_linear_i8(const sgprs_linear_i8_desc_t* d, sgprs_linear_i8_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, d->act);
    if (rc) return rc;
    if (d->m < 0 || d->n <= 0 || d->k <= 0) return fail(SGPRS_ERR_INVALID_ARG, "m %d, n %d, k %d: need m >= 0, n > 0, k > 0", d->m, d->n, d->k);
    if (d->k > 131071) return fail(SGPRS_ERR_UNSUPPORTED, "k %d: sums of more than 131071 products could pass 32 bits", d->k);
    if (d->residual_first != 0 && d->residual_first != 1) return fail(SGPRS_ERR_INVALID_ARG, "residual_first %d is neither 0 nor 1", d->residual_first);
    *full = *d;
    if ((rc = fill_stride("ldx", &full->ldx, d->k)) || (rc = fill_stride("ldw", &full->ldw, d->k)) || (rc = fill_stride("ldr", &full->ldr, d->n)) ||
        (rc = fill_stride("ldy", &full->ldy, d->n)))
        return rc;
    return SGPRS_OK;
}

// One operand's strides between tokens and heads.
static int fill_heads(const char* name, long long* ld, long long* head, int heads, int head_dim, int dtype)
{
    const int vec = 16 / (int)dtype_size(dtype);
    if (*head == 0) *head = head_dim;
    if (*ld == 0) *ld = (long long)heads * head_dim;
    if (*ld < head_dim || *head < head_dim) return fail(SGPRS_ERR_INVALID_ARG, "strides %lld and %lld of %s: less than head_dim", *ld, *head, name);
    if (*ld % vec || *head % vec) return fail(SGPRS_ERR_UNSUPPORTED, "strides %lld and %lld of %s: supported are multiples of 16 bytes", *ld, *head, name);
    if (*ld > kMaxStride || *head > (1ll << 50)) return fail(SGPRS_ERR_UNSUPPORTED, "strides %lld and %lld of %s are too large", *ld, *head, name);
    return SGPRS_OK;
}

// What both operators say of a cache.  (D: a descriptor with these fields)
template <class D> static int check_cache(const D& d, D* full)
{
    if (d.n_seqs <= 0 || d.kv_heads <= 0 || d.head_dim <= 0 || d.n_pages <= 0 || d.page_size <= 0 || d.table_width <= 0)
        return fail(SGPRS_ERR_INVALID_ARG, "non-positive number of sequences, key heads, head channels, pages, positions of a page or table entries");
    if (d.head_dim % 8 || d.head_dim > 128) return fail(SGPRS_ERR_UNSUPPORTED, "head_dim %d: supported are multiples of 8 up to 128", d.head_dim);
    if (d.n_seqs > (1 << 20) || d.kv_heads > 65535) return fail(SGPRS_ERR_UNSUPPORTED, "more than 2^20 sequences or 65535 heads");
    if ((long long)d.table_width * d.page_size > (1 << 30))
        return fail(SGPRS_ERR_UNSUPPORTED, "%d pages of %d: sequences of more than 2^30 positions", d.table_width, d.page_size);
    const int vec = 16 / (int)dtype_size(d.dtype);
    if (full->head_stride == 0) full->head_stride = d.head_dim;
    if (full->token_stride == 0) full->token_stride = (long long)d.kv_heads * d.head_dim;
    if (full->page_stride == 0) full->page_stride = (long long)d.page_size * d.kv_heads * d.head_dim;
    struct { long long stride; int count; } dims[3] = {{full->head_stride, d.kv_heads}, {full->token_stride, d.page_size}, {full->page_stride, d.n_pages}};
    for (auto& s : dims) {
        if (s.stride < d.head_dim) return fail(SGPRS_ERR_INVALID_ARG, "a stride of the cache is %lld: less than head_dim", s.stride);
        if (s.stride % vec) return fail(SGPRS_ERR_UNSUPPORTED, "a stride of the cache is %lld: supported are multiples of 16 bytes", s.stride);
        if ((double)s.stride * s.count > 0x1p50) return fail(SGPRS_ERR_UNSUPPORTED, "a stride of the cache, %lld, is too large", s.stride);
    }
    // the places of two (page, position, head) do not overlap: each stride steps over all that the shorter ones reach
    std::sort(dims, dims + 3, [](auto& a, auto& b) { return a.stride < b.stride; });
    long long reach = d.head_dim;
    for (auto& s : dims) {
        if (s.count == 1) continue;
        if (s.stride < reach) return fail(SGPRS_ERR_INVALID_ARG, "the cache's strides %lld, %lld, %lld let places overlap", full->page_stride, full->token_stride, full->head_stride);
        reach += s.stride * (s.count - 1);
    }
    return SGPRS_OK;
}

int check_paged_append(const sgprs_paged_append_desc_t* d, sgprs_paged_append_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, SGPRS_ACT_NONE);
    if (rc) return rc;
    *full = *d;
    if ((rc = check_cache(*d, full))) return rc;
    if (d->total < 0) return fail(SGPRS_ERR_INVALID_ARG, "total %d: need >= 0", d->total);
    if (d->total > (1 << 30)) return fail(SGPRS_ERR_UNSUPPORTED, "more than 2^30 tokens");
    if ((rc = fill_heads("k", &full->ldk, &full->hk, d->kv_heads, d->head_dim, d->dtype)) || (rc = fill_heads("v", &full->ldv, &full->hv, d->kv_heads, d->head_dim, d->dtype)))
        return rc;
    return SGPRS_OK;
}

int check_paged_attention(const sgprs_paged_attention_desc_t* d, sgprs_paged_attention_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, SGPRS_ACT_NONE);
    if (rc) return rc;
    *full = *d;
    if ((rc = check_cache(*d, full))) return rc;
    if (d->heads <= 0 || d->heads % d->kv_heads) return fail(SGPRS_ERR_INVALID_ARG, "%d heads are no positive multiple of %d key heads", d->heads, d->kv_heads);
    if (d->heads > 65535) return fail(SGPRS_ERR_UNSUPPORTED, "more than 65535 heads");
    if ((long long)d->n_seqs * d->kv_heads * ((d->heads / d->kv_heads + 31) / 32) > (1 << 28))
        return fail(SGPRS_ERR_UNSUPPORTED, "%d sequences of %d key heads: supported are up to 2^28 of both, and of 32 heads each", d->n_seqs, d->kv_heads);
    if (d->window < 0 || d->sinks < 0 || (d->sinks > 0 && d->window == 0))
        return fail(SGPRS_ERR_INVALID_ARG, "window %d, sinks %d: need both >= 0, and a window where there are sinks", d->window, d->sinks);
    if (!(d->scale > -3e38f && d->scale < 3e38f)) return fail(SGPRS_ERR_INVALID_ARG, "scale is not finite");
    if (d->scale < -2e38f || d->scale > 2e38f) return fail(SGPRS_ERR_UNSUPPORTED, "scale %g: supported is up to 2e38 of either sign", (double)d->scale);  // times log2 e
    if (d->scale == 0.f) full->scale = 1.f / sqrtf((float)d->head_dim);
    if ((rc = fill_heads("q", &full->ldq, &full->hq, d->heads, d->head_dim, d->dtype)) || (rc = fill_heads("o", &full->ldo, &full->ho, d->heads, d->head_dim, d->dtype)))
        return rc;
    return SGPRS_OK;
}

}  // namespace sgprs

using namespace sgprs;

extern "C" {

int sgprs_rms_norm(const sgprs_rms_norm_desc_t* d, const void* x, const void* residual, const float* gamma, void* sum, void* y, float* scales,
                   sgprs_pool_t* pool, int partition)
{
    sgprs_rms_norm_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_rms_norm(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.m == 0) return SGPRS_OK;
    const bool i8 = f.out_dtype == SGPRS_I8;
    if (!x || !y || (i8 && !scales)) return fail(SGPRS_ERR_INVALID_ARG, "NULL tensor pointer");
    if (!i8 && scales) return fail(SGPRS_ERR_INVALID_ARG, "scales go with 8-bit rows");
    if (sum && !residual) return fail(SGPRS_ERR_INVALID_ARG, "a sum without a residual");
    const size_t es = dtype_size(f.dtype);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(sum, es) || (!i8 && !aligned(y, es)) || !aligned(gamma, 4) || !aligned(scales, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be aligned to their elements");
    if (y == sum || (i8 && (y == x || y == residual))) return fail(SGPRS_ERR_INVALID_ARG, "y must not alias the sum, 8-bit rows nothing");
    if ((sum == x && f.ldh != f.ldx) || (sum && sum == residual && f.ldh != f.ldr) || (y == x && f.ldy != f.ldx) || (y == residual && f.ldy != f.ldr))
        return fail(SGPRS_ERR_INVALID_ARG, "a result on top of x or the residual needs the same stride");
    return launch_rms_norm(f, x, residual, gamma, sum, y, scales, stream, cus);
}

int sgprs_quantize_i8(const sgprs_quantize_desc_t* d, const void* x, int8_t* y, float* scales, sgprs_pool_t* pool, int partition)
{
    sgprs_quantize_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_quantize(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.m == 0) return SGPRS_OK;
    if (!x || !y || !scales) return fail(SGPRS_ERR_INVALID_ARG, "NULL tensor pointer");
    if (!aligned(x, dtype_size(f.dtype)) || !aligned(scales, 4)) return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be aligned to their elements");
    if (x == (const void*)y) return fail(SGPRS_ERR_INVALID_ARG, "y must not alias x");
    return launch_quantize(f, x, y, scales, stream, cus);
}

int sgprs_linear_i8_workspace(const sgprs_linear_i8_desc_t* d, int partition_cus, size_t* bytes)
{
    sgprs_linear_i8_desc_t f;
    int rc = check_linear_i8(d, &f);
    if (rc || (rc = check_cus(partition_cus, bytes))) return rc;
    *bytes = std::max(linear_i8_workspace_bytes(f, partition_cus), linear_i8_workspace_bytes(f, planning_cus(partition_cus)));
    return SGPRS_OK;
}

int sgprs_linear_i8(const sgprs_linear_i8_desc_t* d, const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales, const float* bias,
                    const void* residual, void* y, void* workspace, size_t workspace_bytes, sgprs_pool_t* pool, int partition)
{
    sgprs_linear_i8_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_linear_i8(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.m == 0) return SGPRS_OK;
    if (!x || !w || !y) return fail(SGPRS_ERR_INVALID_ARG, "NULL tensor pointer");
    const size_t es = dtype_size(f.dtype);
    if (!aligned(residual, es) || !aligned(y, es) || !aligned(bias, 4) || !aligned(x_scales, 4) || !aligned(w_scales, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be aligned to their elements");
    if (y == (const void*)x || y == (const void*)w) return fail(SGPRS_ERR_INVALID_ARG, "y must not alias x or w");
    if (residual == y && f.ldr != f.ldy) return fail(SGPRS_ERR_INVALID_ARG, "y on top of the residual needs the residual's stride");
    if ((rc = check_workspace(workspace, workspace_bytes, linear_i8_workspace_bytes(f, cus)))) return rc;
    return launch_linear_i8(f, x, x_scales, w, w_scales, bias, residual, y, workspace, stream, cus);
}

int sgprs_paged_append(const sgprs_paged_append_desc_t* d, const void* k, const void* v, const int* offsets, const int* table, const int* kv_lens,
                       void* k_cache, void* v_cache, sgprs_pool_t* pool, int partition)
{
    sgprs_paged_append_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_paged_append(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (!offsets && f.total != f.n_seqs)
        return fail(SGPRS_ERR_INVALID_ARG, "%d tokens of %d sequences: without offsets each sequence has one", f.total, f.n_seqs);
    if (f.total == 0) return SGPRS_OK;
    if (!k || !v || !table || !kv_lens || !k_cache || !v_cache) return fail(SGPRS_ERR_INVALID_ARG, "NULL pointer");
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(offsets, 4) || !aligned(table, 4) || !aligned(kv_lens, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned, tables and lengths 4-byte");
    if (k_cache == v_cache || k_cache == k || k_cache == v || v_cache == k || v_cache == v)
        return fail(SGPRS_ERR_INVALID_ARG, "the caches must not alias each other, k or v");
    return launch_paged_append(f, k, v, offsets, table, kv_lens, k_cache, v_cache, stream);
}

int sgprs_paged_attention_workspace(const sgprs_paged_attention_desc_t* d, int partition_cus, size_t* bytes)
{
    sgprs_paged_attention_desc_t f;
    int rc = check_paged_attention(d, &f);
    if (rc || (rc = check_cus(partition_cus, bytes))) return rc;
    *bytes = std::max(paged_attention_workspace_bytes(f, partition_cus), paged_attention_workspace_bytes(f, planning_cus(partition_cus)));
    return SGPRS_OK;
}

int sgprs_paged_attention(const sgprs_paged_attention_desc_t* d, const void* q, const void* k_cache, const void* v_cache, const int* table,
                          const int* kv_lens, void* o, void* workspace, size_t workspace_bytes, sgprs_pool_t* pool, int partition)
{
    sgprs_paged_attention_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_paged_attention(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (!q || !k_cache || !v_cache || !table || !kv_lens || !o) return fail(SGPRS_ERR_INVALID_ARG, "NULL pointer");
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(o, 16) || !aligned(table, 4) || !aligned(kv_lens, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned, tables and lengths 4-byte");
    if (o == q || o == k_cache || o == v_cache) return fail(SGPRS_ERR_INVALID_ARG, "o must not alias q or the caches");
    if ((rc = check_workspace(workspace, workspace_bytes, paged_attention_workspace_bytes(f, cus)))) return rc;
    return launch_paged_attention(f, q, k_cache, v_cache, table, kv_lens, o, workspace, stream, cus);
}

}  // extern "C"
