// Entry points of the attention-block operators: argument validation, then enqueue on the partition's
// stream.  A call that fails validation enqueues nothing.
#include <algorithm>
#include <cmath>

#include "block_ops.h"

namespace sgprs {

constexpr long long kMaxStride = 1 << 20;  // elements between rows: a tile's rows are addressed with 32-bit byte offsets

// Fills in the dense value; the row must hold `width` elements.
static int fill_stride(const char* name, long long* ld, long long width)
{
    if (*ld == 0) *ld = width;
    if (*ld < width) return fail(SGPRS_ERR_INVALID_ARG, "%s %lld is less than the %lld elements of a row", name, *ld, width);
    if (*ld > kMaxStride) return fail(SGPRS_ERR_UNSUPPORTED, "%s %lld: supported are strides up to 2^20 elements", name, *ld);
    return SGPRS_OK;
}

static int check_kind(int dtype, int act)
{
    if (!dtype_ok(dtype)) return fail(SGPRS_ERR_UNSUPPORTED, "dtype %d", dtype);
    if (act < SGPRS_ACT_NONE || act > SGPRS_ACT_SILU) return fail(SGPRS_ERR_UNSUPPORTED, "activation %d", act);
    return SGPRS_OK;
}

int check_linear(const sgprs_linear_desc_t* d, sgprs_linear_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, d->act);
    if (rc) return rc;
    if (d->m < 0 || d->n <= 0 || d->k <= 0) return fail(SGPRS_ERR_INVALID_ARG, "m %d, n %d, k %d: need m >= 0, n > 0, k > 0", d->m, d->n, d->k);
    if (d->residual_first != 0 && d->residual_first != 1) return fail(SGPRS_ERR_INVALID_ARG, "residual_first %d is neither 0 nor 1", d->residual_first);
    *full = *d;
    if ((rc = fill_stride("ldx", &full->ldx, d->k)) || (rc = fill_stride("ldw", &full->ldw, d->k)) || (rc = fill_stride("ldr", &full->ldr, d->n)) ||
        (rc = fill_stride("ldy", &full->ldy, d->n)))
        return rc;
    return SGPRS_OK;
}

int check_group_norm(const sgprs_group_norm_desc_t* d, sgprs_group_norm_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, d->act);
    if (rc) return rc;
    if (d->n < 0 || d->hw <= 0 || d->c <= 0 || d->groups <= 0)
        return fail(SGPRS_ERR_INVALID_ARG, "n %d, hw %d, c %d, groups %d: need n >= 0 and the others > 0", d->n, d->hw, d->c, d->groups);
    if (d->c % d->groups) return fail(SGPRS_ERR_INVALID_ARG, "%d channels do not form %d equal groups", d->c, d->groups);
    if ((long long)(d->c / d->groups) * (long long)dtype_size(d->dtype) > 16384)
        return fail(SGPRS_ERR_UNSUPPORTED, "groups of %d channels: supported are up to 16 KiB of a position", d->c / d->groups);
    if (!(d->eps >= 0.f) || d->eps > 3e38f) return fail(SGPRS_ERR_INVALID_ARG, "eps %g is not a finite number >= 0", (double)d->eps);
    *full = *d;
    if ((rc = fill_stride("ldx", &full->ldx, d->c)) || (rc = fill_stride("ldr", &full->ldr, d->c)) || (rc = fill_stride("ldy", &full->ldy, d->c)))
        return rc;
    return SGPRS_OK;
}

int check_attention(const sgprs_attention_desc_t* d, sgprs_attention_desc_t* full)
{
    if (!d) return fail(SGPRS_ERR_INVALID_ARG, "descriptor is NULL");
    int rc = check_kind(d->dtype, SGPRS_ACT_NONE);
    if (rc) return rc;
    if (d->n_seqs <= 0 || d->total_q < 0 || d->total_kv < 0 || d->heads <= 0 || d->kv_heads <= 0 || d->head_dim <= 0)
        return fail(SGPRS_ERR_INVALID_ARG, "non-positive number of sequences, heads or head channels, or negative number of tokens");
    if (d->max_q < 0 || d->max_q > d->total_q || d->max_kv < 0 || d->max_kv > d->total_kv || (d->total_q > 0 && d->max_q == 0) ||
        (d->total_kv > 0 && d->max_kv == 0))
        return fail(SGPRS_ERR_INVALID_ARG, "longest sequences %d, %d do not fit %d and %d tokens", d->max_q, d->max_kv, d->total_q, d->total_kv);
    if (d->heads % d->kv_heads) return fail(SGPRS_ERR_INVALID_ARG, "%d heads are no multiple of %d key heads", d->heads, d->kv_heads);
    if (d->head_dim % 8 || d->head_dim > 128) return fail(SGPRS_ERR_UNSUPPORTED, "head_dim %d: supported are multiples of 8 up to 128", d->head_dim);
    if (d->n_seqs > (1 << 20) || d->heads > 65535 || d->total_q > (1 << 30) || d->total_kv > (1 << 30))
        return fail(SGPRS_ERR_UNSUPPORTED, "more than 2^20 sequences, 65535 heads or 2^30 tokens");
    if (d->causal != 0 && d->causal != 1) return fail(SGPRS_ERR_INVALID_ARG, "causal %d is neither 0 nor 1", d->causal);
    if (!(d->scale > -3e38f && d->scale < 3e38f)) return fail(SGPRS_ERR_INVALID_ARG, "scale is not finite");
    if (d->scale < -2e38f || d->scale > 2e38f) return fail(SGPRS_ERR_UNSUPPORTED, "scale %g: supported is up to 2e38 of either sign", (double)d->scale);  // times log2 e
    *full = *d;
    if (d->scale == 0.f) full->scale = 1.f / sqrtf((float)d->head_dim);
    const int vec = 16 / (int)dtype_size(d->dtype);
    struct { const char* name; long long *ld, *head; int heads; } s[4] = {{"q", &full->ldq, &full->hq, d->heads},
                                                                            {"k", &full->ldk, &full->hk, d->kv_heads},
                                                                            {"v", &full->ldv, &full->hv, d->kv_heads},
                                                                            {"o", &full->ldo, &full->ho, d->heads}};
    for (auto& t : s) {
        if (*t.head == 0) *t.head = d->head_dim;
        if (*t.ld == 0) *t.ld = (long long)t.heads * d->head_dim;
        if (*t.ld < d->head_dim || *t.head < d->head_dim)
            return fail(SGPRS_ERR_INVALID_ARG, "strides %lld and %lld of %s: less than head_dim", *t.ld, *t.head, t.name);
        if (*t.ld % vec || *t.head % vec) return fail(SGPRS_ERR_UNSUPPORTED, "strides %lld and %lld of %s: supported are multiples of 16 bytes", *t.ld, *t.head, t.name);
        if (*t.ld > kMaxStride || *t.head > (1ll << 50)) return fail(SGPRS_ERR_UNSUPPORTED, "strides %lld and %lld of %s are too large", *t.ld, *t.head, t.name);
    }
    return SGPRS_OK;
}

static bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

static int check_cus(int cus, const size_t* bytes)
{
    if (cus <= 0 || cus > SGPRS_MAX_MASK_WORDS * 32 || !bytes) return fail(SGPRS_ERR_INVALID_ARG, "partition of %d CUs, or NULL result pointer", cus);
    return SGPRS_OK;
}

static int check_workspace(const void* ws, size_t have, size_t need)
{
    if (need && (!ws || have < need || !aligned(ws, 16)))
        return fail(SGPRS_ERR_INVALID_ARG, "workspace of %zu bytes: %zu are needed, 16-byte aligned", ws ? have : (size_t)0, need);
    return SGPRS_OK;
}

}  // namespace sgprs

using namespace sgprs;

extern "C" {

int sgprs_linear_workspace(const sgprs_linear_desc_t* d, int partition_cus, size_t* bytes)
{
    sgprs_linear_desc_t f;
    int rc = check_linear(d, &f);
    if (rc || (rc = check_cus(partition_cus, bytes))) return rc;
    *bytes = std::max(linear_workspace_bytes(f, partition_cus), linear_workspace_bytes(f, planning_cus(partition_cus)));
    return SGPRS_OK;
}

int sgprs_linear(const sgprs_linear_desc_t* d, const void* x, const void* w, const float* bias, const void* residual, void* y, void* workspace,
                 size_t workspace_bytes, sgprs_pool_t* pool, int partition)
{
    sgprs_linear_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_linear(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.m == 0) return SGPRS_OK;
    if (!x || !w || !y) return fail(SGPRS_ERR_INVALID_ARG, "NULL tensor pointer");
    const size_t es = dtype_size(f.dtype);
    if (!aligned(x, es) || !aligned(w, es) || !aligned(residual, es) || !aligned(y, es) || !aligned(bias, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be aligned to their elements");
    if (x == y || w == y) return fail(SGPRS_ERR_INVALID_ARG, "y must not alias x or w");
    if (residual == y && f.ldr != f.ldy) return fail(SGPRS_ERR_INVALID_ARG, "y on top of the residual needs the residual's stride");
    if ((rc = check_workspace(workspace, workspace_bytes, linear_workspace_bytes(f, cus)))) return rc;
    return launch_linear(f, x, w, bias, residual, y, stream, cus);
}

int sgprs_group_norm_workspace(const sgprs_group_norm_desc_t* d, int partition_cus, size_t* bytes)
{
    sgprs_group_norm_desc_t f;
    int rc = check_group_norm(d, &f);
    if (rc || (rc = check_cus(partition_cus, bytes))) return rc;
    *bytes = std::max(group_norm_workspace_bytes(f, partition_cus), group_norm_workspace_bytes(f, planning_cus(partition_cus)));
    return SGPRS_OK;
}

int sgprs_group_norm(const sgprs_group_norm_desc_t* d, const void* x, const float* gamma, const float* beta, const void* residual, void* y,
                     void* workspace, size_t workspace_bytes, sgprs_pool_t* pool, int partition)
{
    sgprs_group_norm_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_group_norm(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.n == 0) return SGPRS_OK;
    if (!x || !y) return fail(SGPRS_ERR_INVALID_ARG, "NULL tensor pointer");
    const size_t es = dtype_size(f.dtype);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(y, es) || !aligned(gamma, 4) || !aligned(beta, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be aligned to their elements");
    if ((x == y && f.ldx != f.ldy) || (residual == y && f.ldr != f.ldy))
        return fail(SGPRS_ERR_INVALID_ARG, "y on top of x or the residual needs the same stride");
    if ((rc = check_workspace(workspace, workspace_bytes, group_norm_workspace_bytes(f, cus)))) return rc;
    return launch_group_norm(f, x, gamma, beta, residual, y, workspace, stream, cus);
}

int sgprs_attention_workspace(const sgprs_attention_desc_t* d, int partition_cus, size_t* bytes)
{
    sgprs_attention_desc_t f;
    int rc = check_attention(d, &f);
    if (rc || (rc = check_cus(partition_cus, bytes))) return rc;
    *bytes = std::max(attention_workspace_bytes(f, partition_cus), attention_workspace_bytes(f, planning_cus(partition_cus)));
    return SGPRS_OK;
}

int sgprs_attention(const sgprs_attention_desc_t* d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                    void* o, void* workspace, size_t workspace_bytes, sgprs_pool_t* pool, int partition)
{
    sgprs_attention_desc_t f;
    hipStream_t stream;
    int cus = 0, rc = check_attention(d, &f);
    if (rc || (rc = resolve_launch(pool, partition, &stream, &cus))) return rc;
    if (f.total_q == 0) return SGPRS_OK;
    if (!q || !o || !q_offsets || !kv_offsets || (f.total_kv > 0 && (!k || !v))) return fail(SGPRS_ERR_INVALID_ARG, "NULL pointer");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(q_offsets, 4) || !aligned(kv_offsets, 4))
        return fail(SGPRS_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned, offsets 4-byte");
    if (o == q || o == k || o == v) return fail(SGPRS_ERR_INVALID_ARG, "o must not alias q, k or v");
    if ((rc = check_workspace(workspace, workspace_bytes, attention_workspace_bytes(f, cus)))) return rc;
    return launch_attention(f, q, k, v, q_offsets, kv_offsets, o, workspace, stream, cus);
}

}  // extern "C"
