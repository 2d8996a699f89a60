// Attention over packed sequences.
//
// One wavefront per query and head: keys are taken one after another with a running maximum m and sum l,
// o <- o exp(m - m') + exp(s - m') v; two of the (up to 128) channels per lane.
#include "block_ops.h"

namespace sgprs {

struct AttentionArgs {
    const void *q, *k, *v;
    void* o;
    const int *q_offsets, *kv_offsets;
    int n_seqs, total_q, total_kv, heads, group, head_dim, causal;
    float scale;
    long long ldq, ldk, ldv, ldo, hq, hk, hv, ho;
};

template <int DT> __global__ __launch_bounds__(256) void attention_kernel(const AttentionArgs a)
{
    typedef typename ElemOf<DT>::type T;
    const int lane = threadIdx.x & 63, head = blockIdx.y;
    const int token = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= a.total_q) return;
    int lo = 0, hi = a.n_seqs;  // the sequence: the last whose first token is not behind this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_offsets[mid] <= token) lo = mid;
        else hi = mid;
    }
    const int nq = a.q_offsets[lo + 1] - a.q_offsets[lo], i = token - a.q_offsets[lo];
    const int k0 = min(max(a.kv_offsets[lo], 0), a.total_kv), nk = min(max(a.kv_offsets[lo + 1], k0), a.total_kv) - k0;
    const int seen = a.causal ? min(nk, i + nk - nq + 1) : nk;
    const T* q = (const T*)a.q + token * a.ldq + head * a.hq;
    const T* k = (const T*)a.k + k0 * a.ldk + head / a.group * a.hk;
    const T* v = (const T*)a.v + k0 * a.ldv + head / a.group * a.hv;
    const int c = 2 * lane;
    const bool live = c < a.head_dim;
    const float q0 = live ? (float)q[c] : 0.f, q1 = live ? (float)q[c + 1] : 0.f;
    float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j = 0; j < seen; ++j) {
        float s = live ? q0 * (float)k[j * a.ldk + c] + q1 * (float)k[j * a.ldk + c + 1] : 0.f;
#pragma unroll
        for (int x = 32; x; x >>= 1) s += __shfl_xor(s, x);
        s *= a.scale;
        const float now = fmaxf(top, s), keep = top == now ? 1.f : __expf(top - now), p = __expf(s - now);
        sum = sum * keep + p;
        if (live) {
            o0 = o0 * keep + p * (float)v[j * a.ldv + c];
            o1 = o1 * keep + p * (float)v[j * a.ldv + c + 1];
        }
        top = now;
    }
    const float inv = sum > 0.f ? 1.f / sum : seen > 0 ? NAN : 0.f;
    if (live) {
        T* o = (T*)a.o + token * a.ldo + head * a.ho;
        o[c] = (T)(o0 * inv);
        o[c + 1] = (T)(o1 * inv);
    }
}

size_t attention_workspace_bytes(const sgprs_attention_desc_t&, int) { return 0; }

int launch_attention(const sgprs_attention_desc_t& d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                     void* o, void* ws, hipStream_t stream, int cus)
{
    const AttentionArgs a = {q, k, v, o, q_offsets, kv_offsets, d.n_seqs, d.total_q, d.total_kv, d.heads, d.heads / d.kv_heads, d.head_dim, d.causal,
                             d.scale, d.ldq, d.ldk, d.ldv, d.ldo, d.hq, d.hk, d.hv, d.ho};
    const dim3 grid((d.total_q + 3) / 4, d.heads);
    if (d.dtype == SGPRS_BF16) SGPRS_LAUNCH(attention_kernel<SGPRS_BF16>, grid, 256, 0, stream, a);
    else SGPRS_LAUNCH(attention_kernel<SGPRS_F32>, grid, 256, 0, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

}  // namespace sgprs
