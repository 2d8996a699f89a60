// Group norm with an activation, channels last.
//
// One workgroup per image and group: mean, then the squares of the deviations, then the results.
#include "block_ops.h"

namespace sgprs {

struct NormArgs {
    const void* x;
    const float *gamma, *beta;
    const void* residual;
    void* y;
    int hw, c, groups;
    float eps;
    long long ldx, ldr, ldy;
};

__device__ __forceinline__ float block_sum(float v, float* parts)
{
#pragma unroll
    for (int s = 32; s; s >>= 1) v += __shfl_xor(v, s);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    return (parts[0] + parts[1]) + (parts[2] + parts[3]);
}

template <int DT, int ACT> __global__ __launch_bounds__(256) void group_norm_kernel(const NormArgs a)
{
    typedef typename ElemOf<DT>::type T;
    __shared__ float parts[4];
    const int per = a.c / a.groups;
    const long long first = (long long)blockIdx.y * a.hw, total = (long long)a.hw * per;
    const int c0 = blockIdx.x * per;
    auto x = [&](long long i) { return (float)((const T*)a.x)[(first + i / per) * a.ldx + c0 + i % per]; };
    float sum = 0.f;
    for (long long i = threadIdx.x; i < total; i += 256) sum += x(i);
    const float mean = block_sum(sum, parts) / (float)total;
    float sq = 0.f;
    for (long long i = threadIdx.x; i < total; i += 256) {
        const float t = x(i) - mean;
        sq += t * t;
    }
    const float inv = 1.f / sqrtf(block_sum(sq, parts) / (float)total + a.eps);
    for (long long i = threadIdx.x; i < total; i += 256) {
        const int c = c0 + (int)(i % per);
        const long long px = first + i / per;
        float z = (x(i) - mean) * inv;
        z = z * (a.gamma ? a.gamma[c] : 1.f) + (a.beta ? a.beta[c] : 0.f);
        if (a.residual) z += (float)((const T*)a.residual)[px * a.ldr + c];
        ((T*)a.y)[px * a.ldy + c] = (T)activate<ACT>(z);
    }
}

size_t group_norm_workspace_bytes(const sgprs_group_norm_desc_t&, int) { return 0; }

template <int DT> static int launch_norm_typed(const NormArgs& a, int n, int act, hipStream_t stream)
{
    const dim3 grid(a.groups, n);
    switch (act) {
    case SGPRS_ACT_RELU: SGPRS_LAUNCH((group_norm_kernel<DT, SGPRS_ACT_RELU>), grid, 256, 0, stream, a); break;
    case SGPRS_ACT_GELU: SGPRS_LAUNCH((group_norm_kernel<DT, SGPRS_ACT_GELU>), grid, 256, 0, stream, a); break;
    case SGPRS_ACT_SILU: SGPRS_LAUNCH((group_norm_kernel<DT, SGPRS_ACT_SILU>), grid, 256, 0, stream, a); break;
    default: SGPRS_LAUNCH((group_norm_kernel<DT, SGPRS_ACT_NONE>), grid, 256, 0, stream, a);
    }
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

int launch_group_norm(const sgprs_group_norm_desc_t& d, const void* x, const float* gamma, const float* beta, const void* residual, void* y,
                      void* ws, hipStream_t stream, int cus)
{
    if (d.n > 65535) return fail(SGPRS_ERR_UNSUPPORTED, "%d images", d.n);
    const NormArgs a = {x, gamma, beta, residual, y, d.hw, d.c, d.groups, d.eps, d.ldx, d.ldr, d.ldy};
    return d.dtype == SGPRS_BF16 ? launch_norm_typed<SGPRS_BF16>(a, d.n, d.act, stream) : launch_norm_typed<SGPRS_F32>(a, d.n, d.act, stream);
}

}  // namespace sgprs
