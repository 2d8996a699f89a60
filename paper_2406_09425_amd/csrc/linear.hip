// y = act(x w^T + bias) + residual.
//
// 64 x 64 outputs per workgroup, operand tiles of 16 inputs through the LDS in fp32, 4 x 4 outputs per thread.
#include "block_ops.h"

namespace sgprs {

struct LinearArgs {
    const void* x;
    const void* w;
    const float* bias;
    const void* residual;
    void* y;
    int m, n, k;
    long long ldx, ldw, ldr, ldy;
    int residual_first;
};

template <int DT, int ACT> __global__ __launch_bounds__(256) void linear_kernel(const LinearArgs a)
{
    typedef typename ElemOf<DT>::type T;
    __shared__ float xs[16][65], ws[16][65];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const long long m0 = (long long)blockIdx.y * 64;
    const int n0 = blockIdx.x * 64;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < a.k; k0 += 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = ty + 16 * i, k = k0 + tx;
            xs[tx][row] = m0 + row < a.m && k < a.k ? (float)((const T*)a.x)[(m0 + row) * a.ldx + k] : 0.f;
            ws[tx][row] = n0 + row < a.n && k < a.k ? (float)((const T*)a.w)[(n0 + row) * a.ldw + k] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_fmaf(xs[k][ty * 4 + i], ws[k][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long row = m0 + ty * 4 + i;
            const int col = n0 + tx * 4 + j;
            if (row >= a.m || col >= a.n) continue;
            float z = acc[i][j] + (a.bias ? a.bias[col] : 0.f);
            const float r = a.residual ? (float)((const T*)a.residual)[row * a.ldr + col] : 0.f;
            z = a.residual_first ? activate<ACT>(z + r) : activate<ACT>(z) + r;
            ((T*)a.y)[row * a.ldy + col] = (T)z;
        }
}

size_t linear_workspace_bytes(const sgprs_linear_desc_t&, int) { return 0; }

template <int DT> static int launch_linear_typed(const LinearArgs& a, int act, hipStream_t stream)
{
    const dim3 grid((a.n + 63) / 64, (a.m + 63) / 64);
    switch (act) {
    case SGPRS_ACT_RELU: SGPRS_LAUNCH((linear_kernel<DT, SGPRS_ACT_RELU>), grid, 256, 0, stream, a); break;
    case SGPRS_ACT_GELU: SGPRS_LAUNCH((linear_kernel<DT, SGPRS_ACT_GELU>), grid, 256, 0, stream, a); break;
    case SGPRS_ACT_SILU: SGPRS_LAUNCH((linear_kernel<DT, SGPRS_ACT_SILU>), grid, 256, 0, stream, a); break;
    default: SGPRS_LAUNCH((linear_kernel<DT, SGPRS_ACT_NONE>), grid, 256, 0, stream, a);
    }
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

int launch_linear(const sgprs_linear_desc_t& d, const void* x, const void* w, const float* bias, const void* residual, void* y, void* ws,
                  hipStream_t stream, int cus)
{
    const LinearArgs a = {x, w, bias, residual, y, d.m, d.n, d.k, d.ldx, d.ldw, d.ldr, d.ldy, d.residual_first};
    if ((d.m + 63) / 64 > 65535) return fail(SGPRS_ERR_UNSUPPORTED, "%d rows", d.m);
    return d.dtype == SGPRS_BF16 ? launch_linear_typed<SGPRS_BF16>(a, d.act, stream) : launch_linear_typed<SGPRS_F32>(a, d.act, stream);
}

}  // namespace sgprs
