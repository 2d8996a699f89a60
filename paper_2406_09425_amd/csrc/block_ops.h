// Internal declarations of the attention-block operators: linear product, group norm, attention.
#pragma once

#include "internal.h"

namespace sgprs {

constexpr long long kMaxStride = 1 << 20;  // elements between rows: a tile's rows are addressed with 32-bit byte offsets

// Checks that the operators' entry points share; 0 or the error that the call returns.
int fill_stride(const char* name, long long* ld, long long width);
int check_kind(int dtype, int act);
int check_cus(int cus, const size_t* bytes);
int check_workspace(const void* ws, size_t have, size_t need);
inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Descriptors with the dense strides filled in and everything checked.
int check_linear(const sgprs_linear_desc_t* d, sgprs_linear_desc_t* full);
int check_group_norm(const sgprs_group_norm_desc_t* d, sgprs_group_norm_desc_t* full);
int check_attention(const sgprs_attention_desc_t* d, sgprs_attention_desc_t* full);

// of a partition planned for `cus` CUs
size_t linear_workspace_bytes(const sgprs_linear_desc_t& d, int cus);
size_t group_norm_workspace_bytes(const sgprs_group_norm_desc_t& d, int cus);
size_t attention_workspace_bytes(const sgprs_attention_desc_t& d, int cus);

int launch_linear(const sgprs_linear_desc_t& d, const void* x, const void* w, const float* bias, const void* residual, void* y,
                  hipStream_t stream, int cus);
int launch_group_norm(const sgprs_group_norm_desc_t& d, const void* x, const float* gamma, const float* beta, const void* residual, void* y,
                      void* ws, hipStream_t stream, int cus);
int launch_attention(const sgprs_attention_desc_t& d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                     void* o, void* ws, hipStream_t stream, int cus);

// ---- device side ------------------------------------------------------------
// GELU of a bf16 result takes erf from Abramowitz and Stegun 7.1.26 (off by at most 1.5e-7): with
// q(t) = 1 - erf(t / sqrt 2) at t = |z| it is max(z, 0) - |z| q / 2 (0 z for 0: a NaN for -infinity, like the formula).  The library's erff took 27 us of a 69 us
// product with 25.7 million outputs, this 2.  Far down the negative side, where bf16 results are below 1e-9, it is off by
// up to 1 %.  SiLU of a bf16 result takes the approximate exponential and reciprocal (1e-6 of the result, 0 below -87).
// fp32 results take neither: 1 + erf would cancel below z = -3 and leave no digit at -6, where erfc keeps them, and
// exp(-z) would overflow below -88.
template <int DT, int ACT> __device__ __forceinline__ float activate(float z)
{
#if __HIP_DEVICE_COMPILE__
    if constexpr (ACT == SGPRS_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == SGPRS_ACT_SILU) {
        if constexpr (DT == SGPRS_BF16) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
        const float e = expf(-fabsf(z));
        const float d = 1.f + e, r = __builtin_amdgcn_rcpf(d);  // d is in [1, 2]: one step takes 1 / d to an ulp
        return (z < 0.f ? z * e : z) * __builtin_fmaf(__builtin_fmaf(-d, r, 1.f), r, r);
    }
    if constexpr (ACT == SGPRS_ACT_GELU) {
        if constexpr (DT == SGPRS_BF16) {
            const float t = fminf(fabsf(z), 40.f), u = __builtin_amdgcn_rcpf(__builtin_fmaf(t, 0.3275911f * 0.70710678f, 1.f));
            float q = __builtin_fmaf(u, 1.061405429f, -1.453152027f);
            q = __builtin_fmaf(q, u, 1.421413741f);
            q = __builtin_fmaf(q, u, -0.284496736f);
            q = __builtin_fmaf(q, u, 0.254829592f) * u;
            return (z < 0.f ? 0.f * z : z) - 0.5f * t * q * __builtin_amdgcn_exp2f(t * t * -0.72134752f);
        }
        return 0.5f * z * erfcf(z * -0.70710678118654752f);
    }
#endif
    return z;
}

}  // namespace sgprs
