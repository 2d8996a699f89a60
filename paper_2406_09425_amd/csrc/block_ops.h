// Internal declarations of the attention-block operators: linear product, group norm, attention.
#pragma once

#include "internal.h"

namespace sgprs {

// Descriptors with the dense strides filled in and everything checked.
int check_linear(const sgprs_linear_desc_t* d, sgprs_linear_desc_t* full);
int check_group_norm(const sgprs_group_norm_desc_t* d, sgprs_group_norm_desc_t* full);
int check_attention(const sgprs_attention_desc_t* d, sgprs_attention_desc_t* full);

// of a partition planned for `cus` CUs
size_t linear_workspace_bytes(const sgprs_linear_desc_t& d, int cus);
size_t group_norm_workspace_bytes(const sgprs_group_norm_desc_t& d, int cus);
size_t attention_workspace_bytes(const sgprs_attention_desc_t& d, int cus);

int launch_linear(const sgprs_linear_desc_t& d, const void* x, const void* w, const float* bias, const void* residual, void* y, void* ws,
                  hipStream_t stream, int cus);
int launch_group_norm(const sgprs_group_norm_desc_t& d, const void* x, const float* gamma, const float* beta, const void* residual, void* y,
                      void* ws, hipStream_t stream, int cus);
int launch_attention(const sgprs_attention_desc_t& d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                     void* o, void* ws, hipStream_t stream, int cus);

// ---- device side ------------------------------------------------------------
// A tensor's element type by its dtype.
template <int DT> struct ElemOf { typedef float type; };
template <> struct ElemOf<SGPRS_BF16> { typedef __bf16 type; };

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == SGPRS_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == SGPRS_ACT_SILU) return z / (1.f + __expf(-z));
    if constexpr (ACT == SGPRS_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    return z;
}

}  // namespace sgprs
