// Internal declarations of the decoding step's operators: norm and rows of 8-bit integers, 8-bit linear product,
// paged cache.
#pragma once

#include "block_ops.h"

namespace sgprs {

// Descriptors with the dense strides filled in and everything checked.
int check_rms_norm(const sgprs_rms_norm_desc_t* d, sgprs_rms_norm_desc_t* full);
int check_quantize(const sgprs_quantize_desc_t* d, sgprs_quantize_desc_t* full);
int check_linear_i8(const sgprs_linear_i8_desc_t* d, sgprs_linear_i8_desc_t* full);
int check_paged_append(const sgprs_paged_append_desc_t* d, sgprs_paged_append_desc_t* full);
int check_paged_attention(const sgprs_paged_attention_desc_t* d, sgprs_paged_attention_desc_t* full);

// Kernels of the 8-bit product, and the one that it is planned by on `cus` CUs.  direct: aligned rows of whole 16-byte chunks.
enum LinearI8Kernel { kTile256, kTile128, kTile64, kDeep128, kDeep64, kStaged128, kStaged64, kStaged32, kSplit16x16, kSplit32x16, kSplit64x16, kSplit32x32, kSplit64x32, kSplit32x64, kSplit64x64, kShort };
int plan_linear_i8(const sgprs_linear_i8_desc_t& d, int cus, bool direct, bool residual);

size_t linear_i8_workspace_bytes(const sgprs_linear_i8_desc_t& d, int cus);
size_t paged_attention_workspace_bytes(const sgprs_paged_attention_desc_t& d, int cus);

int launch_rms_norm(const sgprs_rms_norm_desc_t& d, const void* x, const void* residual, const float* gamma, void* sum, void* y, float* scales,
                    hipStream_t stream, int cus);
int launch_quantize(const sgprs_quantize_desc_t& d, const void* x, int8_t* y, float* scales, hipStream_t stream, int cus);
int launch_linear_i8(const sgprs_linear_i8_desc_t& d, const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales,
                     const float* bias, const void* residual, void* y, void* ws, hipStream_t stream, int cus);
int launch_paged_append(const sgprs_paged_append_desc_t& d, const void* k, const void* v, const int* offsets, const int* table,
                        const int* kv_lens, void* k_cache, void* v_cache, hipStream_t stream);
int launch_paged_attention(const sgprs_paged_attention_desc_t& d, const void* q, const void* k_cache, const void* v_cache, const int* table,
                           const int* kv_lens, void* o, void* ws, hipStream_t stream, int cus);

}  // namespace sgprs
