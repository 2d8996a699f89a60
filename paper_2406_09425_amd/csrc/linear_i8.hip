// y = act(x_scale w_scale sum(x w) + bias) + residual of 8-bit integers on the matrix cores.
//
// w's rows are the MFMA's row operand and x's rows its column operand, so that a lane ends up with four neighbouring
// outputs of one row.  Both operands are walked in k-tiles of 128 bytes a row: eight 16-byte chunks, chunk c of row r in LDS
// slot c ^ (r & 7), so that 16 rows of one chunk meet no bank twice; two 16x16x64 MFMAs a k-tile.  Sums are 32-bit integers
// and exact, so any split of k gives the same bits.
#include <algorithm>
#include <cmath>

#include "decode_ops.h"
#include "linear_tiles.h"

namespace sgprs {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

struct LinearI8Args {
    const unsigned char *x, *w;
    const float *x_scales, *w_scales, *bias;
    const unsigned char* residual;
    unsigned char* y;
    int m, n, k;
    int ldx, ldw, ldr, ldy;  // bytes
    int residual_first;
    int grid_m, grid_n;      // tiles
};

__device__ __forceinline__ i32x4_t mma(u32x4_t a, u32x4_t b, i32x4_t c)
{
#if __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, a), __builtin_bit_cast(i32x4_t, b), c, 0, 0, 0);
#else
    return c;
#endif
}

// What belongs to V neighbouring columns.
template <int V> struct Columns {
    float scale[V], bias[V];
    __device__ __forceinline__ Columns(const LinearI8Args& a, int col)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            scale[e] = a.w_scales && col + e < a.n ? a.w_scales[col + e] : 1.f;
            bias[e] = a.bias && col + e < a.n ? a.bias[col + e] : 0.f;
        }
    }
};
__device__ __forceinline__ float row_scale(const LinearI8Args& a, long long row) { return a.x_scales && row < a.m ? a.x_scales[row] : 1.f; }

// Eight (bf16) or four (fp32) neighbouring outputs of one row.  s: the sums, r: the residual as it lies in memory.
template <int DT, int ACT, int V> __device__ __forceinline__ u32x4_t finish(const LinearI8Args& a, const int* s, float x_scale, const Columns<V>& c, u32x4_t r)
{
    constexpr int ES = 16 / V;
    float o[V];
    auto res = [&](int e) { return ES == 4 ? __uint_as_float(r[e % 4]) : __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16); };
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (float)s[e] * x_scale * c.scale[e] + c.bias[e];
    if (a.residual && a.residual_first) {
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += res(e);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = activate<DT, ACT>(o[e]);
    if (a.residual && !a.residual_first) {
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] += res(e);
    }
    u32x4_t out;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if constexpr (ES == 4) out[p] = __float_as_uint(o[p]);
        else out[p] = pack_bf16x2_relu(o[2 * p], o[2 * p + 1], kNoReluFloor);
    }
    return out;
}

// The same for a row and columns that may lie outside, and rows at any alignment.
template <int DT, int ACT, int V> __device__ __forceinline__ void finish_row(const LinearI8Args& a, long long row, int col, const int* s, const Columns<V>& c)
{
    constexpr int ES = 16 / V;
    if (row >= a.m || col >= a.n) return;
    const unsigned char* rp = a.residual + row * a.ldr + (long long)col * ES;
    unsigned char* yp = a.y + row * a.ldy + (long long)col * ES;
    const int live = min(V, a.n - col);
    const u32x4_t out = finish<DT, ACT>(a, s, row_scale(a, row), c, a.residual ? load_chunk<ES>(rp, live * ES) : u32x4_t{0, 0, 0, 0});
    if (live == V) {
        __builtin_memcpy(yp, &out, 16);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (e >= live) continue;
            if constexpr (ES == 4) ((unsigned*)yp)[e] = out[e];
            else ((unsigned short*)yp)[e] = (unsigned short)(out[e / 2] >> (e % 2 * 16));
        }
    }
}

// A wavefront's 16 TM x 16 TN outputs, from row m0 and column n0 on: 16 rows at a time through LDS of its own (`mine`),
// then V neighbouring outputs a lane.
template <int DT, int TN> struct StagedRows {
    static constexpr int V = DT == SGPRS_BF16 ? 8 : 4, PITCH = TN * 16 + 4;  // values of a staged row
    static constexpr int BYTES = 16 * PITCH * 4;
};
template <int DT, int ACT, int TM, int TN>
__device__ __forceinline__ void store_tile(const LinearI8Args& a, const i32x4_t (&acc)[TN][TM], int* mine, long long m0, int n0)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int V = StagedRows<DT, TN>::V, PITCH = StagedRows<DT, TN>::PITCH;
    constexpr int LPR = TN * 16 / V, RPP = 64 / LPR, PASSES = 16 / RPP;  // lanes of a row, rows of a pass
    const int lane = threadIdx.x & 63, frow = lane & 15, fgrp = lane >> 4, r0 = lane / LPR, c0 = lane % LPR * V, col = n0 + c0;
    const Columns<V> columns(a, col);
    for_each<TM>([&](auto i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *(i32x4_t*)(mine + frow * PITCH + j * 16 + fgrp * 4) = acc[j][i];
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
#pragma unroll 1
        for (int p = 0; p < PASSES; ++p) {
            int s[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) *(i32x4_t*)(s + e) = *(const i32x4_t*)(mine + (p * RPP + r0) * PITCH + c0 + e);
            finish_row<DT, ACT>(a, m0 + i * 16 + p * RPP + r0, col, s, columns);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
    });
#endif
}

// BM x BN outputs, 2 x 2 wavefronts; the k-tile goes through registers to LDS.
template <int DT, int ACT, int BM, int BN> __global__ __launch_bounds__(256) void linear_i8_staged_kernel(const LinearI8Args a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int WM = 2, WN = 2, TM = BM / WM / 16, TN = BN / WN / 16, UNITS = (BM + BN) * 8 / 256;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0), tiles = (a.k + 127) >> 7;
    const unsigned char* xp = a.x + m0 * a.ldx;
    const unsigned char* wp = a.w + (long long)n0 * a.ldw;
    const int chunk = threadIdx.x & 7;
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned slot = (unsigned)((fgrp ^ (frow & 7)) << 4), x_frag = (unsigned)((wm * TM * 16 + frow) * 128) + slot,
                   w_frag = (unsigned)((BM + wn * TN * 16 + frow) * 128) + slot;
    i32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
    for (int t = 0; t < tiles; ++t) {
        u32x4_t unit[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int r = (i * 256 + (int)threadIdx.x) >> 3, at = t * 128 + chunk * 16;
            const bool of_x = r < BM, there = of_x ? r < rows_x : r - BM < rows_w;
            unit[i] = load_chunk<1>((of_x ? xp + (long long)r * a.ldx : wp + (long long)(r - BM) * a.ldw) + at, there ? a.k - at : 0);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int r = (i * 256 + (int)threadIdx.x) >> 3;
            *(u32x4_t*)(smem + r * 128 + ((chunk ^ (r & 7)) << 4)) = unit[i];
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4_t xf[TM], wf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[j] = lds_read((w_frag + j * 2048) ^ (h << 6));
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = lds_read((x_frag + i * 2048) ^ (h << 6));
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] = mma(wf[j], xf[i], acc[j][i]);
        }
    }
    __syncthreads();
    static_assert(4 * StagedRows<DT, TN>::BYTES <= (BM + BN) * 128, "staging fits");
    store_tile<DT, ACT, TM, TN>(a, acc, (int*)(smem + wave * StagedRows<DT, TN>::BYTES), m0 + wm * TM * 16, n0 + wn * TN * 16);
#endif
}

// ---- plans -------------------------------------------------------------------------------------
size_t linear_i8_workspace_bytes(const sgprs_linear_i8_desc_t&, int) { return 0; }

template <auto kernel> static int launch_sized(int lds, const LinearI8Args& a, int threads, hipStream_t stream)
{
    if ((long long)a.grid_m * a.grid_n * threads >= (1ll << 32)) return fail(SGPRS_ERR_UNSUPPORTED, "%d x %d outputs", a.m, a.n);
    SGPRS_LAUNCH(kernel, dim3((unsigned)((long long)a.grid_m * a.grid_n)), threads, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

static LinearI8Args tiled(LinearI8Args a, int bm, int bn)
{
    a.grid_m = (a.m - 1) / bm + 1;  // (m may be the largest int)
    a.grid_n = (a.n - 1) / bn + 1;
    return a;
}

template <int DT, int ACT> static int launch_planned(const LinearI8Args& a, hipStream_t stream)
{
    return launch_sized<linear_i8_staged_kernel<DT, ACT, 64, 64>>(128 * 128, tiled(a, 64, 64), 256, stream);
}

template <int DT> static int launch_act(const LinearI8Args& a, int act, hipStream_t stream)
{
    switch (act) {
    case SGPRS_ACT_RELU: return launch_planned<DT, SGPRS_ACT_RELU>(a, stream);
    case SGPRS_ACT_GELU: return launch_planned<DT, SGPRS_ACT_GELU>(a, stream);
    case SGPRS_ACT_SILU: return launch_planned<DT, SGPRS_ACT_SILU>(a, stream);
    default: return launch_planned<DT, SGPRS_ACT_NONE>(a, stream);
    }
}

int launch_linear_i8(const sgprs_linear_i8_desc_t& d, const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales,
                     const float* bias, const void* residual, void* y, void* ws, hipStream_t stream, int cus)
{
    const int es = (int)dtype_size(d.dtype);
    const LinearI8Args a = {(const unsigned char*)x, (const unsigned char*)w, x_scales, w_scales, bias, (const unsigned char*)residual, (unsigned char*)y,
                            d.m, d.n, d.k, (int)d.ldx, (int)d.ldw, (int)d.ldr * es, (int)d.ldy * es, d.residual_first, 0, 0};
    return d.dtype == SGPRS_BF16 ? launch_act<SGPRS_BF16>(a, d.act, stream) : launch_act<SGPRS_F32>(a, d.act, stream);
}

}  // namespace sgprs
