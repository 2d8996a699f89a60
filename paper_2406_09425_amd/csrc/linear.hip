// y = act(x w^T + bias) + residual on the matrix cores.
//
// w's rows are the MFMA's row operand and x's rows its column operand, so that a lane ends up with four
// neighbouring outputs of one row.  Both operands are walked in k-tiles of 128 bytes a row (64 bf16, 32 fp32):
// eight 16-byte chunks, chunk c of row r in LDS slot c ^ (r & 7), so that 16 rows of one chunk meet no bank
// twice.  A lane's chunk holds 8 consecutive bf16 (one 16x16x32 MFMA) or 4 consecutive fp32 (four 16x16x4; the
// four k groups take elements 4 g + s, for both operands alike, so the order within a k-tile is all that changes).
#include <algorithm>

#include "block_ops.h"

namespace sgprs {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const unsigned char* x;
    const unsigned char* w;
    const float* bias;
    const unsigned char* residual;
    unsigned char* y;
    int m, n, k;
    int ldx, ldw, ldr, ldy;  // bytes
    int residual_first;
    int vector_out;          // outputs, residual and their strides allow 16-byte accesses
    int grid_m, grid_n;      // tiles
};

constexpr unsigned kOutside = 0x80000000u;  // beyond any descriptor's size: reads zeros

template <int DT> __device__ __forceinline__ f32x4_t mma(u32x4_t a, u32x4_t b, f32x4_t c)
{
#if __HIP_DEVICE_COMPILE__
    if constexpr (DT == SGPRS_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c, 0, 0, 0);
        return c;
    }
#else
    return c;
#endif
}

// The same with the accumulator tied to its registers: left to itself, the compiler copies accumulators about where
// there are many.  Its hazard recogniser does not look into the assembly: operands come from loads only, and
// accumulators are read behind settle().
template <int DT> __device__ __forceinline__ void mma_tied(u32x4_t a, u32x4_t b, f32x4_t& c)
{
#if __HIP_DEVICE_COMPILE__
    if constexpr (DT == SGPRS_BF16) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else c = mma<DT>(a, b, c);
#endif
}
template <int N, int M> __device__ __forceinline__ void settle(f32x4_t (&acc)[N][M])
{
#if __HIP_DEVICE_COMPILE__
    asm volatile("s_nop 15");
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < M; ++i) asm volatile("" : "+a"(acc[j][i]));
#endif
}

// 16 bytes at any alignment, of which the first `bytes` (a multiple of ES, may be <= 0) exist; zeros for the others.
template <int ES> __device__ __forceinline__ u32x4_t load_chunk(const unsigned char* p, int bytes)
{
    u32x4_t v = {0, 0, 0, 0};
    if (bytes >= 16) {
        __builtin_memcpy(&v, p, 16);
    } else if (bytes > 0) {
#pragma unroll
        for (int e = 0; e < 16 / ES; ++e) {
            if (e * ES >= bytes) continue;
            if constexpr (ES == 2) v[e / 2] |= (unsigned)*(const unsigned short*)(p + e * 2) << (e % 2 * 16);
            else v[e] = *(const unsigned*)(p + e * 4);
        }
    }
    return v;
}

// Eight (bf16) or four (fp32) neighbouring outputs of one row: epilogue and store.  z: the sums.
template <int DT, int ACT> __device__ __forceinline__ void finish_row(const LinearArgs& a, long long row, int col, const float* z, const float* bias)
{
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    if (row >= a.m || col >= a.n) return;
    const unsigned char* rp = a.residual + row * a.ldr + (long long)col * ES;
    unsigned char* yp = a.y + row * a.ldy + (long long)col * ES;
    const int live = min(V, a.n - col);
    const bool whole = a.vector_out && live == V;
    u32x4_t r = {0, 0, 0, 0};
    if (a.residual) {
        if (whole) r = *(const u32x4_t*)rp;
        else r = load_chunk<ES>(rp, live * ES);
    }
    float o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const float re = ES == 4 ? __uint_as_float(r[e % 4]) : __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
        const float t = z[e] + bias[e];
        o[e] = a.residual_first ? activate<DT, ACT>(t + re) : activate<DT, ACT>(t) + re;
    }
    u32x4_t out;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        if constexpr (ES == 4) out[p] = __float_as_uint(o[p]);
        else out[p] = pack_bf16x2_relu(o[2 * p], o[2 * p + 1], kNoReluFloor);
    }
    if (whole) {
        *(u32x4_t*)yp = out;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (e >= live) continue;
            if constexpr (ES == 4) ((unsigned*)yp)[e] = out[e];
            else ((unsigned short*)yp)[e] = (unsigned short)(out[e / 2] >> (e % 2 * 16));
        }
    }
}

template <int V> __device__ __forceinline__ void load_bias(const LinearArgs& a, int col, float* bias)
{
#pragma unroll
    for (int e = 0; e < V; ++e) bias[e] = a.bias && col + e < a.n ? a.bias[col + e] : 0.f;
}

// Tile of workgroup `id`: workgroups are dealt to the eight dies in turn; each die gets a run of consecutive
// tiles, walked in bands of eight row tiles, so that what a die works on at once shares operands in its L2.
__device__ __forceinline__ void tile_of(int id, int grid_m, int grid_n, int* tm, int* tn)
{
    const int tiles = grid_m * grid_n, per = tiles >> 3, rest = tiles & 7, die = id & 7;
    const int t = die * per + min(die, rest) + (id >> 3);
    const int band = t / (8 * grid_n), in = t - band * 8 * grid_n, rows = min(8, grid_m - band * 8);
    *tn = in / rows;
    *tm = band * 8 + in - *tn * rows;
}

// ---- tiles shared by a workgroup ---------------------------------------------------------------
// BM x BN outputs, WM x WN wavefronts; two k-tiles in LDS.  The barrier of a k-tile stands between its two
// halves: before it the second half's fragments have been read, so that its MFMAs follow the barrier at once
// while the next k-tile's first fragments are read and the one after that is requested into the buffer just left.
// DIRECT: loads that write LDS directly (operands 16-byte aligned, rows whole chunks).  Otherwise chunks go
// through registers, a k-tile earlier.
template <int DT, int ACT, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ __launch_bounds__(WM * WN * 64, BM * BN >= 256 * 128 ? 1 : 2) void linear_tile_kernel(const LinearArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * 128, LA = BM / 8 / NW, LB = BN / 8 / NW, L = LA + LB;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole loads");
    typedef __attribute__((address_space(3))) void* lds_ptr_t;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0);
    const unsigned char* xp = a.x + m0 * a.ldx;
    const unsigned char* wp = a.w + (long long)n0 * a.ldw;
    const int kb = a.k * ES, tiles = (kb + 127) >> 7;
    const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;

    const __amdgpu_buffer_rsrc_t x_rs = __builtin_amdgcn_make_buffer_rsrc((void*)xp, 0, (rows_x - 1) * a.ldx + kb, 0x00020000);
    const __amdgpu_buffer_rsrc_t w_rs = __builtin_amdgcn_make_buffer_rsrc((void*)wp, 0, (rows_w - 1) * a.ldw + kb, 0x00020000);
    const unsigned x_off = (unsigned)((wave * LA * 8 + lrow) * a.ldx + chunk * 16), w_off = (unsigned)((wave * LB * 8 + lrow) * a.ldw + chunk * 16);

    u32x4_t staged[DIRECT ? 1 : L];
    // load i of k-tile t; past the last k-tile everything lies outside
    auto request = [&](int t, int i) {
        const bool live = t * 128 + chunk * 16 < kb;
        if constexpr (DIRECT) {
            unsigned char* st = smem + (t & 1) * STAGE;
            if (i < LA)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rs, (lds_ptr_t)(st + (wave * LA + i) * 1024), 16, live ? x_off + (unsigned)(i * 8 * a.ldx) : kOutside,
                                                         t * 128, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rs, (lds_ptr_t)(st + BM * 128 + (wave * LB + i - LA) * 1024), 16,
                                                         live ? w_off + (unsigned)((i - LA) * 8 * a.ldw) : kOutside, t * 128, 0, 0);
        } else {
            const bool of_x = i < LA;
            const int r = of_x ? (wave * LA + i) * 8 + lrow : (wave * LB + i - LA) * 8 + lrow;
            const int at = t * 128 + chunk * 16;
            const bool row = of_x ? r < rows_x : r < rows_w;
            staged[i] = load_chunk<ES>((of_x ? xp + (long long)r * a.ldx : wp + (long long)r * a.ldw) + at, row ? kb - at : 0);
        }
    };
    auto store_staged = [&](int t) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < L; ++i)
                *(u32x4_t*)(smem + (t & 1) * STAGE + (i < LA ? (wave * LA + i) * 1024 : BM * 128 + (wave * LB + i - LA) * 1024) + lane * 16) = staged[i];
        }
    };
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned slot0 = (unsigned)((fgrp ^ (frow & 7)) << 4);  // chunk fgrp; chunk 4 + fgrp is slot0 ^ 64
    const unsigned x_frag = (unsigned)((wm * TM * 16 + frow) * 128) + slot0, w_frag = (unsigned)(BM * 128 + (wn * TN * 16 + frow) * 128) + slot0;
    auto read = [&](unsigned at) { return *(const lds_u32x4_t*)(unsigned long)at; };

    f32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    u32x4_t xf[2][TM], wf[2][TN];
    // fragment r of half h of k-tile t
    auto read_fragment = [&](int t, int h, int r) {
        const unsigned base = (unsigned)((t & 1) * STAGE);
        if (r < TN) wf[h][r] = read((w_frag + base + r * 2048) ^ (h << 6));
        else xf[h][r - TN] = read((x_frag + base + (r - TN) * 2048) ^ (h << 6));
    };
    constexpr int R = TM + TN, M = TM * TN;
    constexpr int READ_EVERY = M / (R + 1) > 0 ? M / (R + 1) : 1, LOAD_EVERY = M / L > 0 ? M / L : 1;  // MFMAs

#pragma unroll
    for (int i = 0; i < L; ++i) request(0, i);
    store_staged(0);
#pragma unroll
    for (int i = 0; i < L; ++i) request(1, i);
    store_staged(1);
    if constexpr (DIRECT) {
        __builtin_amdgcn_s_waitcnt((L & 15) | ((L >> 4) << 14) | 0x0F70);  // the first k-tile has landed
    } else {
#pragma unroll
        for (int i = 0; i < L; ++i) request(2, i);
        __builtin_amdgcn_s_waitcnt(0xC07F);
    }
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < R; ++r) read_fragment(0, 0, r);
    for (int t = 0; t < tiles; ++t) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = j * TM + i;
                mma_tied<DT>(wf[0][j], xf[0][i], acc[j][i]);
                if (at % READ_EVERY == 0 && at / READ_EVERY < R) read_fragment(t, 1, at / READ_EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
        if constexpr (M < R) {
#pragma unroll
            for (int r = M; r < R; ++r) read_fragment(t, 1, r);
        }
        __builtin_amdgcn_s_waitcnt(DIRECT ? 0x0070 : 0xC07F);  // the next k-tile has landed (DIRECT), the fragments are read
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!DIRECT) store_staged(t);  // k-tile t + 2
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = j * TM + i;
                mma_tied<DT>(wf[1][j], xf[1][i], acc[j][i]);
                if (DIRECT && at % LOAD_EVERY == 0 && at / LOAD_EVERY < L) request(t + 2, at / LOAD_EVERY);
                if (at % READ_EVERY == 0 && at / READ_EVERY < R) read_fragment(t + 1, 0, at / READ_EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
        if constexpr (DIRECT && M < L) {
#pragma unroll
            for (int i = M; i < L; ++i) request(t + 2, i);
        }
        if constexpr (M < R) {
#pragma unroll
            for (int r = M; r < R; ++r) read_fragment(t + 1, 0, r);
        }
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < L; ++i) request(t + 3, i);
        }
    }
    if constexpr (DT == SGPRS_BF16) settle(acc);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();

    // Epilogue: 16 rows at a time through the wavefront's own LDS, then V neighbouring outputs a lane.
    constexpr int SROW = TN * 16 + 4, LPR = TN * 16 / V, RPP = 64 / LPR;  // floats of a staged row; lanes of a row, rows of a pass
    static_assert(NW * 16 * SROW * 4 <= 2 * STAGE, "staging fits");
    float* mine = (float*)smem + wave * 16 * SROW;
    const int col = n0 + wn * TN * 16 + lane % LPR * V;
    float bias[V];
    load_bias<V>(a, col, bias);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *(f32x4_t*)(mine + frow * SROW + j * 16 + fgrp * 4) = acc[j][i];
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
#pragma unroll
        for (int p = 0; p < 16 / RPP; ++p) {
            const int r = p * RPP + lane / LPR;
            float z[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) *(f32x4_t*)(z + e) = *(const f32x4_t*)(mine + r * SROW + lane % LPR * V + e);
            finish_row<DT, ACT>(a, m0 + (wm * TM + i) * 16 + r, col, z, bias);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
    }
#endif
}

// ---- few rows: K split over the wavefronts of a workgroup --------------------------------------
// 16 TM x 16 TN outputs per workgroup; wavefront v takes k-tiles v, v + NW, ..., moves them into an LDS ring of
// its own and meets the others at the end only, where the partial tiles are added in wavefront order.
template <int DT, int ACT, int TM, int TN, int NW, int NS, bool DIRECT>
__global__ __launch_bounds__(NW * 64, 1) void linear_ksplit_kernel(const LinearArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    constexpr int BM = 16 * TM, BN = 16 * TN, STAGE = (BM + BN) * 128, LA = BM / 8, LB = BN / 8, L = LA + LB;
    constexpr int SROW = BN + 4;
    static_assert((NS - 1) * L <= 63, "vmcnt range");
    static_assert(BM * SROW * 4 <= NS * STAGE, "a partial tile fits the ring");
    typedef __attribute__((address_space(3))) void* lds_ptr_t;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0);
    const unsigned char* xp = a.x + m0 * a.ldx;
    const unsigned char* wp = a.w + (long long)n0 * a.ldw;
    const int kb = a.k * ES, tiles = (kb + 127) >> 7;
    const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;
    const unsigned ring = (unsigned)(wave * NS * STAGE);

    const __amdgpu_buffer_rsrc_t x_rs = __builtin_amdgcn_make_buffer_rsrc((void*)xp, 0, (rows_x - 1) * a.ldx + kb, 0x00020000);
    const __amdgpu_buffer_rsrc_t w_rs = __builtin_amdgcn_make_buffer_rsrc((void*)wp, 0, (rows_w - 1) * a.ldw + kb, 0x00020000);
    u32x4_t staged[DIRECT ? 1 : L];
    auto request = [&](int t, int slot) {
        const int at = t * 128 + chunk * 16;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int r = (i < LB ? i : i - LB) * 8 + lrow;
            if constexpr (DIRECT) {
                unsigned char* to = smem + ring + slot * STAGE;
                const unsigned off = at < kb ? (unsigned)(r * (i < LB ? a.ldw : a.ldx) + chunk * 16) : kOutside;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LB ? w_rs : x_rs, (lds_ptr_t)(to + i * 1024), 16, off, t * 128, 0, 0);
            } else {
                const bool row = i < LB ? r < rows_w : r < rows_x;
                staged[i] = load_chunk<ES>((i < LB ? wp + (long long)r * a.ldw : xp + (long long)r * a.ldx) + at, row ? kb - at : 0);
            }
        }
    };
    f32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned w_frag = ring + (unsigned)(frow * 128) + (unsigned)((fgrp ^ (frow & 7)) << 4), x_frag = w_frag + BN * 128;
    auto read = [&](unsigned at) { return *(const lds_u32x4_t*)(unsigned long)at; };
    if constexpr (DIRECT) {
#pragma unroll
        for (int s = 0; s < NS; ++s) request(wave + s * NW, s);
    } else {
        request(wave, 0);
    }
    int slot = 0;
    for (int t = wave; t < tiles; t += NW) {
        if constexpr (DIRECT) {
            constexpr int OUT = (NS - 1) * L;  // requests behind this k-tile's
            __builtin_amdgcn_s_waitcnt((OUT & 15) | ((OUT >> 4) << 14) | 0x0F70);
        } else {
#pragma unroll
            for (int i = 0; i < L; ++i) *(lds_u32x4_t*)(unsigned long)(ring + slot * STAGE + i * 1024 + lane * 16) = staged[i];
            request(t + NW, 0);
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_s_waitcnt(0xC07F);
        }
        __builtin_amdgcn_sched_barrier(0);
        u32x4_t wf[2][TN], xf[2][TM];
        const unsigned base = (unsigned)(slot * STAGE);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[h][j] = read((w_frag + base + j * 2048) ^ (h << 6));
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[h][i] = read((x_frag + base + i * 2048) ^ (h << 6));
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (DIRECT) request(t + NS * NW, slot);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] = mma<DT>(wf[h][j], xf[h][i], acc[j][i]);
        slot = slot + 1 == NS ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(0);  // requests past the end write zeros into the ring
    float* mine = (float*)(smem + ring);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) *(f32x4_t*)(mine + (i * 16 + frow) * SROW + j * 16 + fgrp * 4) = acc[j][i];
    __syncthreads();
    constexpr int LPR = BN / V;
    for (int e0 = threadIdx.x; e0 < BM * LPR; e0 += NW * 64) {
        const int r = e0 / LPR, c = e0 % LPR * V;
        float z[V] = {}, bias[V];
        load_bias<V>(a, n0 + c, bias);
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float* part = (const float*)(smem + v * NS * STAGE) + r * SROW + c;
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] += part[e];
        }
        finish_row<DT, ACT>(a, m0 + r, n0 + c, z, bias);
    }
#endif
}

// ---- plans -------------------------------------------------------------------------------------
enum LinearKernel { kTile256, kTile256x128, kTile128, kTile64, kSplit16, kSplit32x16, kSplit32 };

size_t linear_workspace_bytes(const sgprs_linear_desc_t&, int) { return 0; }

static int plan_linear(const sgprs_linear_desc_t& d, int cus, bool direct)
{
    auto tiles = [&](int bm, int bn) { return (long long)((d.m + bm - 1) / bm) * ((d.n + bn - 1) / bn); };
    if (d.m <= 16) return kSplit16;
    if (d.m <= 32) return tiles(32, 32) >= cus ? kSplit32 : kSplit32x16;
    if (tiles(64, 64) < cus) return kSplit32;
    if (tiles(128, 128) < cus || !direct) return kTile64;
    if (tiles(256, 256) < 2 * cus) return kTile128;
    return kTile256;
}

template <auto kernel> static int launch_sized(int lds, const LinearArgs& a, int threads, hipStream_t stream)
{
    if ((long long)a.grid_m * a.grid_n >= (1ll << 31)) return fail(SGPRS_ERR_UNSUPPORTED, "%d x %d outputs", a.m, a.n);
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    SGPRS_LAUNCH(kernel, dim3((unsigned)((long long)a.grid_m * a.grid_n)), threads, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

template <int DT, int ACT, int BM, int BN, int WM, int WN, bool DIRECT> static int launch_tile(LinearArgs a, hipStream_t stream)
{
    a.grid_m = (a.m + BM - 1) / BM;
    a.grid_n = (a.n + BN - 1) / BN;
    return launch_sized<linear_tile_kernel<DT, ACT, BM, BN, WM, WN, DIRECT>>(2 * (BM + BN) * 128, a, WM * WN * 64, stream);
}

template <int DT, int ACT, int TM, int TN, int NW, int NS, bool DIRECT> static int launch_ksplit(LinearArgs a, hipStream_t stream)
{
    a.grid_m = (a.m + 16 * TM - 1) / (16 * TM);
    a.grid_n = (a.n + 16 * TN - 1) / (16 * TN);
    return launch_sized<linear_ksplit_kernel<DT, ACT, TM, TN, NW, NS, DIRECT>>(NW * NS * (TM + TN) * 2048, a, NW * 64, stream);
}

template <int DT, int ACT, bool DIRECT> static int launch_planned(const LinearArgs& a, int kernel, hipStream_t stream)
{
    switch (kernel) {
    case kTile256: if constexpr (DIRECT && DT == SGPRS_BF16) return launch_tile<DT, ACT, 256, 256, 2, 2, DIRECT>(a, stream);
    case kTile256x128: if constexpr (DIRECT) return launch_tile<DT, ACT, 256, 128, 2, 2, DIRECT>(a, stream);
    case kTile128: if constexpr (DIRECT) return launch_tile<DT, ACT, 128, 128, 2, 2, DIRECT>(a, stream);
    case kTile64: return launch_tile<DT, ACT, 64, 64, 2, 2, DIRECT>(a, stream);
    case kSplit16: return launch_ksplit<DT, ACT, 1, 1, 8, 4, DIRECT>(a, stream);
    case kSplit32x16: return launch_ksplit<DT, ACT, 2, 1, 8, 3, DIRECT>(a, stream);
    default: return launch_ksplit<DT, ACT, 2, 2, 8, 2, DIRECT>(a, stream);
    }
}

template <int DT, bool DIRECT> static int launch_act(const LinearArgs& a, int act, int kernel, hipStream_t stream)
{
    switch (act) {
    case SGPRS_ACT_RELU: return launch_planned<DT, SGPRS_ACT_RELU, DIRECT>(a, kernel, stream);
    case SGPRS_ACT_GELU: return launch_planned<DT, SGPRS_ACT_GELU, DIRECT>(a, kernel, stream);
    case SGPRS_ACT_SILU: return launch_planned<DT, SGPRS_ACT_SILU, DIRECT>(a, kernel, stream);
    default: return launch_planned<DT, SGPRS_ACT_NONE, DIRECT>(a, kernel, stream);
    }
}

int launch_linear(const sgprs_linear_desc_t& d, const void* x, const void* w, const float* bias, const void* residual, void* y, void* ws,
                  hipStream_t stream, int cus)
{
    const int es = (int)dtype_size(d.dtype);
    LinearArgs a = {(const unsigned char*)x, (const unsigned char*)w, bias, (const unsigned char*)residual, (unsigned char*)y, d.m, d.n, d.k,
                    (int)d.ldx * es, (int)d.ldw * es, (int)d.ldr * es, (int)d.ldy * es, d.residual_first, 0, 0, 0};
    a.vector_out = (((uintptr_t)y | (unsigned)a.ldy | (residual ? (uintptr_t)residual | (unsigned)a.ldr : 0)) & 15) == 0;
    const bool direct = (((uintptr_t)x | (uintptr_t)w | (unsigned)a.ldx | (unsigned)a.ldw | (unsigned)(d.k * es)) & 15) == 0;
    const int kernel = plan_linear(d, cus, direct);
    if (d.dtype == SGPRS_BF16)
        return direct ? launch_act<SGPRS_BF16, true>(a, d.act, kernel, stream) : launch_act<SGPRS_BF16, false>(a, d.act, kernel, stream);
    return direct ? launch_act<SGPRS_F32, true>(a, d.act, kernel, stream) : launch_act<SGPRS_F32, false>(a, d.act, kernel, stream);
}

}  // namespace sgprs
