// y = act(x w^T + bias) + residual on the matrix cores.
//
// w's rows are the MFMA's row operand and x's rows its column operand, so that a lane ends up with four
// neighbouring outputs of one row.  Both operands are walked in k-tiles of 128 bytes a row (64 bf16, 32 fp32):
// eight 16-byte chunks, chunk c of row r in LDS slot c ^ (r & 7), so that 16 rows of one chunk meet no bank
// twice.  A lane's chunk holds 8 consecutive bf16 (one 16x16x32 MFMA) or 4 consecutive fp32 (four 16x16x4; the
// four k groups take elements 4 g + s, for both operands alike, so the order within a k-tile is all that changes).
#include <algorithm>
#include <cmath>

#include "linear_tiles.h"

namespace sgprs {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

struct LinearArgs {
    const unsigned char* x;
    const unsigned char* w;
    const float* bias;
    const unsigned char* residual;
    unsigned char* y;
    int m, n, k;
    int ldx, ldw, ldr, ldy;  // bytes
    int residual_first;
    int grid_m, grid_n;      // tiles
};

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

// The bf16 product with the accumulator tied to its registers: left to itself, the compiler copies accumulators about
// where there are many (a 256 x 256 tile then takes four times as long).  Its hazard recogniser does not look into the
// assembly: operands come from loads only, and accumulators are read behind settle().
__device__ __forceinline__ void mma_tied(u32x4_t a, u32x4_t b, f32x4_t& c)
{
#if __HIP_DEVICE_COMPILE__
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
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

// Eight (bf16) or four (fp32) neighbouring outputs of one row.  z: the sums, r: the residual as it lies in memory.
template <int DT, int ACT> __device__ __forceinline__ u32x4_t finish(const LinearArgs& a, const float* z, const float* bias, u32x4_t r)
{
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    float o[V];
    auto res = [&](int e) { return ES == 4 ? __uint_as_float(r[e % 4]) : __uint_as_float(e % 2 ? r[e / 2] & 0xffff0000u : r[e / 2] << 16); };
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = z[e] + bias[e];
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
template <int DT, int ACT> __device__ __forceinline__ void finish_row(const LinearArgs& a, long long row, int col, const float* z, const float* bias)
{
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    if (row >= a.m || col >= a.n) return;
    const unsigned char* rp = a.residual + row * a.ldr + (long long)col * ES;
    unsigned char* yp = a.y + row * a.ldy + (long long)col * ES;
    const int live = min(V, a.n - col);
    const u32x4_t out = finish<DT, ACT>(a, z, bias, a.residual ? load_chunk<ES>(rp, live * ES) : u32x4_t{0, 0, 0, 0});
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

template <int V> __device__ __forceinline__ void load_bias(const LinearArgs& a, int col, float* bias)
{
#pragma unroll
    for (int e = 0; e < V; ++e) bias[e] = a.bias && col + e < a.n ? a.bias[col + e] : 0.f;
}

// A wavefront's 16 TM x 16 TN outputs, from row m0 and column n0 on: 16 rows at a time through LDS of its own (`mine`),
// then V neighbouring outputs a lane.
template <int DT, int TN> struct StagedRows {
    static constexpr int V = DT == SGPRS_BF16 ? 8 : 4, PITCH = TN * 16 + 4;  // floats of a staged row
    static constexpr int BYTES = 16 * PITCH * 4;
};
template <int DT, int ACT, int TM, int TN>
__device__ __forceinline__ void store_tile(const LinearArgs& a, const f32x4_t (&acc)[TN][TM], float* mine, long long m0, int n0)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = StagedRows<DT, TN>::V, PITCH = StagedRows<DT, TN>::PITCH;
    constexpr int LPR = TN * 16 / V, RPP = 64 / LPR, PASSES = 16 / RPP;  // lanes of a row, rows of a pass
    const int lane = threadIdx.x & 63, frow = lane & 15, fgrp = lane >> 4, r0 = lane / LPR, c0 = lane % LPR * V, col = n0 + c0;
    float bias[V];
    load_bias<V>(a, col, bias);
    auto stage = [&](auto i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *(f32x4_t*)(mine + frow * PITCH + j * 16 + fgrp * 4) = acc[j][i];
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
    };
    auto staged = [&](int p, float* z) {
#pragma unroll
        for (int e = 0; e < V; e += 4) *(f32x4_t*)(z + e) = *(const f32x4_t*)(mine + (p * RPP + r0) * PITCH + c0 + e);
    };
    auto read = [] {
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
    };
    if (m0 + 16 * TM <= a.m && n0 + 16 * TN <= a.n) {  // all inside
        unsigned char* yp = a.y + (m0 + r0) * a.ldy + (long long)col * ES;
        const unsigned char* rp = a.residual + (m0 + r0) * a.ldr + (long long)col * ES;
        for_each<TM>([&](auto i) {
            u32x4_t r[PASSES] = {};
            if (a.residual) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p) __builtin_memcpy(&r[p], rp + (long long)(i * 16 + p * RPP) * a.ldr, 16);
            }
            stage(i);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                float z[V];
                staged(p, z);
                const u32x4_t out = finish<DT, ACT>(a, z, bias, r[p]);
                __builtin_memcpy(yp + (long long)(i * 16 + p * RPP) * a.ldy, &out, 16);
            }
            read();
        });
    } else {
        for_each<TM>([&](auto i) {
            stage(i);
#pragma unroll 1
            for (int p = 0; p < PASSES; ++p) {
                float z[V];
                staged(p, z);
                finish_row<DT, ACT>(a, m0 + i * 16 + p * RPP + r0, col, z, bias);
            }
            read();
        });
    }
#endif
}

// ---- tiles shared by a workgroup: aligned bf16 --------------------------------------------------
// BM x BN outputs, 2 x 2 wavefronts; two k-tiles in LDS, filled by loads that write it directly.  The barrier of a
// k-tile stands between its two halves: before it the second half's fragments have been read, so that its MFMAs
// follow the barrier at once while the next k-tile's first fragments are read and the one after that is requested
// into the buffer just left, a load behind every fourth MFMA (one behind every second one: 447 us instead of 409).
// Bound by the matrix cores at the clock they leave: 256 x 256 (one wavefront a SIMD, 256 accumulators; half the LDS
// reads per MFMA of 128 x 128) keeps them 70 % busy at 1.9 GHz, 16384x4096 -> 4096 in 409 to 415 us by card, 1343 to
// 1325 TFLOP/s (with a residual 420 to 424), where a large library product reaches 1529 to 1546.  128 x 128 (two workgroups a CU) is for what 256 x 256 divides badly: a tile's
// beginning and end cost as much as five k-tiles.
template <int ACT, int BM, int BN> __global__ __launch_bounds__(256, BM * BN >= 256 * 128 ? 1 : 2) void linear_tile_kernel(const LinearArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int DT = SGPRS_BF16, V = 8, WM = 2, WN = 2, NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int STAGE = (BM + BN) * 128, LA = BM / 8 / NW, LB = BN / 8 / NW, L = LA + LB;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole loads");
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0);
    const int kb = a.k * 2, tiles = (kb + 127) >> 7;
    const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;
    const __amdgpu_buffer_rsrc_t x_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.ldx), 0, (rows_x - 1) * a.ldx + kb, 0x00020000);
    const __amdgpu_buffer_rsrc_t w_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (long long)n0 * a.ldw), 0, (rows_w - 1) * a.ldw + kb, 0x00020000);
    const unsigned x_off = (unsigned)((wave * LA * 8 + lrow) * a.ldx + chunk * 16), w_off = (unsigned)((wave * LB * 8 + lrow) * a.ldw + chunk * 16);
    // load i of k-tile t; past the last k-tile everything lies outside
    auto request = [&](int t, int i) {
        const bool live = t * 128 + chunk * 16 < kb;
        unsigned char* st = smem + (t & 1) * STAGE;
        if (i < LA)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(x_rs, (lds_ptr_t)(st + (wave * LA + i) * 1024), 16, live ? x_off + (unsigned)(i * 8 * a.ldx) : kOutside,
                                                     t * 128, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rs, (lds_ptr_t)(st + BM * 128 + (wave * LB + i - LA) * 1024), 16,
                                                     live ? w_off + (unsigned)((i - LA) * 8 * a.ldw) : kOutside, t * 128, 0, 0);
    };
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned slot0 = (unsigned)((fgrp ^ (frow & 7)) << 4);  // chunk fgrp; chunk 4 + fgrp is slot0 ^ 64
    const unsigned x_frag = (unsigned)((wm * TM * 16 + frow) * 128) + slot0, w_frag = (unsigned)(BM * 128 + (wn * TN * 16 + frow) * 128) + slot0;

    f32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    u32x4_t xf[2][TM], wf[2][TN];
    // fragment r of half h of k-tile t
    auto read_fragment = [&](int t, int h, int r) {
        const unsigned base = (unsigned)((t & 1) * STAGE);
        if (r < TN) wf[h][r] = lds_read((w_frag + base + r * 2048) ^ (h << 6));
        else xf[h][r - TN] = lds_read((x_frag + base + (r - TN) * 2048) ^ (h << 6));
    };
    constexpr int R = TM + TN, M = TM * TN;
    constexpr int READ_EVERY = M / (R + 1) > 0 ? M / (R + 1) : 1, LOAD_EVERY = M / L > 0 ? M / L : 1;  // MFMAs
    static_assert(M >= R && M >= L, "reads and loads fit behind the MFMAs");

#pragma unroll
    for (int i = 0; i < L; ++i) request(0, i);
#pragma unroll
    for (int i = 0; i < L; ++i) request(1, i);
    __builtin_amdgcn_s_waitcnt((L & 15) | ((L >> 4) << 14) | 0x0F70);  // the first k-tile has landed
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < R; ++r) read_fragment(0, 0, r);
    int t = 0;
    do {  // (k > 0: without a loop that may not run, the accumulators are cleared in one place)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = j * TM + i;
                mma_tied(wf[0][j], xf[0][i], acc[j][i]);
                if (at % READ_EVERY == 0 && at / READ_EVERY < R) read_fragment(t, 1, at / READ_EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
        __builtin_amdgcn_s_waitcnt(0x0070);  // the next k-tile has landed, the fragments are read
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = j * TM + i;
                mma_tied(wf[1][j], xf[1][i], acc[j][i]);
                if (at % LOAD_EVERY == 0 && at / LOAD_EVERY < L) request(t + 2, at / LOAD_EVERY);
                if (at % READ_EVERY == 0 && at / READ_EVERY < R) read_fragment(t + 1, 0, at / READ_EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
    } while (++t < tiles);
    settle(acc);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    static_assert(NW * StagedRows<DT, TN>::BYTES <= 2 * STAGE, "staging fits");
    store_tile<DT, ACT, TM, TN>(a, acc, (float*)(smem + wave * StagedRows<DT, TN>::BYTES), m0 + wm * TM * 16, n0 + wn * TN * 16);
#endif
}

// ---- tiles shared by a workgroup: fp32, and bf16 rows at any alignment --------------------------
// BM x BN outputs, 2 x 2 wavefronts; the next k-tile is on its way to registers while this one, in LDS, is
// multiplied.  A thread brings units of 8 neighbouring inputs of a row.  fp32 goes through the bf16 matrix cores:
// x = h + m + l, each the bf16 nearest to what is left, holds 24 bits, and of the nine products of two such sums the
// six down to 2^-16 are taken (what is left out stays below 2^-23 of a product, and is of either sign); that is six
// MFMAs for 32 inputs instead of eight that take twice as long.  Both operands are multiplied by 2^24 first: so the parts
// of small and subnormal values hold all their bits too, the first one as a normal number (the matrix cores align a
// subnormal operand's products as if they had its leading zeros in front: with 2^16, which takes 2^-149 to bf16's smallest
// number, 2^-149 times ordinary values was off by 2^-17).  A sum that is not finite then (infinities have no such parts;
// operands from 2^104 and sums from 2^80 on pass the range) sends its wavefront through the fp32 matrix cores, with the
// operands as they are.
// 128 x 128, fp32: bound by the splitting (half of the vector units' time) and the MFMAs, 4096x4096 -> 4096 in 700 us,
// 196 TFLOP/s (17 us of it the scaling); fp32 MFMAs on the same tiles reached 142, the rate of the fp32 matrix cores is 157.  Relative error
// against 64 bits 1.6e-7 (plain fp32 chains 2.9e-7 to 7e-7).  64 x 64 with two groups of wavefronts that take every
// other k-tile is for fewer tiles: the second group covers what the first one waits for (fp32 300x700 -> 700 19.9 -> 16.8,
// 3136x512 -> 512 19.8 -> 17.5 us).
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned pack_bf16x2(float lo, float hi)
{
    const f32x2_t f = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2_t));
}
constexpr float kSplitScale = 0x1p24f;
template <int DT> __device__ __forceinline__ void split_unit(const u32x4_t* in, u32x4_t* planes)
{
    if constexpr (DT == SGPRS_BF16) {
        planes[0] = in[0];
    } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float a = __uint_as_float(in[p >> 1][2 * (p & 1)]) * kSplitScale, b = __uint_as_float(in[p >> 1][2 * (p & 1) + 1]) * kSplitScale;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const unsigned v = pack_bf16x2(a, b);
                planes[i][p] = v;
                a -= __uint_as_float(v << 16);  // exact
                b -= __uint_as_float(v & 0xffff0000u);
            }
        }
    }
}

// Drops the first `by` of a unit's eight values (8 or more: all) and fills up with zeros.
template <int DT> __device__ __forceinline__ void shift_unit(u32x4_t* unit, int by)
{
    constexpr int D = DT == SGPRS_BF16 ? 4 : 8;  // dwords
    unsigned v[D];
#pragma unroll
    for (int i = 0; i < D; ++i) v[i] = by >= 8 ? 0u : unit[i / 4][i % 4];
#pragma unroll
    for (int step = 4; step >= 1; step >>= 1) {
        const bool move = by > 0 && (by & step);
        if (DT == SGPRS_BF16 && step == 1) {
#pragma unroll
            for (int i = 0; i < D; ++i) v[i] = move ? v[i] >> 16 | (i + 1 < D ? v[i + 1] << 16 : 0u) : v[i];
        } else {
            const int d = DT == SGPRS_BF16 ? step / 2 : step;
#pragma unroll
            for (int i = 0; i < D; ++i) v[i] = move ? (i + d < D ? v[i + d] : 0u) : v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < D; ++i) unit[i / 4][i % 4] = v[i];
}

// k >= 8
template <int DT, int ACT, int BM, int BN, int AHEAD, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS, 2) void linear_staged_kernel(const LinearArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, WM = 2, WN = 2, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int PLANES = DT == SGPRS_BF16 ? 1 : 3, BK = DT == SGPRS_BF16 ? 64 : 32, STEPS = BK / 32, ROW = BK * 2, UPR = BK / 8;
    constexpr int UNITS = (BM + BN) * UPR / 256, UA = BM * UPR / 256, UC = 8 * ES / 16;  // of a thread, of them x's; 16-byte chunks of a unit
    constexpr int PLANE = (BM + BN) * ROW, BUF = PLANES * PLANE;  // bytes of a group's k-tile
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, thread = threadIdx.x & 255;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) & 3);
    const int wm = wave % WM, wn = wave / WM;
    const unsigned mine = (unsigned)(group * BUF);
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0);
    const unsigned char* xp = a.x + m0 * a.ldx;
    const unsigned char* wp = a.w + (long long)n0 * a.ldw;
    const int rounds = (a.k + BK * GROUPS - 1) / (BK * GROUPS);  // group g takes k-tiles g, g + GROUPS, ...; past the end they are zeros
    // unit i: row (i * 256 + thread) / UPR of x's rows and w's behind them; rows past the end repeat the last one
    const unsigned char* from[UNITS];
    const int octet = thread % UPR;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int r = (i * 256 + thread) / UPR;
        from[i] = i < UA ? xp + (long long)min(r, rows_x - 1) * a.ldx : wp + (long long)min(r - BM, rows_w - 1) * a.ldw;
    }
    u32x4_t staged[AHEAD][UNITS][UC];
    // Loads have no branch (the compiler would then wait for all of them): a unit that begins less than eight inputs
    // before the end of its row, or behind it, is taken from the row's last eight and shifted when it is stored.
    auto request = [&](int round, int set) {
        const long long at = (long long)min((round * GROUPS + group) * BK + octet * 8, a.k - 8) * ES;
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
#pragma unroll
            for (int c = 0; c < UC; ++c) __builtin_memcpy(&staged[set][i][c], from[i] + at + c * 16, 16);
    };
    // slot of octet c of row r: with rows of 64 bytes c ^ (r / 2 & 3), of 128 bytes c ^ (r & 7)
    auto place = [](int r, int c) { return (unsigned)(r * ROW + ((ROW == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7)) << 4)); };
    auto store = [&](int round, int set) {
        const int first = (round * GROUPS + group) * BK;
        if (first + BK > a.k) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) shift_unit<DT>(staged[set][i], first + octet * 8 - (a.k - 8));
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            u32x4_t planes[PLANES];
            split_unit<DT>(staged[set][i], planes);
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
                *(lds_u32x4_t*)(unsigned long)(mine + p * PLANE + place((i * 256 + thread) / UPR, octet)) = planes[p];
        }
    };
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned x_frag = mine + place(wm * TM * 16 + frow, fgrp), w_frag = mine + place(BM + wn * TN * 16 + frow, fgrp);
    f32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&] {
#pragma unroll
        for (int h = 0; h < STEPS; ++h) {
            u32x4_t xf[PLANES][TM], wf[PLANES][TN];
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
#pragma unroll
                for (int j = 0; j < TN; ++j) wf[p][j] = lds_read((w_frag + p * PLANE + j * 16 * ROW) ^ (h << 6));
#pragma unroll
                for (int i = 0; i < TM; ++i) xf[p][i] = lds_read((x_frag + p * PLANE + i * 16 * ROW) ^ (h << 6));
            }
            if constexpr (PLANES == 1) {
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[j][i] = mma<SGPRS_BF16>(wf[0][j], xf[0][i], acc[j][i]);
            } else {
                // 32 inputs' products on their own, the smallest first, then one addition: a sixth of the roundings that
                // reach the long sum.  At least four such chains side by side, or the MFMAs wait for each other.
                constexpr int SIDE = TM >= 4 ? 1 : 4 / TM;
                static_assert(TN % SIDE == 0, "whole steps");
#pragma unroll
                for (int j0 = 0; j0 < TN; j0 += SIDE) {
                    f32x4_t part[SIDE][TM];
#pragma unroll
                    for (int sum = PLANES - 1; sum >= 0; --sum)
#pragma unroll
                        for (int p = 0; p <= sum; ++p)
#pragma unroll
                            for (int j = 0; j < SIDE; ++j)
#pragma unroll
                                for (int i = 0; i < TM; ++i)
                                    part[j][i] = mma<SGPRS_BF16>(wf[sum - p][j0 + j], xf[p][i], sum == PLANES - 1 && p == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : part[j][i]);
#pragma unroll
                    for (int j = 0; j < SIDE; ++j)
#pragma unroll
                        for (int i = 0; i < TM; ++i) acc[j0 + j][i] += part[j][i];
                }
            }
        }
    };
    auto meet = [] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
    // A k-tile's registers are filled again as soon as it is stored, also past the end: with a branch there the compiler
    // could not count the loads behind a k-tile's and would wait for all.
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) request(s, s);
    for (int t = 0; t < rounds; t += AHEAD) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            if (t + s) meet();  // everyone has read the k-tile before
            store(t + s, s);
            meet();
            request(t + s + AHEAD, s);
            multiply();
        }
    }
    __syncthreads();
    if constexpr (GROUPS > 1) {  // the groups' sums, in order
        f32x4_t* sums = (f32x4_t*)smem + wave * TN * TM * 64 + lane;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                if (group) sums[((group - 1) * 4 * TN * TM + j * TM + i) * 64] = acc[j][i];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] += sums[(g * 4 * TN * TM + j * TM + i) * 64];
        __builtin_amdgcn_s_waitcnt(0xC07F);
    }
    if constexpr (DT == SGPRS_F32) {
        bool again = false;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    again |= !(fabsf(acc[j][i][e]) < INFINITY);
                    acc[j][i][e] *= 1.f / (kSplitScale * kSplitScale);
                }
        if (__any(again)) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int k0 = fgrp * 4; k0 < a.k + fgrp * 4; k0 += 16) {
                u32x4_t xf[TM], wf[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    wf[j] = load_chunk<4>(wp + (long long)min(wn * TN * 16 + j * 16 + frow, rows_w - 1) * a.ldw + (long long)k0 * 4, (a.k - k0) * 4);
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    xf[i] = load_chunk<4>(xp + (long long)min(wm * TM * 16 + i * 16 + frow, rows_x - 1) * a.ldx + (long long)k0 * 4, (a.k - k0) * 4);
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[j][i] = mma<SGPRS_F32>(wf[j], xf[i], acc[j][i]);
            }
        }
    }
    // (a wavefront's sums lie in [wave * TN * TM * 1024, + TN * TM * 1024): its rows are staged inside them)
    static_assert(StagedRows<DT, TN>::BYTES <= TN * TM * 1024 && (GROUPS == 1 || 4 * TN * TM * 1024 <= GROUPS * BUF), "staging fits");
    static_assert((GROUPS - 1) * 4 * TN * TM * 1024 <= GROUPS * BUF, "sums fit");
    store_tile<DT, ACT, TM, TN>(a, acc, (float*)(smem + wave * (GROUPS == 1 ? StagedRows<DT, TN>::BYTES : TN * TM * 1024)), m0 + wm * TM * 16, n0 + wn * TN * 16);
#endif
}

// ---- few rows: K split over the wavefronts of a workgroup --------------------------------------
// 16 TM x 16 TN outputs per workgroup; wavefront v takes k-tiles v, v + NW, ..., moves them into an LDS ring of
// its own and meets the others at the end only, where the partial tiles are added in wavefront order.
// Bound by reading w once and by the launch: 24x4096 -> 4096 bf16 in 8.5 us (4 TB/s), 1x512 -> 1000 in 3.8.
template <int DT, int ACT, int TM, int TN, int NW, int NS, bool DIRECT>
__global__ __launch_bounds__(NW * 64, 1) void linear_ksplit_kernel(const LinearArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    constexpr int BM = 16 * TM, BN = 16 * TN, STAGE = (BM + BN) * 128, LA = BM / 8, LB = BN / 8, L = LA + LB;
    constexpr int SROW = BN + 4;
    static_assert((NS - 1) * L <= 63, "vmcnt range");
    static_assert(BM * SROW * 4 <= NS * STAGE, "a partial tile fits the ring");
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
            for (int j = 0; j < TN; ++j) wf[h][j] = lds_read((w_frag + base + j * 2048) ^ (h << 6));
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[h][i] = lds_read((x_frag + base + i * 2048) ^ (h << 6));
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
enum LinearKernel { kTile256, kTile128, kStaged128, kStaged64, kSplit16, kSplit32x16, kSplit32 };

// No kernel splits K over workgroups: with eight wavefronts sharing it, the few tiles where that could pay (K beyond 6000
// at up to 64 rows and 512 outputs: 13 us) leave 4 us of it to gain behind a second launch.
size_t linear_workspace_bytes(const sgprs_linear_desc_t&, int) { return 0; }

// direct: operands whose rows are whole aligned chunks.  Estimates in us, fitted to measurements on 256 CUs (three sets of
// inputs in turn): what a kernel's k-tile and its tile's beginning and end take, times the tiles of a CU.
// bf16, 256 x 256 / 128 x 128 / 64 x 64: 16384x4096 -> 4096 427 / 508 / 800 us, 4096x4096 -> 4096 101 / 119 / 186,
// 12544x512 -> 2048 46 / 42 / 52, 16384x512 -> 512 - / 15.1 / 20.9, 3136x512 -> 512 - / 9.3 / 7.0 (K split over wavefronts
// 21); 300x700 -> 700 18 / 7.2 / 7.6 for 128 x 128 / 64 x 64 / K split.  fp32, 128 x 128 / 64 x 64 / K split:
// 4096x4096 -> 4096 677 / 894 / 1213, 16384x512 -> 512 55 / 71 / 140, 1000x1024 -> 1024 66 / 22 / 28, 300x700 -> 700
// 45 / 17 / 7.2 (before the operands' scaling, which adds up to 3 % to the first two).
static int plan_linear(const sgprs_linear_desc_t& d, int cus, bool direct)
{
    auto tiles = [&](int b, int c) { return (double)((d.m + (long long)b - 1) / b) * ((d.n + c - 1) / c); };
    if (d.m <= 16) return kSplit16;
    if (d.m <= 32) return tiles(32, 32) >= cus ? kSplit32 : kSplit32x16;
    if (d.k < 8 || tiles(64, 64) < cus) return kSplit32;
    const double t64 = tiles(64, 64) / cus, t128 = tiles(128, 128) / (2 * cus), t256 = std::ceil(tiles(256, 256) / cus);
    if (d.dtype == SGPRS_F32) return 2 * t128 >= 1 ? kStaged128 : kStaged64;
    const double kt = std::ceil(d.k / 64.0);
    const double us64 = 2.5 + t64 * (0.27 * kt + 0.4), us128 = std::max(0.7, t128) * (kt + 5.5), us256 = t256 * (1.55 * kt + 10);
    if (us64 < us128) return kStaged64;
    if (!direct) return kStaged128;
    return us128 < us256 ? kTile128 : kTile256;
}

template <auto kernel> static int launch_sized(int lds, const LinearArgs& a, int threads, hipStream_t stream)
{
    if ((long long)a.grid_m * a.grid_n * threads >= (1ll << 32)) return fail(SGPRS_ERR_UNSUPPORTED, "%d x %d outputs", a.m, a.n);
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    SGPRS_LAUNCH(kernel, dim3((unsigned)((long long)a.grid_m * a.grid_n)), threads, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

static LinearArgs tiled(LinearArgs a, int bm, int bn)
{
    a.grid_m = (a.m - 1) / bm + 1;  // (m may be the largest int)
    a.grid_n = (a.n - 1) / bn + 1;
    return a;
}

template <int DT, int ACT, int TM, int TN, int NW, int NS, bool DIRECT> static int launch_ksplit(const LinearArgs& a, hipStream_t stream)
{
    return launch_sized<linear_ksplit_kernel<DT, ACT, TM, TN, NW, NS, DIRECT>>(NW * NS * (TM + TN) * 2048, tiled(a, 16 * TM, 16 * TN), NW * 64, stream);
}

template <int DT, int ACT, bool DIRECT> static int launch_planned(const LinearArgs& a, int kernel, hipStream_t stream)
{
    constexpr int planes = DT == SGPRS_BF16 ? 128 : 3 * 64;  // bytes of a staged row
    switch (kernel) {
    case kTile256:
        if constexpr (DIRECT && DT == SGPRS_BF16) return launch_sized<linear_tile_kernel<ACT, 256, 256>>(2 * 512 * 128, tiled(a, 256, 256), 256, stream);
    case kTile128:
        if constexpr (DIRECT && DT == SGPRS_BF16) return launch_sized<linear_tile_kernel<ACT, 128, 128>>(2 * 256 * 128, tiled(a, 128, 128), 256, stream);
    case kStaged128: return launch_sized<linear_staged_kernel<DT, ACT, 128, 128, 1, 1>>(256 * planes, tiled(a, 128, 128), 256, stream);
    case kStaged64: return launch_sized<linear_staged_kernel<DT, ACT, 64, 64, 1, 2>>(2 * 128 * planes, tiled(a, 64, 64), 512, stream);
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

int launch_linear(const sgprs_linear_desc_t& d, const void* x, const void* w, const float* bias, const void* residual, void* y,
                  hipStream_t stream, int cus)
{
    const int es = (int)dtype_size(d.dtype);
    const LinearArgs a = {(const unsigned char*)x, (const unsigned char*)w, bias, (const unsigned char*)residual, (unsigned char*)y, d.m, d.n, d.k,
                    (int)d.ldx * es, (int)d.ldw * es, (int)d.ldr * es, (int)d.ldy * es, d.residual_first, 0, 0};
    const bool direct = (((uintptr_t)x | (uintptr_t)w | (unsigned)a.ldx | (unsigned)a.ldw | (unsigned)(d.k * es)) & 15) == 0;
    const int kernel = plan_linear(d, cus, direct);
    if (d.dtype == SGPRS_BF16)
        return direct ? launch_act<SGPRS_BF16, true>(a, d.act, kernel, stream) : launch_act<SGPRS_BF16, false>(a, d.act, kernel, stream);
    return direct ? launch_act<SGPRS_F32, true>(a, d.act, kernel, stream) : launch_act<SGPRS_F32, false>(a, d.act, kernel, stream);
}

}  // namespace sgprs
