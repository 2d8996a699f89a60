// y = act(x_scale w_scale sum(x w) + bias) + residual of 8-bit integers on the matrix cores.
//
// w's rows are the MFMA's row operand and x's rows its column operand, so that a lane ends up with four neighbouring
// outputs of one row.  Both operands are walked in k-tiles of 128 bytes a row: eight 16-byte chunks, chunk c of row r in LDS
// slot c ^ (r & 7), so that 16 rows of one chunk meet no bank twice; two 16x16x64 MFMAs a k-tile.  Sums are 32-bit integers
// and exact, so any split of k gives the same bits.
#include <algorithm>
#include <cmath>
#include <type_traits>

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

// What belongs to V neighbouring columns (behind the last one: the last one's).
template <int V> struct Columns {
    float scale[V], bias[V];
    __device__ __forceinline__ Columns() {}
    __device__ __forceinline__ Columns(const LinearI8Args& a, int col)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            scale[e] = 1.f;
            bias[e] = 0.f;
        }
        if (a.w_scales) {
#pragma unroll
            for (int e = 0; e < V; ++e) scale[e] = a.w_scales[min(col + e, a.n - 1)];
        }
        if (a.bias) {
#pragma unroll
            for (int e = 0; e < V; ++e) bias[e] = a.bias[min(col + e, a.n - 1)];
        }
    }
};
__device__ __forceinline__ float row_scale(const LinearI8Args& a, long long row) { return a.x_scales ? a.x_scales[min(row, a.m - 1ll)] : 1.f; }

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
template <int V> __device__ __forceinline__ u32x4_t residual_at(const LinearI8Args& a, long long row, int col)
{
    constexpr int ES = 16 / V;
    const bool live = a.residual && row < a.m && col < a.n;
    return live ? load_chunk<ES>(a.residual + row * a.ldr + (long long)col * ES, min(V, a.n - col) * ES) : u32x4_t{0, 0, 0, 0};
}
template <int DT, int ACT, int V>
__device__ __forceinline__ void finish_row(const LinearI8Args& a, long long row, int col, const int* s, float x_scale, const Columns<V>& c, u32x4_t r)
{
    constexpr int ES = 16 / V;
    if (row >= a.m || col >= a.n) return;
    unsigned char* yp = a.y + row * a.ldy + (long long)col * ES;
    const int live = min(V, a.n - col);
    const u32x4_t out = finish<DT, ACT>(a, s, x_scale, c, r);
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

__device__ __forceinline__ u32x4_t drop_bytes(u32x4_t v, int n)  // the first n of 16 (16: all), zeros behind the others
{
    unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
    if (n >= 8) {
        lo = hi;
        hi = 0;
    }
    const int bits = (n & 7) * 8;
    if (bits) {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    }
    if (n >= 16) lo = 0;
    return u32x4_t{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

// A wavefront's 16 TM x 16 TN outputs, from row m0 and column n0 on: 16 rows at a time through LDS of its own (`mine`),
// then V neighbouring outputs a lane.
template <int DT, int TN> struct StagedRows {
    static constexpr int V = DT == SGPRS_BF16 ? 8 : 4, PITCH = TN * 16 + 4;  // values of a staged row
    static constexpr int BYTES = 16 * PITCH * 4;
};
// What a wavefront's outputs need beside the sums, if it is asked for before they are there: that of the columns and, of a
// tile that lies inside, row scales and the residual.
template <int DT, int TM, int TN> struct Ahead {
    static constexpr int V = StagedRows<DT, TN>::V, ES = 16 / V, LPR = TN * 16 / V, RPP = 64 / LPR, PASSES = 16 / RPP;  // lanes of a row, rows of a pass
    Columns<V> columns;
    u32x4_t r[TM][PASSES];
    float scale[TM][PASSES];
    __device__ __forceinline__ Ahead(const LinearI8Args& a, long long m0, int n0) : columns(a, n0 + (int)(threadIdx.x & 63) % LPR * V)
    {
        if (m0 + 16 * TM > a.m || n0 + 16 * TN > a.n) return;
        const int lane = threadIdx.x & 63;
        const unsigned char* rp = a.residual + (m0 + lane / LPR) * a.ldr + (long long)(n0 + lane % LPR * V) * ES;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                r[i][p] = u32x4_t{0, 0, 0, 0};
                if (a.residual) __builtin_memcpy(&r[i][p], rp + (long long)(i * 16 + p * RPP) * a.ldr, 16);
                scale[i][p] = row_scale(a, m0 + i * 16 + p * RPP + lane / LPR);
            }
    }
};
struct NotAhead {};

template <int DT, int ACT, int TM, int TN, class A>
__device__ __forceinline__ void store_tile(const LinearI8Args& a, const i32x4_t (&acc)[TN][TM], int* mine, long long m0, int n0, const A& ahead)
{
#if __HIP_DEVICE_COMPILE__
    constexpr bool AHEAD = !std::is_same_v<A, NotAhead>;
    constexpr int V = StagedRows<DT, TN>::V, ES = 16 / V, PITCH = StagedRows<DT, TN>::PITCH;
    constexpr int LPR = TN * 16 / V, RPP = 64 / LPR, PASSES = 16 / RPP;  // lanes of a row, rows of a pass
    const int lane = threadIdx.x & 63, frow = lane & 15, fgrp = lane >> 4, r0 = lane / LPR, c0 = lane % LPR * V, col = n0 + c0;
    Columns<V> columns;
    if constexpr (AHEAD) columns = ahead.columns;
    else columns = Columns<V>(a, col);
    auto stage = [&](auto i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) *(i32x4_t*)(mine + frow * PITCH + j * 16 + fgrp * 4) = acc[j][i];
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_s_waitcnt(0xC07F);
    };
    auto staged = [&](int p, int* s) {
#pragma unroll
        for (int e = 0; e < V; e += 4) *(i32x4_t*)(s + e) = *(const i32x4_t*)(mine + (p * RPP + r0) * PITCH + c0 + e);
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
            float scale[PASSES];
            if (!AHEAD && a.residual) {
#pragma unroll
                for (int p = 0; p < PASSES; ++p) __builtin_memcpy(&r[p], rp + (long long)(i * 16 + p * RPP) * a.ldr, 16);
            }
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                if constexpr (AHEAD) {
                    r[p] = ahead.r[i][p];
                    scale[p] = ahead.scale[i][p];
                } else {
                    scale[p] = row_scale(a, m0 + i * 16 + p * RPP + r0);
                }
            }
            stage(i);
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                int s[V];
                staged(p, s);
                const u32x4_t out = finish<DT, ACT>(a, s, scale[p], columns, r[p]);
                __builtin_memcpy(yp + (long long)(i * 16 + p * RPP) * a.ldy, &out, 16);
            }
            read();
        });
    } else {
        for_each<TM>([&](auto i) {
            stage(i);
#pragma unroll 1
            for (int p = 0; p < PASSES; ++p) {
                int s[V];
                staged(p, s);
                const long long row = m0 + i * 16 + p * RPP + r0;
                finish_row<DT, ACT>(a, row, col, s, row_scale(a, row), columns, residual_at<V>(a, row, col));
            }
            read();
        });
    }
#endif
}

// The product with the accumulator tied to its registers: left to itself, the compiler copies accumulators about where
// there are many.  Its hazard recogniser does not look into the assembly: operands come from loads only, and
// accumulators are read behind settle().
__device__ __forceinline__ void mma_tied(u32x4_t a, u32x4_t b, i32x4_t& c)
{
#if __HIP_DEVICE_COMPILE__
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
#endif
}
template <int N, int M> __device__ __forceinline__ void settle(i32x4_t (&acc)[N][M])
{
#if __HIP_DEVICE_COMPILE__
    asm volatile("s_nop 15");
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < M; ++i) asm volatile("" : "+a"(acc[j][i]));
#endif
}

// ---- tiles shared by a workgroup: aligned rows --------------------------------------------------
// BM x BN outputs, 2 x 2 wavefronts; two k-tiles (or NS) in LDS, filled by loads that write it directly.  The barrier of a k-tile
// stands between its two halves: before it the second half's fragments have been read, so that its MFMAs follow the barrier
// at once while the next k-tile's first fragments are read and the one after that is requested into the buffer just left.
// NS k-tiles in LDS: four where few tiles leave it free, 1024x4096 -> 4096 by 128x128 tiles 26 -> 22 us, 256x4096 -> 4096 by
// 64x64 18 -> 10.6; where several workgroups share a CU two are faster (2048x4096 -> 4096 35 for 42).
// 16384x4096 -> 4096 in 238 to 262 us, by card (2.1 to 2.3 PFLOP/s; the library's product of integers alone 259 to 270): bound
// by the MFMAs and the clock under them (of 30 launches without a pause the first five take 256 to 265, the others 271 to 292).  32x32x32 MFMAs took 255 for 237, a ring of four half k-tiles 258 for 255.
template <int DT, int ACT, int BM, int BN, int NS> __global__ __launch_bounds__(256, BM * BN >= 256 * 128 ? 1 : 2) void linear_i8_tile_kernel(const LinearI8Args a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int WM = 2, WN = 2, NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
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
    const int tiles = (a.k + 127) >> 7;
    const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;
    const __amdgpu_buffer_rsrc_t x_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.ldx), 0, (rows_x - 1) * a.ldx + a.k, 0x00020000);
    const __amdgpu_buffer_rsrc_t w_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (long long)n0 * a.ldw), 0, (rows_w - 1) * a.ldw + a.k, 0x00020000);
    const unsigned x_off = (unsigned)((wave * LA * 8 + lrow) * a.ldx + chunk * 16), w_off = (unsigned)((wave * LB * 8 + lrow) * a.ldw + chunk * 16);
    // load i of k-tile t; past the last k-tile everything lies outside
    auto request = [&](int t, int i) {
        const bool live = t * 128 + chunk * 16 < a.k;
        unsigned char* st = smem + (t & (NS - 1)) * STAGE;
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

    i32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
    u32x4_t xf[2][TM], wf[2][TN];
    // fragment r of half h of k-tile t
    auto read_fragment = [&](int t, int h, int r) {
        const unsigned base = (unsigned)((t & (NS - 1)) * STAGE);
        if (r < TN) wf[h][r] = lds_read((w_frag + base + r * 2048) ^ (h << 6));
        else xf[h][r - TN] = lds_read((x_frag + base + (r - TN) * 2048) ^ (h << 6));
    };
    constexpr int R = TM + TN, M = TM * TN;
    constexpr int READ_EVERY = M / (R + 1) > 0 ? M / (R + 1) : 1, LOAD_EVERY = M / L > 0 ? M / L : 1;  // MFMAs
    static_assert(M >= R && M >= L, "reads and loads fit behind the MFMAs");
    static_assert((NS & (NS - 1)) == 0 && (NS - 1) * L <= 63, "slots by masks, vmcnt range");

    const long long mw = m0 + wm * TM * 16;
    const int nw = n0 + wn * TN * 16;
    const auto ahead = [&] {  // in bf16 3136x512 -> 512 with a residual 6.2 -> 5.6 us, 5000x256 -> 256 4.8 -> 4.4; in fp32 it cost 0.3
        if constexpr (BM == 64 && DT == SGPRS_BF16) return Ahead<DT, TM, TN>(a, mw, nw);
        else return NotAhead();
    }();
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < L; ++i) request(s, i);
    constexpr int BEHIND = (NS - 1) * L, NEXT = (NS - 2) * L;  // requests behind the first k-tile, and behind the next one
    __builtin_amdgcn_s_waitcnt((BEHIND & 15) | ((BEHIND >> 4) << 14) | 0x0F70);  // the first k-tile has landed
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
        __builtin_amdgcn_s_waitcnt((NEXT & 15) | ((NEXT >> 4) << 14) | 0x0070);  // the next k-tile has landed, the fragments are read
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = j * TM + i;
                mma_tied(wf[1][j], xf[1][i], acc[j][i]);
                if (at % LOAD_EVERY == 0 && at / LOAD_EVERY < L) request(t + NS, at / LOAD_EVERY);
                if (at % READ_EVERY == 0 && at / READ_EVERY < R) read_fragment(t + 1, 0, at / READ_EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
    } while (++t < tiles);
    settle(acc);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    static_assert(NW * StagedRows<DT, TN>::BYTES <= NS * STAGE, "staging fits");
    store_tile<DT, ACT, TM, TN>(a, acc, (int*)(smem + wave * StagedRows<DT, TN>::BYTES), mw, nw, ahead);
#endif
}

// ---- tiles shared by a workgroup: rows at any alignment -----------------------------------------
// BM x BN outputs, 2 x 2 wavefronts; the next k-tile is on its way to registers while this one, in one of two LDS buffers, is
// multiplied.  k >= 16: loads have no branch; a chunk that reaches past the end of its row is taken from the row's
// last 16 bytes and shifted when it is stored, rows past the end repeat the last one.
// Few tiles are 32 rows high: 700x700 -> 701 in bf16 5.4 us, by 64x64 tiles 6.1, 1500x300 -> 300 in fp32 with a residual 4.8 for
// 6.0, 3137x250 -> 509 6.6 for 7.6, without a residual 6.4 for 6.2.
// 3137x517 -> 509 in fp32 in 8 us, with a residual 9.1 (by 64x64 tiles 9.8): few k-tiles, each a round trip to memory.  Of
// 64x64 tiles two k-tiles on their way took 8.6 for 7.5; residuals and scales asked for before the k loop 8.5 for 7.9.
template <int DT, int ACT, int BM, int BN> __global__ __launch_bounds__(256, 2) void linear_i8_staged_kernel(const LinearI8Args a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int WM = 2, WN = 2, TM = BM / WM / 16, TN = BN / WN / 16, UNITS = (BM + BN) * 8 / 256, STAGE = (BM + BN) * 128;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0), tiles = (a.k + 127) >> 7;
    const int chunk = threadIdx.x & 7;
    const unsigned char* from[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int r = (i * 256 + (int)threadIdx.x) >> 3;
        from[i] = i < BM / 32 ? a.x + (m0 + min(r, rows_x - 1)) * a.ldx : a.w + (long long)(n0 + min(r - BM, rows_w - 1)) * a.ldw;
    }
    u32x4_t unit[UNITS];
    auto request = [&](int t) {
        const int at = min(t * 128 + chunk * 16, a.k - 16);
#pragma unroll
        for (int i = 0; i < UNITS; ++i) __builtin_memcpy(&unit[i], from[i] + at, 16);
    };
    auto store = [&](int t) {
        if (t * 128 + 128 > a.k) {
            const int over = min(max(t * 128 + chunk * 16 + 16 - a.k, 0), 16);
#pragma unroll
            for (int i = 0; i < UNITS; ++i) unit[i] = drop_bytes(unit[i], over);
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int r = (i * 256 + (int)threadIdx.x) >> 3;
            *(u32x4_t*)(smem + (t & 1) * STAGE + r * 128 + ((chunk ^ (r & 7)) << 4)) = unit[i];
        }
    };
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned slot = (unsigned)((fgrp ^ (frow & 7)) << 4), x_frag = (unsigned)((wm * TM * 16 + frow) * 128) + slot,
                   w_frag = (unsigned)((BM + wn * TN * 16 + frow) * 128) + slot;
    i32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
    request(0);
    for (int t = 0; t < tiles; ++t) {
        store(t);  // (everyone has left this buffer: it was read before the last barrier)
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        request(t + 1);
        const unsigned base = (unsigned)((t & 1) * STAGE);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4_t xf[TM], wf[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[j] = lds_read((w_frag + base + j * 2048) ^ (h << 6));
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = lds_read((x_frag + base + i * 2048) ^ (h << 6));
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] = mma(wf[j], xf[i], acc[j][i]);
        }
    }
    __syncthreads();
    static_assert(4 * StagedRows<DT, TN>::BYTES <= 2 * STAGE, "staging fits");
    store_tile<DT, ACT, TM, TN>(a, acc, (int*)(smem + wave * StagedRows<DT, TN>::BYTES), m0 + wm * TM * 16, n0 + wn * TN * 16, NotAhead());
#endif
}

// The same for k < 16: one k-tile, byte by byte where there are less than 16.
template <int DT, int ACT> __global__ __launch_bounds__(256) void linear_i8_short_kernel(const LinearI8Args a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int BM = 64, BN = 64, TM = 2, TN = 2;
    __shared__ __align__(16) int staged[4][StagedRows<DT, TN>::BYTES / 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1, frow = lane & 15;
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM + wm * TM * 16;
    const int n0 = tile_n * BN + wn * TN * 16, live = lane < 16 ? a.k : 0;
    i32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const u32x4_t w = load_chunk<1>(a.w + (long long)min(n0 + j * 16 + frow, a.n - 1) * a.ldw, live);
            const u32x4_t x = load_chunk<1>(a.x + min(m0 + i * 16 + frow, a.m - 1ll) * a.ldx, live);
            acc[j][i] = mma(w, x, i32x4_t{0, 0, 0, 0});
        }
    store_tile<DT, ACT, TM, TN>(a, acc, staged[wave], m0, n0, NotAhead());
#endif
}

// ---- few tiles: K split over the wavefronts of a workgroup ---------------------------------------
// 16 TM x 16 TN outputs per workgroup; wavefront v takes k-tiles v, v + NW, ..., moves them into an LDS ring of its own and
// meets the others at the end only, where the partial tiles are added.  Bound by the L2 -> CU path (about 105 GB/s a CU here)
// and, for the fewest rows, the memory: 24x4096 -> 4096 in 6.3 us, 24x4096 -> 16384 in 12.9 (5.2 TB/s), 256x4096 -> 4096 in 10.6.
// (Fragments straight from memory to registers, without LDS: 7.9, 26 and 45 us: 64 bytes of a row at a time.)
// Aligned rows by loads that write LDS directly; others (k >= 16) through registers, the next k-tile on its way.
template <int DT, int ACT, int TM, int TN, int NW, int NS, bool DIRECT> __global__ __launch_bounds__(NW * 64, 1) void linear_i8_ksplit_kernel(const LinearI8Args a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int V = DT == SGPRS_BF16 ? 8 : 4, BM = 16 * TM, BN = 16 * TN, STAGE = (BM + BN) * 128, LA = BM / 8, LB = BN / 8, L = LA + LB;
    constexpr int SROW = BN + 4, LPR = BN / V;
    static_assert((NS - 1) * L <= 63, "vmcnt range");
    static_assert(BM * SROW * 4 <= NS * STAGE, "a partial tile fits the ring");
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tile_m, tile_n;
    tile_of(blockIdx.x, a.grid_m, a.grid_n, &tile_m, &tile_n);
    const long long m0 = (long long)tile_m * BM;
    const int n0 = tile_n * BN, tiles = (a.k + 127) >> 7;
    const int rows_x = (int)min((long long)BM, a.m - m0), rows_w = min(BN, a.n - n0);
    const int lrow = lane >> 3, chunk = (lane & 7) ^ lrow;
    const unsigned ring = (unsigned)(wave * NS * STAGE);
    const __amdgpu_buffer_rsrc_t x_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + m0 * a.ldx), 0, (rows_x - 1) * a.ldx + a.k, 0x00020000);
    const __amdgpu_buffer_rsrc_t w_rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + (long long)n0 * a.ldw), 0, (rows_w - 1) * a.ldw + a.k, 0x00020000);
    u32x4_t unit[DIRECT ? 1 : L];
    auto request = [&](int t, int slot) {
        if constexpr (DIRECT) {
            const bool live = t * 128 + chunk * 16 < a.k;
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int r = (i < LB ? i : i - LB) * 8 + lrow;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LB ? w_rs : x_rs, (lds_ptr_t)(smem + ring + slot * STAGE + i * 1024), 16,
                                                         live ? (unsigned)(r * (i < LB ? a.ldw : a.ldx) + chunk * 16) : kOutside, t * 128, 0, 0);
            }
        } else {  // rows past the end repeat the last one; a chunk that reaches past the end of its row is its last 16 bytes
            const int at = min(t * 128 + chunk * 16, a.k - 16);
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const unsigned char* from = i < LB ? a.w + (long long)(n0 + min(i * 8 + lrow, rows_w - 1)) * a.ldw : a.x + (m0 + min((i - LB) * 8 + lrow, rows_x - 1)) * a.ldx;
                __builtin_memcpy(&unit[i], from + at, 16);
            }
        }
    };
    i32x4_t acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
    const int frow = lane & 15, fgrp = lane >> 4;
    const unsigned w_frag = ring + (unsigned)(frow * 128) + (unsigned)((fgrp ^ (frow & 7)) << 4), x_frag = w_frag + BN * 128;
    // what this thread's first outputs need beside the sums (asked for behind the k loop: 24x4096 -> 16384 13.4 us for 12.9)
    const int c0 = (int)threadIdx.x % LPR * V, r0 = (int)threadIdx.x / LPR;
    const Columns<V> columns(a, n0 + c0);
    const float scale0 = row_scale(a, m0 + r0);
    const u32x4_t res0 = residual_at<V>(a, m0 + r0, n0 + c0);
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
            if (t * 128 + 128 > a.k) {
                const int over = min(max(t * 128 + chunk * 16 + 16 - a.k, 0), 16);
#pragma unroll
                for (int i = 0; i < L; ++i) unit[i] = drop_bytes(unit[i], over);
            }
#pragma unroll
            for (int i = 0; i < L; ++i) *(lds_u32x4_t*)(unsigned long)(ring + slot * STAGE + i * 1024 + lane * 16) = unit[i];
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
                for (int i = 0; i < TM; ++i) acc[j][i] = mma(wf[h][j], xf[h][i], acc[j][i]);
        slot = slot + 1 == NS ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(0);  // requests past the end write zeros into the ring
    int* mine = (int*)(smem + ring);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) *(i32x4_t*)(mine + (i * 16 + frow) * SROW + j * 16 + fgrp * 4) = acc[j][i];
    __syncthreads();
    static_assert(NW * 64 % LPR == 0, "a thread keeps its columns");
    for (int r = r0; r < BM; r += NW * 64 / LPR) {
        i32x4_t total[V / 4] = {};
#pragma unroll
        for (int v = 0; v < NW; ++v)
#pragma unroll
            for (int e = 0; e < V / 4; ++e) total[e] += *(const i32x4_t*)((const int*)(smem + v * NS * STAGE) + r * SROW + c0 + 4 * e);
        finish_row<DT, ACT>(a, m0 + r, n0 + c0, (const int*)total, r == r0 ? scale0 : row_scale(a, m0 + r), columns, r == r0 ? res0 : residual_at<V>(a, m0 + r, n0 + c0));
    }
#endif
}

// ---- plans -------------------------------------------------------------------------------------
// Integers are summed exactly in any order, but no kernel splits k over workgroups: with a join in a second launch 128x4096
// -> 4096 took 17 us, where the wavefronts of a workgroup split it in 8.5.
size_t linear_i8_workspace_bytes(const sgprs_linear_i8_desc_t&, int) { return 0; }

// direct: operands whose rows are whole aligned chunks.  The kernel with the least estimate, in us, fitted to measurements on
// 256 CUs (three sets of inputs in turn): what a launch takes, and what the busiest CU's tiles do, by their k-tiles.
// 256 / 128 / 64 square tiles, 64x64 / 32x32 / 16x16 with k split: 16384x4096 -> 4096 237 / 283 / 430 us, 12544x512 -> 2048
// 33 / 30 / 39, 2048x1024 -> 1024 19 / 9.5 / 7.1 / 10.8, 256x4096 -> 4096 43 / 23 (17 with four k-tiles) / 18 (10.6) / 10.6 / 22, 64x4096 ->
// 4096 42 / 23 / 17 / 9.9 / 7.3 / 17, 1x4096 -> 4096 39 / 21 / 16 / 8.8 / 6.2 / 5.7.
int plan_linear_i8(const sgprs_linear_i8_desc_t& d, int cus, bool direct, bool residual)
{
    if (d.k < 16) return kShort;
    const double kt = (d.k + 127) / 128;
    // k_alone, end_alone: of one tile with a CU to itself, k_shared, end: of each where CUs have several.  A tile alone waits
    // for its residual and twice the bytes of fp32; 4100x130 -> 520 in fp32 with a residual 128 / 64 square tiles 14.0 / 7.9 us.
    struct Tile { int kernel, b, bn; double k_alone, end_alone, k_shared, end; };
    static const Tile tiled[3] = {{kTile256, 256, 256, 1.0, 8, 1.5, 9}, {kTile128, 128, 128, 0.54, 2.9, 0.43, 2.6}, {kTile64, 64, 64, 0.42, 1.3, 0.2, 0.6}};
    static const Tile staged[3] = {{kStaged128, 128, 128, 1.6, 3, 0.9, 1.5}, {kStaged64, 64, 64, 0.87, 1.4, 0.42, 0.9}, {kStaged32, 32, 64, 0.5, 0.6, 0.35, 0.45}};
    const double wait = 1 + (d.dtype == SGPRS_F32 ? 0.5 : 0) + (residual ? 0.8 : 0);
    struct Split { int kernel, bm, bn; };
    static const Split split[7] = {{kSplit64x64, 64, 64}, {kSplit64x32, 64, 32}, {kSplit32x64, 32, 64}, {kSplit32x32, 32, 32}, {kSplit64x16, 64, 16}, {kSplit32x16, 32, 16}, {kSplit16x16, 16, 16}};
    auto tiles = [&](int bm, int bn) { return (double)((d.m + (long long)bm - 1) / bm) * ((d.n + bn - 1) / bn); };
    int best = direct ? kTile256 : kStaged128;
    double least = 1e300;
    auto offer = [&](int kernel, double us) {
        if (us >= least) return;
        least = us;
        best = kernel;
    };
    for (const Tile& t : tiled) {
        const double share = tiles(t.b, t.bn) / cus;
        if (direct) offer(t.kernel, 2.6 + std::max(kt * t.k_alone + t.end_alone * wait, (t.b == 256 ? std::ceil(share) : share) * (kt * t.k_shared + t.end)));
    }
    // four k-tiles in LDS instead of two, for a workgroup (128) or two (64) on a CU: alone, a k-tile is a round trip
    const double on128 = tiles(128, 128) / cus, on64 = std::ceil(tiles(64, 64) / cus);
    if (direct && kt > 4 && on128 <= 1) offer(kDeep128, 2.6 + kt * (0.34 + 0.18 * on128) + 3 * wait);
    if (direct && kt > 4 && on64 <= 2) offer(kDeep64, 2.6 + kt * 0.195 * on64 + 1.6 * wait);
    for (const Tile& t : staged)
        if (!direct) offer(t.kernel, 2.6 + std::max(kt * t.k_alone + t.end_alone * wait, tiles(t.b, t.bn) / cus * (kt * t.k_shared + t.end)));
    for (const Split& s : split)
        if (direct || s.kernel == kSplit64x64 || s.kernel == kSplit32x32 || s.kernel == kSplit16x16)
            offer(s.kernel, 3 + std::ceil(tiles(s.bm, s.bn) / cus) * (0.8 * (wait - 1) + (direct ? 2.3 + (s.bm + s.bn) * kt * 128 / 105e3 : 0.2 + (s.bm + s.bn) / 53. + (s.bm + s.bn) * kt * 128 / 45e3)));
    return best;
}

// By tiles of bm x bn outputs.  A launch has less than 2^32 threads: rows in bands.  (n is at most 2^20, so that a band has 127 row
// tiles or more.)
template <auto kernel> static int launch_sized(int lds, LinearI8Args a, int bm, int bn, int threads, hipStream_t stream)
{
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    a.grid_n = (a.n - 1) / bn + 1;
    const long long band = ((1ll << 32) - 1) / threads / a.grid_n * bm, m = a.m;
    for (long long done = 0; done < m; done += band) {
        a.m = (int)std::min(m - done, band);
        a.grid_m = (a.m - 1) / bm + 1;  // (m may be the largest int)
        SGPRS_LAUNCH(kernel, dim3((unsigned)((long long)a.grid_m * a.grid_n)), threads, lds, stream, a);
        SGPRS_HIP(hipGetLastError());
        a.x += band * a.ldx;
        a.y += band * a.ldy;
        if (a.x_scales) a.x_scales += band;
        if (a.residual) a.residual += band * a.ldr;
    }
    return SGPRS_OK;
}

template <int DT, int ACT, int BM, int BN, int NS> static int launch_tile(const LinearI8Args& a, hipStream_t stream)
{
    return launch_sized<linear_i8_tile_kernel<DT, ACT, BM, BN, NS>>(NS * (BM + BN) * 128, a, BM, BN, 256, stream);
}
template <int DT, int ACT, int BM, int BN> static int launch_staged(const LinearI8Args& a, hipStream_t stream)
{
    return launch_sized<linear_i8_staged_kernel<DT, ACT, BM, BN>>(2 * (BM + BN) * 128, a, BM, BN, 256, stream);
}
template <int DT, int ACT, bool DIRECT, int TM, int TN, int NW, int NS> static int launch_ksplit(const LinearI8Args& a, hipStream_t stream)
{
    return launch_sized<linear_i8_ksplit_kernel<DT, ACT, TM, TN, NW, NS, DIRECT>>(NW * NS * (TM + TN) * 2048, a, 16 * TM, 16 * TN, NW * 64, stream);
}

template <int DT, int ACT, bool DIRECT> static int launch_planned(const LinearI8Args& a, int kernel, hipStream_t stream)
{
    if (kernel == kShort) return launch_sized<linear_i8_short_kernel<DT, ACT>>(0, a, 64, 64, 256, stream);
    if constexpr (DIRECT) {
        switch (kernel) {
        case kTile256: return launch_tile<DT, ACT, 256, 256, 2>(a, stream);
        case kTile128: return launch_tile<DT, ACT, 128, 128, 2>(a, stream);
        case kTile64: return launch_tile<DT, ACT, 64, 64, 2>(a, stream);
        case kDeep128: return launch_tile<DT, ACT, 128, 128, 4>(a, stream);
        case kDeep64: return launch_tile<DT, ACT, 64, 64, 4>(a, stream);
        case kSplit32x16: return launch_ksplit<DT, ACT, true, 2, 1, 8, 3>(a, stream);
        case kSplit64x16: return launch_ksplit<DT, ACT, true, 4, 1, 4, 3>(a, stream);
        case kSplit64x32: return launch_ksplit<DT, ACT, true, 4, 2, 4, 3>(a, stream);
        case kSplit32x64: return launch_ksplit<DT, ACT, true, 2, 4, 4, 3>(a, stream);
        }
    } else {
        switch (kernel) {
        case kStaged128: return launch_staged<DT, ACT, 128, 128>(a, stream);
        case kStaged64: return launch_staged<DT, ACT, 64, 64>(a, stream);
        case kStaged32: return launch_staged<DT, ACT, 32, 64>(a, stream);
        }
    }
    switch (kernel) {
    case kSplit16x16: return launch_ksplit<DT, ACT, DIRECT, 1, 1, 8, DIRECT ? 4 : 1>(a, stream);
    case kSplit32x32: return launch_ksplit<DT, ACT, DIRECT, 2, 2, 8, DIRECT ? 2 : 1>(a, stream);
    case kSplit64x64: return launch_ksplit<DT, ACT, DIRECT, 4, 4, 4, 2>(a, stream);
    }
    return fail(SGPRS_ERR_UNSUPPORTED, "kernel %d", kernel);
}

template <int DT, bool DIRECT> static int launch_act(const LinearI8Args& a, int act, int kernel, hipStream_t stream)
{
    switch (act) {
    case SGPRS_ACT_RELU: return launch_planned<DT, SGPRS_ACT_RELU, DIRECT>(a, kernel, stream);
    case SGPRS_ACT_GELU: return launch_planned<DT, SGPRS_ACT_GELU, DIRECT>(a, kernel, stream);
    case SGPRS_ACT_SILU: return launch_planned<DT, SGPRS_ACT_SILU, DIRECT>(a, kernel, stream);
    default: return launch_planned<DT, SGPRS_ACT_NONE, DIRECT>(a, kernel, stream);
    }
}

int launch_linear_i8(const sgprs_linear_i8_desc_t& d, const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales,
                     const float* bias, const void* residual, void* y, void* ws, hipStream_t stream, int cus)
{
    const int es = (int)dtype_size(d.dtype);
    const LinearI8Args a = {(const unsigned char*)x, (const unsigned char*)w, x_scales, w_scales, bias, (const unsigned char*)residual, (unsigned char*)y,
                            d.m, d.n, d.k, (int)d.ldx, (int)d.ldw, (int)d.ldr * es, (int)d.ldy * es, d.residual_first, 0, 0};
    const bool direct = (((uintptr_t)x | (uintptr_t)w | (unsigned)a.ldx | (unsigned)a.ldw | (unsigned)a.k) & 15) == 0;
    const int kernel = plan_linear_i8(d, cus, direct, residual != nullptr);
    if (d.dtype == SGPRS_BF16)
        return direct ? launch_act<SGPRS_BF16, true>(a, d.act, kernel, stream) : launch_act<SGPRS_BF16, false>(a, d.act, kernel, stream);
    return direct ? launch_act<SGPRS_F32, true>(a, d.act, kernel, stream) : launch_act<SGPRS_F32, false>(a, d.act, kernel, stream);
}

}  // namespace sgprs
