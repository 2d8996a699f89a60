// Group norm with an activation (and residual), channels last.
//
// Bound by the memory: x in, y out.  A thread keeps to one vector of 16 bytes of channels and takes every
// step-th position of it, so that whatever the groups' width, rows are read whole and what a thread knows of
// its channels (mean, scale, shift) stays in registers.  Statistics are two passes over values in registers
// (sum, then squares of the deviations from the mean), so nothing cancels, whatever the mean:
//   * one launch where an image's positions of a slice of whole groups fit one workgroup's registers;
//   * else one launch for the statistics of chunks of positions (mean and sum of squares of each group, in the
//     workspace) and one that merges an image's chunks and writes the results; with many chunks, which every
//     workgroup would have to read, a launch between the two merges them;
//   * a norm over all channels of single positions (layer norm) is a wavefront per row.
// 64 images of 112 x 112 x 64 bf16 with residual and SiLU: 79 us, of launches of 19 (statistics, x once, 5.4 TB/s), 5 (the
// chunks) and 48 (results: x from the caches, residual, y, 6.4 TB/s).  12544 layer norms of 512 bf16 channels 6.6 us
// (3.9 TB/s; a copy of as much 4.2 at the rate of larger ones, 5 by itself); one map of 49 positions 3.6 to 4.2 us, a launch.
#include <algorithm>
#include <type_traits>

#include "block_ops.h"

namespace sgprs {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

struct NormArgs {
    const unsigned char* x;
    const float *gamma, *beta;
    const unsigned char* residual;
    unsigned char* y;
    float2* partial;         // [image][chunk][group]: mean, sum of the squared deviations
    float2* merged;          // [image][group]: mean, 1 / deviation; NULL: each workgroup merges the chunks itself
    int n, hw, c, groups, per;
    unsigned per_mul;
    int per_sh;              // channel / per
    long long ldx, ldr, ldy; // bytes
    float eps;
    int slice, vectors, step;  // channels of a slice, vectors of 16 bytes in it, positions that a workgroup takes at once
    unsigned vec_mul;
    int vec_sh;              // thread / vectors
    int slice_groups;
    int share_log2;          // lanes that add up a group
    int chunks;              // of an image's positions
};

// 1 / sqrt(v).  The instruction takes subnormal numbers, variances of values below 2^-63, for 0.
__device__ __forceinline__ float inverse_root(float v)
{
#if __HIP_DEVICE_COMPILE__
    const bool small = v < 0x1p-100f;
    return __builtin_amdgcn_rsqf(small ? v * 0x1p60f : v) * (small ? 0x1p30f : 1.f);
#else
    return v;
#endif
}

__device__ __forceinline__ int div_magic(int m, unsigned mul, int sh) { return (int)(__umulhi(2u * (unsigned)m, mul) >> sh); }

// WHOLE: the channels of every slice are whole vectors.  16-byte accesses need no alignment beyond the element's.
template <int DT, bool WHOLE> struct NormVec {
    static constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    // the first `live` of V channels at p
    static __device__ __forceinline__ u32x4_t load(const unsigned char* p, int live)
    {
        u32x4_t v = {0, 0, 0, 0};
        if (WHOLE || live == V) {
            __builtin_memcpy(&v, p, 16);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (e >= live) continue;
                if constexpr (ES == 2) v[e / 2] |= (unsigned)((const unsigned short*)p)[e] << (e % 2 * 16);
                else v[e] = ((const unsigned*)p)[e];
            }
        }
        return v;
    }
    static __device__ __forceinline__ void store(unsigned char* p, u32x4_t v, int live)
    {
        if (WHOLE || live == V) {
            __builtin_memcpy(p, &v, 16);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (e >= live) continue;
                if constexpr (ES == 2) ((unsigned short*)p)[e] = (unsigned short)(v[e / 2] >> (e % 2 * 16));
                else ((unsigned*)p)[e] = v[e];
            }
        }
    }
    // V floats of a per-channel array (NULL: `other`)
    static __device__ __forceinline__ void per_channel(const float* p, int live, float other, float* out)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = other;
        if (!p) return;
        if (WHOLE || live == V) {
            __builtin_memcpy(out, p, V * 4);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < live) out[e] = p[e];
        }
    }
    static __device__ __forceinline__ float get(const u32x4_t& v, int e)
    {
        if constexpr (ES == 4) return __uint_as_float(v[e]);
        else return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    }
    static __device__ __forceinline__ u32x4_t pack(const float* f)
    {
        u32x4_t v;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if constexpr (ES == 4) v[p] = __float_as_uint(f[p]);
            else v[p] = pack_bf16x2_relu(f[2 * p], f[2 * p + 1], kNoReluFloor);
        }
        return v;
    }
};

// (x - mean) * scale + shift (+ residual), activated and stored, for one vector.
template <int DT, int ACT, bool WHOLE>
__device__ __forceinline__ void finish_vector(const NormArgs& a, const u32x4_t& x, const u32x4_t& r, const float* mean, const float* scale,
                                              const float* shift, unsigned char* y, int live)
{
    typedef NormVec<DT, WHOLE> N;
    float o[N::V];
#pragma unroll
    for (int e = 0; e < N::V; ++e) {
        float z = (N::get(x, e) - mean[e]) * scale[e] + shift[e];
        if (a.residual) z += N::get(r, e);
        o[e] = activate<DT, ACT>(z);
    }
    N::store(y, N::pack(o), live);
}

// Sum over `share` neighbouring lanes (a power of two up to 64), in all of them.  Within 16 lanes by data-parallel
// moves: neighbours, pairs, then mirrored halves, which hold the same sums as the lanes beside them.
__device__ __forceinline__ float lanes_sum(float v, int share)
{
#if __HIP_DEVICE_COMPILE__
    auto moved = [](float x, auto control) {
        return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), decltype(control)::value, 0xf, 0xf, true));
    };
    if (share > 1) v += moved(v, std::integral_constant<int, 0xB1>());   // quad_perm 1 0 3 2
    if (share > 2) v += moved(v, std::integral_constant<int, 0x4E>());   // quad_perm 2 3 0 1
    if (share > 4) v += moved(v, std::integral_constant<int, 0x141>());  // row_half_mirror
    if (share > 8) v += moved(v, std::integral_constant<int, 0x140>());  // row_mirror
    if (share > 16) v += __shfl_xor(v, 16);
    if (share > 32) v += __shfl_xor(v, 32);
#endif
    return v;
}

// Sums over a workgroup, group by group: thread (s, v) brings V values of vector v (zeros for channels that do
// not exist); total[g] gets the sum of group g of the slice.  scratch: a float for every value.  All threads call it;
// `share` neighbouring lanes add up a group, in a fixed order.
template <int V>
__device__ __forceinline__ void group_sums(const NormArgs& a, const float* value, int groups, float* scratch, float* total)
{
    const int tid = threadIdx.x, T = blockDim.x;
    const bool whole = a.per % V == 0;  // a vector lies within one group
    if (whole) {
        float s = value[0];
#pragma unroll
        for (int e = 1; e < V; ++e) s += value[e];
        scratch[tid] = s;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) scratch[tid * V + e] = value[e];
    }
    __syncthreads();
    const int row = whole ? a.vectors : a.vectors * V, width = whole ? a.per / V : a.per;  // of a position's values, of a group's
    const int share = 1 << a.share_log2, part = tid & (share - 1);
    for (int g0 = 0; g0 < groups; g0 += T >> a.share_log2) {
        const int g = g0 + (tid >> a.share_log2);
        float s = 0.f;
        if (g < groups) {
            const float* at = scratch + g * width;
            if (width == 1) {
#pragma unroll 4
                for (int p = part; p < a.step; p += share) s += at[p * row];
            } else if (width == 2) {
#pragma unroll 4
                for (int p = part; p < a.step; p += share) s += at[p * row] + at[p * row + 1];
            } else {
                for (int p = part; p < a.step; p += share)
#pragma unroll 4
                    for (int i = 0; i < width; ++i) s += at[p * row + i];
            }
        }
        s = lanes_sum(s, share);
        if (g < groups && part == 0) total[g] = s;
    }
    __syncthreads();
}

// A workgroup's share: positions `first` and on of an image, channels c0 and on; a thread's vector and first position.
// Loads of positions past the end repeat the last one, so that they need no branch; threads beyond the last whole
// step repeat vector 0.
template <int DT, bool WHOLE, int NV> struct NormShare {
    typedef NormVec<DT, WHOLE> N;
    int c0, channels, groups, image, first, rows, s, v, live;
    long long row0;
    __device__ __forceinline__ NormShare(const NormArgs& a)
    {
        const int tid = threadIdx.x;
        c0 = blockIdx.y * a.slice;
        channels = min(a.slice, a.c - c0);
        groups = a.slice_groups;
        if (channels < a.slice) groups = channels / a.per;
        image = blockIdx.z;
        first = blockIdx.x * a.step * NV;
        rows = min(a.step * NV, a.hw - first);
        s = div_magic(tid, a.vec_mul, a.vec_sh);
        v = tid - s * a.vectors;
        live = s < a.step ? min(N::V, channels - v * N::V) : 0;
        if (WHOLE && channels < a.slice && v * N::V >= channels) live = 0;
        row0 = (long long)image * a.hw + first;
    }
    __device__ __forceinline__ bool has(const NormArgs& a, int k) const { return live > 0 && s + k * a.step < rows; }
    __device__ __forceinline__ void load(const NormArgs& a, const unsigned char* base, long long ld, u32x4_t* x) const
    {
        const unsigned char* p = base + row0 * ld + (long long)(c0 + (live > 0 ? v * N::V : 0)) * N::ES;
#pragma unroll
        for (int k = 0; k < NV; ++k) x[k] = N::load(p + min(s + k * a.step, rows - 1) * ld, live);
    }
};

// Statistics of a chunk of positions and a slice of channels, NV positions a thread; with FUSED the chunk is the
// image and the results follow from the registers.
template <int DT, int ACT, bool WHOLE, int NV, bool FUSED> __global__ __launch_bounds__(1024) void group_norm_chunk_kernel(const NormArgs a)
{
    typedef NormVec<DT, WHOLE> N;
    constexpr int V = N::V;
    extern __shared__ __align__(16) float lds[];
    const int tid = threadIdx.x, T = blockDim.x;
    const NormShare<DT, WHOLE, NV> m(a);
    float* total = lds + T * V;  // per group of the slice
    constexpr bool EARLY = FUSED && NV < 8;  // the residual is requested with x where there are registers for it
    u32x4_t x[NV], r[EARLY ? NV : 1];
    m.load(a, a.x, a.ldx, x);
    if constexpr (EARLY) {
        if (a.residual) m.load(a, a.residual, a.ldr, r);
    }
    float gamma[V], beta[V];
    const int c = m.c0 + (m.live > 0 ? m.v * V : 0);
    if constexpr (FUSED) {
        N::per_channel(a.gamma ? a.gamma + c : nullptr, m.live, 1.f, gamma);
        N::per_channel(a.beta ? a.beta + c : nullptr, m.live, 0.f, beta);
    }
    float sum[V], sq[V], mean[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = sq[e] = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = __builtin_fmaf(N::get(x[k], e), m.has(a, k) ? 1.f : 0.f, sum[e]);  // (what a load repeats is of the same group)
    group_sums<V>(a, sum, m.groups, lds, total);
    const float inv_count = 1.f / ((float)m.rows * (float)a.per);
    int group[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        group[e] = div_magic(max(0, min(m.v * V + e, m.channels - 1)), a.per_mul, a.per_sh);
        mean[e] = total[group[e]] * inv_count;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float t = N::get(x[k], e) - mean[e];
            sq[e] = __builtin_fmaf((WHOLE || e < m.live) && m.has(a, k) ? t : 0.f, t, sq[e]);
        }
    float2* partial = a.partial + ((long long)m.image * a.chunks + blockIdx.x) * a.groups + blockIdx.y * a.slice_groups;
    if constexpr (!FUSED) {
        for (int g = tid; g < m.groups; g += T) partial[g].x = total[g] * inv_count;
    }
    __syncthreads();  // total has been read and is written again
    group_sums<V>(a, sq, m.groups, lds, total);
    if constexpr (!FUSED) {
        for (int g = tid; g < m.groups; g += T) partial[g].y = total[g];
    } else if (m.live > 0) {
#pragma unroll
        for (int e = 0; e < V; ++e) gamma[e] *= inverse_root(total[group[e]] * inv_count + a.eps);
        unsigned char* yp = a.y + m.row0 * a.ldy + (long long)c * N::ES;
        const unsigned char* rp = a.residual + m.row0 * a.ldr + (long long)c * N::ES;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!m.has(a, k)) continue;
            if constexpr (!EARLY) {
                if (a.residual) r[0] = N::load(rp + (m.s + k * a.step) * a.ldr, m.live);
            }
            finish_vector<DT, ACT, WHOLE>(a, x[k], r[EARLY ? k : 0], mean, gamma, beta, yp + (m.s + k * a.step) * a.ldy, m.live);
        }
    }
}

// Merges the chunks of a group of an image, over the lanes of a workgroup in a fixed order; all but the last chunk
// count `full` positions.
__global__ __launch_bounds__(256) void group_norm_merge_kernel(const NormArgs a, int full)
{
    __shared__ float sums[8];
    const int tid = threadIdx.x, group = blockIdx.x, image = blockIdx.y, last = a.hw - (a.chunks - 1) * full;
    const float2* from = a.partial + (long long)image * a.chunks * a.groups + group;
    const float inv_hw = 1.f / (float)a.hw;
    auto count = [&](int k) { return (float)(k == a.chunks - 1 ? last : full); };
    auto all = [&](float v, float* s) {
        v = lanes_sum(v, 64);
        if ((tid & 63) == 0) s[tid >> 6] = v;
        __syncthreads();
        return (s[0] + s[1]) + (s[2] + s[3]);
    };
    float mean = 0.f, m2 = 0.f;
#pragma unroll 4
    for (int k = tid; k < a.chunks; k += 256) mean += from[(long long)k * a.groups].x * count(k);
    mean = all(mean, sums) * inv_hw;
#pragma unroll 4
    for (int k = tid; k < a.chunks; k += 256) {
        const float2 one = from[(long long)k * a.groups];
        m2 += one.y + (one.x - mean) * (one.x - mean) * (count(k) * (float)a.per);
    }
    m2 = all(m2, sums + 4);
    if (tid == 0) a.merged[(long long)image * a.groups + group] = make_float2(mean, inverse_root(m2 * inv_hw / (float)a.per + a.eps));
}

// Merges an image's chunks, if that is not done, and writes the results of one of them.
template <int DT, int ACT, bool WHOLE, int NV> __global__ __launch_bounds__(1024) void group_norm_apply_kernel(const NormArgs a)
{
    typedef NormVec<DT, WHOLE> N;
    constexpr int V = N::V;
    extern __shared__ __align__(16) float lds[];
    const int tid = threadIdx.x, T = blockDim.x;
    const NormShare<DT, WHOLE, NV> m(a);
    const int groups = m.groups, full = a.step * NV;
    u32x4_t x[NV], r[NV];
    m.load(a, a.x, a.ldx, x);
    if (a.residual) m.load(a, a.residual, a.ldr, r);
    float gamma[V], beta[V], mean[V];
    const int c = m.c0 + (m.live > 0 ? m.v * V : 0);
    N::per_channel(a.gamma ? a.gamma + c : nullptr, m.live, 1.f, gamma);
    N::per_channel(a.beta ? a.beta + c : nullptr, m.live, 0.f, beta);
    // Chunks of a group: `share` neighbouring lanes, in order.  All chunks but the last count `full` positions.
    const float2* partial = a.partial + (long long)m.image * a.chunks * a.groups + blockIdx.y * a.slice_groups;
    float *means = lds, *scales = means + groups;
    const float inv_hw = 1.f / (float)a.hw;
    const int last = a.hw - (a.chunks - 1) * full;
    const int share = 1 << a.share_log2, part = tid & (share - 1);
    if (a.merged) {
        const float2* merged = a.merged + (long long)m.image * a.groups + blockIdx.y * a.slice_groups;
        for (int g = tid; g < groups; g += T) {
            means[g] = merged[g].x;
            scales[g] = merged[g].y;
        }
    }
    for (int g0 = a.merged ? groups : 0; g0 < groups; g0 += T >> a.share_log2) {
        const int g = g0 + (tid >> a.share_log2);
        const float2* from = partial + min(g, groups - 1);
        float mean = 0.f, m2 = 0.f;
#pragma unroll 4
        for (int k = part; k < a.chunks; k += share) mean += from[(long long)k * a.groups].x * (float)(k == a.chunks - 1 ? last : full);
        mean = lanes_sum(mean, share) * inv_hw;
#pragma unroll 4
        for (int k = part; k < a.chunks; k += share) {
            const float2 one = from[(long long)k * a.groups];
            m2 += one.y + (one.x - mean) * (one.x - mean) * ((float)(k == a.chunks - 1 ? last : full) * (float)a.per);
        }
        m2 = lanes_sum(m2, share);
        if (g < groups && part == 0) {
            means[g] = mean;
            scales[g] = inverse_root(m2 * inv_hw / (float)a.per + a.eps);
        }
    }
    __syncthreads();
    if (m.live <= 0) return;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int g = div_magic(min(m.v * V + e, m.channels - 1), a.per_mul, a.per_sh);
        mean[e] = means[g];
        gamma[e] *= scales[g];
    }
    unsigned char* yp = a.y + m.row0 * a.ldy + (long long)c * N::ES;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (m.has(a, k)) finish_vector<DT, ACT, WHOLE>(a, x[k], r[k], mean, gamma, beta, yp + (m.s + k * a.step) * a.ldy, m.live);
}

// One group over single positions: a wavefront per row, NV vectors a lane, the next row requested before this one's sums.
template <int DT, int ACT, bool WHOLE, int NV> __global__ __launch_bounds__(256) void row_norm_kernel(const NormArgs a)
{
    typedef NormVec<DT, WHOLE> N;
    constexpr int V = N::V;
    const int lane = threadIdx.x & 63;
    int c[NV], live[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        live[k] = max(0, min(V, a.c - (lane + 64 * k) * V));
        c[k] = live[k] ? (lane + 64 * k) * V : 0;
    }
    auto load = [&](const unsigned char* base, long long ld, long long row, u32x4_t* x) {
#pragma unroll
        for (int k = 0; k < NV; ++k) x[k] = N::load(base + row * ld + c[k] * N::ES, live[k]);
    };
    const long long step = (long long)gridDim.x * 4;
    long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.n) return;
    u32x4_t x[NV], r[NV];
    load(a.x, a.ldx, row, x);
    if (a.residual) load(a.residual, a.ldr, row, r);
    float gamma[NV][V], beta[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        N::per_channel(a.gamma ? a.gamma + c[k] : nullptr, live[k], 1.f, gamma[k]);
        N::per_channel(a.beta ? a.beta + c[k] : nullptr, live[k], 0.f, beta[k]);
    }
    const float inv_c = 1.f / (float)a.c;
    for (;;) {
        const long long next = row + step;
        u32x4_t x1[NV], r1[NV];
        if (next < a.n) {
            load(a.x, a.ldx, next, x1);
            if (a.residual) load(a.residual, a.ldr, next, r1);
        }
        float sum = 0.f, sq = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sum += live[k] ? N::get(x[k], e) : 0.f;
        const float mean1 = lanes_sum(sum, 64) * inv_c;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float t = N::get(x[k], e) - mean1;
                sq += (WHOLE ? live[k] > 0 : e < live[k]) ? t * t : 0.f;
            }
        const float inv = inverse_root(lanes_sum(sq, 64) * inv_c + a.eps);
        float mean[V];
#pragma unroll
        for (int e = 0; e < V; ++e) mean[e] = mean1;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float scale[V];
#pragma unroll
            for (int e = 0; e < V; ++e) scale[e] = inv * gamma[k][e];
            if (live[k]) finish_vector<DT, ACT, WHOLE>(a, x[k], r[k], mean, scale, beta[k], a.y + row * a.ldy + c[k] * N::ES, live[k]);
        }
        if (next >= a.n) return;
        row = next;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            x[k] = x1[k];
            r[k] = r1[k];
        }
    }
}

// ---- plans -------------------------------------------------------------------------------------
struct NormPlan {
    int rows;      // vectors a lane of the row kernel, 0: another kernel
    bool fused, merge;
    int threads, nv, slice, vectors, step, chunks, slices;
};

static NormPlan plan_norm(const sgprs_group_norm_desc_t& d, int cus)
{
    NormPlan p = {};
    const int V = 16 / (int)dtype_size(d.dtype), per = d.c / d.groups;
    if (d.hw == 1 && d.groups == 1 && d.c <= 64 * V * 8) {
        const int need = (d.c + 64 * V - 1) / (64 * V);
        p.rows = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
        return p;
    }
    auto vectors = [&](int slice) { return (slice + V - 1) / V; };
    auto slice_of = [&](int bytes) {  // whole groups, at least so many bytes, whole vectors where that is possible
        int s = (bytes / (int)dtype_size(d.dtype) + per - 1) / per * per;
        for (int i = 0; i < V && s % V && s < d.c; ++i) s += per;
        return std::min(s, d.c);
    };
    // One launch: the widest slices of up to 512 bytes a position that give every CU a workgroup and fit its registers
    // (8192 vectors), else slices of 64 bytes; those up to 2048 vectors, beyond which half lines and one workgroup's own
    // speed cost more than a second launch (64 images of 784 positions, 128 channels bf16: 18.4 us against 14.9; one
    // image 14.2 against 9.5; in slices of 128 bytes, fp32, 12.3 against 16.5).
    for (int bytes : {512, 256, 128, 64}) {
        const int s = slice_of(bytes), v = vectors(s), count = (d.c + s - 1) / s;
        if (v > 1024) continue;
        if (d.hw > (1024 / v) * 8 || (bytes == 64 && (long long)d.hw * v > 2048)) continue;
        if (bytes > 64 && (long long)count * d.n < cus) continue;
        p.fused = true;
        p.slice = s;
        break;
    }
    if (!p.fused) {
        p.slice = d.c;
        if (vectors(d.c) > 512) p.slice = std::max(per, 512 * V / per * per);
    }
    p.vectors = vectors(p.slice);
    p.slices = (d.c + p.slice - 1) / p.slice;
    if (p.fused) {
        p.threads = 64;
        auto holds = [&](int threads, int nv) { return threads >= p.vectors && (long long)(threads / p.vectors) * nv >= d.hw; };
        while (p.threads < 1024 && !holds(p.threads, p.threads < 256 ? 1 : p.threads < 512 ? 2 : 4)) p.threads *= 2;
        p.nv = 1;
        while (p.nv < 8 && !holds(p.threads, p.nv)) p.nv *= 2;
    } else {
        p.threads = p.vectors > 512 ? 1024 : p.vectors > 256 ? 512 : 256;
        p.nv = 8;
    }
    p.step = std::max(1, p.threads / p.vectors);
    p.chunks = (d.hw - 1) / (p.step * p.nv) + 1;  // (hw may be the largest int)
    // Workgroups that merge the chunks themselves read n slices chunks^2 groups pairs from the caches, twice; a launch of its
    // own for that costs 3 us.  Worth it from 40 KB a CU on; without it / with it, 256 CUs, 32 groups: one image of 12544
    // positions, 64 channels bf16 (1 MB) 10.4 / 11.7 us, 8 of them (10 MB) 15.1 / 15.1, 64 (79 MB) 90.7 / 78.6; one of 3136,
    // 512 channels fp32 (20 MB) 12.8 / 11.5, of 12544 (315 MB) 77 / 18.7.
    p.merge = !p.fused && 16.0 * d.n * p.slices * p.chunks * p.chunks * (p.slice / per) > 40e3 * cus;
    return p;
}

size_t group_norm_workspace_bytes(const sgprs_group_norm_desc_t& d, int cus)
{
    const NormPlan p = plan_norm(d, cus);
    return p.rows || p.fused ? 0 : (size_t)d.n * (p.chunks + (p.merge ? 1 : 0)) * d.groups * sizeof(float2);
}

template <int DT, int ACT, bool WHOLE> static int launch_norm(const NormArgs& a, const NormPlan& p, int cus, hipStream_t stream)
{
    constexpr int V = NormVec<DT, WHOLE>::V;
    if (p.rows) {
        const dim3 grid(std::min((a.n - 1) / 4 + 1, 8 * cus));
        switch (p.rows) {
        case 1: SGPRS_LAUNCH((row_norm_kernel<DT, ACT, WHOLE, 1>), grid, 256, 0, stream, a); break;
        case 2: SGPRS_LAUNCH((row_norm_kernel<DT, ACT, WHOLE, 2>), grid, 256, 0, stream, a); break;
        case 4: SGPRS_LAUNCH((row_norm_kernel<DT, ACT, WHOLE, 4>), grid, 256, 0, stream, a); break;
        default: SGPRS_LAUNCH((row_norm_kernel<DT, ACT, WHOLE, 8>), grid, 256, 0, stream, a);
        }
    } else {
        const dim3 grid(p.chunks, p.slices, a.n);
        const size_t lds = sizeof(float) * ((size_t)p.threads * V + 2 * a.slice_groups);
        if (p.fused) {
            switch (p.nv) {
            case 1: SGPRS_LAUNCH((group_norm_chunk_kernel<DT, ACT, WHOLE, 1, true>), grid, p.threads, lds, stream, a); break;
            case 2: SGPRS_LAUNCH((group_norm_chunk_kernel<DT, ACT, WHOLE, 2, true>), grid, p.threads, lds, stream, a); break;
            case 4: SGPRS_LAUNCH((group_norm_chunk_kernel<DT, ACT, WHOLE, 4, true>), grid, p.threads, lds, stream, a); break;
            default: SGPRS_LAUNCH((group_norm_chunk_kernel<DT, ACT, WHOLE, 8, true>), grid, p.threads, lds, stream, a);
            }
        } else {
            SGPRS_LAUNCH((group_norm_chunk_kernel<DT, SGPRS_ACT_NONE, WHOLE, 8, false>), grid, p.threads, lds, stream, a);
            if (p.merge) SGPRS_LAUNCH(group_norm_merge_kernel, dim3(a.groups, a.n), 256, 0, stream, a, p.step * p.nv);
            SGPRS_LAUNCH((group_norm_apply_kernel<DT, ACT, WHOLE, 8>), grid, p.threads, lds, stream, a);
        }
    }
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

template <int DT, bool WHOLE> static int launch_norm_act(const NormArgs& a, const NormPlan& p, int act, int cus, hipStream_t stream)
{
    switch (act) {
    case SGPRS_ACT_RELU: return launch_norm<DT, SGPRS_ACT_RELU, WHOLE>(a, p, cus, stream);
    case SGPRS_ACT_GELU: return launch_norm<DT, SGPRS_ACT_GELU, WHOLE>(a, p, cus, stream);
    case SGPRS_ACT_SILU: return launch_norm<DT, SGPRS_ACT_SILU, WHOLE>(a, p, cus, stream);
    default: return launch_norm<DT, SGPRS_ACT_NONE, WHOLE>(a, p, cus, stream);
    }
}

// Images that a launch takes: its grid's third dimension.
constexpr int kMaxImages = 65535;

int launch_group_norm(const sgprs_group_norm_desc_t& d, const void* x, const float* gamma, const float* beta, const void* residual, void* y,
                      void* ws, hipStream_t stream, int cus)
{
    const NormPlan p = plan_norm(d, cus);
    if (!p.rows && (p.slices > 65535 || (long long)p.chunks * p.threads >= (1ll << 32)))
        return fail(SGPRS_ERR_UNSUPPORTED, "%d images of %d positions and %d channels", d.n, d.hw, d.c);
    const long long es = (long long)dtype_size(d.dtype);
    const int V = 16 / (int)es;
    NormArgs a = {(const unsigned char*)x, gamma, beta, (const unsigned char*)residual, (unsigned char*)y, (float2*)ws,
                  p.merge ? (float2*)ws + (size_t)d.n * p.chunks * d.groups : nullptr, d.n, d.hw, d.c, d.groups,
                  d.c / d.groups, 0, 0, d.ldx * es, d.ldr * es, d.ldy * es, d.eps, p.slice, p.vectors, p.step, 0, 0, 0, 0, p.chunks};
    div_constants(a.per, &a.per_mul, &a.per_sh);
    if (!p.rows) {
        div_constants(p.vectors, &a.vec_mul, &a.vec_sh);
        a.slice_groups = p.slice / a.per;
        while (a.share_log2 < 6 && (2 << a.share_log2) * a.slice_groups <= p.threads) ++a.share_log2;
    }
    const bool whole = d.c % V == 0 && (p.rows || p.slice % V == 0);
    for (long long first = 0; first < d.n; first += kMaxImages) {
        NormArgs part = a;
        if (!p.rows) {
            const long long positions = first * d.hw;
            part.n = (int)std::min<long long>(kMaxImages, d.n - first);
            part.x += positions * a.ldx;
            if (a.residual) part.residual += positions * a.ldr;
            part.y += positions * a.ldy;
            part.partial += first * p.chunks * d.groups;
            if (p.merge) part.merged += first * d.groups;
        }
        int rc;
        if (d.dtype == SGPRS_BF16)
            rc = whole ? launch_norm_act<SGPRS_BF16, true>(part, p, d.act, cus, stream) : launch_norm_act<SGPRS_BF16, false>(part, p, d.act, cus, stream);
        else
            rc = whole ? launch_norm_act<SGPRS_F32, true>(part, p, d.act, cus, stream) : launch_norm_act<SGPRS_F32, false>(part, p, d.act, cus, stream);
        if (rc || p.rows) return rc;
    }
    return SGPRS_OK;
}

}  // namespace sgprs
