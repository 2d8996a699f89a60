// Root-mean-square norm of rows with the residual's addition, and rows of 8-bit integers with a scale each.
//
// A row is read once and kept in the registers of a wavefront or a workgroup (rows beyond that are read twice).  The sum of
// squares and the largest value are held in 64 bits, where no square of a 32-bit number overflows or vanishes.
// With t = h gamma a row's integers are 127 t / max|t|: the norm's factor cancels, so they need no statistics but the
// maximum, and in 64 bits t is exact, so that they are those of the definition whatever the order of anything.
#include <algorithm>

#include "decode_ops.h"

namespace sgprs {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

enum RowKind { kNorm, kNormI8, kQuantize };

struct RowArgs {
    const unsigned char *x, *residual;
    const float* gamma;
    unsigned char *sum, *y;
    float* scales;
    int m, c;
    long long ldx, ldr, ldh, ldy;  // bytes
    float eps;
};

// Vectors of 16 bytes of a row, of which the last one may be cut; rows at any alignment of their elements.
template <int DT> struct RowVec {
    static constexpr int ES = DT == SGPRS_BF16 ? 2 : 4, V = 16 / ES;
    static __device__ __forceinline__ u32x4_t load(const unsigned char* p, int live)
    {
        u32x4_t v = {0, 0, 0, 0};
        if (live >= V) {
            __builtin_memcpy(&v, p, 16);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (e >= live) continue;
                if constexpr (ES == 2) v[e / 2] |= (unsigned)*(const unsigned short*)(p + e * 2) << (e % 2 * 16);
                else v[e] = *(const unsigned*)(p + e * 4);
            }
        }
        return v;
    }
    static __device__ __forceinline__ void store(unsigned char* p, u32x4_t v, int live)
    {
        if (live >= V) {
            __builtin_memcpy(p, &v, 16);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (e >= live) continue;
                if constexpr (ES == 2) *(unsigned short*)(p + e * 2) = (unsigned short)(v[e / 2] >> (e % 2 * 16));
                else *(unsigned*)(p + e * 4) = v[e];
            }
        }
    }
    static __device__ __forceinline__ float get(u32x4_t v, int e)
    {
        if constexpr (ES == 2) return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
        else return __uint_as_float(v[e]);
    }
    static __device__ __forceinline__ u32x4_t pack(const float* z)
    {
        u32x4_t v;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if constexpr (ES == 2) v[p] = pack_bf16x2_relu(z[2 * p], z[2 * p + 1], kNoReluFloor);
            else v[p] = __float_as_uint(z[p]);
        }
        return v;
    }
    static __device__ __forceinline__ void store_i8(unsigned char* p, const int* q, int live)
    {
        unsigned w[V / 4];
#pragma unroll
        for (int d = 0; d < V / 4; ++d)
            w[d] = (q[4 * d] & 255u) | (q[4 * d + 1] & 255u) << 8 | (q[4 * d + 2] & 255u) << 16 | (unsigned)q[4 * d + 3] << 24;
        if (live >= V) {
            __builtin_memcpy(p, w, V);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < live) p[e] = (unsigned char)(w[e / 4] >> (e % 4 * 8));
        }
    }
};

// What a row comes to, joined over its THREADS threads in a fixed order.
struct RowStat {
    double squares, most;
    int odd;  // an infinity or a NaN among the t
};
template <int THREADS> __device__ __forceinline__ RowStat join(RowStat s, RowStat* shared)
{
#if __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int x = 32; x; x >>= 1) {
        s.squares += __shfl_xor(s.squares, x);
        s.most = fmax(s.most, __shfl_xor(s.most, x));
    }
    s.odd = __any(s.odd);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
        __syncthreads();
        s = shared[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) {
            s.squares += shared[w].squares;
            s.most = fmax(s.most, shared[w].most);
            s.odd |= shared[w].odd;
        }
    }
#endif
    return s;
}

// THREADS threads a row (a wavefront: four rows a workgroup), VPT vectors of it each; VPT 0: as many as it takes, read twice.
template <int DT, int KIND, int THREADS, int VPT> __global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void rms_norm_kernel(const RowArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef RowVec<DT> Vec;
    constexpr int V = Vec::V, ES = Vec::ES;
    __shared__ RowStat shared[THREADS / 64];
    const int thread = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int row = THREADS == 64 ? blockIdx.x * 4 + (int)(threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.m) return;
    const unsigned char* xp = a.x + row * a.ldx;
    const unsigned char* rp = KIND != kQuantize && a.residual ? a.residual + row * a.ldr : nullptr;
    unsigned char* hp = KIND != kQuantize && a.sum ? a.sum + row * a.ldh : nullptr;
    unsigned char* yp = a.y + row * a.ldy;
    const int vectors = (a.c + V - 1) / V;

    auto stream = [&](int v) {  // h
        const int live = a.c - v * V;
        u32x4_t h = Vec::load(xp + (long long)v * 16, live);
        if (rp) {
            const u32x4_t r = Vec::load(rp + (long long)v * 16, live);
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = Vec::get(h, e) + Vec::get(r, e);
            h = Vec::pack(z);
        }
        return h;
    };
    auto load_gamma = [&](int v, float* g) {
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = KIND != kQuantize && a.gamma && v * V + e < a.c ? a.gamma[v * V + e] : 1.f;
    };
    RowStat stat = {0.0, 0.0, 0};
    auto take = [&](int v, u32x4_t h) {
        if (hp) Vec::store(hp + (long long)v * 16, h, a.c - v * V);
        float g[V];
        if constexpr (KIND == kNormI8) load_gamma(v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double f = Vec::get(h, e);
            if constexpr (KIND != kQuantize) stat.squares = __builtin_fma(f, f, stat.squares);
            if constexpr (KIND != kNorm) {
                const double t = KIND == kNormI8 ? f * (double)g[e] : f;
                stat.most = fmax(stat.most, fabs(t));
                stat.odd |= !(fabs(t) < (double)INFINITY);
            }
        }
    };
    u32x4_t kept[VPT > 0 ? VPT : 1];
    if constexpr (VPT > 0) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) kept[i] = thread + i * THREADS < vectors ? stream(thread + i * THREADS) : u32x4_t{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (thread + i * THREADS < vectors) take(thread + i * THREADS, kept[i]);
    } else {
        for (int v = thread; v < vectors; v += THREADS) take(v, stream(v));
    }
    stat = join<THREADS>(stat, shared);

    double factor = 1.0;  // 1 / root mean square
    if constexpr (KIND != kQuantize) factor = 1.0 / sqrt(stat.squares / a.c + (double)a.eps);
    const bool odd = KIND != kNorm && (stat.odd || !(stat.squares < (double)INFINITY));
    if constexpr (KIND != kNorm) {
        if (thread == 0) a.scales[row] = odd ? NAN : (float)(stat.most * factor / 127.0);
    }
    // h * factor in 32 bits: the factor as a power of two, which takes h to its place, and a number of 1 to 2
    int power = 0;
    float scale = 1.f;
    if constexpr (KIND == kNorm) {
        const bool fine = factor > 0.0 && factor < (double)INFINITY;
        power = fine ? ilogb(factor) : 0;
        scale = (float)(fine ? ldexp(factor, -power) : factor);
    }
    const double step = KIND != kNorm && stat.most > 0.0 ? 127.0 / stat.most : 0.0;
    auto finish = [&](int v, u32x4_t h) {
        const int live = a.c - v * V;
        float g[V];
        load_gamma(v, g);
        if constexpr (KIND == kNorm) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = __builtin_amdgcn_ldexpf(Vec::get(h, e), power) * scale * g[e];
            Vec::store(yp + (long long)v * 16, Vec::pack(z), live);
        } else {
            int q[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const double t = KIND == kNormI8 ? (double)Vec::get(h, e) * (double)g[e] : (double)Vec::get(h, e);
                const double u = t * step, whole = rint(u);
                // u is off by less than 2^-45: next to a border between two integers the quotient itself decides
                q[e] = odd ? 0 : (int)(fabs(u - whole) > 0.5 - 0x1p-40 ? rint(127.0 * t / stat.most) : whole);
            }
            Vec::store_i8(yp + (long long)v * V, q, live);
        }
    };
    if constexpr (VPT > 0) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (thread + i * THREADS < vectors) finish(thread + i * THREADS, kept[i]);
    } else {
        for (int v = thread; v < vectors; v += THREADS) finish(v, hp ? Vec::load(hp + (long long)v * 16, a.c - v * V) : stream(v));
    }
#endif
}

template <int DT, int KIND, int THREADS, int VPT> static int launch_rows_as(const RowArgs& a, hipStream_t stream)
{
    const int grid = THREADS == 64 ? (a.m - 1) / 4 + 1 : a.m;
    // a launch has less than 2^32 threads: rows in runs
    constexpr int kRun = THREADS == 64 ? 1 << 23 : 1 << 21;
    for (int done = 0; done < grid;) {
        const int now = std::min(grid - done, kRun);
        RowArgs part = a;
        const long long rows = (long long)done * (THREADS == 64 ? 4 : 1);
        part.x += rows * a.ldx;
        if (a.residual) part.residual += rows * a.ldr;
        if (a.sum) part.sum += rows * a.ldh;
        part.y += rows * a.ldy;
        if (a.scales) part.scales += rows;
        part.m = (int)(a.m - rows);
        SGPRS_LAUNCH((rms_norm_kernel<DT, KIND, THREADS, VPT>), dim3((unsigned)now), THREADS == 64 ? 256 : THREADS, 0, stream, part);
        SGPRS_HIP(hipGetLastError());
        done += now;
    }
    return SGPRS_OK;
}

template <int DT, int KIND> static int launch_rows(const RowArgs& a, hipStream_t stream, int cus)
{
    constexpr int V = RowVec<DT>::V;
    const int vectors = (a.c - 1) / V + 1;
    if (vectors > 8192) return launch_rows_as<DT, KIND, 1024, 0>(a, stream);
    if (vectors > 2048) return launch_rows_as<DT, KIND, 1024, 8>(a, stream);
    if (vectors > 1024) return launch_rows_as<DT, KIND, 256, 8>(a, stream);
    if (a.m < 4 * cus && vectors > 64) return launch_rows_as<DT, KIND, 256, 4>(a, stream);
    if (vectors > 512) return launch_rows_as<DT, KIND, 64, 16>(a, stream);
    if (vectors > 128) return launch_rows_as<DT, KIND, 64, 8>(a, stream);
    return launch_rows_as<DT, KIND, 64, 2>(a, stream);
}

int launch_rms_norm(const sgprs_rms_norm_desc_t& d, const void* x, const void* residual, const float* gamma, void* sum, void* y, float* scales,
                    hipStream_t stream, int cus)
{
    const long long es = (long long)dtype_size(d.dtype);
    const bool i8 = d.out_dtype == SGPRS_I8;
    const RowArgs a = {(const unsigned char*)x, (const unsigned char*)residual, gamma, (unsigned char*)sum, (unsigned char*)y, scales, d.m, d.c,
                       d.ldx * es, d.ldr * es, d.ldh * es, i8 ? d.ldy : d.ldy * es, d.eps};
    if (d.dtype == SGPRS_BF16) return i8 ? launch_rows<SGPRS_BF16, kNormI8>(a, stream, cus) : launch_rows<SGPRS_BF16, kNorm>(a, stream, cus);
    return i8 ? launch_rows<SGPRS_F32, kNormI8>(a, stream, cus) : launch_rows<SGPRS_F32, kNorm>(a, stream, cus);
}

int launch_quantize(const sgprs_quantize_desc_t& d, const void* x, int8_t* y, float* scales, hipStream_t stream, int cus)
{
    const RowArgs a = {(const unsigned char*)x, nullptr, nullptr, nullptr, (unsigned char*)y, scales, d.m, d.c,
                       d.ldx * (long long)dtype_size(d.dtype), 0, 0, d.ldy, 0.f};
    return d.dtype == SGPRS_BF16 ? launch_rows<SGPRS_BF16, kQuantize>(a, stream, cus) : launch_rows<SGPRS_F32, kQuantize>(a, stream, cus);
}

}  // namespace sgprs
