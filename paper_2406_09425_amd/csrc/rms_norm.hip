// Root-mean-square norm of rows with the residual's addition, and rows of 8-bit integers with a scale each.
//
// Bound by the memory.  A row is read once and kept in the registers of a wavefront or a workgroup (rows beyond that are
// read twice).  With t = h gamma a row's integers are 127 t / max|t|: the norm's factor cancels, so they need no
// statistics but the maximum, and they are to be those of the definition whatever the order of anything.  So they are
// worked out in 32 bits, which leaves a quotient (up to 127, three roundings) off by less than 2^-15, and those within
// 2^-15 of a border between two integers are decided in 64 bits, in which t is exact.  Rows whose squares or products could leave the range of
// 32-bit numbers, and rows that are not finite, go through 64 bits altogether.
//
// 16384 rows of 4096 in bf16 with a residual, their sum and 8-bit results 83 us (470 MB, 5.6 TB/s; every integer decided in 64
// bits took 255); 8-bit rows of 4093x4099 in fp32 15 (84 MB, 5.6 TB/s); a row or 24 of 4096 3.6, which a launch takes.
#include <algorithm>
#include <type_traits>

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
    double per_channel;            // 1 / c
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
    // q: integers in the low bytes
    static __device__ __forceinline__ void store_i8(unsigned char* p, const unsigned* q, int live)
    {
        unsigned w[V / 4];
#if __HIP_DEVICE_COMPILE__
#pragma unroll
        for (int d = 0; d < V / 4; ++d)
            w[d] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * d + 3], q[4 * d + 2], 0x0c0c0400u), __builtin_amdgcn_perm(q[4 * d + 1], q[4 * d], 0x0c0c0400u), 0x05040100u);
#endif
        if (live >= V) {
            __builtin_memcpy(p, w, V);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < live) p[e] = (unsigned char)(w[e / 4] >> (e % 4 * 8));
        }
    }
    // V factors from channel c on, of which `live` exist
    static __device__ __forceinline__ void load_factors(const float* p, int live, float* g)
    {
        if (live >= V) {
            __builtin_memcpy(g, p, V * 4);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = e < live ? p[e] : 1.f;
        }
    }
};

// Sums and maxima over a row's threads, in a fixed order.
template <int THREADS> struct RowJoin {
    double squares[THREADS / 64], most[THREADS / 64];
    unsigned bits[THREADS / 64];
};
struct Add {
    template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Most {
    template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; }
};
template <class Op, class T> __device__ __forceinline__ T over_wavefront(T v, Op op)
{
#if __HIP_DEVICE_COMPILE__
    if constexpr (sizeof(T) == 4) {  // the 16 lanes of a row by rotations, then rows and halves
        auto with = [&](auto turn) { v = op(v, __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x120 + decltype(turn)::value, 0xf, 0xf, true))); };
        with(std::integral_constant<int, 8>());
        with(std::integral_constant<int, 4>());
        with(std::integral_constant<int, 2>());
        with(std::integral_constant<int, 1>());
        v = op(v, __shfl_xor(v, 16));
        v = op(v, __shfl_xor(v, 32));
    } else {
#pragma unroll
        for (int x = 32; x; x >>= 1) v = op(v, __shfl_xor(v, x));
    }
#endif
    return v;
}
template <int WAVES, class Op, class T> __device__ __forceinline__ T over_wavefronts(const T* all, Op op)
{
    T v = all[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = op(v, all[w]);
    return v;
}

// THREADS threads a row (a wavefront: four rows a workgroup), VPT vectors of it each; VPT 0: as many as it takes, read twice.
template <int DT, int KIND, int THREADS, int VPT> __global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void rms_norm_kernel(const RowArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef RowVec<DT> Vec;
    constexpr int V = Vec::V, WAVES = THREADS / 64;
    __shared__ RowJoin<THREADS> joined;
    const int thread = THREADS == 64 ? threadIdx.x & 63 : threadIdx.x, wave = THREADS == 64 ? 0 : threadIdx.x >> 6;
    const int row = THREADS == 64 ? blockIdx.x * 4 + (int)(threadIdx.x >> 6) : blockIdx.x;
    if (row >= a.m) return;
    const unsigned char* xp = a.x + row * a.ldx;
    const unsigned char* rp = KIND != kQuantize && a.residual ? a.residual + row * a.ldr : nullptr;
    unsigned char* hp = KIND != kQuantize && a.sum ? a.sum + row * a.ldh : nullptr;
    unsigned char* yp = a.y + row * a.ldy;
    const float* gamma = KIND != kQuantize ? a.gamma : nullptr;
    const int vectors = (a.c + V - 1) / V;

    auto added = [&](u32x4_t x, u32x4_t r) {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = Vec::get(x, e) + Vec::get(r, e);
        return Vec::pack(z);
    };
    auto load_gamma = [&](int v, float* g) {
        if (gamma) {
            Vec::load_factors(gamma + v * V, a.c - v * V, g);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = 1.f;
        }
    };
    auto in_64_bits = [&](float h, float g) { return KIND == kQuantize ? (double)h : (double)h * (double)g; };
    // 127 t / most, rounded; step: 127 / most, off by less than 2^-49 of it: next to a border the quotient itself decides
    auto integer = [&](double t, double most, double step) {
        const double u = t * step, whole = rint(u);
        return (unsigned)(int)(fabs(u - whole) > 0.5 - 0x1p-40 ? rint(127.0 * t / most) : whole);
    };

    u32x4_t kept[VPT > 0 ? VPT : 1];
    if constexpr (VPT > 0) {
        constexpr bool ONCE = VPT * V <= 16;  // gamma stays in registers
        float g_kept[ONCE ? VPT : 1][V];
        auto factors = [&](int i, float* g) {
            if constexpr (ONCE) {
#pragma unroll
                for (int e = 0; e < V; ++e) g[e] = g_kept[i][e];
            } else {
                load_gamma(thread + i * THREADS, g);
            }
        };
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = thread + i * THREADS;
            kept[i] = v < vectors ? Vec::load(xp + (long long)v * 16, a.c - v * V) : u32x4_t{0, 0, 0, 0};
        }
        if (rp) {
            u32x4_t r[VPT];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int v = thread + i * THREADS;
                r[i] = v < vectors ? Vec::load(rp + (long long)v * 16, a.c - v * V) : u32x4_t{0, 0, 0, 0};
            }
            if constexpr (ONCE && KIND != kQuantize) {
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    if (thread + i * THREADS < vectors) load_gamma(thread + i * THREADS, g_kept[i]);
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) kept[i] = added(kept[i], r[i]);
        } else if constexpr (ONCE && KIND != kQuantize) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (thread + i * THREADS < vectors) load_gamma(thread + i * THREADS, g_kept[i]);
        }
        float lane_squares = 0.f;
        unsigned most_of[VPT], most = 0;  // bits of the largest |t| without the sign, twice: NaNs are above infinity
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = thread + i * THREADS;
            most_of[i] = 0;
            if (v >= vectors) continue;
            if (hp) Vec::store(hp + (long long)v * 16, kept[i], a.c - v * V);
            float g[V], sum = 0.f;
            if constexpr (KIND == kNormI8) factors(i, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = Vec::get(kept[i], e);
                if constexpr (KIND != kQuantize) sum = __builtin_fmaf(h, h, sum);
                if constexpr (KIND != kNorm) most_of[i] = max(most_of[i], __float_as_uint(KIND == kNormI8 ? h * g[e] : h) << 1);
            }
            most = max(most, most_of[i]);
            lane_squares += sum;
        }
        // (eight squares, eight sums, six levels of lanes: off by at most 22 roundings, the factor by half of that)
        double squares = 0.0;
        if constexpr (KIND != kQuantize) squares = over_wavefront(lane_squares, Add());
        if constexpr (KIND != kNorm) most = over_wavefront(most, Most());
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                joined.squares[wave] = squares;
                joined.bits[wave] = most;
            }
            __syncthreads();
            if constexpr (KIND != kQuantize) squares = over_wavefronts<WAVES>(joined.squares, Add());
            if constexpr (KIND != kNorm) most = over_wavefronts<WAVES>(joined.bits, Most());
        }
        bool fast = KIND == kQuantize || (squares >= 0x1p-60 && squares <= 0x1p120);
        if constexpr (KIND != kNorm) fast = fast && most >= __float_as_uint(0x1p-90f) << 1 && most <= __float_as_uint(0x1p90f) << 1;
        fast = __all(fast);
        if (fast) {
            float factor = 1.f;
            double wide = 1.0;
            if constexpr (KIND != kQuantize) {
                const double mean = __builtin_fma(squares, a.per_channel, (double)a.eps);
                wide = __builtin_amdgcn_rsq(mean);  // 2^-23 or better, of which a step makes 2^-44
                wide = __builtin_fma(wide * 0.5, __builtin_fma(-mean * wide, wide, 1.0), wide);
                factor = (float)wide;
            }
            if constexpr (KIND == kNorm) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int v = thread + i * THREADS;
                    if (v >= vectors) continue;
                    float g[V], z[V];
                    factors(i, g);
#pragma unroll
                    for (int e = 0; e < V; ++e) z[e] = Vec::get(kept[i], e) * factor * g[e];
                    Vec::store(yp + (long long)v * 16, Vec::pack(z), a.c - v * V);
                }
                return;
            }
            // the largest |t| itself, among what 32 bits have close to it
            double largest = __uint_as_float(most >> 1);
            if constexpr (KIND == kNormI8) {
                largest = 0.0;
                const unsigned close = most - 8;  // four steps of a 32-bit number: t is off by half of one
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    if (most_of[i] < close) continue;
                    float g[V];
                    factors(i, g);
#pragma unroll
                    for (int e = 0; e < V; ++e) largest = fmax(largest, thread * V + i * THREADS * V + e < a.c ? fabs(in_64_bits(Vec::get(kept[i], e), g[e])) : 0.0);
                }
                const unsigned long long found = __ballot(largest > 0.0);  // (most often one lane)
                if (__popcll(found) == 1) {
                    const int from = __ffsll(found) - 1;
                    const unsigned long long bits = __builtin_bit_cast(unsigned long long, largest);
                    largest = __builtin_bit_cast(double, (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)bits, from) |
                                                             (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), from) << 32);
                } else if (found) {
                    largest = over_wavefront(largest, Most());
                }
                if constexpr (WAVES > 1) {
                    if ((threadIdx.x & 63) == 0) joined.most[wave] = largest;
                    __syncthreads();
                    largest = over_wavefronts<WAVES>(joined.most, Most());
                }
            }
            if (thread == 0) a.scales[row] = (float)(largest * wide * (1.0 / 127.0));
            double inverse = __builtin_amdgcn_rcp(largest);  // as above
            inverse = __builtin_fma(inverse, __builtin_fma(-largest, inverse, 1.0), inverse);
            inverse = __builtin_fma(inverse, __builtin_fma(-largest, inverse, 1.0), inverse);
            const double exact_step = 127.0 * inverse;
            const float step = (float)exact_step;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int v = thread + i * THREADS;
                if (v >= vectors) continue;
                float g[V], far = 0.f;
                if constexpr (KIND == kNormI8) factors(i, g);
                unsigned q[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float h = Vec::get(kept[i], e), u = (KIND == kNormI8 ? h * g[e] : h) * step;
                    const float placed = u + 0x1.8p23f;  // u, rounded, in the low bits
                    q[e] = __float_as_uint(placed);
                    far = fmaxf(far, fabsf(u - (placed - 0x1.8p23f)));
                }
                if (far > 0.5f - 0x1p-15f) {
#pragma unroll
                    for (int e = 0; e < V; ++e) q[e] = integer(in_64_bits(Vec::get(kept[i], e), KIND == kNormI8 ? g[e] : 1.f), largest, exact_step);
                }
                Vec::store_i8(yp + (long long)v * V, q, a.c - v * V);
            }
            return;
        }
        if constexpr (WAVES > 1) __syncthreads();  // (before the sums are written again)
    }

    // ---- in 64 bits, where no square of a 32-bit number overflows or vanishes ----
    double squares = 0.0, most = 0.0;
    unsigned odd = 0;  // an infinity or a NaN among the t
    auto stream = [&](int v) {
        const int live = a.c - v * V;
        const u32x4_t x = Vec::load(xp + (long long)v * 16, live);
        return rp ? added(x, Vec::load(rp + (long long)v * 16, live)) : x;
    };
    auto take = [&](int v, u32x4_t h) {
        float g[V];
        if constexpr (KIND == kNormI8) load_gamma(v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (v * V + e >= a.c) continue;
            const double f = Vec::get(h, e), t = KIND == kNormI8 ? f * (double)g[e] : f;
            if constexpr (KIND != kQuantize) squares = __builtin_fma(f, f, squares);
            if constexpr (KIND != kNorm) {
                most = fmax(most, fabs(t));
                odd |= !(fabs(t) < (double)INFINITY);
            }
        }
    };
    if constexpr (VPT > 0) {
#pragma unroll 1
        for (int i = 0; i < VPT; ++i) {
            u32x4_t h = kept[0];
#pragma unroll
            for (int j = 1; j < VPT; ++j) h = i == j ? kept[j] : h;
            if (thread + i * THREADS < vectors) take(thread + i * THREADS, h);
        }
    } else {
        for (int v = thread; v < vectors; v += THREADS) {
            const u32x4_t h = stream(v);
            if (hp) Vec::store(hp + (long long)v * 16, h, a.c - v * V);
            take(v, h);
        }
    }
    squares = over_wavefront(squares, Add());
    most = over_wavefront(most, Most());
    odd = over_wavefront(odd, Most());
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
            joined.squares[wave] = squares;
            joined.most[wave] = most;
            joined.bits[wave] = odd;
        }
        __syncthreads();
        squares = over_wavefronts<WAVES>(joined.squares, Add());
        most = over_wavefronts<WAVES>(joined.most, Most());
        odd = over_wavefronts<WAVES>(joined.bits, Most());
    }
    double factor = 1.0;
    if constexpr (KIND != kQuantize) factor = 1.0 / sqrt(squares / a.c + (double)a.eps);
    if (!(squares < (double)INFINITY)) odd = 1;
    if constexpr (KIND != kNorm) {
        if (thread == 0) a.scales[row] = odd ? NAN : (float)(most * factor / 127.0);
    }
    // h * factor in 32 bits: the factor as a power of two, which takes h to its place, and a number of 1 to 2
    const bool fine = factor > 0.0 && factor < (double)INFINITY;
    const int power = fine ? ilogb(factor) : 0;
    const float scale = (float)(fine ? ldexp(factor, -power) : factor);
    const double step = 127.0 / most;
    auto finish = [&](int v, u32x4_t h) {
        float g[V];
        load_gamma(v, g);
        if constexpr (KIND == kNorm) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] = __builtin_amdgcn_ldexpf(Vec::get(h, e), power) * scale * g[e];
            Vec::store(yp + (long long)v * 16, Vec::pack(z), a.c - v * V);
        } else {
            unsigned q[V];
#pragma unroll
            for (int e = 0; e < V; ++e) q[e] = odd || most == 0.0 ? 0u : integer(in_64_bits(Vec::get(h, e), g[e]), most, step);
            Vec::store_i8(yp + (long long)v * V, q, a.c - v * V);
        }
    };
    if constexpr (VPT > 0) {
#pragma unroll 1
        for (int i = 0; i < VPT; ++i) {
            u32x4_t h = kept[0];
#pragma unroll
            for (int j = 1; j < VPT; ++j) h = i == j ? kept[j] : h;
            if (thread + i * THREADS < vectors) finish(thread + i * THREADS, h);
        }
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

// Threads of a row by its vectors of 16 bytes: so many that a row is two or four vectors of each, since all of them wait for
// the slowest; a wavefront only where that would leave it idle.  Of one sweep (events around 30 calls on a stream, 1 to 2 us a
// call above the figures at the top): 16384 rows of bf16 with residual and 8-bit results, us:
// 4096 channels by 256 threads 85 (5.5 TB/s), by 64 98, by 512 99; 2048 by 256 46, by 64 52; 1024 by 64 28, by 256 34.
// 4000 rows of 16384 by 1024 threads 90, by 512 96, by 256 98; one row of 4096 by 256 4.3, by 64 9.3.
template <int DT, int KIND> static int launch_rows(const RowArgs& a, hipStream_t stream, int cus)
{
    constexpr int V = RowVec<DT>::V;
    const int vectors = (a.c - 1) / V + 1;
    if (vectors > 8192) return launch_rows_as<DT, KIND, 1024, 0>(a, stream);
    if (vectors > 4096) return launch_rows_as<DT, KIND, 1024, 8>(a, stream);
    if (vectors > 2048) return launch_rows_as<DT, KIND, 1024, 4>(a, stream);
    if (vectors > 1536) return launch_rows_as<DT, KIND, 1024, 2>(a, stream);
    if (vectors > 1024) return launch_rows_as<DT, KIND, 512, 4>(a, stream);
    if (vectors > 512) return launch_rows_as<DT, KIND, 256, 4>(a, stream);
    if (vectors > 256) return launch_rows_as<DT, KIND, 256, 2>(a, stream);
    if (vectors > 128 || (vectors > 64 && a.m < 4 * cus)) return launch_rows_as<DT, KIND, 256, 1>(a, stream);
    return vectors > 64 ? launch_rows_as<DT, KIND, 64, 2>(a, stream) : launch_rows_as<DT, KIND, 64, 1>(a, stream);
}

int launch_rms_norm(const sgprs_rms_norm_desc_t& d, const void* x, const void* residual, const float* gamma, void* sum, void* y, float* scales,
                    hipStream_t stream, int cus)
{
    const long long es = (long long)dtype_size(d.dtype);
    const bool i8 = d.out_dtype == SGPRS_I8;
    const RowArgs a = {(const unsigned char*)x, (const unsigned char*)residual, gamma, (unsigned char*)sum, (unsigned char*)y, scales, d.m, d.c,
                       d.ldx * es, d.ldr * es, d.ldh * es, i8 ? d.ldy : d.ldy * es, d.eps, 1.0 / d.c};
    if (d.dtype == SGPRS_BF16) return i8 ? launch_rows<SGPRS_BF16, kNormI8>(a, stream, cus) : launch_rows<SGPRS_BF16, kNorm>(a, stream, cus);
    return i8 ? launch_rows<SGPRS_F32, kNormI8>(a, stream, cus) : launch_rows<SGPRS_F32, kNorm>(a, stream, cus);
}

int launch_quantize(const sgprs_quantize_desc_t& d, const void* x, int8_t* y, float* scales, hipStream_t stream, int cus)
{
    const RowArgs a = {(const unsigned char*)x, nullptr, nullptr, nullptr, (unsigned char*)y, scales, d.m, d.c,
                       d.ldx * (long long)dtype_size(d.dtype), 0, 0, d.ldy, 0.f, 1.0 / d.c};
    return d.dtype == SGPRS_BF16 ? launch_rows<SGPRS_BF16, kQuantize>(a, stream, cus) : launch_rows<SGPRS_F32, kQuantize>(a, stream, cus);
}

}  // namespace sgprs
