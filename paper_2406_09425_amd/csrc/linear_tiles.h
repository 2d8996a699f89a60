// What the linear products share: loads of rows at any alignment, and the order of a launch's tiles.
#pragma once

#include <type_traits>
#include <utility>

#include "block_ops.h"

namespace sgprs {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr unsigned kOutside = 0x80000000u;  // beyond any descriptor's size: reads zeros

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
            if constexpr (ES == 1) v[e / 4] |= (unsigned)p[e] << (e % 4 * 8);
            else if constexpr (ES == 2) v[e / 2] |= (unsigned)*(const unsigned short*)(p + e * 2) << (e % 2 * 16);
            else v[e] = *(const unsigned*)(p + e * 4);
        }
    }
    return v;
}

#if __HIP_DEVICE_COMPILE__
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
__device__ __forceinline__ u32x4_t lds_read(unsigned at) { return *(const lds_u32x4_t*)(unsigned long)at; }
#endif

// for_each<N>(f): f(0), ..., f(N - 1) as constants.  (A loop over accumulators that the compiler finds too long to unroll
// would put them in memory.)
template <class F, int... I> __device__ __forceinline__ void for_each(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F> __device__ __forceinline__ void for_each(F f) { for_each(f, std::make_integer_sequence<int, N>()); }

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

}  // namespace sgprs
