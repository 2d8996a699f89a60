// Tiles of keys and the running softmax over them, shared by the attention kernels: one block of 32 queries (or
// query heads of a key head) a wavefront against 32 keys at a time.
#pragma once

#include "block_ops.h"

namespace sgprs {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

constexpr unsigned kOutside = 0x80000000u;  // beyond any descriptor's size: reads zeros
constexpr float kKeepMax = 8.f;

// Tiles of keys in LDS: rows of HD channels, 16-byte chunk c of row r in slot c ^ swizzle(r): 16 rows of one chunk
// (k as the row operand) meet no bank twice, nor do the four rows of a transpose read or the two of an fp32 one.
template <int DT, int HD> struct KvTile {
    static constexpr int ES = DT == SGPRS_BF16 ? 2 : 4;
    static constexpr int ROW = (HD <= 32 ? 32 : HD <= 64 ? 64 : 128) * ES;  // bytes
    static constexpr int CHUNKS = ROW / 16;
    static constexpr int KEYS = DT == SGPRS_BF16 ? 64 : 32;
    static constexpr int BYTES = KEYS * ROW;
    // (linear in the bits of r: what is fixed of a read's row and chunk goes in as one exclusive or)
    static __host__ __device__ constexpr int swizzle(int r)
    {
        if constexpr (ROW == 64) return (r >> 2) & 3;
        if constexpr (ROW == 128) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
        if constexpr (DT == SGPRS_BF16 && ROW == 256) return (r & 3) << 2 | ((r >> 2) & 3);
        return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
    }
};

#if __HIP_DEVICE_COMPILE__
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef __attribute__((address_space(3))) unsigned lds_u32_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Where a lane reads: its own row and chunk of a tile, to which a read adds fixed ones.  Hidden from the compiler in
// every tile, or it would keep the sums for all reads in registers.
template <int DT, int HD> struct LanePlaces {
    typedef KvTile<DT, HD> Tile;
    unsigned k, v;
    __device__ __forceinline__ LanePlaces()
    {
        const int lane = threadIdx.x & 63, h = lane >> 5, s = lane & 15, g = (lane >> 4) & 1;
        k = place(lane & 31, h);
        if constexpr (DT == SGPRS_BF16) v = place(h * 4 + (s >> 2), g * 2 + ((s & 3) >> 1)) + (s & 1) * 8;
        else v = place(h * 4, (lane & 31) >> 2) + (lane & 3) * 4;
    }
    static __device__ __forceinline__ unsigned place(int r, int chunk) { return (unsigned)(r * Tile::ROW + ((chunk ^ Tile::swizzle(r)) << 4)); }
    static __device__ __forceinline__ unsigned hidden(unsigned base)
    {
        asm volatile("" : "+v"(base));
        return base;
    }
    // row and chunk must not share bits with the lane's
    static __device__ __forceinline__ unsigned plus(unsigned base, int r, int chunk) { return (base ^ (unsigned)((chunk ^ Tile::swizzle(r)) << 4)) + (unsigned)(r * Tile::ROW); }
};

// Scores of BLOCKS blocks of 32 keys with this lane's query, as two chains of MFMAs that alternate: the two blocks', or
// one block's even and odd steps.  Two blocks' first MFMAs are inline assembly for the constant 0 as addend (the compiler
// would clear 32 registers); their results are first used two MFMAs on.
template <int DT, int HD, int BLOCKS> __device__ __forceinline__ void scores(unsigned k_base, const u32x4_t* q, f32x16_t* s)
{
    typedef KvTile<DT, HD> Tile;
    constexpr int STEPS = HD * Tile::ES / 32;  // two chunks each
    auto chunk = [&](int b, int c) { return *(const lds_u32x4_t*)(unsigned long)LanePlaces<DT, HD>::plus(k_base, b * 32, 2 * c); };
    auto add = [&](f32x16_t& sum, u32x4_t k, int c) {
        if constexpr (DT == SGPRS_BF16) {
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q[c]), sum, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), sum, 0, 0, 0);
        }
    };
    if constexpr (BLOCKS == 2) {
        static_assert(DT == SGPRS_BF16, "the assembly's type");
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const u32x4_t k = chunk(b, c);
                if (c == 0) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(s[b]) : "v"(k), "v"(q[c]));
                else add(s[b], k, c);
            }
    } else {
        f32x16_t even = {}, odd = {};
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
            const u32x4_t k = chunk(0, c);
            if constexpr (DT == SGPRS_BF16) {
                add(c % 2 ? odd : even, k, c);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x16_t& sum = e % 2 ? odd : even;
                    sum = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), sum, 0, 0, 0);
                }
            }
        }
        s[0] = even + odd;
    }
}

// v of channels 32 d and on at keys 16 u of a block, as the row operand (bf16)
template <int HD> __device__ __forceinline__ u32x4_t value_fragment(unsigned v_base, int block, int u, int d)
{
    u32x4_t f;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const s16x4_t t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_t*)(unsigned long)LanePlaces<SGPRS_BF16, HD>::plus(v_base, block * 32 + u * 16 + a * 8, d * 4));
        const u32x2_t w = __builtin_bit_cast(u32x2_t, t);
        f[2 * a] = w[0];
        f[2 * a + 1] = w[1];
    }
    return f;
}

// o += V^T P^T for one block of 32 keys; p: this lane's 16 weights.  bf16: they are rounded to bf16, as the matrix cores
// take them beside v (their sum is of the fp32 ones); errors of a result rise from 1.6e-3, its own rounding, to 2.1e-3,
// where weights in two parts would double the products with v.  CLEAN: some keys are not seen, and where v holds
// infinities or NaNs 0 * v would be NaN: such values are left out (*odd: there are some) for add_not_finite.
template <int DT, int HD, bool CLEAN>
__device__ __forceinline__ void add_values(f32x16_t* o, const float* p, unsigned v_base, int block, bool* odd)
{
    constexpr int DB = HD / 32;
    if constexpr (DT == SGPRS_BF16) {
        u32x4_t w[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) w[u][e] = pack_bf16x2_relu(p[8 * u + 2 * e], p[8 * u + 2 * e + 1], kNoReluFloor);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4_t f = value_fragment<HD>(v_base, block, u, d);
                if constexpr (CLEAN) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool lo = (f[e] & 0x7f80u) == 0x7f80u, hi = (f[e] & 0x7f800000u) == 0x7f800000u;
                        f[e] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                        *odd |= lo | hi;
                    }
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, w[u]), o[d], 0, 0, 0);
            }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                float f = __uint_as_float(*(const lds_u32_t*)(unsigned long)LanePlaces<DT, HD>::plus(v_base, block * 32 + (i >> 2) * 8 + (i & 3), d * 8));
                if constexpr (CLEAN) {
                    const bool not_finite = !(fabsf(f) < INFINITY);
                    f = not_finite ? 0.f : f;
                    *odd |= not_finite;
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(f, p[i], o[d], 0, 0, 0);
            }
        }
    }
}

// The same for bf16 with all of a block's fragments read at once.  The reads are inline assembly, waited for inside it: before
// the builtins' the compiler waits for every load that writes LDS, the next tile's too.
//
// Weights are two bf16 parts: the bits that fit, and what is left, rounded, so that they are off by 2^-15 of them and a result
// by little more than its own rounding.  The kernel that calls this is bound by the memory: 16 caches of 1 to 32768 tokens
// 60.5 us for 60.2 with rounded weights, 128 of 300 37.6 for 36.9.  Where v is infinite 0 * v or a
// negative part would make a NaN of it, so the first part is cut off, not rounded, and 2^-20 of the weight is added to the
// second, which is then above zero wherever the weight is.
template <int HD> __device__ __forceinline__ void add_values_at_once(f32x16_t* o, const float* p, unsigned v_base)
{
    typedef KvTile<SGPRS_BF16, HD> Tile;
    constexpr int DB = HD / 32;
    u32x4_t w[2], rest[2];
    auto left = [](float z) { return __builtin_fmaf(z, 1.f + 0x1p-20f, -__uint_as_float(__float_as_uint(z) & 0xffff0000u)); };
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float even = p[8 * u + 2 * e], odd = p[8 * u + 2 * e + 1];
            w[u][e] = __builtin_amdgcn_perm(__float_as_uint(odd), __float_as_uint(even), 0x07060302u);
            rest[u][e] = pack_bf16x2_relu(left(even), left(odd), kNoReluFloor);
        }
#pragma unroll
    for (int d0 = 0; d0 < DB; d0 += 2) {
        constexpr int N = DB > 1 ? 2 : 1;
        u32x2_t f[2][2][2];  // [d][u][a]
        unsigned at[2][2];
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int a = 0; a < 2; ++a) at[d][a] = LanePlaces<SGPRS_BF16, HD>::plus(v_base, a * 8, (min(d0 + d, DB - 1)) * 4);
        if constexpr (N == 2)
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %2, %8 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                         "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %11\n\tds_read_b64_tr_b16 %6, %10 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(f[0][0][0]), "=&v"(f[0][0][1]), "=&v"(f[0][1][0]), "=&v"(f[0][1][1]), "=&v"(f[1][0][0]), "=&v"(f[1][0][1]), "=&v"(f[1][1][0]), "=&v"(f[1][1][1])
                         : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "n"(16 * Tile::ROW)
                         : "memory");
        else
            asm volatile("ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\tds_read_b64_tr_b16 %2, %4 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(f[0][0][0]), "=&v"(f[0][0][1]), "=&v"(f[0][1][0]), "=&v"(f[0][1][1])
                         : "v"(at[0][0]), "v"(at[0][1]), "n"(16 * Tile::ROW)
                         : "memory");
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (d0 + d >= DB) continue;
                const u32x4_t v = {f[d][u][0][0], f[d][u][0][1], f[d][u][1][0], f[d][u][1][1]};
                o[d0 + d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, w[u]), o[d0 + d], 0, 0, 0);
                o[d0 + d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, rest[u]), o[d0 + d], 0, 0, 0);
            }
    }
}

// Of a tile's keys, a lane sees those below this, counted from its half's first one.
__device__ __forceinline__ int keys_left(int key0, int first_unseen)
{
    int left = first_unseen - key0 - (int)((threadIdx.x & 63) >> 5) * 4;
    asm volatile("" : "+v"(left));  // compared with constants, not taken from 32 sums kept in registers
    return left;
}

// What add_values left out of a block: infinities and NaNs reach the queries that see their key.  They are counted in
// a product with 1 for a key that is seen and 0 for one that is not: infinities, + 2^8 for -infinities, + 2^16 for NaNs.
template <int DT, int HD> __device__ __forceinline__ void add_not_finite(f32x16_t* o, unsigned v_base, int block, int key0, int first_unseen)
{
    const int mine = keys_left(key0, first_unseen);
    auto seen = [&](int i) { return block * 32 + (i >> 2) * 8 + (i & 3) < mine ? 1.f : 0.f; };
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
        f32x16_t count = {};
        if constexpr (DT == SGPRS_BF16) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4_t f = value_fragment<HD>(v_base, block, u, d);
                u32x4_t kind, w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    kind[e] = 0;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const unsigned v = f[e] >> (16 * half) & 0xffffu, k = v & 0x7fu ? 0x4780u : v & 0x8000u ? 0x4380u : 0x3f80u;
                        kind[e] |= ((v & 0x7f80u) == 0x7f80u ? k : 0u) << (16 * half);
                    }
                    w[e] = pack_bf16x2_relu(seen(8 * u + 2 * e), seen(8 * u + 2 * e + 1), kNoReluFloor);
                }
                count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kind), __builtin_bit_cast(bf16x8_t, w), count, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float f = __uint_as_float(*(const lds_u32_t*)(unsigned long)LanePlaces<DT, HD>::plus(v_base, block * 32 + (i >> 2) * 8 + (i & 3), d * 8));
                count = __builtin_amdgcn_mfma_f32_32x32x2f32(fabsf(f) < INFINITY ? 0.f : f != f ? 65536.f : f < 0.f ? 256.f : 1.f, seen(i), count, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const unsigned n = (unsigned)count[i];
            o[d][i] += !n ? 0.f : n >> 16 || (n >> 8 && n & 0xffu) ? NAN : n >> 8 ? -INFINITY : INFINITY;
        }
    }
}

// A query's running softmax: maximum (of scores as they are multiplied, in base 2), sum of the weights, results.
template <int DT, int HD> struct Running {
    static constexpr int DB = HD / 32;
    f32x16_t o[DB];
    float top, sum;  // sum: of this half's keys
    LanePlaces<DT, HD> place;
    __device__ __forceinline__ void start()
    {
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
    }
    __device__ __forceinline__ float total() const { return sum + other_half(sum); }
    // BLOCKS blocks of 32 keys from key0 on, in LDS at k_at and v_at; keys from first_unseen on are not seen.  k_done
    // is called when k has been read, v_ready before v is.
    // ZEROS: v holds zeros at keys that are not seen, so that only the scores need a mask.
    template <int BLOCKS, bool MASKED, bool ZEROS = false, class KDone, class VReady>
    __device__ __forceinline__ void tile(const u32x4_t* q, float scale_log2, unsigned k_at, unsigned v_at, int key0, int first_unseen, KDone k_done, VReady v_ready)
    {
        const unsigned k_base = place.hidden(place.k + k_at), v_base = place.hidden(place.v + v_at);
        f32x16_t s[BLOCKS];
        scores<DT, HD, BLOCKS>(k_base, q, s);
        k_done();
        const int mine = MASKED ? keys_left(key0, first_unseen) : 0;
        float most = -INFINITY;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            if constexpr (MASKED) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = b * 32 + (i >> 2) * 8 + (i & 3) < mine ? s[b][i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[b][i]);
        }
        most = fmaxf(most, other_half(most)) * scale_log2;
        if (__any(most > top + kKeepMax)) {
            const float now = fmaxf(top, most), keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= keep;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= keep;
        }
        const float base = top == -INFINITY ? 0.f : top + kKeepMax;  // weights stay below 1, so sums with large v keep their range
        v_ready();
        bool odd = false;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale_log2, -base));
                sum += p[i];
            }
            if constexpr (ZEROS && DT == SGPRS_BF16) {
                static_assert(BLOCKS == 1, "a block at a time");
                add_values_at_once<HD>(o, p, v_base);
            } else {
                add_values<DT, HD, MASKED && !ZEROS>(o, p, v_base, b, &odd);
            }
        }
        if constexpr (MASKED && !ZEROS) {
            static_assert(BLOCKS == 1, "a block at a time");
            if (__any(odd)) add_not_finite<DT, HD>(o, v_base, 0, key0, first_unseen);
        }
    }
};
#endif

// 1 / the sum of the weights; without a key the result is zero, and where all scores are -inf there is none.
__device__ __forceinline__ float normaliser(float sum, bool any_key) { return sum > 0.f ? 1.f / sum : any_key ? NAN : 0.f; }

// four channels of a result, from channel c on
template <int DT> __device__ __forceinline__ void store4(unsigned char* row, int c, const float* z)
{
    if constexpr (DT == SGPRS_BF16)
        *(u32x2_t*)(row + c * 2) = u32x2_t{pack_bf16x2_relu(z[0], z[1], kNoReluFloor), pack_bf16x2_relu(z[2], z[3], kNoReluFloor)};
    else
        *(float4*)(row + c * 4) = make_float4(z[0], z[1], z[2], z[3]);
}

#if __HIP_DEVICE_COMPILE__
// The last sequence s of n with key(offsets[s], s) <= value, for keys that do not fall: 64 of them are looked at at once.
template <class Key> __device__ __forceinline__ int last_not_above(const int* offsets, int n, int value, Key key)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, at = min(lo + lane * step, hi - 1);
        const int below = (int)__popcll(__ballot(lo + lane * step < hi && key(offsets[at], at) <= value));
        const int to = max(below - 1, 0);
        hi = min(hi, lo + (to + 1) * step);
        lo += to * step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
#endif

}  // namespace sgprs
