// Attention over packed sequences: o = softmax(scale q k^T) v in one pass over the keys.
//
// Scores are computed transposed, S^T = K Q^T with MFMA 32x32: a lane then holds 16 keys' scores of ONE query,
// so the running maximum and sum of a query are lane arithmetic plus one exchange between the wavefront's halves,
// and the weights are already the column operand of O^T = V^T P^T: they never leave the registers.  A half of the
// wavefront holds keys 8 a + 4 h + b (h: which half); the products with v take the keys in that order, which for
// bf16 is what the LDS transpose read delivers from rows of v (four keys of one channel a lane), for fp32 a plain
// read.  The running maximum moves only when a tile's scores pass it by 2^8: until then the accumulators need no
// touching.  Weights are taken relative to 2^8 times the maximum, so that none is above 1.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "block_ops.h"

namespace sgprs {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

struct AttentionArgs {
    const unsigned char *q, *k, *v;
    unsigned char* o;
    const int *q_offsets, *kv_offsets;
    int n_seqs, total_q, total_kv, heads, kv_heads, group, head_dim, causal;
    float scale_log2;                // |scale| log2 e
    unsigned q_flip;                 // sign bits of a dword of q, where the scale is negative
    int ldq, ldk, ldv, ldo;          // bytes
    long long hq, hk, hv, ho;        // bytes
    int slots;                       // query tiles, with room for each sequence's last one
    int chunk, chunks;               // keys that a workgroup takes of a sequence; of the longest one
    int tile_rows;                   // of a prompt's tile, 0 for single tokens
    int row_blocks;                  // of 32 rows (queries x heads of a key head)
    float* part_o;                   // [chunk][token][head][head_dim], weights relative to part_stat
    float2* part_stat;               // [chunk][token][head]: maximum, sum
};

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

// One of the `parts` wavefronts' share of a tile: rows of a tensor that starts at p, `rows` of them, into LDS at `to`.
template <int DT, int HD, int KEYS> __device__ __forceinline__ void request_tile(const unsigned char* p, int ld, int rows, int row_bytes, unsigned char* to, int part, int parts)
{
    typedef KvTile<DT, HD> Tile;
    constexpr int RPI = 1024 / Tile::ROW, LOADS = KEYS * Tile::ROW / 1024;  // rows of a load
    unsigned lane = threadIdx.x & 63;
    if constexpr (HD > 32) asm volatile("" : "+v"(lane));  // the offsets are worked out in every tile rather than kept in registers
    const int lrow = (int)(lane / Tile::CHUNKS), slot = (int)(lane % Tile::CHUNKS) ^ Tile::swizzle(lrow);
    const int size = __builtin_amdgcn_readfirstlane(rows > 0 ? (rows - 1) * ld + row_bytes : 0);  // (a clamp is vector arithmetic)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, size, 0x00020000);
    const unsigned first = (unsigned)(lrow * ld);
#pragma unroll
    for (int i = 0; i < LOADS / parts; ++i) {
        const int r = (i * parts + part) * RPI, chunk = (slot ^ Tile::swizzle(r)) << 4;  // r: of the load's first row
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t)(to + (i * parts + part) * 1024), 16,
                                                 chunk < row_bytes ? first + (unsigned)(r * ld) + (unsigned)chunk : kOutside, 0, 0, 0);
    }
}

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
    template <int BLOCKS, bool MASKED, class KDone, class VReady>
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
            add_values<DT, HD, MASKED>(o, p, v_base, b, &odd);
        }
        if constexpr (MASKED) {
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
// First token and length of a sequence, inside the tensor whatever the offsets say; in scalar registers, since buffer
// descriptors are made of them.
__device__ __forceinline__ void range_of(const int* offsets, int seq, int total, int* first, int* count)
{
    const int from = min(max(offsets[seq], 0), total), to = min(max(offsets[seq + 1], from), total);
    *first = __builtin_amdgcn_readfirstlane(from);
    *count = __builtin_amdgcn_readfirstlane(to - from);
}
#endif

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

// Sequence and tile of a slot: a sequence's tiles start at slot q_offsets[s] / BM + s, which leaves each its own.
__device__ __forceinline__ bool tile_of_slot(const AttentionArgs& a, int slot, int bm, int* seq, int* row, int* q0, int* nq)
{
#if __HIP_DEVICE_COMPILE__
    *seq = last_not_above(a.q_offsets, a.n_seqs, slot, [=](int offset, int s) { return offset / bm + s; });
    range_of(a.q_offsets, *seq, a.total_q, q0, nq);
    const int tile = __builtin_amdgcn_readfirstlane(slot - (a.q_offsets[*seq] / bm + *seq));
    *row = tile * bm;
    return tile >= 0 && tile < (1 << 23) && *row < *nq;
#else
    return false;
#endif
}

constexpr int kPromptRows = 128;
// Chunks of keys that the queries of one workgroup were split into; one: the result was written at once.  (tile_rows:
// queries of a prompt's tile; 0 for single tokens.)
__device__ __forceinline__ int chunks_of(const AttentionArgs& a, int query, int nq, int nk)
{
    int keys = nk;
    if (a.tile_rows && a.causal) keys = min(nk, min(query / a.tile_rows * a.tile_rows + a.tile_rows, nq) + nk - nq);
    return min(a.chunks, max(1, (keys + a.chunk - 1) / a.chunk));
}

// ---- prompts -----------------------------------------------------------------------------------
// 128 queries of one head per workgroup, 32 per wavefront; tiles of keys in an LDS ring of two or three stages.
// bf16: bound by the vector units' softmax and what the two (heads of 64: three) wavefronts of a SIMD cannot hide of it
// behind each other's MFMAs: heads of 128, 59 % of their time and 35 % of the matrix cores'; 2 x 4096 tokens, 16 heads of
// 128: 321 us, 857 TFLOP/s; 8192 tokens, 16 heads of 64: 362 us, 759.  fp32 by fp32 MFMAs: 4 x 1024 tokens, 8 heads of
// 128: 170 us, 101 TFLOP/s.  Registers decide: what the compiler would keep of addresses and masks is worked out in every
// tile, since one spilled register waits for all keys on their way (heads of 128: 714 -> 849 TFLOP/s).
template <int DT, int HD> struct PromptShape {
    static constexpr int STAGE = 2 * KvTile<DT, HD>::BYTES, STAGES = STAGE <= 16384 ? 3 : 2;
};
template <int DT, int HD> __global__ __launch_bounds__(256, (DT == SGPRS_F32 && HD > 64 ? 1 : DT == SGPRS_BF16 && HD <= 64 ? 3 : 2)) void attention_prompt_kernel(const AttentionArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef KvTile<DT, HD> Tile;
    constexpr int ES = Tile::ES, STEPS = HD * ES / 32, BM = kPromptRows;
    typedef PromptShape<DT, HD> Shape;
    constexpr int NS = Shape::STAGES, LOADS = Shape::STAGE / 1024 / 4;  // of a wavefront for a tile
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // heavy tiles (the last ones under the causal mask) first; heads that share keys on one die where there are eight of them
    const int item = blockIdx.x % (a.slots * a.heads), chunk = blockIdx.x / (a.slots * a.heads);
    const int j = item % a.heads, slot = a.slots - 1 - item / a.heads;
    const int kv_head = j % a.kv_heads, head = kv_head * a.group + j / a.kv_heads;
    int seq, row0, q0, nq;
    if (!tile_of_slot(a, slot, BM, &seq, &row0, &q0, &nq)) return;
    int k0, nk;
    range_of(a.kv_offsets, seq, a.total_kv, &k0, &nk);
    const int row = row0 + wave * 32 + (lane & 31);       // of the sequence
    const int last_row = min(row0 + BM, nq) - 1;
    const int all_keys = a.causal ? max(0, min(nk, last_row + nk - nq + 1)) : nk;  // that anyone here sees
    const int begin = chunk * a.chunk, keys = min(all_keys - begin, a.chunk);       // of this chunk
    if (chunk > 0 && keys <= 0) return;
    const int my_row = min(row, nq - 1);
    const int first_unseen = a.causal ? min(nk, my_row + nk - nq + 1) : nk;
    const int wave_first = min(row0 + wave * 32, nq - 1);
    const int wave_all = a.causal ? min(nk, wave_first + nk - nq + 1) : nk;      // keys that every query of the wavefront sees
    const int wave_any = row0 + wave * 32 < nq ? (a.causal ? min(nk, min(row0 + wave * 32 + 32, nq) + nk - nq) : nk) : 0;
    const int row_bytes = a.head_dim * ES;

    u32x4_t q[STEPS];
    const unsigned char* qp = a.q + (long long)(q0 + my_row) * a.ldq + head * a.hq;
#pragma unroll
    for (int c = 0; c < STEPS; ++c) {
        q[c] = (2 * c + h) * 16 < row_bytes ? *(const u32x4_t*)(qp + (2 * c + h) * 16) : u32x4_t{0, 0, 0, 0};
        q[c] ^= a.q_flip;
    }
    const unsigned char* kp = a.k + (long long)(k0 + begin) * a.ldk + kv_head * a.hk;
    const unsigned char* vp = a.v + (long long)(k0 + begin) * a.ldv + kv_head * a.hv;
    auto request = [&](int t) {
        unsigned char* to = smem + t % NS * Shape::STAGE;
        const int rows = max(0, min(Tile::KEYS, nk - begin - t * Tile::KEYS));  // (none behind the last tile)
        request_tile<DT, HD, Tile::KEYS>(kp + (long long)t * Tile::KEYS * a.ldk, a.ldk, rows, row_bytes, to, wave, 4);
        request_tile<DT, HD, Tile::KEYS>(vp + (long long)t * Tile::KEYS * a.ldv, a.ldv, rows, row_bytes, to + Tile::BYTES, wave, 4);
    };
    Running<DT, HD> run;
    run.start();
    const int tiles = (keys + Tile::KEYS - 1) / Tile::KEYS;
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) request(t);
    for (int t = 0; t < tiles; ++t) {
        constexpr int BEHIND = (NS - 2) * LOADS;
        __builtin_amdgcn_s_waitcnt((BEHIND & 15) | ((BEHIND >> 4) << 14) | 0x0F70);  // this tile has landed
        __builtin_amdgcn_s_barrier();  // everyone's, and everyone has left the buffer of the tile before
        __builtin_amdgcn_sched_barrier(0);
        request(t + NS - 1);
        const unsigned at = (unsigned)(t % NS * Shape::STAGE);
        const int key0 = begin + t * Tile::KEYS;
        if (key0 < wave_any) {
            auto nothing = [] {};
            const unsigned v_at = at + Tile::BYTES;
            if (key0 + Tile::KEYS <= wave_all) {
                run.template tile<Tile::KEYS / 32, false>(q, a.scale_log2, at, v_at, key0, first_unseen, nothing, nothing);
            } else {  // block by block, those that somebody here sees
#pragma unroll 1
                for (int b = 0; b < Tile::KEYS && key0 + b < wave_any; b += 32)
                    run.template tile<1, true>(q, a.scale_log2, at + b * Tile::ROW, v_at + b * Tile::ROW, key0 + b, first_unseen, nothing, nothing);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // requests behind the last tile write zeros
    if (row >= nq) return;
    const float sum = run.total();
    if (a.chunks > 1 && all_keys > a.chunk) {
        const long long at = ((long long)chunk * a.total_q + q0 + row) * a.heads + head;
        if (h == 0) a.part_stat[at] = make_float2(run.top, sum);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int c = d * 32 + (i >> 2) * 8 + h * 4;
                if (c < a.head_dim)
                    *(float4*)(a.part_o + at * a.head_dim + c) = make_float4(run.o[d][i], run.o[d][i + 1], run.o[d][i + 2], run.o[d][i + 3]);
            }
        return;
    }
    const float inv = normaliser(sum, first_unseen > 0);
    unsigned char* op = a.o + (long long)(q0 + row) * a.ldo + head * a.ho;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int c = d * 32 + (i >> 2) * 8 + h * 4;
            if (c >= a.head_dim) continue;
            float z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = run.o[d][i + e] * inv;
            store4<DT>(op, c, z);
        }
#endif
}

// ---- single tokens -----------------------------------------------------------------------------
// Few queries against many keys: bound by reading k and v.  The queries of all heads that share a key head are one
// block of 32 columns (or several), so k and v are read once for them; a workgroup takes a chunk of a sequence's
// keys, its wavefronts every NW-th tile of 32 keys, each through LDS buffers of its own.  The wavefronts' sums meet
// in LDS; those of several chunks in the workspace, joined by attention_join_kernel.  One buffer for k and one for v, so
// that two workgroups share a CU: with two of each and one workgroup, 16 caches of 2048 tokens took 44 us instead of 32
// (4.2 TB/s, join included).
template <int DT, int HD> struct DecodeShape {
    static constexpr int HALF = 32 * KvTile<DT, HD>::ROW, STAGE = 2 * HALF;  // k, and v behind it
    static constexpr int NW = 4;
    static constexpr int SROW = HD + 4;                                       // floats of a row where the sums meet
    static constexpr int JOIN = NW * (32 * SROW + 64) * 4, LDS = NW * STAGE > JOIN ? NW * STAGE : JOIN;
};

template <int DT, int HD> __global__ __launch_bounds__((DecodeShape<DT, HD>::NW * 64), (DecodeShape<DT, HD>::LDS > 81920 ? 1 : 2)) void attention_decode_kernel(const AttentionArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef KvTile<DT, HD> Tile;
    typedef DecodeShape<DT, HD> Shape;
    constexpr int ES = Tile::ES, STEPS = HD * ES / 32, NW = Shape::NW, LOADS = Shape::HALF / 1024;  // of k, of v
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int item = blockIdx.x;
    const int kv_head = item % a.kv_heads;
    item /= a.kv_heads;
    const int block = item % a.row_blocks;
    item /= a.row_blocks;
    const int seq = item % a.n_seqs, chunk = item / a.n_seqs;
    int q0, nq;
    range_of(a.q_offsets, seq, a.total_q, &q0, &nq);
    int k0, nk;
    range_of(a.kv_offsets, seq, a.total_kv, &k0, &nk);
    const int rows = nq * a.group - block * 32;  // (query, head of the group), heads fastest
    if (rows <= 0 || (chunk > 0 && chunk * a.chunk >= nk)) return;
    const int my = block * 32 + min(col, rows - 1), query = my / a.group, head = kv_head * a.group + my - query * a.group;
    const int last_query = min(nq * a.group - 1, block * 32 + 31) / a.group;
    const int first_unseen = a.causal ? min(nk, query + nk - nq + 1) : nk;
    const int begin = chunk * a.chunk, end = max(begin, min(begin + a.chunk, a.causal ? min(nk, last_query + nk - nq + 1) : nk));
    const int all = a.causal ? min(nk, block * 32 / a.group + nk - nq + 1) : nk;  // keys that every query of the block sees
    const int row_bytes = a.head_dim * ES;

    u32x4_t q[STEPS];
    const unsigned char* qp = a.q + (long long)(q0 + query) * a.ldq + head * a.hq;
#pragma unroll
    for (int c = 0; c < STEPS; ++c) {
        q[c] = (2 * c + h) * 16 < row_bytes ? *(const u32x4_t*)(qp + (2 * c + h) * 16) : u32x4_t{0, 0, 0, 0};
        q[c] ^= a.q_flip;
    }
    const unsigned char* kp = a.k + (long long)(k0 + begin) * a.ldk + kv_head * a.hk;
    const unsigned char* vp = a.v + (long long)(k0 + begin) * a.ldv + kv_head * a.hv;
    const int tiles = (end - begin + 31) >> 5;
    // One buffer for k and one for v: the next k is requested when the scores are there, the next v behind the products.
    unsigned char* mine = smem + wave * Shape::STAGE;
    const unsigned at = (unsigned)(wave * Shape::STAGE);
    auto request_k = [&](int t) {
        request_tile<DT, HD, 32>(kp + (long long)t * 32 * a.ldk, a.ldk, max(0, min(32, end - begin - t * 32)), row_bytes, mine, 0, 1);
    };
    auto request_v = [&](int t) {
        request_tile<DT, HD, 32>(vp + (long long)t * 32 * a.ldv, a.ldv, max(0, min(32, end - begin - t * 32)), row_bytes, mine + Shape::HALF, 0, 1);
    };
    auto landed = [] {  // all but the last LOADS requests
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((LOADS & 15) | ((LOADS >> 4) << 14) | 0x0F70);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto read = [] {  // what was read from LDS has arrived, the buffer may be written
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_sched_barrier(0);
    };
    Running<DT, HD> run;
    run.start();
    request_k(wave);
    request_v(wave);
    for (int t = wave; t < tiles; t += NW) {
        landed();
        const int key0 = begin + t * 32;
        auto k_done = [&] {
            read();
            request_k(t + NW);
        };
        if (key0 + 32 <= all) run.template tile<1, false>(q, a.scale_log2, at, at + Shape::HALF, key0, first_unseen, k_done, landed);
        else run.template tile<1, true>(q, a.scale_log2, at, at + Shape::HALF, key0, first_unseen, k_done, landed);
        read();
        request_v(t + NW);
    }
    __builtin_amdgcn_s_waitcnt(0);  // requests past the end write zeros
    __syncthreads();
    float* sums = (float*)smem;  // [wavefront][column][channel], then [wavefront][column] maxima and sums
    float* tops = sums + NW * 32 * Shape::SROW;
    float* totals = tops + NW * 32;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *(float4*)(sums + (wave * 32 + col) * Shape::SROW + d * 32 + (i >> 2) * 8 + h * 4) = make_float4(run.o[d][i], run.o[d][i + 1], run.o[d][i + 2], run.o[d][i + 3]);
    const float sum = run.total();
    if (h == 0) {
        tops[wave * 32 + col] = run.top;
        totals[wave * 32 + col] = sum;
    }
    __syncthreads();
    const int live = min(rows, 32), vecs = a.head_dim >> 2;
    const bool whole = a.chunks == 1 || nk <= a.chunk;  // (a sequence longer than max_kv has no room for partial sums)
    for (int e = threadIdx.x; e < live * vecs; e += NW * 64) {
        const int r = e / vecs, c = (e - r * vecs) * 4;
        float top = tops[r], total = 0.f, z[4] = {};
#pragma unroll
        for (int v = 1; v < NW; ++v) top = fmaxf(top, tops[v * 32 + r]);
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float t = tops[v * 32 + r], w = t == top ? 1.f : __builtin_amdgcn_exp2f(t - top);  // (both may be -inf: sums of 0)
            total = __builtin_fmaf(totals[v * 32 + r], w, total);
#pragma unroll
            for (int x = 0; x < 4; ++x) z[x] = __builtin_fmaf(sums[(v * 32 + r) * Shape::SROW + c + x], w, z[x]);
        }
        const int row = block * 32 + r, qi = row / a.group, hd = kv_head * a.group + row - qi * a.group;
        if (whole) {
            const float inv = normaliser(total, (a.causal ? min(nk, qi + nk - nq + 1) : nk) > 0);
#pragma unroll
            for (int x = 0; x < 4; ++x) z[x] *= inv;
            store4<DT>(a.o + (long long)(q0 + qi) * a.ldo + hd * a.ho, c, z);
        } else {
            const long long at = ((long long)chunk * a.total_q + q0 + qi) * a.heads + hd;
            *(float4*)(a.part_o + at * a.head_dim + c) = make_float4(z[0], z[1], z[2], z[3]);
            if (c == 0) a.part_stat[at] = make_float2(top, total);
        }
    }
#endif
}

// Joins the chunks of what has several: 256 / ROWS threads per query and head, four channels a lane, 8 / ROWS chunks at
// a time, added in a fixed order.
constexpr int kMaxChunks = 576, kMaxPromptChunks = 64;  // of plan_attention: a few more than the 512 CUs of the largest partition
template <int DT, int ROWS> __global__ __launch_bounds__(256) void attention_join_kernel(const AttentionArgs a)
{
#if __HIP_DEVICE_COMPILE__
    constexpr int THREADS = 256 / ROWS, GROUPS = THREADS / 32;
    static_assert(ROWS == 1 || ROWS == 4, "a workgroup or a wavefront");
    __shared__ float weights[ROWS][ROWS == 1 ? kMaxChunks : kMaxPromptChunks];
    __shared__ float stat[8];
    __shared__ float4 part[8][32];
    const int tid = threadIdx.x % THREADS, lane = tid & 31, group = tid >> 5;
    const long long item = (long long)blockIdx.x * ROWS + threadIdx.x / THREADS;
    const int token = (int)(item / a.heads), head = (int)(item - (long long)token * a.heads);
    if (token >= a.total_q) return;
    const int seq = last_not_above(a.q_offsets, a.n_seqs, token, [](int offset, int) { return offset; });
    int q0, nq, k0, nk;
    range_of(a.q_offsets, seq, a.total_q, &q0, &nq);
    range_of(a.kv_offsets, seq, a.total_kv, &k0, &nk);
    const int query = token - q0, n = query < 0 || query >= nq ? 1 : chunks_of(a, query, nq, nk);
    if (n == 1) return;
    const long long step = (long long)a.total_q * a.heads;
    float* weight = weights[threadIdx.x / THREADS];
    // what other lanes write to LDS is read behind it: a wavefront's own LDS operations run in order, as long as the compiler
    // leaves them so
    auto meet = [] {
        if constexpr (ROWS == 1) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    // maximum, weights and sum
    float top = -INFINITY, total = 0.f;
    for (int s = tid; s < n; s += THREADS) top = fmaxf(top, a.part_stat[s * step + item].x);
#pragma unroll
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    if constexpr (ROWS == 1) {
        if ((tid & 63) == 0) stat[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(stat[0], stat[1]), fmaxf(stat[2], stat[3]));
    }
    for (int s = tid; s < n; s += THREADS) {
        const float2 st = a.part_stat[s * step + item];
        const float w = st.x == top ? 1.f : __builtin_amdgcn_exp2f(st.x - top);
        weight[s] = w;
        total = __builtin_fmaf(st.y, w, total);
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) total += __shfl_xor(total, x);
    if constexpr (ROWS == 1) {
        if ((tid & 63) == 0) stat[4 + (tid >> 6)] = total;
    }
    meet();
    if constexpr (ROWS == 1) total = (stat[4] + stat[5]) + (stat[6] + stat[7]);
    float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
    const int c = lane * 4;
    if (c < a.head_dim) {
        const float* p = a.part_o + item * a.head_dim + c;
#pragma unroll 4
        for (int s = group; s < n; s += GROUPS) {
            const float w = weight[s];
            const float4 o = *(const float4*)(p + s * step * a.head_dim);
            z = make_float4(__builtin_fmaf(o.x, w, z.x), __builtin_fmaf(o.y, w, z.y), __builtin_fmaf(o.z, w, z.z), __builtin_fmaf(o.w, w, z.w));
        }
    }
    float4(*parts)[32] = part + threadIdx.x / THREADS * GROUPS;
    parts[group][lane] = z;
    meet();
    if (group || c >= a.head_dim) return;
    float out[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) {
        const float4 t = parts[g][lane];
        out[0] += t.x;
        out[1] += t.y;
        out[2] += t.z;
        out[3] += t.w;
    }
    const float inv = normaliser(total, (a.causal ? min(nk, query + nk - nq + 1) : nk) > 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] *= inv;
    store4<DT>(a.o + (long long)token * a.ldo + head * a.ho, c, out);
#endif
}

// ---- plans -------------------------------------------------------------------------------------
struct AttentionPlan {
    bool decode;
    int chunk, chunks, row_blocks;
};

static AttentionPlan plan_attention(const sgprs_attention_desc_t& d, int cus)
{
    AttentionPlan p = {};
    // Few queries, or keys enough that reading them once for a key head's whole group is what counts.  This way / as
    // prompts: 16 queries against 4000 keys, 8 sequences, 16/4 heads of 128, 30 / 50 us; 64 queries 46 / 58; 128 against
    // 4000, 2 sequences, 8 heads of 64, 16.4 / 20.0; 256 sequences of 32, 8 heads of 64, 17.8 / 17.6, but of 64 32 / 23.6.
    const int group = d.heads / d.kv_heads;
    p.decode = d.max_q <= 32 || ((long long)d.max_q * group <= 256 && d.max_kv >= 16ll * d.max_q);
    p.chunk = std::max(1, d.max_kv);
    p.chunks = 1;
    if (!p.decode) {
        // Where the tiles leave workgroup slots idle (one a CU for wide fp32 heads, else two), a tile's keys may be split,
        // 128 or more for a workgroup; under the causal mask half of the chunks lie behind what their queries see.  Worth
        // it where the estimate, in us, says so: a workgroup's keys one after another, against a second launch and partial
        // sums written and read.  Split / whole, 256 CUs: 4096 causal tokens, 4 heads of 128, 57 / 112 us; 1000, 2 of 64,
        // 13 / 22; ragged fp32, 6/2 of 72, 39 / 92; but 8 x 600, 8 of 128, 43 / 31; 2 x 1000, 8 of 64, 30 / 22.
        const double tiles = (d.total_q / (double)kPromptRows + 0.5 * d.n_seqs) * d.heads;
        const bool f32 = d.dtype == SGPRS_F32;
        const double slots = (f32 && d.head_dim > 64 ? 1.0 : 2.0) * cus * (d.causal ? 2 : 1);
        const int most = std::min({(int)std::lround(std::min(slots / tiles, 1000.0)), (d.max_kv + 127) / 128, kMaxPromptChunks});
        const double keys_us = d.max_kv * (f32 ? 0.001 * d.head_dim : 0.006 + 0.00015 * d.head_dim);
        const double chunk_us = 2.0 * 4 * d.total_q * d.heads * d.head_dim / 2.5e6;
        auto us = [&](int c) { return keys_us / c + (c > 1 ? 6 + (d.causal ? 0.5 * (c + 1) : c) * chunk_us : 0.0); };
        int best = 1;
        for (int c = 2; c <= most; ++c)
            if (us(c) < us(best)) best = c;
        if (best > 1) {
            p.chunk = ((d.max_kv + best - 1) / best + 63) / 64 * 64;
            p.chunks = (d.max_kv + p.chunk - 1) / p.chunk;
        }
    } else {
        p.row_blocks = (d.max_q * group + 31) / 32;
        // Chunks of keys for a workgroup a CU, 128 keys (a tile for each wavefront) or more: 16 caches of 2048 tokens,
        // 32/8 heads of 128, take 31.6 us so, 32.9 with two and 34.9 with three (more partial sums to join); one cache
        // of 8192 12.7, 13.7 and 13.7.
        const long long want = (long long)d.total_kv * d.kv_heads * p.row_blocks / cus;
        p.chunk = (int)std::min<long long>(std::max<long long>(want + 127, 128) / 128 * 128, 1 << 30);
        p.chunks = std::max(1, (d.max_kv + p.chunk - 1) / p.chunk);
    }
    return p;
}

size_t attention_workspace_bytes(const sgprs_attention_desc_t& d, int cus)
{
    const AttentionPlan p = plan_attention(d, cus);
    return p.chunks > 1 ? (size_t)p.chunks * d.total_q * d.heads * (d.head_dim * sizeof(float) + sizeof(float2)) : 0;
}

constexpr long long kMaxGrid = (1ll << 24) - 1;  // workgroups of 256 threads: a launch has less than 2^32 threads
static int too_large(const AttentionArgs& a)
{
    return fail(SGPRS_ERR_UNSUPPORTED, "%d sequences of %d tokens and %d heads", a.n_seqs, a.total_q, a.heads);
}

template <auto kernel> static int launch_sized(long long grid, int threads, int lds, const AttentionArgs& a, hipStream_t stream)
{
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    SGPRS_LAUNCH(kernel, dim3((unsigned)grid), threads, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

template <int DT, int HD> static int launch_shape(AttentionArgs a, bool decode, hipStream_t stream)
{
    if (!decode) {
        a.slots = a.total_q / kPromptRows + a.n_seqs;
        a.tile_rows = kPromptRows;
        const long long grid = (long long)a.chunks * a.slots * a.heads, join = ((long long)a.total_q * a.heads + 3) / 4;
        if (grid > kMaxGrid || (a.chunks > 1 && join > kMaxGrid)) return too_large(a);  // (before anything is enqueued)
        const int rc = launch_sized<attention_prompt_kernel<DT, HD>>(grid, 256, PromptShape<DT, HD>::STAGES * PromptShape<DT, HD>::STAGE, a, stream);
        if (rc || a.chunks == 1) return rc;
        return launch_sized<attention_join_kernel<DT, 4>>(join, 256, 0, a, stream);
    }
    typedef DecodeShape<DT, HD> Shape;
    static_assert(Shape::NW * 64 == 256, "kMaxGrid's workgroups");
    const long long grid = (long long)a.chunks * a.n_seqs * a.row_blocks * a.kv_heads, join = (long long)a.total_q * a.heads;
    if (grid > kMaxGrid || (a.chunks > 1 && join > kMaxGrid)) return too_large(a);
    const int rc = launch_sized<attention_decode_kernel<DT, HD>>(grid, Shape::NW * 64, Shape::LDS, a, stream);
    if (rc || a.chunks == 1) return rc;
    return launch_sized<attention_join_kernel<DT, 1>>(join, 256, 0, a, stream);
}

template <int DT> static int launch_typed(const AttentionArgs& a, bool decode, hipStream_t stream)
{
    if (a.head_dim <= 32) return launch_shape<DT, 32>(a, decode, stream);
    if (a.head_dim <= 64) return launch_shape<DT, 64>(a, decode, stream);
    if (a.head_dim <= 96) return launch_shape<DT, 96>(a, decode, stream);
    return launch_shape<DT, 128>(a, decode, stream);
}

int launch_attention(const sgprs_attention_desc_t& d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                     void* o, void* ws, hipStream_t stream, int cus)
{
    const long long es = (long long)dtype_size(d.dtype);
    const AttentionPlan p = plan_attention(d, cus);
    AttentionArgs a = {(const unsigned char*)q, (const unsigned char*)k, (const unsigned char*)v, (unsigned char*)o, q_offsets, kv_offsets,
                             d.n_seqs, d.total_q, d.total_kv, d.heads, d.kv_heads, d.heads / d.kv_heads, d.head_dim, d.causal,
                             std::fabs(d.scale) * 1.4426950408889634f, d.scale >= 0.f ? 0u : d.dtype == SGPRS_BF16 ? 0x80008000u : 0x80000000u,
                             (int)(d.ldq * es), (int)(d.ldk * es), (int)(d.ldv * es), (int)(d.ldo * es), d.hq * es, d.hk * es, d.hv * es, d.ho * es, 0, p.chunk, p.chunks, 0, p.row_blocks, nullptr, nullptr};
    a.part_o = (float*)ws;  // first, so that its vectors of four lie on multiples of 16 bytes
    a.part_stat = (float2*)(a.part_o + (size_t)p.chunks * d.total_q * d.heads * d.head_dim);
    return d.dtype == SGPRS_BF16 ? launch_typed<SGPRS_BF16>(a, p.decode, stream) : launch_typed<SGPRS_F32>(a, p.decode, stream);
}

}  // namespace sgprs
