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
    static __device__ __forceinline__ int swizzle(int r)
    {
        if constexpr (ROW == 64) return (r >> 2) & 3;
        if constexpr (ROW == 128) return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
        if constexpr (DT == SGPRS_BF16) return (r & 3) << 2 | ((r >> 2) & 3);
        return ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 | (r & 3);
    }
};

#if __HIP_DEVICE_COMPILE__
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
typedef __attribute__((address_space(3))) unsigned lds_u32_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// One of the `parts` wavefronts' share of a tile: rows of a tensor that starts at p, `rows` of them, into LDS at `to`.
template <int DT, int HD> __device__ __forceinline__ void request_tile(const unsigned char* p, int ld, int rows, int row_bytes, unsigned char* to, int part, int parts)
{
    typedef KvTile<DT, HD> Tile;
    constexpr int RPI = 1024 / Tile::ROW, LOADS = Tile::BYTES / 1024;  // rows of a load
    const int lane = threadIdx.x & 63, lrow = lane / Tile::CHUNKS, slot = lane % Tile::CHUNKS;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, rows > 0 ? (rows - 1) * ld + row_bytes : 0, 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS / parts; ++i) {
        const int r = (i * parts + part) * RPI + lrow, chunk = slot ^ Tile::swizzle(r);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t)(to + (i * parts + part) * 1024), 16,
                                                 chunk * 16 < row_bytes ? (unsigned)(r * ld + chunk * 16) : kOutside, 0, 0, 0);
    }
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// scores of 32 keys (rows `block` * 32 and on of the tile at `at`) with this lane's query
template <int DT, int HD> __device__ __forceinline__ f32x16_t scores(unsigned at, int block, const u32x4_t* q)
{
    typedef KvTile<DT, HD> Tile;
    constexpr int STEPS = HD * Tile::ES / 32;  // two chunks each
    const int lane = threadIdx.x & 63, r = block * 32 + (lane & 31), h = lane >> 5;
    f32x16_t s = {};
#pragma unroll
    for (int c = 0; c < STEPS; ++c) {
        const u32x4_t k = *(const lds_u32x4_t*)(unsigned long)(at + r * Tile::ROW + (((2 * c + h) ^ Tile::swizzle(r)) << 4));
        if constexpr (DT == SGPRS_BF16) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q[c]), s, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(q[c][e]), s, 0, 0, 0);
        }
    }
    return s;
}

// v of channels 32 d and on at keys 16 u of a block, as the row operand (bf16)
template <int HD> __device__ __forceinline__ u32x4_t value_fragment(unsigned at, int block, int u, int d)
{
    typedef KvTile<SGPRS_BF16, HD> Tile;
    const int lane = threadIdx.x & 63, s = lane & 15, h = lane >> 5, g = (lane >> 4) & 1;
    u32x4_t f;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const int r = block * 32 + u * 16 + a * 8 + h * 4 + (s >> 2), chunk = d * 4 + g * 2 + ((s & 3) >> 1);
        const s16x4_t t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(unsigned long)(at + r * Tile::ROW + ((chunk ^ Tile::swizzle(r)) << 4) + (s & 1) * 8));
        const u32x2_t w = __builtin_bit_cast(u32x2_t, t);
        f[2 * a] = w[0];
        f[2 * a + 1] = w[1];
    }
    return f;
}

// o += V^T P^T for one block of 32 keys; p: this lane's 16 weights.  `masked`: some weights are zero because their
// keys are not seen; should v hold infinities or NaNs there, 0 * v would be NaN, so such values are taken out of the
// product and counted, in a second one, for the queries that see them.  seen: 1 or 0 for each weight.
template <int DT, int HD>
__device__ __forceinline__ void add_values(f32x16_t* o, const float* p, unsigned at, int block, bool masked, const float* seen)
{
    typedef KvTile<DT, HD> Tile;
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
                u32x4_t f = value_fragment<HD>(at, block, u, d);
                if (masked) {
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= (f[e] & 0x7f80u) == 0x7f80u || (f[e] & 0x7f800000u) == 0x7f800000u;
                    if (__any(odd)) {
                        u32x4_t kind, sw;  // of each value that is not finite: 1 for inf, 2^8 for -inf, 2^16 for NaN
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            kind[e] = 0;
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const unsigned v = f[e] >> (16 * half) & 0xffffu;
                                if ((v & 0x7f80u) != 0x7f80u) continue;
                                kind[e] |= (v & 0x7fu ? 0x4780u : v & 0x8000u ? 0x4380u : 0x3f80u) << (16 * half);
                                f[e] &= ~(0xffffu << (16 * half));
                            }
                            sw[e] = pack_bf16x2_relu(seen[8 * u + 2 * e], seen[8 * u + 2 * e + 1], kNoReluFloor);
                        }
                        f32x16_t count = {};
                        count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kind), __builtin_bit_cast(bf16x8_t, sw), count, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const unsigned n = (unsigned)count[i];
                            if (n) o[d][i] += n >> 16 || (n >> 8 && n & 0xffu) ? NAN : n >> 8 ? -INFINITY : INFINITY;
                        }
                    }
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, w[u]), o[d], 0, 0, 0);
            }
    } else {
        const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = block * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int chunk = d * 8 + ((lane & 31) >> 2);
                float f = __uint_as_float(*(const lds_u32_t*)(unsigned long)(at + r * Tile::ROW + ((chunk ^ Tile::swizzle(r)) << 4) + (lane & 3) * 4));
                if (masked) {
                    const bool odd = !(fabsf(f) < INFINITY);
                    if (__any(odd)) {
                        f32x16_t count = {};
                        count = __builtin_amdgcn_mfma_f32_32x32x2f32(odd ? f != f ? 65536.f : f < 0.f ? 256.f : 1.f : 0.f, seen[i], count, 0, 0, 0);
                        if (odd) f = 0.f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const unsigned n = (unsigned)count[j];
                            if (n) o[d][j] += n >> 16 || (n >> 8 && n & 0xffu) ? NAN : n >> 8 ? -INFINITY : INFINITY;
                        }
                    }
                }
                o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(f, p[i], o[d], 0, 0, 0);
            }
        }
    }
}

// A query's running softmax: maximum (of scores as they are multiplied, in base 2), sum of the weights, results.
template <int DT, int HD> struct Running {
    static constexpr int DB = HD / 32;
    f32x16_t o[DB];
    float top, sum;
    __device__ __forceinline__ void start()
    {
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
    }
    // keys from `key` on are not seen; BLOCKS blocks of 32 from key0 on, at LDS address k_at and v_at
    template <int BLOCKS> __device__ __forceinline__ void tile(const u32x4_t* q, float scale_log2, unsigned k_at, unsigned v_at, int key0, int first_unseen, bool masked)
    {
        const int h = (threadIdx.x & 63) >> 5;
        f32x16_t s[BLOCKS];
        float most = -INFINITY;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            s[b] = scores<DT, HD>(k_at, b, q);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + b * 32 + (i >> 2) * 8 + h * 4 + (i & 3) >= first_unseen) s[b][i] = -INFINITY;
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
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            float p[16], seen[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale_log2, -base));
                sum += p[i];
                seen[i] = key0 + b * 32 + (i >> 2) * 8 + h * 4 + (i & 3) < first_unseen ? 1.f : 0.f;
            }
            add_values<DT, HD>(o, p, v_at, b, masked, seen);
        }
    }
};
#endif

// Sequence and tile of a slot: a sequence's tiles start at slot q_offsets[s] / BM + s, which leaves each its own.
__device__ __forceinline__ bool tile_of_slot(const AttentionArgs& a, int slot, int bm, int* seq, int* row, int* q0, int* nq)
{
    int lo = 0, hi = a.n_seqs;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_offsets[mid] / bm + mid <= slot) lo = mid;
        else hi = mid;
    }
    const int first = min(max(a.q_offsets[lo], 0), a.total_q), end = min(max(a.q_offsets[lo + 1], first), a.total_q);
    const int tile = slot - (a.q_offsets[lo] / bm + lo);
    *seq = lo;
    *q0 = first;
    *nq = end - first;
    *row = tile * bm;
    return tile >= 0 && tile < (1 << 24) && *row < *nq;
}

// ---- prompts -----------------------------------------------------------------------------------
// 128 queries of one head per workgroup, 32 per wavefront; tiles of keys double buffered in LDS.
template <int DT, int HD> __global__ __launch_bounds__(256, 2) void attention_prompt_kernel(const AttentionArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef KvTile<DT, HD> Tile;
    constexpr int ES = Tile::ES, STEPS = HD * ES / 32, BM = 128, LPW = Tile::BYTES / 1024 / 4;
    static_assert(2 * LPW <= 63, "vmcnt range");
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // heavy tiles (the last ones under the causal mask) first; heads that share keys on one die where there are eight of them
    const int item = blockIdx.x, j = item % a.heads, slot = a.slots - 1 - item / a.heads;
    const int kv_head = j % a.kv_heads, head = kv_head * a.group + j / a.kv_heads;
    int seq, row0, q0, nq;
    if (!tile_of_slot(a, slot, BM, &seq, &row0, &q0, &nq)) return;
    const int k0 = min(max(a.kv_offsets[seq], 0), a.total_kv), nk = min(max(a.kv_offsets[seq + 1], k0), a.total_kv) - k0;
    const int row = row0 + wave * 32 + (lane & 31);       // of the sequence
    const int last_row = min(row0 + BM, nq) - 1;
    const int keys = a.causal ? max(0, min(nk, last_row + nk - nq + 1)) : nk;  // that anyone here sees
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
    const unsigned char* kp = a.k + (long long)k0 * a.ldk + kv_head * a.hk;
    const unsigned char* vp = a.v + (long long)k0 * a.ldv + kv_head * a.hv;
    auto request = [&](int t) {
        unsigned char* to = smem + (t & 1) * 2 * Tile::BYTES;
        const int rows = max(0, min(Tile::KEYS, nk - t * Tile::KEYS));
        request_tile<DT, HD>(kp + (long long)t * Tile::KEYS * a.ldk, a.ldk, rows, row_bytes, to, wave, 4);
        request_tile<DT, HD>(vp + (long long)t * Tile::KEYS * a.ldv, a.ldv, rows, row_bytes, to + Tile::BYTES, wave, 4);
    };
    Running<DT, HD> run;
    run.start();
    const int tiles = (keys + Tile::KEYS - 1) / Tile::KEYS;
    if (tiles > 0) request(0);
    for (int t = 0; t < tiles; ++t) {
        __builtin_amdgcn_s_waitcnt(0x0F70);  // this tile has landed
        __builtin_amdgcn_s_barrier();        // everyone's, and everyone has left the other buffer
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < tiles) request(t + 1);
        const unsigned at = (unsigned)((t & 1) * 2 * Tile::BYTES);
        const int key0 = t * Tile::KEYS;
        if (key0 < wave_any) {
            if (key0 + Tile::KEYS <= wave_all) run.template tile<Tile::KEYS / 32>(q, a.scale_log2, at, at + Tile::BYTES, key0, first_unseen, false);
            else run.template tile<Tile::KEYS / 32>(q, a.scale_log2, at, at + Tile::BYTES, key0, first_unseen, true);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
    }
    if (row >= nq) return;
    const float sum = run.sum + other_half(run.sum);
    const float inv = sum > 0.f ? 1.f / sum : first_unseen > 0 ? NAN : 0.f;
    unsigned char* op = a.o + (long long)(q0 + row) * a.ldo + head * a.ho;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int c = d * 32 + (i >> 2) * 8 + h * 4;
            if (c >= a.head_dim) continue;
            if constexpr (DT == SGPRS_BF16) {
                *(u32x2_t*)(op + c * 2) = u32x2_t{pack_bf16x2_relu(run.o[d][i] * inv, run.o[d][i + 1] * inv, kNoReluFloor),
                                                  pack_bf16x2_relu(run.o[d][i + 2] * inv, run.o[d][i + 3] * inv, kNoReluFloor)};
            } else {
                u32x4_t w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(run.o[d][i + e] * inv);
                *(u32x4_t*)(op + c * 4) = w;
            }
        }
#endif
}

// ---- plans -------------------------------------------------------------------------------------
size_t attention_workspace_bytes(const sgprs_attention_desc_t&, int) { return 0; }

template <int DT, int HD> static int launch_prompt(AttentionArgs a, hipStream_t stream)
{
    constexpr int lds = 4 * KvTile<DT, HD>::BYTES;
    a.slots = a.total_q / 128 + a.n_seqs;
    const long long grid = (long long)a.slots * a.heads;
    if (grid >= (1ll << 31)) return fail(SGPRS_ERR_UNSUPPORTED, "%d sequences of %d tokens and %d heads", a.n_seqs, a.total_q, a.heads);
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)attention_prompt_kernel<DT, HD>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    SGPRS_LAUNCH((attention_prompt_kernel<DT, HD>), dim3((unsigned)grid), 256, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

template <int DT> static int launch_typed(const AttentionArgs& a, hipStream_t stream)
{
    if (a.head_dim <= 32) return launch_prompt<DT, 32>(a, stream);
    if (a.head_dim <= 64) return launch_prompt<DT, 64>(a, stream);
    if (a.head_dim <= 96) return launch_prompt<DT, 96>(a, stream);
    return launch_prompt<DT, 128>(a, stream);
}

int launch_attention(const sgprs_attention_desc_t& d, const void* q, const void* k, const void* v, const int* q_offsets, const int* kv_offsets,
                     void* o, void* ws, hipStream_t stream, int cus)
{
    const long long es = (long long)dtype_size(d.dtype);
    const AttentionArgs a = {(const unsigned char*)q, (const unsigned char*)k, (const unsigned char*)v, (unsigned char*)o, q_offsets, kv_offsets,
                             d.n_seqs, d.total_q, d.total_kv, d.heads, d.kv_heads, d.heads / d.kv_heads, d.head_dim, d.causal,
                             std::fabs(d.scale) * 1.4426950408889634f, d.scale >= 0.f ? 0u : d.dtype == SGPRS_BF16 ? 0x80008000u : 0x80000000u,
                             (int)(d.ldq * es), (int)(d.ldk * es), (int)(d.ldv * es), (int)(d.ldo * es), d.hq * es, d.hk * es, d.hv * es, d.ho * es, 0};
    return d.dtype == SGPRS_BF16 ? launch_typed<SGPRS_BF16>(a, stream) : launch_typed<SGPRS_F32>(a, stream);
}

}  // namespace sgprs
