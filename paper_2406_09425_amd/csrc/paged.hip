// A cache of pages: new keys and values to their places, and attention of one new token of each sequence over them.
//
// Attention is bound by reading the cache.  The queries of all heads that share a key head are one block of 32 columns (or
// several), so a key is read once for them.  An item is a sequence, a key head and a block; its visible positions, one
// behind the other (first tokens, then the window), form units of 128.  All items in a row are divided into runs of equal
// cost, one for each workgroup, which may begin and end inside items: however different the lengths are, all workgroups
// have the same to do.  An item that several of them share is joined by a second launch from partial sums, two at most of a
// workgroup, in a fixed order.  Wavefront v of four takes every fourth tile of 32 keys of an item, k and v through LDS
// buffers of its own, each row from wherever its page is.  Its requests run on over the end of an item: table entries come
// two tiles ahead, the next item's first tile is on its way while this one's sums meet.
//
// Measured, both launches, 256 CUs: 16 caches of 1 to 32768 tokens, 32/8 heads of 128 in bf16, 60 us (55 and 5; 265 MB, 4.5
// TB/s); 16 of 4096, 8 heads of 128 in fp32, 102 (5.3 TB/s).  With a run for each wavefront instead of each workgroup 16 equal
// caches took 69 for 61: four times the partial sums.  Few short caches are a chain of latencies (lengths, table, keys, the
// join's launch): three of up to 700 in 8.7 us, one of 2048 in 11.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>
#include <utility>

#include "attention_tiles.h"
#include "decode_ops.h"

namespace sgprs {

struct JoinRecord {
    int seq, item, last, unused;  // what begins in a workgroup's run and ends in that of workgroup `last` (-1: nothing)
};

struct PagedArgs {
    const unsigned char *q, *k, *v;
    unsigned char* o;
    const int *table, *lens;
    int n_seqs, heads, kv_heads, group, head_dim;
    int n_pages, page_size, table_width;
    unsigned page_mul;
    int page_sh;                     // position / page_size
    int window, sinks;
    float scale_log2;                // |scale| log2 e
    unsigned q_flip;                 // sign bits of a dword of q, where the scale is negative
    int ldq, ldo;                    // bytes
    long long hq, ho;                // bytes
    long long page_stride, token_stride, head_stride;  // bytes
    int row_blocks, rows;            // blocks of 32 heads of a key head; rows of the largest
    int items;                       // of a sequence
    unsigned heads_mul, grid_mul;
    int heads_sh, grid_sh;           // item / kv_heads, cost / workgroups
    int unit_log2;                   // tiles of a unit
    float* part_o;                   // [workgroup][item that goes on, item that begins][row][head_dim], weights relative to part_stat
    float2* part_stat;               // [workgroup][item that goes on, item that begins][row]: maximum, sum
    JoinRecord* records;             // [workgroup]
};

constexpr int kWaves = 4;            // of a workgroup
constexpr int kMaxWorkgroups = 2 * SGPRS_MAX_MASK_WORDS * 32;
constexpr int kItemCost = 1;         // what an item costs beside its units, in units
constexpr int kMeetRows = 4;         // rows whose sums meet in LDS at once

__device__ __align__(16) unsigned paged_zeros[128] = {};  // a row that is loaded for positions behind the last

__device__ __forceinline__ int quotient(int n, unsigned mul, int sh) { return (int)(__umulhi(2u * (unsigned)n, mul) >> sh); }

// The positions that a sequence's new token sees: n of them, the i-th at i or, from `sinks` on, at i + gap.
struct Seen {
    int n, sinks, gap;
    __device__ __forceinline__ int units(const PagedArgs& a) const { return max(1, (((n + 31) >> 5) + (1 << a.unit_log2) - 1) >> a.unit_log2); }  // (one to write zeros)
    __device__ __forceinline__ int cost(const PagedArgs& a) const { return units(a) + kItemCost; }
};
__device__ __forceinline__ Seen seen_of(const PagedArgs& a, int length)
{
    const int len = min(max(length, 0), a.table_width * a.page_size);
    const int first = a.window > 0 && len > a.window ? len - a.window : 0;
    const int sinks = min(a.sinks, first);
    return {sinks + len - first, sinks, first - sinks};
}

__device__ __forceinline__ int kv_head_of(const PagedArgs& a, int item) { return item - quotient(item, a.heads_mul, a.heads_sh) * a.kv_heads; }

// Runs of an equal cost (up to one): the first unit of workgroup w's, and whose a unit is.
struct Runs {
    int per, rest;
    __device__ __forceinline__ Runs(const PagedArgs& a, int cost, int runs) : per(quotient(cost, a.grid_mul, a.grid_sh)), rest(cost - per * runs) {}
    __device__ __forceinline__ int first(int w) const { return w * per + min(w, rest); }
    __device__ __forceinline__ int owner(int u) const
    {
        const unsigned longer = rest * (per + 1u);
        return (unsigned)u < longer ? (unsigned)u / (per + 1u) : rest + ((unsigned)u - longer) / (unsigned)per;
    }
};

#if __HIP_DEVICE_COMPILE__
// The running softmax of up to 4 SETS query heads in fp32 over tiles of 32 keys, with the same parts as Running.  MFMAs of 16
// blocks of 4 x 4 x 1: a block's rows are four keys and its columns four queries, so that few queries leave no column idle
// (32 x 32 x 2 takes eight times as long for them).  A row of a tile is CHUNKS chunks of four channels.
//   scores: lane l brings key l % 32 and the even (lanes below 32) or odd chunks; it ends up with the scores of query
//           l % 4 with keys 4 (l / 4 % 8) + r, half of the channels in each half of the wavefront.
//   values: a read brings PK keys, CHUNKS lanes each; the weights reach the lanes as row operands, where the instruction
//           hands those of one block in each group of blocks to all of the group.  Lane l ends up with channels
//           4 (l % CHUNKS) + e of all four queries, summed over every PK-th key.
// 16 caches of 4096, 8/8 heads of 128, when this was written: 111 us, by 32 x 32 x 2 MFMAs 151 (now 102).
template <int HD, int SETS> struct RunningNarrow {
    typedef KvTile<SGPRS_F32, HD> Tile;
    static constexpr int CHUNKS = Tile::CHUNKS, PK = 64 / CHUNKS, GROUP_LOG2 = CHUNKS == 32 ? 3 : CHUNKS == 16 ? 2 : 1;  // blocks of a group
    static constexpr int Q = CHUNKS / 2;  // vectors of q
    typedef float f32x4_t __attribute__((ext_vector_type(4)));
    f32x4_t o[SETS][4];  // [.][e][query]
    float top[SETS], sum[SETS];
    unsigned k_place, v_place;
    __device__ __forceinline__ RunningNarrow()
    {
        const int lane = threadIdx.x & 63, row = lane & 31, group = lane / CHUNKS;
        k_place = LanePlaces<SGPRS_F32, HD>::place(row, lane >> 5);
        // key of group g at step (block, r): 4 (g * blocks of a group + block) % 32 + r, the upper half one further
        v_place = LanePlaces<SGPRS_F32, HD>::place((group << (GROUP_LOG2 + 2)) % 32 + (lane >> 5), lane % CHUNKS);
    }
    __device__ __forceinline__ void start()
    {
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            top[s] = -INFINITY;
            sum[s] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[s][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
    // of query l % 4 of a set, in all lanes
    __device__ __forceinline__ float total(int s) const
    {
        float v = sum[s];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) v += __shfl_xor(v, x);
        return v;
    }
    // channels 4 (l % CHUNKS) + e of a set's query i, in all lanes
    __device__ __forceinline__ float4 result(int s, int i) const
    {
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            z[e] = o[s][e][i];
#pragma unroll
            for (int x = CHUNKS; x < 64; x <<= 1) z[e] += __shfl_xor(z[e], x);
        }
        return make_float4(z[0], z[1], z[2], z[3]);
    }
    static __device__ __forceinline__ float of_query(float v, int i)
    {
        const int w = __float_as_int(v);
        switch (i) {
        case 0: return __int_as_float(__builtin_amdgcn_mov_dpp(w, 0x00, 0xf, 0xf, true));
        case 1: return __int_as_float(__builtin_amdgcn_mov_dpp(w, 0x55, 0xf, 0xf, true));
        case 2: return __int_as_float(__builtin_amdgcn_mov_dpp(w, 0xaa, 0xf, 0xf, true));
        default: return __int_as_float(__builtin_amdgcn_mov_dpp(w, 0xff, 0xf, 0xf, true));
        }
    }
    template <class KDone, class VReady>
    __device__ __forceinline__ void tile(const u32x4_t (*q)[Q], float scale_log2, unsigned k_at, unsigned v_at, int key0, int first_unseen, KDone k_done, VReady v_ready)
    {
        const unsigned k_base = LanePlaces<SGPRS_F32, HD>::hidden(k_place + k_at), v_base = LanePlaces<SGPRS_F32, HD>::hidden(v_place + v_at);
        f32x4_t s[2 * SETS];  // (two chains of MFMAs that alternate)
#pragma unroll
        for (int n = 0; n < 2 * SETS; ++n) s[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < Q; ++c) {
            const u32x4_t k = *(const lds_u32x4_t*)(unsigned long)(k_base ^ (unsigned)(c << 5));
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int n = 0; n < SETS; ++n)
                    s[e % 2 * SETS + n] = __builtin_amdgcn_mfma_f32_4x4x1f32(__uint_as_float(k[e]), __uint_as_float(q[n][c][e]), s[e % 2 * SETS + n], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < SETS; ++n) s[n] += s[SETS + n];
        k_done();
        const int lane = threadIdx.x & 63, mine = first_unseen - key0 - ((lane >> 2) & 7) * 4;
        float p[SETS][4];
#pragma unroll
        for (int n = 0; n < SETS; ++n) {
            float most = -INFINITY;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[n][r] += __shfl_xor(s[n][r], 32);
                s[n][r] = r < mine ? s[n][r] : -INFINITY;
                most = fmaxf(most, s[n][r]);
            }
            most *= scale_log2;
            if (__any(most > top[n] + kKeepMax)) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) most = fmaxf(most, __shfl_xor(most, x));
                const float now = fmaxf(top[n], most), keep = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[n] - now);
                top[n] = now;
                sum[n] *= keep;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float k = of_query(keep, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[n][e][i] *= k;
                }
            }
            const float base = top[n] == -INFINITY ? 0.f : top[n] + kKeepMax;  // weights stay below 1, so sums with large v keep their range
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], scale_log2, -base));
                sum[n] += p[n][r];
            }
            const float odd0 = p[n][1], odd2 = p[n][3];  // the upper half takes the odd keys
            if (lane >= 32) {
                p[n][0] = odd0;
                p[n][2] = odd2;
            }
        }
        v_ready();
        all_values(v_base, p, std::make_integer_sequence<int, 1 << GROUP_LOG2>());
    }
    template <int... B> __device__ __forceinline__ void all_values(unsigned v_base, const float (*p)[4], std::integer_sequence<int, B...>) { (values<B>(v_base, p), ...); }
    template <int B> __device__ __forceinline__ void values(unsigned v_base, const float (*p)[4])
    {
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const u32x4_t v = *(const lds_u32x4_t*)(unsigned long)LanePlaces<SGPRS_F32, HD>::plus(v_base, 4 * B + r, 0);
#pragma unroll
            for (int n = 0; n < SETS; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = __builtin_amdgcn_mfma_f32_4x4x1f32(p[n][r], __uint_as_float(v[e]), o[n][e], GROUP_LOG2, B, 0);
        }
    }
};
#endif

template <int DT, int HD> struct PagedShape {
    static constexpr int HALF = 32 * KvTile<DT, HD>::ROW, STAGE = 2 * HALF;  // k, and v behind it
    static constexpr int SROW = HD + 4;                                       // floats of a row where the sums meet
    static constexpr int ROWS_AT = kWaves * STAGE, MEET = ROWS_AT + kWaves * 256, LDS = MEET + kWaves * kMeetRows * (SROW + 2) * 4;
    static constexpr int PER_CU = LDS > 81920 ? 1 : 2;
};

#if __HIP_DEVICE_COMPILE__
// What a run has of an item, the same for all lanes.
struct Segment {
    int seq, item, n, sinks, gap;  // item: of the sequence; n: positions
    int first, end, tiles;         // tiles that it has, of so many
    __device__ __forceinline__ bool begins() const { return first == 0; }
    __device__ __forceinline__ bool ends() const { return end == tiles; }
};
#endif

// SETS: of four heads of a key head, in fp32; 0: up to 32 heads.
// No vector register is spilled; of the scalars (some 50 dwords of arguments, segments, masks of padded chunks) 58 to 183 live in
// lanes of vector registers.  Channels 65 to 96 in fp32 take rows of 128 in LDS (138624 bytes, one workgroup of a CU).
template <int DT, int HD, int SETS> __global__ __launch_bounds__(256, (PagedShape<DT, HD>::PER_CU)) void paged_attention_kernel(const PagedArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef KvTile<DT, HD> Tile;
    typedef PagedShape<DT, HD> Shape;
    constexpr int ES = Tile::ES, STEPS = HD * ES / 32, NW = kWaves, LOADS = Shape::HALF / 1024, RPI = 1024 / Tile::ROW;
    extern __shared__ __align__(16) unsigned char smem[];  // (all of the LDS, from address 0 on)
    int* scratch = (int*)(smem + Shape::MEET);
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // ---- this workgroup's run, and the sequence that it begins in ----
    int seq, start, length, cost;  // start: the cost of the sequences before it
    if (a.n_seqs <= 64) {
        length = lane < a.n_seqs ? a.lens[lane] : 0;
        const int mine = lane < a.n_seqs ? seen_of(a, length).cost(a) * a.items : 0;
        int upto = mine;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int left = __shfl_up(upto, x);
            if (lane >= x) upto += left;
        }
        cost = __builtin_amdgcn_readlane(upto, 63);
        const int begin = Runs(a, cost, gridDim.x).first(blockIdx.x);
        seq = min((int)__popcll(__ballot(upto <= begin)), a.n_seqs - 1);  // (the costs rise, and those behind the last one are its)
        start = __builtin_amdgcn_readlane(upto - mine, seq);
        length = __builtin_amdgcn_readlane(length, seq);
    } else {
        const int share = (a.n_seqs + 255) >> 8, s0 = min((int)threadIdx.x * share, a.n_seqs), s1 = min(s0 + share, a.n_seqs);
        int mine = 0;
        for (int s = s0; s < s1; ++s) mine += seen_of(a, a.lens[s]).cost(a) * a.items;
        int upto = mine;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int left = __shfl_up(upto, x);
            if (lane >= x) upto += left;
        }
        if (lane == 63) scratch[wave] = upto;
        if (threadIdx.x == 0) scratch[NW] = a.n_seqs;
        __syncthreads();
        cost = 0;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            if (v == wave) upto += cost;
            cost += scratch[v];
        }
        const int begin = Runs(a, cost, gridDim.x).first(blockIdx.x);
        if (upto - mine <= begin && begin < upto) {
            int s = s0, before = upto - mine;
            for (; s < s1; ++s) {
                length = a.lens[s];
                const int c = seen_of(a, length).cost(a) * a.items;
                if (begin < before + c) break;
                before += c;
            }
            scratch[NW] = s;
            scratch[NW + 1] = before;
            scratch[NW + 2] = length;
        }
        __syncthreads();
        cost = __builtin_amdgcn_readfirstlane(cost);
        seq = __builtin_amdgcn_readfirstlane(scratch[NW]);
        start = __builtin_amdgcn_readfirstlane(scratch[NW + 1]);
        length = __builtin_amdgcn_readfirstlane(scratch[NW + 2]);
        __syncthreads();
    }
    const Runs runs(a, cost, gridDim.x);
    int at = runs.first(blockIdx.x);
    const int run_end = runs.first(blockIdx.x + 1);
    if (threadIdx.x == 0) a.records[blockIdx.x] = {0, 0, -1, 0};
    if (at >= run_end || seq >= a.n_seqs) return;

    Seen seen = seen_of(a, length);
    int item_cost = seen.cost(a), item = (int)((unsigned)(at - start) / (unsigned)item_cost), offset = at - start - item * item_cost;
    // The next item of the run that has tiles in it; false at the run's end.
    auto next_segment = [&](Segment& s) {
        while (at < run_end) {
            if (item == a.items) {
                item = 0;
                if (++seq >= a.n_seqs) return false;
                // (a scalar load: a vector load's wait would be for the keys on their way, too)
                seen = seen_of(a, *(const __attribute__((address_space(4))) int*)(unsigned long)(a.lens + seq));
                item_cost = seen.cost(a);
            }
            const int here = min(run_end - at, item_cost - offset), tiles = max(1, (seen.n + 31) >> 5);
            const int first = max(offset - kItemCost, 0) << a.unit_log2, end = min(max(offset + here - kItemCost, 0) << a.unit_log2, tiles);
            s = {seq, item, seen.n, seen.sinks, seen.gap, first, end, tiles};
            at += here;
            offset = 0;
            ++item;
            if (first < end) return true;
        }
        return false;
    };

    const int row_bytes = a.head_dim * ES;
    const int lrow = lane / Tile::CHUNKS, slot = (lane % Tile::CHUNKS) ^ Tile::swizzle(lrow);
    unsigned char* buffers = smem + wave * Shape::STAGE;
    const unsigned buffers_at = (unsigned)(wave * Shape::STAGE);
    auto landed = [](auto behind) {  // all but the last `behind` requests
        constexpr int N = decltype(behind)::value;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto read = [] {  // what was read from LDS has arrived, the buffer may be written
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        __builtin_amdgcn_sched_barrier(0);
    };
    // lane l looks after key l of a tile: its page first, then its place (-1 behind the segment's last key)
    auto position = [&](const Segment& s, int t) {
        const int i = max(min(t * 32 + col, s.n - 1), 0);
        return i < s.sinks ? i : i + s.gap;
    };
    auto entry_of = [&](const Segment& s, int t) {
        return s.n > 0 ? a.table[(long long)s.seq * a.table_width + quotient(position(s, t), a.page_mul, a.page_sh)] : 0;
    };
    auto place_of = [&](const Segment& s, int t, int entry) {
        const int p = position(s, t), page = min((unsigned)entry, (unsigned)a.n_pages - 1u);
        const int in = p - quotient(p, a.page_mul, a.page_sh) * a.page_size;
        const long long place = page * a.page_stride + in * a.token_stride + kv_head_of(a, s.item) * a.head_stride;
        return t < s.end && t * 32 + col < s.n ? place : -1;
    };
    // Addresses go through LDS from the lanes that worked them out to those that load: eight bytes a row.
    typedef __attribute__((address_space(3))) unsigned long long lds_u64_t;
    const unsigned rows_at = (unsigned)(Shape::ROWS_AT + wave * 256);
    const bool padded = row_bytes < Tile::ROW;
    auto request = [&](const unsigned char* cache, unsigned char* to, long long place) {
        *(lds_u64_t*)(unsigned long)(rows_at + col * 8) = (unsigned long long)(place >= 0 ? cache + place : (const unsigned char*)paged_zeros);
        unsigned from = rows_at + lrow * 8, first = slot << 4;
        asm volatile("" : "+v"(from), "+v"(first));  // what follows from them is worked out in every tile rather than kept in registers
        unsigned long long row[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) row[i] = *(const lds_u64_t*)(unsigned long)(from + i * RPI * 8);
        if (padded) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int chunk = first ^ (Tile::swizzle(i * RPI) << 4);
                row[i] = chunk < row_bytes ? row[i] + chunk : (unsigned long long)paged_zeros;
            }
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) row[i] += first ^ (Tile::swizzle(i * RPI) << 4);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)row[i], (lds_ptr_t)(to + i * 1024), 16, 0, 0);
    };
    constexpr int ROWS = SETS > 0 ? SETS : 1, Q = SETS > 0 ? HD * ES / 32 + (HD == 96) * 4 : STEPS;
    u32x4_t q[ROWS][Q];
    auto load_row = [&](u32x4_t* to, const unsigned char* from) {
#pragma unroll
        for (int c = 0; c < Q; ++c) to[c] = *(const u32x4_t*)(padded && (2 * c + h) * 16 >= row_bytes ? (const unsigned char*)paged_zeros : from + (2 * c + h) * 16);
    };
    auto load_q = [&](const Segment& s) {
        const int kv_head = kv_head_of(a, s.item), block = quotient(s.item, a.heads_mul, a.heads_sh);
        if constexpr (SETS > 0) {
#pragma unroll
            for (int n = 0; n < SETS; ++n) {
                const unsigned char* qp = a.q + (long long)s.seq * a.ldq + (kv_head * a.group + min(n * 4 + (lane & 3), a.group - 1)) * a.hq;
                load_row(q[n], qp);
            }
            return;
        }
        const unsigned char* qp = a.q + (long long)s.seq * a.ldq + (kv_head * a.group + min(block * 32 + col, a.group - 1)) * a.hq;
        load_row(q[0], qp);
    };

    Segment now = {}, next = {};
    if (!next_segment(now)) return;
    int t = now.first + wave;
    const int first_entry = entry_of(now, t);
    int entry = entry_of(now, t + NW), next_entry = 0;
    load_q(now);
    long long place = place_of(now, t, first_entry);
    __builtin_amdgcn_sched_barrier(0);
    request(a.k, buffers, place);
    request(a.v, buffers + Shape::HALF, place);
    for (;;) {
        const bool more = next_segment(next);
        const int next_t = next.first + wave;
        int next_place_entry = 0;
        if (more) {
            next_place_entry = entry_of(next, next_t);
            next_entry = entry_of(next, next_t + NW);
        }
#pragma unroll
        for (int n = 0; n < ROWS; ++n)
#pragma unroll
            for (int c = 0; c < Q; ++c) q[n][c] ^= a.q_flip;
        std::conditional_t<(SETS > 0), RunningNarrow<HD, ROWS>, Running<DT, HD>> run;
        run.start();
        // a tile for each wavefront at least, if only one without keys
        do {
            landed(std::integral_constant<int, LOADS>());  // k, before v
            auto k_done = [&] {
                read();
                if (t + NW < now.end) {
                    place = place_of(now, t + NW, entry);
                    entry = entry_of(now, t + 2 * NW);
                } else {
                    place = more ? place_of(next, next_t, next_place_entry) : -1;
                }
                __builtin_amdgcn_sched_barrier(0);
                request(a.k, buffers, place);
            };
            auto v_ready = [&] { landed(std::integral_constant<int, LOADS>()); };  // v, before the next k
            const int unseen = min(now.n, now.end * 32);
            if constexpr (SETS > 0) run.tile(q, a.scale_log2, buffers_at, buffers_at + Shape::HALF, t * 32, unseen, k_done, v_ready);
            else run.template tile<1, true, true>(q[0], a.scale_log2, buffers_at, buffers_at + Shape::HALF, t * 32, unseen, k_done, v_ready);
            read();
            request(a.v, buffers + Shape::HALF, place);
            t += NW;
        } while (t < now.end);
        if (more) load_q(next);

        // ---- the wavefronts' sums meet ----
        const int kv_head = kv_head_of(a, now.item), block = quotient(now.item, a.heads_mul, a.heads_sh);
        const int rows = min(32, a.group - block * 32), first_head = kv_head * a.group + block * 32, vecs = a.head_dim >> 2;
        const bool whole = now.begins() && now.ends();
        const long long part = ((long long)blockIdx.x * 2 + now.begins()) * a.rows;
        float sum = 0.f;
        if constexpr (SETS == 0) sum = run.total();
        // [wavefront][row][channel], then [wavefront][row] maxima and sums: by numbers, since before LDS accesses through
        // pointers the compiler waits for every load that writes LDS, the next tile's too
        typedef __attribute__((address_space(3))) float lds_f32_t;
        typedef __attribute__((address_space(3))) u32x4_t lds_vec_t;
        auto sums = [](int r) { return (unsigned)(Shape::MEET + r * Shape::SROW * 4); };
        auto tops = [](int r) { return (lds_f32_t*)(unsigned long)(unsigned)(Shape::MEET + NW * kMeetRows * Shape::SROW * 4 + r * 4); };
        auto sum_of = [&](int r) { return tops(NW * kMeetRows + r); };
        auto put = [&](int r, int c, float x, float y, float z, float w) {
            *(lds_vec_t*)(unsigned long)(sums(r) + c * 4) = u32x4_t{__float_as_uint(x), __float_as_uint(y), __float_as_uint(z), __float_as_uint(w)};
        };
        auto meet = [] {  // (without waiting for what is on its way from memory)
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F);
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int r0 = 0; r0 < rows; r0 += kMeetRows) {
            meet();
            if constexpr (SETS > 0) {
#pragma unroll
                for (int n = 0; n < SETS; ++n) {
                    if (n * 4 != r0) continue;
                    const float all = run.total(n);
                    if (lane < 4) {
                        *tops(wave * kMeetRows + lane) = run.top[n];
                        *sum_of(wave * kMeetRows + lane) = all;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 z = run.result(n, i);
                        if (lane < RunningNarrow<HD, ROWS>::CHUNKS && lane * 4 < HD) put(wave * kMeetRows + i, lane * 4, z.x, z.y, z.z, z.w);
                    }
                }
            } else if (col >= r0 && col < r0 + kMeetRows) {
                const int r = wave * kMeetRows + col - r0;
#pragma unroll
                for (int d = 0; d < HD / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        put(r, d * 32 + (i >> 2) * 8 + h * 4, run.o[d][i], run.o[d][i + 1], run.o[d][i + 2], run.o[d][i + 3]);
                *tops(r) = run.top;
                *sum_of(r) = sum;
            }
            meet();
            for (int e = threadIdx.x; e < min(kMeetRows, rows - r0) * 32; e += NW * 64) {
                const int r = e >> 5, c = (e & 31) * 4;
                if (c >= a.head_dim) continue;
                float top = *tops(r), total = 0.f, z[4] = {};
#pragma unroll
                for (int v = 1; v < NW; ++v) top = fmaxf(top, *tops(v * kMeetRows + r));
#pragma unroll
                for (int v = 0; v < NW; ++v) {
                    const float m = *tops(v * kMeetRows + r), w = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);  // (both may be -inf: sums of 0)
                    total = __builtin_fmaf(*sum_of(v * kMeetRows + r), w, total);
                    const u32x4_t o = *(const lds_vec_t*)(unsigned long)(sums(v * kMeetRows + r) + c * 4);
#pragma unroll
                    for (int x = 0; x < 4; ++x) z[x] = __builtin_fmaf(__uint_as_float(o[x]), w, z[x]);
                }
                if (whole) {
                    const float inv = normaliser(total, now.n > 0);
#pragma unroll
                    for (int x = 0; x < 4; ++x) z[x] *= inv;
                    store4<DT>(a.o + (long long)now.seq * a.ldo + (first_head + r0 + r) * a.ho, c, z);
                } else {
                    *(float4*)(a.part_o + (part + r0 + r) * a.head_dim + c) = make_float4(z[0], z[1], z[2], z[3]);
                    if (c == 0) a.part_stat[part + r0 + r] = make_float2(top, total);
                }
            }
        }
        if (now.begins() && !now.ends() && threadIdx.x == 0) {
            const int units = (now.tiles + (1 << a.unit_log2) - 1) >> a.unit_log2;  // the run's end is behind unit end of them
            a.records[blockIdx.x] = {now.seq, now.item, min(runs.owner(run_end + units - (now.end >> a.unit_log2) - 1), (int)gridDim.x - 1), 0};
        }
        if (!more) break;
        now = next;
        t = next_t;
        entry = next_entry;
    }
    __builtin_amdgcn_s_waitcnt(0);  // the last requests bring zeros
#endif
}

// Joins what begins in the run of workgroup blockIdx.x and ends in another's: 32 lanes of four channels take every eighth
// partial sum, each with its maximum, and meet in a fixed order.  The first of each are asked for before it is known whether
// there is something to join.
template <int DT> __global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a)
{
#if __HIP_DEVICE_COMPILE__
    __shared__ float4 parts[8][32];
    __shared__ float tops[8], totals[8];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c = min(lane * 4, a.head_dim - 4);
    auto part = [&](int p, int r) { return (min((int)blockIdx.x + p, (int)gridDim.x - 1) * 2ll + (p == 0)) * a.rows + r; };
    const JoinRecord record = a.records[blockIdx.x];
    const float2 first_stat = a.part_stat[part(group, blockIdx.y)];
    const float4 first = *(const float4*)(a.part_o + part(group, blockIdx.y) * a.head_dim + c);
    if (record.last < 0) return;
    const int n = record.last - (int)blockIdx.x + 1;
    const int kv_head = kv_head_of(a, record.item), block = quotient(record.item, a.heads_mul, a.heads_sh), rows = min(32, a.group - block * 32);
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        float top = -INFINITY, total = 0.f, z[4] = {};
        auto add = [&](float2 stat, float4 o) {
            const float now = fmaxf(top, stat.x), keep = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), w = stat.x == now ? 1.f : __builtin_amdgcn_exp2f(stat.x - now);
            top = now;
            total = __builtin_fmaf(total, keep, stat.y * w);
            z[0] = __builtin_fmaf(z[0], keep, o.x * w);
            z[1] = __builtin_fmaf(z[1], keep, o.y * w);
            z[2] = __builtin_fmaf(z[2], keep, o.z * w);
            z[3] = __builtin_fmaf(z[3], keep, o.w * w);
        };
        constexpr int AHEAD = 4;
        int p0 = group;
        if (r == (int)blockIdx.y) {
            if (group < n) add(first_stat, first);
            p0 += 8;
        }
        for (; p0 < n; p0 += 8 * AHEAD) {
            float2 stat[AHEAD];
            float4 o[AHEAD];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const long long at = part(min(p0 + e * 8, n - 1), r);
                stat[e] = a.part_stat[at];
                o[e] = *(const float4*)(a.part_o + at * a.head_dim + c);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e)
                if (p0 + e * 8 < n) add(stat[e], o[e]);
        }
        parts[group][lane] = make_float4(z[0], z[1], z[2], z[3]);
        if (lane == 0) {
            tops[group] = top;
            totals[group] = total;
        }
        __syncthreads();
        if (group == 0 && lane * 4 < a.head_dim) {
#pragma unroll
            for (int g = 1; g < 8; ++g)
                if (g < n) add(make_float2(tops[g], totals[g]), parts[g][lane]);
            const float inv = normaliser(total, true);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] *= inv;
            store4<DT>(a.o + (long long)record.seq * a.ldo + (kv_head * a.group + block * 32 + r) * a.ho, c, z);
        }
        __syncthreads();
    }
#endif
}

// ---- new keys and values -----------------------------------------------------------------------
struct AppendArgs {
    const unsigned char *k, *v;
    const int *offsets, *table, *lens;
    unsigned char *k_cache, *v_cache;
    int n_seqs, total, kv_heads, n_pages, page_size, table_width;
    unsigned page_mul;
    int page_sh;
    int chunks, row_chunks;          // of 16 bytes: of a head, of a token
    unsigned chunk_mul;
    int chunk_sh;                    // chunk / chunks
    int lanes;                       // of a wavefront for a token: 64, or the power of two that holds row_chunks
    long long ldk, ldv, hk, hv, page_stride, token_stride, head_stride;  // bytes
};

// A wavefront copies a token at a time, or several where a token is less than 64 chunks.  Bound by the memory: 48 MB of four
// prompts read and 48 written in 19 us (5 TB/s).  Data asked for before its place is known took 20, several tokens in turn 21.
__global__ __launch_bounds__(256) void paged_append_kernel(const AppendArgs a)
{
#if __HIP_DEVICE_COMPILE__
    const int lane = threadIdx.x & 63, per = 64 / a.lanes, capacity = a.table_width * a.page_size;
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), waves = gridDim.x * 4;
    for (int first = wave * per; first < a.total; first += waves * per) {
        const int token = first + lane / a.lanes;
        int seq = token, count = 1, at = 0;
        bool there = token < a.total;
        if (a.offsets) {
            seq = last_not_above(a.offsets, a.n_seqs, first, [](int offset, int) { return offset; });
            while (there && seq + 1 < a.n_seqs && a.offsets[seq + 1] <= token) ++seq;
            const int begin = a.offsets[seq], end = a.offsets[seq + 1];
            there = there && begin >= 0 && token >= begin && token < end;
            count = end - begin;
            at = token - begin;
        }
        if (!there) continue;
        const int len = min(max(a.lens[seq], 0), capacity);
        const long long position = (long long)len - count + at;
        if (position < 0) continue;
        const int nth = quotient((int)position, a.page_mul, a.page_sh), page = a.table[(long long)seq * a.table_width + nth];
        if (page < 0 || page >= a.n_pages) continue;
        const long long place = page * a.page_stride + ((int)position - nth * a.page_size) * a.token_stride;
        for (int c = lane & (a.lanes - 1); c < a.row_chunks; c += a.lanes) {
            const int head = quotient(c, a.chunk_mul, a.chunk_sh), in = (c - head * a.chunks) * 16;
            const u32x4_t k = *(const u32x4_t*)(a.k + token * a.ldk + head * a.hk + in), v = *(const u32x4_t*)(a.v + token * a.ldv + head * a.hv + in);
            *(u32x4_t*)(a.k_cache + place + head * a.head_stride + in) = k;
            *(u32x4_t*)(a.v_cache + place + head * a.head_stride + in) = v;
        }
    }
#endif
}

// ---- plans -------------------------------------------------------------------------------------
struct PagedPlan {
    int workgroups, row_blocks, rows, unit_log2;
    bool join;
};

static PagedPlan plan_paged(const sgprs_paged_attention_desc_t& d, int cus)
{
    PagedPlan p;
    const int group = d.heads / d.kv_heads;
    p.row_blocks = (group + 31) / 32;
    p.rows = std::min(32, group);
    long long most = (long long)d.table_width * d.page_size;  // positions that a token can see
    if (d.window > 0) most = std::min(most, (long long)d.window + d.sinks);
    const long long tiles = std::max(1ll, (most + 31) / 32), items = (long long)d.n_seqs * d.kv_heads * p.row_blocks;
    const bool wide = d.dtype == SGPRS_F32 && d.head_dim > 64;  // (LDS for one workgroup of a CU)
    const long long slots = std::min(kMaxWorkgroups, (wide ? 1 : 2) * cus);
    // A tile for each wavefront; more where the cost of all items could pass 2^31.  Items of at most 512 keys that have a
    // workgroup each, and are half of the CUs or more, stay whole, which saves the join: 32/8 heads x 128 in bf16, 128 items of
    // 300 keys 14.1 -> 10.2 us, 256 of 300 16.7 -> 11.8, of 1 to 512 16.7 -> 12.7, one of 512 and 255 of 60 12.5 -> 10.8; in
    // fp32 256 of 300 20.2 -> 18.7.  Fewer or longer ones lose by it: 64 items, one of 512 10.0 -> 11.0, 128 of 2048 34 -> 40.
    p.unit_log2 = tiles <= 16 && items * 2 >= cus && items <= slots ? 4 : 2;
    while (items * (((tiles - 1) >> p.unit_log2) + 1 + kItemCost) >= (1ll << 31)) ++p.unit_log2;
    const long long units = ((tiles - 1) >> p.unit_log2) + 1;
    p.workgroups = (int)std::min(slots, units > 1 ? items * (units + kItemCost) : items);
    p.join = units > 1;
    return p;
}

static size_t part_rows(const PagedPlan& p) { return (size_t)p.workgroups * 2 * p.rows; }

size_t paged_attention_workspace_bytes(const sgprs_paged_attention_desc_t& d, int cus)
{
    const PagedPlan p = plan_paged(d, cus);
    return p.workgroups * sizeof(JoinRecord) + part_rows(p) * (d.head_dim * sizeof(float) + sizeof(float2));
}

template <auto kernel> static int launch_sized(dim3 grid, int lds, const PagedArgs& a, hipStream_t stream)
{
    static std::atomic<bool> raised{false};  // more than the default 64 KiB of dynamic LDS needs an opt-in per kernel
    if (lds > 65536 && !raised) {
        SGPRS_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        raised = true;
    }
    SGPRS_LAUNCH(kernel, grid, 256, lds, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

template <int DT> static int launch_typed(const PagedArgs& a, const PagedPlan& p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.workgroups);
    auto sized = [&](auto sets) {
        constexpr int SETS = decltype(sets)::value;
        if (a.head_dim <= 32) return launch_sized<paged_attention_kernel<DT, 32, SETS>>(grid, PagedShape<DT, 32>::LDS, a, stream);
        if (a.head_dim <= 64) return launch_sized<paged_attention_kernel<DT, 64, SETS>>(grid, PagedShape<DT, 64>::LDS, a, stream);
        if (a.head_dim <= 96) return launch_sized<paged_attention_kernel<DT, 96, SETS>>(grid, PagedShape<DT, 96>::LDS, a, stream);
        return launch_sized<paged_attention_kernel<DT, 128, SETS>>(grid, PagedShape<DT, 128>::LDS, a, stream);
    };
    int rc;
    if constexpr (DT == SGPRS_F32)
        rc = a.group <= 4 ? sized(std::integral_constant<int, 1>()) : a.group <= 8 ? sized(std::integral_constant<int, 2>()) : sized(std::integral_constant<int, 0>());
    else
        rc = sized(std::integral_constant<int, 0>());
    if (rc || !p.join) return rc;
    return launch_sized<paged_join_kernel<DT>>(dim3((unsigned)p.workgroups, (unsigned)std::min(p.rows, 8)), 0, a, stream);
}

int launch_paged_attention(const sgprs_paged_attention_desc_t& d, const void* q, const void* k_cache, const void* v_cache, const int* table,
                           const int* kv_lens, void* o, void* ws, hipStream_t stream, int cus)
{
    const long long es = (long long)dtype_size(d.dtype);
    const PagedPlan p = plan_paged(d, cus);
    PagedArgs a = {};
    a.q = (const unsigned char*)q;
    a.k = (const unsigned char*)k_cache;
    a.v = (const unsigned char*)v_cache;
    a.o = (unsigned char*)o;
    a.table = table;
    a.lens = kv_lens;
    a.n_seqs = d.n_seqs;
    a.heads = d.heads;
    a.kv_heads = d.kv_heads;
    a.group = d.heads / d.kv_heads;
    a.head_dim = d.head_dim;
    a.n_pages = d.n_pages;
    a.page_size = d.page_size;
    a.table_width = d.table_width;
    div_constants(d.page_size, &a.page_mul, &a.page_sh);
    a.window = d.window;
    a.sinks = d.sinks;
    a.scale_log2 = std::fabs(d.scale) * 1.4426950408889634f;
    a.q_flip = d.scale >= 0.f ? 0u : d.dtype == SGPRS_BF16 ? 0x80008000u : 0x80000000u;
    a.ldq = (int)(d.ldq * es);
    a.ldo = (int)(d.ldo * es);
    a.hq = d.hq * es;
    a.ho = d.ho * es;
    a.page_stride = d.page_stride * es;
    a.token_stride = d.token_stride * es;
    a.head_stride = d.head_stride * es;
    a.row_blocks = p.row_blocks;
    a.rows = p.rows;
    a.items = d.kv_heads * p.row_blocks;
    div_constants(d.kv_heads, &a.heads_mul, &a.heads_sh);
    div_constants(p.workgroups, &a.grid_mul, &a.grid_sh);
    a.unit_log2 = p.unit_log2;
    a.records = (JoinRecord*)ws;
    a.part_o = (float*)(a.records + p.workgroups);
    a.part_stat = (float2*)(a.part_o + part_rows(p) * d.head_dim);
    return d.dtype == SGPRS_BF16 ? launch_typed<SGPRS_BF16>(a, p, stream) : launch_typed<SGPRS_F32>(a, p, stream);
}

int launch_paged_append(const sgprs_paged_append_desc_t& d, const void* k, const void* v, const int* offsets, const int* table,
                        const int* kv_lens, void* k_cache, void* v_cache, hipStream_t stream)
{
    const long long es = (long long)dtype_size(d.dtype);
    AppendArgs a = {};
    a.k = (const unsigned char*)k;
    a.v = (const unsigned char*)v;
    a.offsets = offsets;
    a.table = table;
    a.lens = kv_lens;
    a.k_cache = (unsigned char*)k_cache;
    a.v_cache = (unsigned char*)v_cache;
    a.n_seqs = d.n_seqs;
    a.total = d.total;
    a.kv_heads = d.kv_heads;
    a.n_pages = d.n_pages;
    a.page_size = d.page_size;
    a.table_width = d.table_width;
    div_constants(d.page_size, &a.page_mul, &a.page_sh);
    a.chunks = (int)(d.head_dim * es / 16);
    a.row_chunks = a.chunks * d.kv_heads;
    div_constants(a.chunks, &a.chunk_mul, &a.chunk_sh);
    for (a.lanes = 1; a.lanes < 64 && a.lanes < a.row_chunks;) a.lanes *= 2;
    a.ldk = d.ldk * es;
    a.ldv = d.ldv * es;
    a.hk = d.hk * es;
    a.hv = d.hv * es;
    a.page_stride = d.page_stride * es;
    a.token_stride = d.token_stride * es;
    a.head_stride = d.head_stride * es;
    const int grid = std::min((d.total - 1) / (4 * (64 / a.lanes)) + 1, 1 << 20);
    SGPRS_LAUNCH(paged_append_kernel, dim3((unsigned)grid), 256, 0, stream, a);
    SGPRS_HIP(hipGetLastError());
    return SGPRS_OK;
}

}  // namespace sgprs
