// A cache of pages: new keys and values to their places, and attention of one new token of each sequence over them.
//
// Attention is bound by reading the cache.  The queries of all heads that share a key head are one block of 32 columns (or
// several), so a key is read once for them.  An item is a sequence, a key head and a block; its visible positions, one
// behind the other (first tokens, then the window), form units of 128.  Every workgroup finds the sum of all sequences'
// units and takes an equal run of them, which may begin and end inside items: however different the lengths are, all
// workgroups have the same to do.  An item that several of them share is joined by a second launch from partial sums, two
// at most of a workgroup, in a fixed order.  Wavefront v of four takes every fourth tile of 32 keys of a run, k and v through
// LDS buffers of its own, each row from wherever its page is: the table's entries come two tiles ahead of the loads.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "attention_tiles.h"
#include "decode_ops.h"

namespace sgprs {

struct JoinRecord {
    int seq, item, last, unused;  // what begins in a workgroup and ends in workgroup `last` (-1: nothing)
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
    float* part_o;                   // [workgroup][continued, begun][row][head_dim], weights relative to part_stat
    float2* part_stat;               // [workgroup][continued, begun][row]: maximum, sum
    JoinRecord* records;             // [workgroup]
};

constexpr int kUnit = 128;           // positions: a tile of 32 for each wavefront
constexpr int kMaxWorkgroups = 2 * SGPRS_MAX_MASK_WORDS * 32;

__device__ __align__(16) unsigned paged_zeros[4] = {0, 0, 0, 0};  // what is loaded for positions behind the last

__device__ __forceinline__ int quotient(int n, unsigned mul, int sh) { return (int)(__umulhi(2u * (unsigned)n, mul) >> sh); }

__device__ __forceinline__ long long uniform(long long v)
{
#if __HIP_DEVICE_COMPILE__
    return (long long)(unsigned)__builtin_amdgcn_readfirstlane((int)v) | (long long)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
#else
    return v;
#endif
}

// The positions that a sequence's new token sees: n of them, the i-th at i or, from `sinks` on, at i + gap.
struct Seen {
    int n, sinks, gap;
    __device__ __forceinline__ int units() const { return max(1, (n + kUnit - 1) / kUnit); }  // (one to write zeros)
};
__device__ __forceinline__ Seen seen_of(const PagedArgs& a, int seq)
{
    const int len = min(max(a.lens[seq], 0), a.table_width * a.page_size);
    const int first = a.window > 0 && len > a.window ? len - a.window : 0;
    const int sinks = min(a.sinks, first);
    return {sinks + len - first, sinks, first - sinks};
}

// Runs of an equal number of units (up to one): the first of workgroup w, and whose unit u is.
struct Runs {
    long long per, rest;
    __device__ __forceinline__ Runs(long long units, int workgroups) : per(units / workgroups), rest(units % workgroups) {}
    __device__ __forceinline__ long long first(int w) const { return w * per + min((long long)w, rest); }
    __device__ __forceinline__ int owner(long long u) const { return (int)(u < rest * (per + 1) ? u / (per + 1) : rest + (u - rest * (per + 1)) / per); }
};

template <int DT, int HD> struct PagedShape {
    static constexpr int HALF = 32 * KvTile<DT, HD>::ROW, STAGE = 2 * HALF;  // k, and v behind it
    static constexpr int NW = 4;
    static constexpr int SROW = HD + 4;                                       // floats of a row where the sums meet
    static constexpr int JOIN = NW * (32 * SROW + 64) * 4, LDS = NW * STAGE > JOIN ? NW * STAGE : JOIN;
    static constexpr int PER_CU = LDS > 81856 ? 1 : 2;
};

template <int DT, int HD> __global__ __launch_bounds__(256, (PagedShape<DT, HD>::PER_CU)) void paged_attention_kernel(const PagedArgs a)
{
#if __HIP_DEVICE_COMPILE__
    typedef KvTile<DT, HD> Tile;
    typedef PagedShape<DT, HD> Shape;
    constexpr int ES = Tile::ES, STEPS = HD * ES / 32, NW = Shape::NW, LOADS = Shape::HALF / 1024, RPI = 1024 / Tile::ROW;
    extern __shared__ __align__(16) unsigned char smem[];  // (all of the LDS, from address 0 on)
    long long* totals = (long long*)(smem + Shape::LDS);
    long long& found_start = totals[4];
    int& found_seq = *(int*)(totals + 5);
    const int lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads_and_blocks = a.kv_heads * a.row_blocks;

    // ---- this workgroup's run of units, and the sequence it begins in ----
    const int share = (a.n_seqs + 255) >> 8, s0 = min((int)threadIdx.x * share, a.n_seqs), s1 = min(s0 + share, a.n_seqs);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) mine += seen_of(a, s).units();
    long long upto = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        const long long left = __shfl_up(upto, x);
        if (lane >= x) upto += left;
    }
    if (lane == 63) totals[wave] = upto;
    if (threadIdx.x == 0) found_seq = a.n_seqs;
    __syncthreads();
    long long units = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
        if (v == wave) upto += units;
        units += totals[v];
    }
    const Runs runs(units * heads_and_blocks, gridDim.x);
    const long long run_begin = uniform(runs.first(blockIdx.x)), run_end = uniform(runs.first(blockIdx.x + 1));
    if (threadIdx.x == 0) a.records[blockIdx.x] = {0, 0, -1, 0};
    if (run_begin >= run_end) return;
    if ((upto - mine) * heads_and_blocks <= run_begin && run_begin < upto * heads_and_blocks) {
        long long start = upto - mine;
        int s = s0;
        for (; s + 1 < s1; ++s) {
            const int n = seen_of(a, s).units();
            if (run_begin < (start + n) * heads_and_blocks) break;
            start += n;
        }
        found_seq = s;
        found_start = start * heads_and_blocks;
    }
    __syncthreads();

    const int row_bytes = a.head_dim * ES;
    const int lrow = lane / Tile::CHUNKS, slot = (lane % Tile::CHUNKS) ^ Tile::swizzle(lrow);
    unsigned char* buffers = smem + wave * Shape::STAGE;
    const unsigned at = (unsigned)(wave * Shape::STAGE);
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

    int seq = __builtin_amdgcn_readfirstlane(found_seq);
    long long seq_start = uniform(found_start), unit = run_begin;
    while (unit < run_end && seq < a.n_seqs) {
        const Seen seen = seen_of(a, seq);
        const int n_units = seen.units();
        if (unit - seq_start >= (long long)n_units * heads_and_blocks) {
            seq_start += (long long)n_units * heads_and_blocks;
            ++seq;
            continue;
        }
        const int item = (int)((unit - seq_start) / n_units), unit0 = (int)(unit - seq_start - (long long)item * n_units);
        const int take = (int)min(run_end - unit, (long long)(n_units - unit0));
        const int kv_head = item % a.kv_heads, block = item / a.kv_heads;
        const int rows = min(32, a.group - block * 32);
        const int first_head = kv_head * a.group + block * 32, head = first_head + min(col, rows - 1);
        const int begin = unit0 * kUnit, end = min(seen.n, (unit0 + take) * kUnit);
        const int tiles = (end - begin + 31) >> 5;
        const int* table = a.table + (long long)seq * a.table_width;
        const unsigned char* kp = a.k + kv_head * a.head_stride;
        const unsigned char* vp = a.v + kv_head * a.head_stride;

        // lane l looks after key l of a tile: its page first, then its place
        auto position = [&](int t) {
            const int i = min(begin + t * 32 + col, end - 1);
            return i < seen.sinks ? i : i + seen.gap;
        };
        auto entry_of = [&](int t) { return table[quotient(position(t), a.page_mul, a.page_sh)]; };
        auto place_of = [&](int t, int entry) {  // -1 behind the last key
            const int p = position(t), page = min((unsigned)entry, (unsigned)a.n_pages - 1u);
            const int in = p - quotient(p, a.page_mul, a.page_sh) * a.page_size;
            return begin + t * 32 + col < end ? page * a.page_stride + in * a.token_stride : -1;
        };
        auto request = [&](const unsigned char* from, unsigned char* to, long long place) {
            int lane_row = lrow;
            asm volatile("" : "+v"(lane_row));  // what follows from it is worked out in every tile rather than kept in registers
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int chunk = (slot ^ Tile::swizzle(i * RPI)) << 4;
                const long long at = __shfl(place, i * RPI + lane_row);
                const unsigned char* p = at >= 0 && chunk < row_bytes ? from + at + chunk : (const unsigned char*)paged_zeros;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, (lds_ptr_t)(to + i * 1024), 16, 0, 0);
            }
        };

        Running<DT, HD> run;
        run.start();
        if (tiles > 0) {
            u32x4_t q[STEPS];
            const unsigned char* qp = a.q + (long long)seq * a.ldq + head * a.hq;
#pragma unroll
            for (int c = 0; c < STEPS; ++c) {
                q[c] = (2 * c + h) * 16 < row_bytes ? *(const u32x4_t*)(qp + (2 * c + h) * 16) : u32x4_t{0, 0, 0, 0};
                q[c] ^= a.q_flip;
            }
            long long place = place_of(wave, entry_of(wave));
            int entry = entry_of(wave + NW);
            request(kp, buffers, place);
            request(vp, buffers + Shape::HALF, place);
            for (int t = wave; t < tiles; t += NW) {
                landed(std::integral_constant<int, LOADS>());  // k, before v
                const int key0 = begin + t * 32;
                auto k_done = [&] {
                    read();
                    place = place_of(t + NW, entry);
                    entry = entry_of(t + 2 * NW);
                    __builtin_amdgcn_sched_barrier(0);
                    request(kp, buffers, place);
                };
                auto v_ready = [&] { landed(std::integral_constant<int, LOADS + 1>()); };  // v, before an entry and the next k
                if (key0 + 32 <= end) run.template tile<1, false>(q, a.scale_log2, at, at + Shape::HALF, key0, end, k_done, v_ready);
                else run.template tile<1, true>(q, a.scale_log2, at, at + Shape::HALF, key0, end, k_done, v_ready);
                read();
                request(vp, buffers + Shape::HALF, place);
            }
            __builtin_amdgcn_s_waitcnt(0);  // requests past the end bring zeros
        }
        __syncthreads();
        float* sums = (float*)smem;  // [wavefront][column][channel], then [wavefront][column] maxima and sums
        float* tops = sums + NW * 32 * Shape::SROW;
        float* sum_of = tops + NW * 32;
        if (col < rows) {
#pragma unroll
            for (int d = 0; d < HD / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *(float4*)(sums + (wave * 32 + col) * Shape::SROW + d * 32 + (i >> 2) * 8 + h * 4) = make_float4(run.o[d][i], run.o[d][i + 1], run.o[d][i + 2], run.o[d][i + 3]);
        }
        const float sum = run.total();
        if (h == 0) {
            tops[wave * 32 + col] = run.top;
            sum_of[wave * 32 + col] = sum;
        }
        __syncthreads();
        const int vecs = a.head_dim >> 2;
        const bool whole = take == n_units;
        const long long part = ((long long)blockIdx.x * 2 + (unit0 == 0)) * a.rows;
        for (int e = threadIdx.x; e < rows * vecs; e += NW * 64) {
            const int r = e / vecs, c = (e - r * vecs) * 4;
            float top = tops[r], total = 0.f, z[4] = {};
#pragma unroll
            for (int v = 1; v < NW; ++v) top = fmaxf(top, tops[v * 32 + r]);
#pragma unroll
            for (int v = 0; v < NW; ++v) {
                const float t = tops[v * 32 + r], w = t == top ? 1.f : __builtin_amdgcn_exp2f(t - top);  // (both may be -inf: sums of 0)
                total = __builtin_fmaf(sum_of[v * 32 + r], w, total);
#pragma unroll
                for (int x = 0; x < 4; ++x) z[x] = __builtin_fmaf(sums[(v * 32 + r) * Shape::SROW + c + x], w, z[x]);
            }
            if (whole) {
                const float inv = normaliser(total, seen.n > 0);
#pragma unroll
                for (int x = 0; x < 4; ++x) z[x] *= inv;
                store4<DT>(a.o + (long long)seq * a.ldo + (first_head + r) * a.ho, c, z);
            } else {
                *(float4*)(a.part_o + (part + r) * a.head_dim + c) = make_float4(z[0], z[1], z[2], z[3]);
                if (c == 0) a.part_stat[part + r] = make_float2(top, total);
            }
        }
        if (!whole && unit0 == 0 && threadIdx.x == 0) a.records[blockIdx.x] = {seq, item, runs.owner(unit + n_units - 1), 0};
        unit += take;
        __syncthreads();  // the buffers are free again
    }
#endif
}

// Joins what begins in workgroup blockIdx.x of the first launch and ends in another: 32 lanes of four channels, eight
// partial sums at a time.
template <int DT> __global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a)
{
#if __HIP_DEVICE_COMPILE__
    __shared__ float weights[kMaxWorkgroups];
    __shared__ float stat[8];
    __shared__ float4 parts[8][32];
    const JoinRecord record = a.records[blockIdx.x];
    if (record.last < 0) return;
    const int n = record.last - (int)blockIdx.x + 1;
    const int kv_head = record.item % a.kv_heads, block = record.item / a.kv_heads, rows = min(32, a.group - block * 32);
    const int tid = threadIdx.x, lane = tid & 31, group = tid >> 5, c = lane * 4;
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        auto part = [&](int p) { return ((long long)(blockIdx.x + p) * 2 + (p == 0)) * a.rows + r; };
        float top = -INFINITY, total = 0.f;
        for (int p = tid; p < n; p += 256) top = fmaxf(top, a.part_stat[part(p)].x);
#pragma unroll
        for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
        if ((tid & 63) == 0) stat[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(stat[0], stat[1]), fmaxf(stat[2], stat[3]));
        for (int p = tid; p < n; p += 256) {
            const float2 st = a.part_stat[part(p)];
            const float w = st.x == top ? 1.f : __builtin_amdgcn_exp2f(st.x - top);
            weights[p] = w;
            total = __builtin_fmaf(st.y, w, total);
        }
#pragma unroll
        for (int x = 32; x; x >>= 1) total += __shfl_xor(total, x);
        if ((tid & 63) == 0) stat[4 + (tid >> 6)] = total;
        __syncthreads();
        total = (stat[4] + stat[5]) + (stat[6] + stat[7]);
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < a.head_dim) {
#pragma unroll 4
            for (int p = group; p < n; p += 8) {
                const float w = weights[p];
                const float4 o = *(const float4*)(a.part_o + part(p) * a.head_dim + c);
                z = make_float4(__builtin_fmaf(o.x, w, z.x), __builtin_fmaf(o.y, w, z.y), __builtin_fmaf(o.z, w, z.z), __builtin_fmaf(o.w, w, z.w));
            }
        }
        parts[group][lane] = z;
        __syncthreads();
        if (group == 0 && c < a.head_dim) {
            float out[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
            for (int g = 1; g < 8; ++g) {
                const float4 t = parts[g][lane];
                out[0] += t.x;
                out[1] += t.y;
                out[2] += t.z;
                out[3] += t.w;
            }
            const float inv = normaliser(total, true);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] *= inv;
            store4<DT>(a.o + (long long)record.seq * a.ldo + (kv_head * a.group + block * 32 + r) * a.ho, c, out);
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

// A wavefront copies a token at a time, or several where a token is less than 64 chunks.  Bound by the memory.
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
    int workgroups, row_blocks, rows;
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
    const long long units = (most + kUnit - 1) / kUnit, items = (long long)d.n_seqs * d.kv_heads * p.row_blocks;
    const bool wide = d.dtype == SGPRS_F32 && d.head_dim > 64;
    p.workgroups = (int)std::min<long long>(std::min(kMaxWorkgroups, (wide ? 1 : 2) * cus), (double)units * items > 1e6 ? 1000000 : units * items);
    p.join = units > 1;
    return p;
}

static size_t part_floats(const sgprs_paged_attention_desc_t& d, const PagedPlan& p) { return (size_t)p.workgroups * 2 * p.rows * d.head_dim; }

size_t paged_attention_workspace_bytes(const sgprs_paged_attention_desc_t& d, int cus)
{
    const PagedPlan p = plan_paged(d, cus);
    return p.workgroups * sizeof(JoinRecord) + part_floats(d, p) * 4 + (size_t)p.workgroups * 2 * p.rows * sizeof(float2);
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
    int rc;
    if (a.head_dim <= 32) rc = launch_sized<paged_attention_kernel<DT, 32>>(grid, PagedShape<DT, 32>::LDS + 64, a, stream);
    else if (a.head_dim <= 64) rc = launch_sized<paged_attention_kernel<DT, 64>>(grid, PagedShape<DT, 64>::LDS + 64, a, stream);
    else if (a.head_dim <= 96) rc = launch_sized<paged_attention_kernel<DT, 96>>(grid, PagedShape<DT, 96>::LDS + 64, a, stream);
    else rc = launch_sized<paged_attention_kernel<DT, 128>>(grid, PagedShape<DT, 128>::LDS + 64, a, stream);
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
    a.records = (JoinRecord*)ws;
    a.part_o = (float*)(a.records + p.workgroups);
    a.part_stat = (float2*)(a.part_o + part_floats(d, p));
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
