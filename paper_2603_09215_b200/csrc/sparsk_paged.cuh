// A page pool's bookkeeping: which pages a step's new rows get, and the rows themselves into them.
#pragma once

#include <cuda_fp8.h>

#include "../../include/sparsk.h"
#include "sparsk_common.cuh"
#include "sparsk_warp.cuh"

namespace sparsk {

// ------------------------------------------------------------------ page map
// With had = ceil(len / P), has = ceil((len + rows) / P): three running sums over the sequences (rows,
// pages taken, pages given back) say everything; each entry written is then found on its own, by a
// binary search for its sequence.  Nothing a block reads is written by another (a new row's page is read from
// the queue and not from the table), so every block works the sums out for itself
// and the blocks share the rows and pages without waiting for one another: one launch.
// Latency is all there is to it (a step of 64 sequences writes about a kilobyte): two trips to the memory and the
// sums between them, so no 64-bit division, and a row a thread.  64 sequences of one row: 3.6 us (6.4 with 64-bit sums and
// divisions), 300 sequences with 24 prompts, 33,000 rows: 6 us (11.8 with four rows a thread).
constexpr int PM_THREADS = 1024;
constexpr uint32_t PM_MOST = 0x7fffffffu;  // sums end here: whatever the lengths say, none of them wraps

struct PageMapArgs {
    sparsk_page_map_args a;
    int shift;  // page_size = 2^shift, or -1
};
__device__ __forceinline__ uint32_t pm_add(uint32_t x, uint32_t y) { return min(x + y, PM_MOST); }

// The largest i in [0, n) with first[i] <= x (first[0] = 0, ascending).
__device__ __forceinline__ int pm_find(const int *first, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

static __global__ void __launch_bounds__(PM_THREADS) page_map_kernel(const PageMapArgs p)
{
    extern __shared__ int pm_first[];  // [3][n_seqs]: rows, pages taken, pages given back of the sequences before; [n_seqs]: lengths
    __shared__ uint32_t warp_sum[3][PM_THREADS / 32];
    __shared__ int warp_bad[PM_THREADS / 32];
    const sparsk_page_map_args &a = p.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.n_seqs, P = a.page_size;
    int *first_row = pm_first, *first_grow = pm_first + n, *first_back = pm_first + 2 * n, *lens = pm_first + 3 * n;
    const auto page_of = [&](uint32_t pos) { return p.shift >= 0 ? pos >> p.shift : pos / (uint32_t)P; };
    const auto blocks = [&](int len) { return page_of((uint32_t)len + (uint32_t)P - 1u); };

    // a thread's sequences lie side by side
    const int per = (n + PM_THREADS - 1) / PM_THREADS, used = (n + per - 1) / per, warps = (used + 31) >> 5;
    const int beg = min(tid * per, n), end = min(beg + per, n);
    const int head = a.queue[0], count = a.queue[1];
    uint32_t sum[3] = {0, 0, 0};
    int bad = 0;
    for (int i = beg; i < end; i++) {
        const int len = a.seq_len[i], rows = a.seq_rows[i];
        lens[i] = len;
        if (len < 0 || rows < -1) {
            bad |= SPARSK_PAGES_BAD;
            continue;
        }
        const long long after = (long long)len + (rows > 0 ? rows : 0), room = (long long)a.max_blocks * P;
        if (after > room || after > INT_MAX) {
            bad |= SPARSK_PAGES_TABLE;
            continue;
        }
        const uint32_t had = blocks(len);
        sum[0] = pm_add(sum[0], rows > 0 ? rows : 0);
        if (rows >= 0) sum[1] = pm_add(sum[1], blocks((int)after) - had);
        else sum[2] = pm_add(sum[2], had);
    }
    // sums of the threads before
    uint32_t upto[3] = {sum[0], sum[1], sum[2]};
    if (warp < warps) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto[0], o), y = __shfl_up_sync(0xffffffffu, upto[1], o),
                           z = __shfl_up_sync(0xffffffffu, upto[2], o);
            if (lane >= o) {
                upto[0] = pm_add(upto[0], x);
                upto[1] = pm_add(upto[1], y);
                upto[2] = pm_add(upto[2], z);
            }
        }
        bad = __reduce_or_sync(0xffffffffu, bad);
        if (lane == 31) {
#pragma unroll
            for (int q = 0; q < 3; q++) warp_sum[q][warp] = upto[q];
            warp_bad[warp] = bad;
        }
    }
    __syncthreads();
    uint32_t before[3] = {0, 0, 0}, total[3] = {0, 0, 0};
    bad = 0;
    for (int w = 0; w < warps; w++) {
#pragma unroll
        for (int q = 0; q < 3; q++) {
            if (w == warp) before[q] = total[q];
            total[q] = pm_add(total[q], warp_sum[q][w]);
        }
        bad |= warp_bad[w];
    }
    if (head < 0 || head >= a.ring_size || count < 0 || count > a.ring_size) bad |= SPARSK_PAGES_BAD;
    else {
        if (total[1] > (uint32_t)count) bad |= SPARSK_PAGES_SHORT;
        if (total[2] > (uint32_t)(a.ring_size - count)) bad |= SPARSK_PAGES_BAD;  // more pages than the ring has places
    }
    if (total[0] > (uint32_t)a.max_rows || total[0] == PM_MOST) bad |= SPARSK_PAGES_ROWS;

    const int step = gridDim.x * PM_THREADS, at = blockIdx.x * PM_THREADS + tid;
    if (bad) {
        for (int i = at; i < n; i += step) a.seq_len_out[i] = a.seq_len[i];
        for (int i = at; i <= n; i += step) a.row_start[i] = 0;
        for (int r = at; r < a.max_rows; r += step) {
            a.row_seq[r] = a.row_pos[r] = -1;
            a.slot_map[r] = -1;
        }
        if (at == 0) {
            a.queue_out[0] = head;
            a.queue_out[1] = count;
            *a.status = bad;
        }
        return;
    }
    {
        // (nothing is at its end here: the sums are what they say)
        int b0 = (int)(before[0] + upto[0] - sum[0]), b1 = (int)(before[1] + upto[1] - sum[1]), b2 = (int)(before[2] + upto[2] - sum[2]);
        for (int i = beg; i < end; i++) {
            const int len = lens[i], rows = a.seq_rows[i], more = max(rows, 0), had = (int)blocks(len);
            first_row[i] = b0;
            first_grow[i] = b1;
            first_back[i] = b2;
            if (blockIdx.x == 0) {
                a.row_start[i] = b0;
                a.seq_len_out[i] = rows < 0 ? 0 : len + more;
            }
            b0 += more;
            if (rows >= 0) b1 += (int)blocks(len + more) - had;
            else b2 += had;
        }
    }
    const int n_rows = (int)total[0], n_grow = (int)total[1], n_back = (int)total[2];
    const auto around = [&](uint32_t i) { return i >= (uint32_t)a.ring_size ? i - (uint32_t)a.ring_size : i; };  // (never twice around)
    if (at == 0) {
        a.row_start[n] = n_rows;
        a.queue_out[0] = (int)around((uint32_t)head + n_grow);
        a.queue_out[1] = count - n_grow + n_back;
        *a.status = 0;
    }
    __syncthreads();
    for (int r = at; r < a.max_rows; r += step) {
        int seq = -1, pos = -1;
        long long slot = -1;
        if (r < n_rows) {
            seq = pm_find(first_row, n, r);
            const int len = lens[seq];
            pos = len + (r - first_row[seq]);
            const int block = (int)page_of((uint32_t)pos), had = (int)blocks(len);
            const int page = block < had ? a.block_table[seq * a.table_stride + block] : a.ring[around((uint32_t)head + (first_grow[seq] + block - had))];
            slot = (long long)page * P + (pos - block * P);
        }
        a.row_seq[r] = seq;
        a.row_pos[r] = pos;
        a.slot_map[r] = slot;
    }
    for (int t = at; t < n_grow; t += step) {
        const int seq = pm_find(first_grow, n, t);
        a.block_table[seq * a.table_stride + (int)blocks(lens[seq]) + (t - first_grow[seq])] = a.ring[around((uint32_t)head + t)];
    }
    for (int t = at; t < n_back; t += step) {
        const int seq = pm_find(first_back, n, t);
        a.ring[around(around((uint32_t)head + count) + t)] = a.block_table[seq * a.table_stride + (t - first_back[seq])];
    }
}

// ------------------------------------------------------------------ rows into pages
// A thread takes eight pairs (j, j + head_dim / 2) of one head of one row: two 16-byte reads and two writes of a
// 16-bit type, and the pairs' cosines and sines once.  Every number is read and written once; what bounds it is latency, in a decode step
// one trip after another, with many rows six waves of blocks whose threads wait for a row, its slot and the table's entry in turn.
// 4,001 rows of 36 heads of 128 (bf16, 32 of them queries, into e4m3 pages): 74 MB in 20.9 us (11.3 at the rate of a large copy; torch's
// copy of as many bytes 26).  Four heads a thread, turned by the same factors: 20.7, two: 21.9; numbers asked for only when it was
// known where they go: 23.4.  Rows that do not start at 16 bytes, rising positions: 21 us for 17.7, fp32 28 (read number by number 23 and 33).
constexpr int PA_THREADS = 256;

template <int TYPE>
__device__ __forceinline__ void pa_store8(void *p, const float (&v)[8], bool vec)
{
    if constexpr (TYPE == SPARSK_E4M3) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[i * 4], v[i * 4 + 1]), __NV_SATFINITE, __NV_E4M3);
            const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[i * 4 + 2], v[i * 4 + 3]), __NV_SATFINITE, __NV_E4M3);
            w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
        }
        *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            w[i] = TYPE == SPARSK_BF16 ? pack_bf16x2(v[i * 2], v[i * 2 + 1]) : pack_h2(pa_clamp_fp16(v[i * 2]), pa_clamp_fp16(v[i * 2 + 1]));
        if (vec) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                reinterpret_cast<uint16_t *>(p)[i * 2] = (uint16_t)w[i];
                reinterpret_cast<uint16_t *>(p)[i * 2 + 1] = (uint16_t)(w[i] >> 16);
            }
        }
    }
}
// Eight numbers as they lie in memory, and as floats.
template <int TYPE>
struct PaRaw {
    static constexpr int N = TYPE == SPARSK_FP32 ? 8 : 4;
    uint32_t w[N];
    __device__ __forceinline__ void load(const void *base, long long at, bool vec)
    {
        if (vec) {
            const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(base) + at * (TYPE == SPARSK_FP32 ? 4 : 2));
#pragma unroll
            for (int i = 0; i < N / 4; i++) {
                const uint4 x = p[i];
                w[i * 4] = x.x; w[i * 4 + 1] = x.y; w[i * 4 + 2] = x.z; w[i * 4 + 3] = x.w;
            }
        } else {
            // The 16-byte blocks that they lie in (each holds a byte of them, so none is read that the row has no part in), put
            // together by shifts.
            const char *p = reinterpret_cast<const char *>(base) + at * (TYPE == SPARSK_FP32 ? 4 : 2);
            const unsigned m = (unsigned)((uintptr_t)p & 15);
            const uint4 *b = reinterpret_cast<const uint4 *>(p - m);
            uint32_t x[N + 4];
#pragma unroll
            for (int i = 0; i <= N / 4; i++) {
                const uint4 y = i < N / 4 || m ? b[i] : make_uint4(0u, 0u, 0u, 0u);
                x[i * 4] = y.x; x[i * 4 + 1] = y.y; x[i * 4 + 2] = y.z; x[i * 4 + 3] = y.w;
            }
#pragma unroll
            for (int i = 0; i < N + 2; i++) x[i] = m & 8 ? x[i + 2] : x[i];
#pragma unroll
            for (int i = 0; i < N + 1; i++) x[i] = m & 4 ? x[i + 1] : x[i];
#pragma unroll
            for (int i = 0; i < N; i++) w[i] = TYPE == SPARSK_FP32 ? x[i] : __funnelshift_r(x[i], x[i + 1], (m & 2) * 8);
        }
    }
    __device__ __forceinline__ void floats(float (&v)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if constexpr (TYPE == SPARSK_FP32) v[i] = __uint_as_float(w[i]);
            else if constexpr (TYPE == SPARSK_BF16) v[i] = i & 1 ? bf_hi(w[i / 2]) : bf_lo(w[i / 2]);
            else v[i] = __half2float(__ushort_as_half((unsigned short)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu)));
        }
    }
};

// vec bits: 1 keys, 2 values, 4 queries, 8 turned queries may be read and written 16 bytes at a time, 16 the table.
template <int XT, int CT>
static __global__ void __launch_bounds__(PA_THREADS) paged_append_kernel(const sparsk_paged_append_args a, int row0, unsigned n_items, int vec)
{
    const unsigned idx = blockIdx.x * PA_THREADS + threadIdx.x;
    if (idx >= n_items) return;
    const int half = a.pool.head_dim >> 1, oct = half >> 3, Hk = a.pool.n_kv_heads, Hq = a.q ? a.n_q_heads : 0;
    const unsigned per_row = (unsigned)(Hq + 2 * Hk) * oct;
    const int row = row0 + (int)(idx / per_row), c = (int)(idx % per_row);
    int head = c / oct;
    const int j = (c % oct) * 8;
    const int what = head < Hq ? 0 : head < Hq + Hk ? 1 : 2;  // query, key, value
    head -= what == 0 ? 0 : what == 1 ? Hq : Hq + Hk;
    // the numbers are asked for before it is known where they go: what would wait is the memory
    const void *src = what == 0 ? a.q : what == 1 ? a.k : a.v;
    const long long at = row * (what == 0 ? a.q_row_stride : what == 1 ? a.k_row_stride : a.v_row_stride) +
                         head * (what == 0 ? a.q_head_stride : what == 1 ? a.k_head_stride : a.v_head_stride) + j;
    const bool wide = vec & (what == 0 ? 4 : what == 1 ? 1 : 2);
    PaRaw<XT> raw[2];
    raw[0].load(src, at, wide);
    raw[1].load(src, at + half, wide);
    const long long slot = what == 0 ? 0 : a.slot_map[row];
    const int pos = a.rope ? a.row_pos[row] : 0;
    if (slot < 0 || slot >= (long long)a.pool.n_pages * a.pool.page_size || (a.rope && (pos < 0 || pos >= a.rope_len))) return;
    float x[8], y[8];
    raw[0].floats(x);
    raw[1].floats(y);
    if (a.rope && what != 2) {
        const float *cs = a.rope + ((long long)pos * half + j) * 2;
        float t[16];
        if (vec & 16) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float4 f = reinterpret_cast<const float4 *>(cs)[i];
                t[i * 4] = f.x; t[i * 4 + 1] = f.y; t[i * 4 + 2] = f.z; t[i * 4 + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++) t[i] = cs[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float u = x[i] * t[2 * i] - y[i] * t[2 * i + 1];
            y[i] = y[i] * t[2 * i] + x[i] * t[2 * i + 1];
            x[i] = u;
        }
    }
    if (what == 0) {
        uint16_t *q = reinterpret_cast<uint16_t *>(a.q_out) + row * a.q_out_row_stride + head * a.q_out_head_stride + j;
        if (a.q_out_type == SPARSK_BF16) {
            pa_store8<SPARSK_BF16>(q, x, vec & 8);
            pa_store8<SPARSK_BF16>(q + half, y, vec & 8);
        } else {
            pa_store8<SPARSK_FP16>(q, x, vec & 8);
            pa_store8<SPARSK_FP16>(q + half, y, vec & 8);
        }
        return;
    }
    const float *scale = what == 1 ? a.pool.k_scale : a.pool.v_scale;
    if (scale) {
        const float s = scale[head];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            x[i] = __fdiv_rn(x[i], s);
            y[i] = __fdiv_rn(y[i], s);
        }
    }
    const long long page = (slot >> 32) ? slot / a.pool.page_size : (long long)((unsigned)slot / (unsigned)a.pool.page_size);
    const int off = (int)(slot - page * a.pool.page_size);
    constexpr int ES = CT == SPARSK_E4M3 ? 1 : 2;
    char *dst = reinterpret_cast<char *>(what == 1 ? a.pool.k : a.pool.v) +
                (page * a.pool.page_stride + head * a.pool.head_stride + off * a.pool.pos_stride + j) * ES;
    pa_store8<CT>(dst, x, true);
    pa_store8<CT>(dst + half * ES, y, true);
}

}  // namespace sparsk
