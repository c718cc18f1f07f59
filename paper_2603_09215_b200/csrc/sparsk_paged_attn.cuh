// Attention of a step's new rows over a paged cache, split over the cache's length and joined.
//
//   out = sum_p w_p v_p / sum_p w_p,  w_p = exp(scale q.k_p - max), the maximum and both sums running (one pass).
//
// A segment is (sequence, block of 16 MT query vectors, kv head): the rows' query heads of that kv head are the M dimension of
// m16n8k16 products (as in sparsk_attn.cuh), so that one read of the head's keys and values serves all of them.
// All segments, laid end to end in boxes of 16 positions (plus a few boxes' worth for a segment's set-up and end), are cut into equal
// shares, one for each CTA of a grid that is resident at once: nobody knows the lengths but the device, and
// every CTA adds them up for itself.  A share begins and ends anywhere; a segment that lies in one share is written
// out at once, others leave a partial (sums and maxima) at either end of a share, which
// a second kernel joins in order.
//
// Within a CTA one warp brings boxes of 16 positions by TMA (a tensor map of the pool: dimensions, positions of a page, halves of
// the head, heads, pages, whichever of heads and positions lies outside; a box never leaves its page, whose size is a multiple of 16) into
// a ring of stages of 64 positions, and four warps take boxes from it: with MT = 1 a box each, with MT = 2 two boxes
// each for one of two blocks of 16 query vectors, with MT = 4 all four for one of four.  Every warp keeps the softmax of
// its own positions; the warps of one block meet at the segment's end only.  8-bit pages are widened to fp16 in
// registers, between the shared memory and the product.
// Bound by HBM: a position of a head of 128 fp16 numbers is 512 bytes, 23 of which come per clock and SM, so 16 positions
// may take 350 clocks of an SM.
#pragma once

#include <cuda_fp8.h>

#include "sparsk_attn.cuh"
#include "sparsk_paged.cuh"

namespace sparsk {

constexpr int PT_THREADS = 160, PT_WARPS = 4;  // four warps compute, the fifth brings the boxes
constexpr int PT_BOX = 16, PT_STAGE = 64;      // positions
constexpr int PT_CTAS = 2;                     // resident on an SM
constexpr int PT_MAX_SHARES = 2 * 160;         // CTAs of a launch (the scratch is sized for them)
constexpr int PT_END_BOXES = 3;                // what a segment's set-up and end cost, in boxes
constexpr int PT_WHOLE = 8;                    // a segment of up to so many boxes is never cut
constexpr int PT_MIN_SHARE = 7;                // boxes
constexpr int PT_RING_BYTES = 96 * 1024;
constexpr int PJ_THREADS = 256;

// A share's partials for the join: bit 0 its last segment goes on in the next share, bits 1..2 its first one began in an
// earlier share and 1 goes on, 2 ends here; and which segment the last one is.
struct PtRecord {
    int flags, row0, rows, qblk, head, pad[3];
};
struct PtStage {  // what the computing warps have to know of a stage
    int p0, end;  // its first position; the piece's positions end here
    int flags;    // PT_*, and in bits 8..11 which boxes it holds
    int row0, rows, len, qblk, head;
};
enum { PT_FIRST = 1, PT_LAST = 2, PT_STOP = 4, PT_HEAD_PART = 16, PT_TAIL_PART = 32 };

struct PtArgs {
    const void *q;
    void *out;
    float *lse;
    const int *block_table, *seq_len, *row_start;
    const float *k_scale, *v_scale;
    PtRecord *records;  // [shares]
    float4 *part_o;     // [shares][2][MT][HD / 8][32 lanes]: accumulators as the lanes hold them
    float2 *part_ml;    // [shares][2][16 MT]: maximum in powers of two, sum
    long long table_stride, q_row_stride, q_head_stride, out_row_stride, out_head_stride;
    float scale_log2;
    int q_type, n_rows, n_seqs, max_blocks, page_size, n_pages, Hk, G;
    int whole_boxes;    // segments of up to so many boxes are never cut
};

template <int HD, int CT>
struct PtForm {
    static constexpr int ES = CT == SPARSK_E4M3 ? 1 : 2;
    static constexpr int RB = HD * ES;                          // bytes of a position
    static constexpr int STAGE = 2 * PT_STAGE * RB;             // keys, then values
    static constexpr int NS = PT_RING_BYTES / STAGE;
    static constexpr int MEET = PT_WARPS * (HD / 16) * 32 * 16; // the warps' sums, half of the dimensions at a time
    static constexpr int SMEM = NS * STAGE + MEET + NS * (16 + (int)sizeof(PtStage)) + PT_WARPS * 16 * 8 + 80;
    // byte offset of 16-byte chunk c of row r inside a box
    __device__ __forceinline__ static int at(int r, int c)
    {
        if (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
        return (RB > 128 ? (c >> 3) * (PT_BOX * 128) : 0) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    }
};

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int y, int head, int page)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %3, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(y), "r"(head), "r"(page)
        : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int CT>
__device__ __forceinline__ void pt_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (CT == SPARSK_BF16) mma_bf16(d, a, b0, b1);
    else mma_f16(d, a, b0, b1);
}
// two e4m3 numbers -> two fp16 numbers (exact)
__device__ __forceinline__ uint32_t pt_widen(uint32_t two)
{
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(r) : "r"(two));
    return r;
}
// Two query numbers in the type that meets the pool's: a number beyond fp16 as its largest.
template <int CT>
__device__ __forceinline__ uint32_t pt_query2(const uint16_t *p, int q_type)
{
    const uint32_t w = (uint32_t)p[0] | ((uint32_t)p[1] << 16);
    if (CT == SPARSK_BF16 || q_type == SPARSK_FP16) return w;
    return pack_h2(pa_clamp_fp16(bf_lo(w)), pa_clamp_fp16(bf_hi(w)));
}
template <int CT>
__device__ __forceinline__ uint32_t pt_pack2(float a, float b)
{
    return CT == SPARSK_BF16 ? pack_bf16x2(a, b) : pack_h2(a, b);
}
// what the rounding to 16 bits left over
template <int CT>
__device__ __forceinline__ uint32_t pt_rest2(float a, float b, uint32_t hi)
{
    if (CT == SPARSK_BF16) return pack_bf16x2(a - bf_lo(hi), b - bf_hi(hi));
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    return pack_h2(a - f.x, b - f.y);
}
// One byte or half of a value that is not finite, in a word of them: cleared.
template <int CT>
__device__ __forceinline__ bool pt_not_finite16(uint32_t h)  // fp16 or bf16 bits
{
    constexpr uint32_t E = CT == SPARSK_BF16 ? 0x7f80u : 0x7c00u;
    return (h & E) == E;
}
template <int CT>
__device__ __forceinline__ uint32_t pt_finite2(uint32_t w)
{
    if (pt_not_finite16<CT>(w & 0xffffu)) w &= 0xffff0000u;
    if (pt_not_finite16<CT>(w >> 16)) w &= 0xffffu;
    return w;
}

// ------------------------------------------------------------------ the lengths, and a CTA's share of them
struct PtSeq {
    int row0, rows, len;  // first row, rows, positions
};
__device__ __forceinline__ PtSeq pt_seq(const PtArgs &a, int i)
{
    PtSeq s;
    const int r0 = a.row_start ? min(max(__ldcg(a.row_start + i), 0), a.n_rows) : i;
    const int r1 = a.row_start ? min(max(__ldcg(a.row_start + i + 1), 0), a.n_rows) : i + 1;
    s.row0 = r0;
    s.rows = max(r1 - r0, 0);
    s.len = max(__ldcg(a.seq_len + i), 0);  // as it was given; a table that ends earlier cuts it where it is used
    return s;
}
template <int MT>
__device__ __forceinline__ int pt_blocks_of(const PtArgs &a, int rows) { return (int)(((long long)rows * a.G + 16 * MT - 1) / (16 * MT)); }

template <int HD, int CT, int MT, bool P2>
static __global__ void __launch_bounds__(PT_THREADS, PT_CTAS)
paged_attn_kernel(const PtArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv)
{
    typedef PtForm<HD, CT> F;
    constexpr int NS = F::NS, RB = F::RB, KS = HD / 16, NT = HD / 8, PG = PT_WARPS / MT;
    constexpr float LN2 = 0.6931471805599453f;
    extern __shared__ __align__(1024) unsigned char pt_smem[];
    unsigned char *ring = pt_smem;
    float4 *meet = reinterpret_cast<float4 *>(pt_smem + NS * F::STAGE);
    uint64_t *full = reinterpret_cast<uint64_t *>(pt_smem + NS * F::STAGE + F::MEET), *empty = full + NS;
    PtStage *stages = reinterpret_cast<PtStage *>(empty + NS);
    float2 *meet_ml = reinterpret_cast<float2 *>(stages + NS);
    long long *plan = reinterpret_cast<long long *>(meet_ml + PT_WARPS * 16);  // [5 sums of warps], first sequence and its begin
    uint64_t *meeting = reinterpret_cast<uint64_t *>(plan + 7);
    volatile int *giving_up = reinterpret_cast<volatile int *>(plan + 8);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    griddep_launch();
    if (tid == 0) {
        for (int s = 0; s < NS; s++) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], PT_WARPS);
        }
        mbar_init(meeting, PT_WARPS);
        giving_up[0] = giving_up[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    griddep_wait();

    // this CTA's share [beg, end) of all segments' boxes
    const int cap = a.max_blocks * a.page_size;
    const auto cost_of = [&](const PtSeq &s) { return (min(s.len, cap) + PT_BOX - 1) / PT_BOX + PT_END_BOXES; };
    const int per = (a.n_seqs + PT_THREADS - 1) / PT_THREADS, s_beg = min(tid * per, a.n_seqs), s_end = min(s_beg + per, a.n_seqs);
    long long mine = 0;
    for (int i = s_beg; i < s_end; i++) {
        const PtSeq s = pt_seq(a, i);
        mine += (long long)pt_blocks_of<MT>(a, s.rows) * a.Hk * cost_of(s);
    }
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
    }
    if (lane == 31) plan[warp] = upto;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < PT_WARPS + 1; w++) {
        if (w < warp) upto += plan[w];
        total += plan[w];
    }
    const long long share = max((total + gridDim.x - 1) / gridDim.x, (long long)(PT_MIN_SHARE + PT_END_BOXES));
    const long long beg = share * blockIdx.x, end = min(beg + share, total);
    if (beg >= end) {
        if (tid == 0) a.records[blockIdx.x].flags = 0;
        return;
    }
    if (mine > 0 && upto - mine <= beg && beg < upto) {  // the sequence in which it begins is one of this thread's
        long long at = upto - mine;
        for (int i = s_beg; i < s_end; i++) {
            const PtSeq s = pt_seq(a, i);
            const long long c = (long long)pt_blocks_of<MT>(a, s.rows) * a.Hk * cost_of(s);
            if (beg < at + c) {
                plan[5] = i;
                plan[6] = at;
                break;
            }
            at += c;
        }
    }
    __syncthreads();

    if (warp == PT_WARPS) {
        // ---------------------------------------------------------------- the warp that brings the boxes
        int seq = (int)plan[5], base = -64, it = 0, issued = 0, flags = 0;
        long long at = plan[6], x = beg;
        PtSeq ahead{};  // of sequence base + lane
        PtRecord rec{};
        bool ok = true;
        const auto next_stage = [&]() {
            const int s = it % NS;
            if (it >= NS) ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], ((it / NS) - 1) & 1, giving_up, nullptr));
            it++;
            return s;
        };
        const int page_boxes = a.page_size / PT_BOX;
        while (ok && x < end) {
            if (seq - base >= 32) {
                base = seq;
                if (seq + lane < a.n_seqs) ahead = pt_seq(a, seq + lane);
            }
            PtSeq s;
            s.row0 = __shfl_sync(0xffffffffu, ahead.row0, seq - base);
            s.rows = __shfl_sync(0xffffffffu, ahead.rows, seq - base);
            s.len = __shfl_sync(0xffffffffu, ahead.len, seq - base);
            const int cost = cost_of(s), boxes = cost - PT_END_BOXES;
            const long long all = (long long)pt_blocks_of<MT>(a, s.rows) * a.Hk * cost;
            if (x >= at + all) {
                at += all;
                seq++;
                continue;
            }
            const long long seg = (x - at) / cost;
            const int from = (int)(x - at - seg * cost);
            int to = (int)min((long long)cost, from + (end - x));
            x += to - from;
            if (boxes <= a.whole_boxes) {
                if (from > 0) continue;  // the share before this one has it
                to = cost;
            }
            const int b0 = min(from, boxes), b1 = min(to, boxes);
            if (b0 >= b1 && !(boxes == 0 && from == 0)) continue;
            const int qblk = (int)(seg / a.Hk), head = (int)(seg % a.Hk);
            int part = 0;
            if (b0 > 0) {
                part = PT_HEAD_PART;
                flags |= b1 == boxes ? 4 : 2;
            } else if (b1 < boxes) {
                part = PT_TAIL_PART;
                flags |= 1;
                rec.row0 = s.row0;
                rec.rows = s.rows;
                rec.qblk = qblk;
                rec.head = head;
            }
            const int pos_end = min(min(s.len, cap), b1 * PT_BOX);
            int page = -1;
            for (int b = b0; ok && (b < b1 || b == b0); b += 4) {
                const int chunk = (b - b0) & 31;
                if (chunk == 0) {  // the pages of the next 32 boxes
                    const int mine_b = b + lane;
                    page = mine_b < b1 ? __ldcg(a.block_table + seq * a.table_stride + mine_b / page_boxes) : -1;
                    if (page >= a.n_pages) page = -1;
                }
                const int n_box = min(4, b1 - b), j = lane >> 1;
                const int my_page = __shfl_sync(0xffffffffu, page, (chunk + j) & 31);
                const bool copy = lane < 8 && j < n_box && my_page >= 0;
                const uint32_t have = __ballot_sync(0xffffffffu, copy) & 0x55u;
                const int st = next_stage();
                if (!ok) break;
                if (lane == 0) {
                    PtStage &d = stages[st];
                    d.p0 = b * PT_BOX;
                    d.end = pos_end;
                    d.flags = (b == b0 ? PT_FIRST : 0) | (b + 4 >= b1 ? PT_LAST : 0) | part |
                              ((have & 1u) << 8) | ((have & 4u) << 7) | ((have & 16u) << 6) | ((have & 64u) << 5);
                    d.row0 = s.row0;
                    d.rows = s.rows;
                    d.len = s.len;
                    d.qblk = qblk;
                    d.head = head;
                    mbar_expect_tx(&full[st], (uint32_t)__popc(have) * 2u * PT_BOX * RB);
                }
                __syncwarp();
                if (copy) {
                    const int box = b + j, y = (box % page_boxes) * PT_BOX;
                    const uint32_t dst = smem_u32(ring + st * F::STAGE + (lane & 1) * (PT_STAGE * RB) + j * (PT_BOX * RB));
                    tma_load_5d(dst, (lane & 1) ? &mv : &mk, &full[st], y, head, my_page);
                }
                issued = it;
            }
        }
        if (ok) {
            const int st = next_stage();
            if (lane == 0 && ok) {
                stages[st].flags = PT_STOP;
                mbar_arrive(&full[st]);
            }
        }
        if (lane == 0) {
            rec.flags = flags;
            a.records[blockIdx.x] = rec;
        }
        // someone has given up: no copy may land in shared memory that is another CTA's by then
        if (!ok)
            for (int k = max(0, issued - NS); k < issued; k++) mbar_wait(&full[k % NS], (k / NS) & 1, giving_up + 1, nullptr);
        return;
    }

    // -------------------------------------------------------------------- the warps that compute
    const int mt = warp % MT, pg = warp / MT, t4 = lane & 3;
    uint32_t qa[KS][4];
    float o[NT][4], m_run[2], l_run[2], c_log2 = 0.f;
    int limit[2], lim_min = 0, meetings = 0;
    // all four warps; like every wait here it ends by itself when another warp has given up
    const auto meet_here = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(meeting);
        return __all_sync(0xffffffffu, mbar_wait(meeting, meetings++ & 1, giving_up, nullptr));
    };
    for (int it = 0;; it++) {
        const int st = it % NS;
        if (!__all_sync(0xffffffffu, mbar_wait(&full[st], (it / NS) & 1, giving_up, nullptr))) return;
        const PtStage d = stages[st];
        if (d.flags & PT_STOP) break;
        const int v0 = (d.qblk * MT + mt) * 16, n_vec = d.rows * a.G;  // this warp's query vectors: v0 .. v0 + 15, as far as there are
        if (d.flags & PT_FIRST) {
            c_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[d.head] : 1.f);
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int e = 0; e < 4; e++) o[nt][e] = 0.f;
            lim_min = d.len - d.rows + v0 / a.G;
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                const int v = v0 + (lane >> 2) + hf * 8;
                const bool have = v < n_vec;
                const int r = have ? v / a.G : 0, h = have ? v % a.G : 0;
                m_run[hf] = -INFINITY;
                l_run[hf] = 0.f;
                limit[hf] = have ? d.len - d.rows + r : -1;  // the last position that this vector sees
                const uint16_t *q = reinterpret_cast<const uint16_t *>(a.q) + (d.row0 + r) * a.q_row_stride + (d.head * a.G + h) * a.q_head_stride;
#pragma unroll
                for (int ks = 0; ks < KS; ks++) {
                    // 8-bit keys come four dimensions to a lane, 16-bit keys two and two
                    const int d0 = ks * 16 + (F::ES == 1 ? t4 * 4 : t4 * 2), d1 = d0 + (F::ES == 1 ? 2 : 8);
                    qa[ks][hf] = have ? pt_query2<CT>(q + d0, a.q_type) : 0u;
                    qa[ks][2 + hf] = have ? pt_query2<CT>(q + d1, a.q_type) : 0u;
                }
            }
        }
        bool wrote = false;
#pragma unroll 1
        for (int b = pg; b < 4; b += PG) {
            const int p0 = d.p0 + b * PT_BOX;
            if (!(d.flags >> (8 + b) & 1)) continue;
            const unsigned char *K = ring + st * F::STAGE + b * (PT_BOX * RB), *V = K + PT_STAGE * RB;
            // S = Q K^T for 16 positions, two chains
            float s[2][4], s2[2][4];
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int e = 0; e < 4; e++) s[nt][e] = s2[nt][e] = 0.f;
            const int krow = (lane & 7) + ((lane >> 4) << 3), kch = (lane >> 3) & 1;
            if constexpr (F::ES == 2) {
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    uint32_t kb[4], kb2[4];
                    ldsm_x4(kb, K + F::at(krow, ks * 2 + kch));
                    ldsm_x4(kb2, K + F::at(krow, (ks + 1) * 2 + kch));
                    pt_mma<CT>(s[0], qa[ks], kb[0], kb[1]);
                    pt_mma<CT>(s[1], qa[ks], kb[2], kb[3]);
                    pt_mma<CT>(s2[0], qa[ks + 1], kb2[0], kb2[1]);
                    pt_mma<CT>(s2[1], qa[ks + 1], kb2[2], kb2[3]);
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    uint32_t kb[4];
                    ldsm_x4(kb, K + F::at(krow, ks + kch));
                    pt_mma<CT>(s[0], qa[ks], pt_widen(kb[0]), pt_widen(kb[0] >> 16));
                    pt_mma<CT>(s2[0], qa[ks + 1], pt_widen(kb[1]), pt_widen(kb[1] >> 16));
                    pt_mma<CT>(s[1], qa[ks], pt_widen(kb[2]), pt_widen(kb[2] >> 16));
                    pt_mma<CT>(s2[1], qa[ks + 1], pt_widen(kb[3]), pt_widen(kb[3] >> 16));
                }
            }
            // a box that every vector sees whole needs no mask
            const bool whole = p0 + PT_BOX <= d.end && p0 + PT_BOX - 1 <= lim_min;
            uint32_t pa[4], pr[4];
            float alpha[2];
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                float v[4], top = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < 2; nt++)
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int p = p0 + nt * 8 + t4 * 2 + e;
                        const bool see = whole || (p < d.end && p <= limit[hf]);
                        v[nt * 2 + e] = see ? (s[nt][hf * 2 + e] + s2[nt][hf * 2 + e]) * c_log2 : -INFINITY;
                        top = fmaxf(top, v[nt * 2 + e]);
                    }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const float m_new = fmaxf(m_run[hf], top);
                const float m_use = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet: every weight is 2^-inf = 0
                alpha[hf] = exp2f(m_run[hf] - m_use);
                if (m_run[hf] == m_new) alpha[hf] = 1.f;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    v[i] = exp2f(v[i] - m_use);
                    sum += v[i];
                }
                l_run[hf] = l_run[hf] * alpha[hf] + sum;  // a lane's own positions; lanes are summed at the end
                m_run[hf] = m_new;
                pa[hf] = pt_pack2<CT>(v[0], v[1]);
                pa[2 + hf] = pt_pack2<CT>(v[2], v[3]);
                if (P2) {
                    pr[hf] = pt_rest2<CT>(v[0], v[1], pa[hf]);
                    pr[2 + hf] = pt_rest2<CT>(v[2], v[3], pa[2 + hf]);
                }
            }
            if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                    o[nt][0] *= alpha[0];
                    o[nt][1] *= alpha[0];
                    o[nt][2] *= alpha[1];
                    o[nt][3] *= alpha[1];
                }
            }
            // Values that nobody sees meet a weight of zero, which must not meet an infinity or a NaN: rows behind the end are
            // cleared.  Rows that some vectors of a causal block see and others do not are looked at first.
            bool odd_values = false;
            if (!whole) {
                constexpr int CH = RB / 16;
                for (int i = lane; i < PT_BOX * CH; i += 32) {
                    const int r = i / CH;
                    uint4 *w = reinterpret_cast<uint4 *>(const_cast<unsigned char *>(V) + F::at(r, i % CH));
                    if (p0 + r >= d.end) {
                        *w = make_uint4(0u, 0u, 0u, 0u);
                        wrote = true;
                    } else if (p0 + r > lim_min) {
                        const uint32_t x[4] = {w->x, w->y, w->z, w->w};
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            if (F::ES == 1) {
#pragma unroll
                                for (int y = 0; y < 4; y++) odd_values |= ((x[k] >> (8 * y)) & 0x7fu) == 0x7fu;
                            } else odd_values |= pt_not_finite16<CT>(x[k] & 0xffffu) || pt_not_finite16<CT>(x[k] >> 16);
                        }
                    }
                }
                odd_values = __any_sync(0xffffffffu, odd_values);  // (also: the cleared rows are written)
            }
            // O += P V
            const int vrow = (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
            for (int np = 0; np < HD * F::ES / 32; np++) {
                uint32_t vb[4], w[F::ES == 1 ? 8 : 4];
                ldsm_x4_t(vb, V + F::at(vrow, np * 2 + (lane >> 4)));
                constexpr int N = F::ES == 1 ? 4 : 2;  // products of eight dimensions each
                if constexpr (F::ES == 1) {
                    // a word holds two positions of two dimensions: dimension by dimension
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint32_t x = __byte_perm(vb[i], 0, 0x3120);
                        w[(i >> 1) * 4 + (i & 1)] = pt_widen(x);
                        w[(i >> 1) * 4 + 2 + (i & 1)] = pt_widen(x >> 16);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++) w[i] = vb[i];
                }
                if (odd_values) {
#pragma unroll
                    for (int i = 0; i < 2 * N; i++) w[i] = pt_finite2<CT>(w[i]);
                }
#pragma unroll
                for (int i = 0; i < N; i++) {
                    pt_mma<CT>(o[np * N + i], pa, w[2 * i], w[2 * i + 1]);
                    if (P2) pt_mma<CT>(o[np * N + i], pr, w[2 * i], w[2 * i + 1]);
                }
            }
            if (odd_values) {
                // the numbers left out above, one by one, to the vectors that see them
#pragma unroll 1
                for (int j = 0; j < PT_BOX; j++) {
                    const uint32_t w0 = __shfl_sync(0xffffffffu, j < 8 ? pa[0] : pa[2], (lane & ~3) + (j % 8) / 2);
                    const uint32_t w1 = __shfl_sync(0xffffffffu, j < 8 ? pa[1] : pa[3], (lane & ~3) + (j % 8) / 2);
                    float pj[2];
#pragma unroll
                    for (int hf = 0; hf < 2; hf++) {
                        const uint32_t h = (hf ? w1 : w0) >> (16 * (j & 1)) & 0xffffu;
                        pj[hf] = CT == SPARSK_BF16 ? bf_lo(h) : __half2float(__ushort_as_half((unsigned short)h));
                    }
                    if (p0 + j >= d.end) break;
#pragma unroll
                    for (int nt = 0; nt < NT; nt++)
#pragma unroll
                        for (int e = 0; e < 2; e++) {
                            const int dim = F::ES == 1 ? (nt >> 1) * 16 + t4 * 4 + e * 2 + (nt & 1) : nt * 8 + t4 * 2 + e;
                            const unsigned char *at_v = V + F::at(j, dim * F::ES / 16) + dim * F::ES % 16;
                            uint32_t h;
                            if (F::ES == 1) h = pt_widen(*at_v);
                            else h = *reinterpret_cast<const uint16_t *>(at_v);
                            h &= 0xffffu;
                            if (!pt_not_finite16<CT>(h)) continue;
                            const float f = CT == SPARSK_BF16 ? bf_lo(h) : __half2float(__ushort_as_half((unsigned short)h));
#pragma unroll
                            for (int hf = 0; hf < 2; hf++)
                                if (p0 + j <= limit[hf]) o[nt][hf * 2 + e] += pj[hf] * f;
                        }
                }
            }
        }
        if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[st]);
        if (!(d.flags & PT_LAST)) continue;

        // ---------------------------------------------------------------- the piece's end
        float l[2], m[2] = {m_run[0], m_run[1]};
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            l[hf] = l_run[hf];
            l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 1);
            l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 2);
        }
        if (PG > 1) {
            // the warps of one block of vectors: to a common maximum
            if (t4 == 0) {
                meet_ml[warp * 16 + (lane >> 2)] = make_float2(m[0], l[0]);
                meet_ml[warp * 16 + (lane >> 2) + 8] = make_float2(m[1], l[1]);
            }
            if (!meet_here()) return;
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                float top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int g = 0; g < PG; g++) top = fmaxf(top, meet_ml[(g * MT + mt) * 16 + (lane >> 2) + hf * 8].x);
                const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int g = 0; g < PG; g++) {
                    const float2 x = meet_ml[(g * MT + mt) * 16 + (lane >> 2) + hf * 8];
                    sum += x.y * exp2f(x.x - use);
                }
                const float f = exp2f(m[hf] - use);
                if (f != 1.f) {
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        o[nt][hf * 2] *= f;
                        o[nt][hf * 2 + 1] *= f;
                    }
                }
                m[hf] = top;
                l[hf] = sum;
            }
        }
        const bool part = d.flags & (PT_HEAD_PART | PT_TAIL_PART);
        const size_t cell = ((size_t)blockIdx.x * 2 + (d.flags & PT_TAIL_PART ? 1 : 0)) * MT + mt;
        float inv[2];
        long long to[2];
        bool have[2];
        const float vs = a.v_scale ? a.v_scale[d.head] : 1.f;
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            const int v = v0 + (lane >> 2) + hf * 8;
            have[hf] = v < n_vec;
            const int r = have[hf] ? v / a.G : 0, h = d.head * a.G + (have[hf] ? v % a.G : 0);
            to[hf] = (d.row0 + r) * a.out_row_stride + h * a.out_head_stride;
            inv[hf] = l[hf] == 0.f ? 0.f : __fdividef(vs, l[hf]);
            if (t4 == 0 && pg == 0) {
                if (part) a.part_ml[cell * 16 + (lane >> 2) + hf * 8] = make_float2(m[hf], l[hf]);
                else if (a.lse && have[hf]) a.lse[(long long)(d.row0 + r) * a.Hk * a.G + h] = l[hf] == 0.f ? -INFINITY : (m[hf] + log2f(l[hf])) * LN2;
            }
        }
        const auto put = [&](int nt, const float4 &x) {
            if (part) {
                a.part_o[(cell * NT + nt) * 32 + lane] = x;
                return;
            }
            const float y[4] = {x.x * inv[0], x.y * inv[0], x.z * inv[1], x.w * inv[1]};
#pragma unroll
            for (int hf = 0; hf < 2; hf++)
                if (have[hf]) {
#pragma unroll
                    for (int e = 0; e < 2; e++) {
                        const int dim = F::ES == 1 ? (nt >> 1) * 16 + t4 * 4 + e * 2 + (nt & 1) : nt * 8 + t4 * 2 + e;
                        if (a.q_type == SPARSK_BF16) reinterpret_cast<bf16 *>(a.out)[to[hf] + dim] = __float2bfloat16(y[hf * 2 + e]);
                        else reinterpret_cast<__half *>(a.out)[to[hf] + dim] = __float2half(y[hf * 2 + e]);
                    }
                }
        };
        if (PG == 1) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++) put(nt, make_float4(o[nt][0], o[nt][1], o[nt][2], o[nt][3]));
        } else {
#pragma unroll
            for (int ph = 0; ph < 2; ph++) {  // half of the dimensions at a time
#pragma unroll
                for (int i = 0; i < NT / 2; i++)
                    meet[(warp * (NT / 2) + i) * 32 + lane] =
                        make_float4(o[ph * NT / 2 + i][0], o[ph * NT / 2 + i][1], o[ph * NT / 2 + i][2], o[ph * NT / 2 + i][3]);
                if (!meet_here()) return;
                for (int i = pg; i < NT / 2; i += PG) {
                    float4 x = meet[(mt * (NT / 2) + i) * 32 + lane];
#pragma unroll
                    for (int g = 1; g < PG; g++) {
                        const float4 y = meet[((g * MT + mt) * (NT / 2) + i) * 32 + lane];
                        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                    }
                    put(ph * (NT / 2) + i, x);
                }
                if (!meet_here()) return;
            }
        }
    }
}

// ------------------------------------------------------------------ the join
// Share `blockIdx.x` ends in the middle of a segment: its last partial and the first ones of the shares behind it, up to
// the one in which the segment ends.  blockIdx.y: which block of 16 vectors, and which quarter of the accumulators.
template <int HD, int CT, int MT>
static __global__ void __launch_bounds__(PJ_THREADS) paged_join_kernel(const PtArgs a, int shares)
{
    constexpr int NT = HD / 8, QN = NT / 4, COLS = QN * 32, GROUPS = PJ_THREADS / COLS;
    constexpr float LN2 = 0.6931471805599453f;
    __shared__ float weight[PT_MAX_SHARES][16], red[PJ_THREADS / 16][16], sums[PJ_THREADS / 16][16];
    __shared__ float4 acc[GROUPS][COLS];
    __shared__ int count;
    griddep_wait();
    const int w0 = blockIdx.x, mt = blockIdx.y >> 2, quarter = blockIdx.y & 3, tid = threadIdx.x;
    PtRecord rec;
    rec.flags = __ldcg(&a.records[w0].flags);
    if (!(rec.flags & 1)) return;
    rec.row0 = __ldcg(&a.records[w0].row0);
    rec.rows = __ldcg(&a.records[w0].rows);
    rec.qblk = __ldcg(&a.records[w0].qblk);
    rec.head = __ldcg(&a.records[w0].head);
    const int v0 = (rec.qblk * MT + mt) * 16, n_vec = rec.rows * a.G;
    if (v0 >= n_vec) return;
    if (tid < 32) {
        int n = 1;
        for (int w = w0 + 1; w < shares; w += 32) {
            const bool last = w + tid < shares && (__ldcg(&a.records[w + tid].flags) & 4);
            const uint32_t b = __ballot_sync(0xffffffffu, last);
            if (b) {
                n += __ffs(b);
                break;
            }
            n += min(32, shares - w);
        }
        if (tid == 0) count = n;
    }
    __syncthreads();
    const int n = count;
    const auto cell = [&](int i) { return ((size_t)(w0 + i) * 2 + (i == 0 ? 1 : 0)) * MT + mt; };
    // weights of the partials for each vector
    const int v = tid & 15, i0 = tid >> 4;
    float top = -INFINITY;
    for (int i = i0; i < n; i += PJ_THREADS / 16) {
        const float2 x = __ldcg(&a.part_ml[cell(i) * 16 + v]);
        weight[i][v] = x.x;
        top = fmaxf(top, x.x);
    }
    red[i0][v] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PJ_THREADS / 16; i++) top = fmaxf(top, red[i][v]);
    const float use = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int i = i0; i < n; i += PJ_THREADS / 16) {
        const float f = exp2f(weight[i][v] - use);
        weight[i][v] = f;
        sum += f * __ldcg(&a.part_ml[cell(i) * 16 + v]).y;
    }
    sums[i0][v] = sum;
    __syncthreads();
    const int col = tid % COLS, grp = tid / COLS, lane = col & 31, nt = quarter * QN + col / 32;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = grp; i < n; i += GROUPS) {
        const float4 y = __ldcg(&a.part_o[(cell(i) * NT + nt) * 32 + lane]);
        const float f0 = weight[i][lane >> 2], f1 = weight[i][(lane >> 2) + 8];
        x.x += f0 * y.x; x.y += f0 * y.y; x.z += f1 * y.z; x.w += f1 * y.w;
    }
    acc[grp][col] = x;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; g++) {
        const float4 y = acc[g][col];
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    const float vs = a.v_scale ? a.v_scale[rec.head] : 1.f;
    const float val[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int hf = 0; hf < 2; hf++) {
        const int vec = (lane >> 2) + hf * 8;
        if (v0 + vec >= n_vec) continue;
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < PJ_THREADS / 16; i++) l += sums[i][vec];
        const int r = (v0 + vec) / a.G, h = rec.head * a.G + (v0 + vec) % a.G;
        const float inv = l == 0.f ? 0.f : __fdividef(vs, l);
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int dim = CT == SPARSK_E4M3 ? (nt >> 1) * 16 + (lane & 3) * 4 + e * 2 + (nt & 1) : nt * 8 + (lane & 3) * 2 + e;
            const long long at = (rec.row0 + r) * a.out_row_stride + h * a.out_head_stride + dim;
            if (a.q_type == SPARSK_BF16) reinterpret_cast<bf16 *>(a.out)[at] = __float2bfloat16(val[hf * 2 + e] * inv);
            else reinterpret_cast<__half *>(a.out)[at] = __float2half(val[hf * 2 + e] * inv);
        }
        if (a.lse && quarter == 0 && nt == 0 && (lane & 3) == 0) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < PJ_THREADS / 16; i++) m = fmaxf(m, red[i][vec]);
            a.lse[(long long)(rec.row0 + r) * a.Hk * a.G + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
        }
    }
}

}  // namespace sparsk
