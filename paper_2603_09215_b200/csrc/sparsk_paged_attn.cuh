// Attention of a step's new rows over a paged cache, split over the cache's length and joined.
//
//   out = sum_p w_p v_p / sum_p w_p,  w_p = exp(scale q.k_p - max), the maximum and both sums running (one pass).
//
// A segment is (sequence, block of up to 64 query vectors, kv head): the rows' query heads of that kv head are the M dimension of
// m16n8k16 products (as in sparsk_attn.cuh), so that one read of the head's keys and values serves all of them.
// All segments, laid end to end in boxes of 16 positions (plus a few boxes' worth for a segment's set-up and end), are cut into equal
// shares, one for each CTA of a grid that is resident at once: nobody knows the lengths but the device, and
// every CTA adds them up.  A share begins and ends anywhere; a segment that lies in one share is written
// out at once, others leave a partial (sums and maxima) at either end of a share, which
// a second kernel joins in order.
//
// Within a CTA one warp brings boxes of 16 positions by TMA (a tensor map of the pool: dimensions, positions of a page, halves of
// the head, heads, pages, whichever of heads and positions lies outside; a box never leaves its page, whose size is a multiple of 16) into
// a ring of stages of 64 positions, and four warps take boxes from it: a box each where the segment has up to 16 query
// vectors, two boxes each for one of two tiles of 16 where it has up to 32, else all four for one of four.  Every warp
// keeps the softmax of its own positions; the warps of one tile meet at the segment's end only.  8-bit pages are widened to fp16 in
// registers, between the shared memory and the product.
// Bound by HBM where a segment has one tile of query vectors: a position of a head of 128 fp16 numbers is 512 bytes, 23 of which
// come per clock and SM, so 16 positions may take 350 clocks of an SM; eight computing warps need about 240.  64 sequences of
// 8,192 positions (32 heads on 2, bf16): 537 MB in 92 us, 5.8 TB/s of 6.5 that a copy reaches; 64 of 256 to 2,048 (28 on 4, fp16): 152 MB
// in 35.8 us, of which the first copies take 3, the segments' ends and the join 5.  With three or four tiles the warps' instructions
// bound it (about 330 a box and tile, widening of 8-bit pages among them): 48 refresh blocks of up to four rows, 32 heads on 2:
// 60 MB of e4m3 in 45 us, 120 MB of fp16 in 42.  Two boxes side by side in a warp were 4 % faster there over e4m3, and slower
// elsewhere (single rows 4 %).  Single rows over 8-bit pages are bound by instructions as well: half the bytes leave 175 clocks for 16
// positions, and their numbers are widened besides: 64 sequences of 8,192 (32 on 2) 74 us, 41 of them bytes; fp16 92 of 82.
// A block of vectors is sent every box of its sequence, those behind its last row too, which are masked: a refresh block has one or two
// of them, but of the rows of a prompt from nothing half the boxes are such (four of 1,000 rows, 28 on 4: 734 us, 39 TFLOP/s).
// What a share waits for at its start is instructions that no warp of the SM has met yet, more than memory: divisions
// out of line, one code for all tile counts.
#pragma once

#include <cstdint>
#include <type_traits>

#include "../../include/sparsk.h"
#include "sparsk_common.cuh"
#include "sparsk_warp.cuh"

namespace sparsk {

constexpr int PT_THREADS = 256, PT_WARPS = 4, PT_Q_WARPS = 3;  // four warps compute, one brings the boxes, three the queries
// Registers are given out by fours of warps, and the four that compute take most of what the others were launched with.
constexpr int PT_REGS = 200, PT_REGS_BRING = 56;  // (times 128 threads each: the launch's 128 times 256)
constexpr int PT_BOX = 16, PT_STAGE = 64;      // positions
constexpr int PT_CTAS = 2;                     // resident on an SM
constexpr int PT_MAX_SHARES = 2 * 160;         // CTAs of a launch (the scratch is sized for them)
constexpr int PT_END_COST = 24;                // a segment's set-up and end, in the unit of PtForm::box_cost (16 or 36: 1 to 2 % more)
constexpr int PT_WHOLE = 8;                    // a segment of up to so many boxes is never cut
constexpr int PT_MIN_SHARE = 20;               // the same unit (40 puts two short segments into one share: 7.1 us for 5.1; one of 1,500
                                               // positions 11.2 us, with 40 13.1, with 80 16.5)
constexpr float PT_LAG = 8.f;                  // in powers of two, and these
constexpr float PT_UP = 7.f;                   // weights that are fp16 numbers lie so much higher: 2^15 at most
constexpr float PT_DEEP = 12.f, PT_LIFT = 64.f; // a box whose largest weight is below 2^-PT_DEEP is raised further, 2^PT_LIFT at most
constexpr int PT_RING_BYTES = 112 * 1024;      // of a CTA's shared memory: boxes, queries, sums that meet
constexpr int PJ_THREADS = 256;

// A share's partials for the join: bit 0 its last segment goes on in the next share, bits 1..2 its first one began in an
// earlier share and 1 goes on, 2 ends here; and which segment the last one is.
struct __align__(16) PtRecord {
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
    float4 *part_o;     // [shares][2][tiles][HD / 8][32 lanes]: accumulators as the lanes hold them
    float2 *part_ml;    // [shares][2][tiles][16]: maximum in powers of two, sum
    int *status;        // or NULL
    long long table_stride, q_row_stride, q_head_stride, out_row_stride, out_head_stride;
    float scale_log2;
    float up;           // PtForm::UP
    int q_type, n_rows, n_seqs, max_blocks, page_size, n_pages, Hk, G;
    int tiles;          // of 16 query vectors, in a segment at most (1, 2 or 4)
    int page_shift;     // a page has 2^page_shift boxes, or -1
    int whole_boxes;    // segments of up to so many boxes are never cut
    int short_copy;     // of which CTA (from 1) the stages wait for more bytes than come; 0: of none
    uint32_t g_inverse, g_limit;  // ceil(2^32 / G), and below which numbers it divides by G exactly
    int q_wide, out_words;      // queries may be read sixteen bytes at a time, outputs written two numbers at a time
};

template <int HD, int CT>
struct PtForm {
    static constexpr int ES = CT == SPARSK_E4M3 ? 1 : 2;
    static constexpr int RB = HD * ES;                          // bytes of a position
    static constexpr int STAGE = 2 * PT_STAGE * RB;             // keys, then values
    static constexpr int SUMS = PT_WARPS * (HD / 8) * 32 * 16;  // the warps' accumulators
    static constexpr int MEET = SUMS > STAGE ? SUMS - STAGE : 0; // what of them a stage does not hold
    static constexpr int QTILE = 16 * HD * 2;                   // a tile's queries
    static constexpr int FIT = (PT_RING_BYTES - MEET - 4 * QTILE) / STAGE, NS = FIT < 11 ? FIT : 11;
    static constexpr int SMEM = NS * STAGE + MEET + 4 * QTILE + NS * (16 + (int)sizeof(PtStage)) + 160 + PT_WARPS * 16 * 8 + 16;
    static_assert(PT_CTAS * (SMEM + 1024) <= 228 * 1024, "two CTAs share an SM");
    // What a box costs where the segment has one tile of vectors (the stage's boxes go to four warps), two (two by two) or more
    // (every box to every warp).  48 refresh blocks over e4m3 / fp16 pages, us: 2, 3, 5 47.2 / 41.3 (44.8 / 42.3 since); 2, 3, 6 50.1 / 43.5; 2, 3, 8 56.6 / 49.9; 2,
    // 2, 5 56.5 / 48.4; 2, 4, 6 48.9 / 43.7 (and 28 vectors in fp16 56.1 for 51.9).
    static constexpr int PT_C2 = 3, PT_C4 = 5;
    static constexpr float UP = CT == SPARSK_BF16 ? 0.f : PT_UP;  // (bf16 weights have the range of fp32)
    __device__ __forceinline__ static int box_cost(int vectors) { return vectors <= 16 ? 2 : vectors <= 32 ? PT_C2 : PT_C4; }
    // byte offset of 16-byte chunk c of row r inside a box
    __device__ __forceinline__ static int at(int r, int c)
    {
        if (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
        return (RB > 128 ? (c >> 3) * (PT_BOX * 128) : 0) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
    }
    // the same inside a tile of queries
    __device__ __forceinline__ static int at_q(int r, int c) { return r * HD * 2 + ((c & ~7) << 4) + (((c & 7) ^ (r & 7)) << 4); }
    // at(r, c0 + c) from at(r, c0), c0 below 2 and c even
    __device__ __forceinline__ static int turn(int at0, int c) { return (at0 ^ ((c & 7) << 4)) + (c >> 3) * (PT_BOX * 128); }
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
// 2^n, exactly (exp2f is not)
__device__ __forceinline__ float pt_power(int n) { return __int_as_float((127 + n) << 23); }
// two e4m3 numbers -> two fp16 numbers (exact)
__device__ __forceinline__ uint32_t pt_widen(uint32_t two)
{
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(r) : "r"(two));
    return r;
}
// four of them at once
__device__ __forceinline__ void pt_widen4(uint32_t four, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(four));
}
// Two query numbers in the type that meets the pool's: a number beyond fp16 as its largest.
template <int CT>
__device__ __forceinline__ uint32_t pt_query2(uint32_t w, int q_type)
{
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

// Values that nobody sees meet a weight of zero, which must not meet an infinity or a NaN: the box's rows behind `end` are
// cleared (`wrote`).  True (in all lanes) if rows that some vectors of a causal block see and others do not, those behind
// lim_min, hold such numbers.
template <int HD, int CT>
__device__ __forceinline__ bool pt_clean(unsigned char *V, int p0, int end, int lim_min, int lane, bool &wrote)
{
    typedef PtForm<HD, CT> F;
    constexpr int CH = F::RB / 16;
    bool odd = false;
#pragma unroll 1
    for (int i = lane; i < PT_BOX * CH; i += 32) {
        const int r = i / CH;
        uint4 *w = reinterpret_cast<uint4 *>(V + F::at(r, i % CH));
        if (p0 + r >= end) {
            *w = make_uint4(0u, 0u, 0u, 0u);
            wrote = true;
        } else if (p0 + r > lim_min) {
            const uint32_t x[4] = {w->x, w->y, w->z, w->w};
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (F::ES == 1) {
#pragma unroll
                    for (int y = 0; y < 4; y++) odd |= ((x[k] >> (8 * y)) & 0x7fu) == 0x7fu;
                } else odd |= pt_not_finite16<CT>(x[k] & 0xffffu) || pt_not_finite16<CT>(x[k] >> 16);
            }
        }
    }
    __syncwarp();  // the warp's other lanes read the cleared rows (a vote orders no memory)
    return __any_sync(0xffffffffu, odd);
}

// O += P V for one box.  ODD: numbers that are not finite are left out of the products and given one by one to the vectors
// that see them.
template <int HD, int CT, bool P2, bool ODD>
__device__ __forceinline__ void pt_values(float (&o)[HD / 8][4], const uint32_t (&pa)[4], const uint32_t (&pr)[4], const unsigned char *V,
                                          int v_at, int lane, int p0, int end, const int (&limit)[2])
{
    typedef PtForm<HD, CT> F;
    constexpr int N = F::ES == 1 ? 4 : 2;  // products of eight dimensions a load
#pragma unroll
    for (int np = 0; np < HD / 8 / N; np++) {
        uint32_t vb[4], w[2 * N];
        ldsm_x4_t(vb, V + F::turn(v_at, np * 2));
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (F::ES == 1) {
                // a word holds two positions of two dimensions: dimension by dimension
                pt_widen4(__byte_perm(vb[i], 0, 0x3120), w[(i >> 1) * 4 + (i & 1)], w[(i >> 1) * 4 + 2 + (i & 1)]);
            } else w[i] = vb[i];
        }
        if (ODD) {
#pragma unroll
            for (int i = 0; i < 2 * N; i++) w[i] = pt_finite2<CT>(w[i]);
        }
#pragma unroll
        for (int i = 0; i < N; i++) {
            pt_mma<CT>(o[np * N + i], pa, w[2 * i], w[2 * i + 1]);
            if (P2) pt_mma<CT>(o[np * N + i], pr, w[2 * i], w[2 * i + 1]);
        }
    }
    if (!ODD) return;
    const int t4 = lane & 3;
#pragma unroll 1
    for (int j = 0; j < PT_BOX && p0 + j < end; j++) {
        const uint32_t w0 = __shfl_sync(0xffffffffu, j < 8 ? pa[0] : pa[2], (lane & ~3) + (j % 8) / 2);
        const uint32_t w1 = __shfl_sync(0xffffffffu, j < 8 ? pa[1] : pa[3], (lane & ~3) + (j % 8) / 2);
        float pj[2];
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            const uint32_t h = (hf ? w1 : w0) >> (16 * (j & 1)) & 0xffffu;
            pj[hf] = CT == SPARSK_BF16 ? bf_lo(h) : __half2float(__ushort_as_half((unsigned short)h));
        }
#pragma unroll
        for (int nt = 0; nt < HD / 8; nt++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int dim = F::ES == 1 ? (nt >> 1) * 16 + t4 * 4 + e * 2 + (nt & 1) : nt * 8 + t4 * 2 + e;
                const unsigned char *at_v = V + F::at(j, dim * F::ES / 16) + dim * F::ES % 16;
                const uint32_t h = (F::ES == 1 ? pt_widen(*at_v) : *reinterpret_cast<const uint16_t *>(at_v)) & 0xffffu;
                if (!pt_not_finite16<CT>(h)) continue;
                const float f = CT == SPARSK_BF16 ? bf_lo(h) : __half2float(__ushort_as_half((unsigned short)h));
#pragma unroll
                for (int hf = 0; hf < 2; hf++)
                    if (p0 + j <= limit[hf]) o[nt][hf * 2 + e] += pj[hf] * f;
            }
    }
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
// segments of a sequence
__device__ __forceinline__ int pt_segments(const PtArgs &a, int rows)
{
    const int shift = a.tiles == 1 ? 4 : a.tiles == 2 ? 5 : 6;
    return ((rows * a.G + (1 << shift) - 1) >> shift) * a.Hk;  // (rows times query heads fit 31 bits)
}
// x / y for x >= 0, y > 0: almost always of 32 bits, which divide several times as fast
static __device__ __noinline__ long long pt_div_wide(long long x, int y) { return x / y; }
__device__ __forceinline__ long long pt_div(long long x, int y)
{
    return (x >> 32) == 0 ? (long long)((unsigned)x / (unsigned)y) : pt_div_wide(x, y);
}
// a CTA's share of the sum of all costs
__device__ __forceinline__ long long pt_share(long long total) { return max(pt_div(total + gridDim.x - 1, gridDim.x), (long long)PT_MIN_SHARE); }
// v / G for a query vector's number
__device__ __forceinline__ int pt_row_of(const PtArgs &a, int v)
{
    return (uint32_t)v < a.g_limit ? (int)__umulhi((uint32_t)v, a.g_inverse) : v / a.G;
}
// A wait that ends: the hardware's own, again and again until the phase is over, somebody has given up or two seconds have gone.
__device__ __forceinline__ bool pt_wait(uint64_t *bar, uint32_t parity, volatile int *giving_up)
{
    const uint32_t at = smem_u32(bar);
    unsigned long long t0 = 0;
    for (uint32_t spin = 0;; spin++) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(at), "r"(parity)
            : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
        if ((spin & 63u) == 63u) {
            bool stop = *giving_up;
            const unsigned long long now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > WAIT_TIMEOUT_NS) stop = true;
            if (__any_sync(0xffffffffu, stop)) {
                *giving_up = 1;
                return false;
            }
        }
    }
}

// A warp that is done (its copies have landed) and leaves; those that compute wait for all.
__device__ __forceinline__ void pt_left() { asm volatile("barrier.arrive 1, %0;" ::"n"(PT_THREADS) : "memory"); }

// The outputs of one vector from two neighbouring products: two and two numbers side by side, or, where the products took
// even and odd dimensions (8-bit pages), four.
template <int ES>
__device__ __forceinline__ void pt_put(const PtArgs &a, long long to, int nt, int t4, float e0, float e1, float o0, float o1)
{
    const auto two = [&](float x, float y) { return a.q_type == SPARSK_BF16 ? pack_bf16x2(x, y) : pack_h2(x, y); };
    const uint32_t w0 = ES == 1 ? two(e0, o0) : two(e0, e1), w1 = ES == 1 ? two(e1, o1) : two(o0, o1);
    uint16_t *p0 = reinterpret_cast<uint16_t *>(a.out) + to + nt * 8 + t4 * (ES == 1 ? 4 : 2), *p1 = p0 + (ES == 1 ? 2 : 8);
    if (a.out_words) {
        *reinterpret_cast<uint32_t *>(p0) = w0;
        *reinterpret_cast<uint32_t *>(p1) = w1;
    } else {
        p0[0] = (uint16_t)w0;
        p0[1] = (uint16_t)(w0 >> 16);
        p1[0] = (uint16_t)w1;
        p1[1] = (uint16_t)(w1 >> 16);
    }
}

template <int HD, int CT, bool P2>
static __global__ void __launch_bounds__(PT_THREADS, PT_CTAS)
paged_attn_kernel(const PtArgs a, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv)
{
    typedef PtForm<HD, CT> F;
    constexpr int NS = F::NS, RB = F::RB, KS = HD / 16, NT = HD / 8;
    constexpr float LN2 = 0.6931471805599453f;
    extern __shared__ __align__(1024) unsigned char pt_smem[];
    unsigned char *ring = pt_smem;
    float4 *meet = reinterpret_cast<float4 *>(pt_smem + NS * F::STAGE);
    unsigned char *queries = pt_smem + NS * F::STAGE + F::MEET;  // four tiles: of four, two segments or one
    uint64_t *full = reinterpret_cast<uint64_t *>(queries + 4 * F::QTILE), *empty = full + NS, *q_full = empty + NS, *q_empty = q_full + 4, *q_told = q_empty + 4;
    int4 *segments = reinterpret_cast<int4 *>(q_told + 4);
    PtStage *stages = reinterpret_cast<PtStage *>(segments + 4);
    float2 *meet_ml = reinterpret_cast<float2 *>(stages + NS);
    uint64_t *meeting = reinterpret_cast<uint64_t *>(meet_ml + PT_WARPS * 16);
    volatile int *giving_up = reinterpret_cast<volatile int *>(meeting + 1);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    griddep_launch();
    if (tid == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mk) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&mv) : "memory");
    }
    if (tid == 0) {
        for (int s = 0; s < NS; s++) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], PT_WARPS);
        }
        for (int s = 0; s < 4; s++) {
            mbar_init(&q_full[s], PT_Q_WARPS * 32);
            mbar_init(&q_empty[s], PT_WARPS);
            mbar_init(&q_told[s], 1);
        }
        mbar_init(meeting, PT_WARPS);
        giving_up[0] = giving_up[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    griddep_wait();

    // This CTA's share [beg, end) of all segments' boxes.  What a thread's sequences cost, and what those before them do:
    const int cap = a.max_blocks * a.page_size;
    const auto boxes_of = [&](const PtSeq &s) { return (min(s.len, cap) + PT_BOX - 1) / PT_BOX; };
    const auto box_cost = [&](const PtSeq &s) { return F::box_cost(min(s.rows * a.G, a.tiles * 16)); };
    const auto cost_of = [&](const PtSeq &s) { return boxes_of(s) * box_cost(s) + PT_END_COST; };
    const int per = (a.n_seqs + PT_THREADS - 1) / PT_THREADS;
    long long *plan = reinterpret_cast<long long *>(queries);           // [256]: up to and with a thread's sequences, in its warp
    PtSeq *plan_seq = reinterpret_cast<PtSeq *>(plan + PT_THREADS);     // [256], where a thread has one sequence
    {
        long long mine = 0;
#pragma unroll 1
        for (int i = tid * per; i < min((tid + 1) * per, a.n_seqs); i++) {
            // (the lines of the tables on their way to the L2 meanwhile, one for each CTA)
            if ((int)blockIdx.x * 32 < a.max_blocks) prefetch_l2(a.block_table + i * a.table_stride + blockIdx.x * 32);
            const PtSeq s = pt_seq(a, i);
            mine += (long long)pt_segments(a, s.rows) * cost_of(s);
            plan_seq[tid] = s;
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, mine, o);
            if (lane >= o) mine += y;
        }
        plan[tid] = mine;
    }
    __syncthreads();
    const int q_shift = a.tiles == 1 ? 2 : a.tiles == 2 ? 1 : 0, q_slots = 1 << q_shift;
    if (warp >= PT_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PT_REGS_BRING));
        if (warp > PT_WARPS) {
            // ------------------------------------------------------------ the warps that bring the queries, sixteen bytes a lane
            // and copy.  (Read by the computing warps themselves, as the lanes hold them, they cost four times the sectors in each of
            // four warps and a trip to the memory at every segment's start.)
            for (int segs = 0;; segs++) {
                const int slot = segs & (q_slots - 1);
                if (!pt_wait(&q_told[slot], (segs >> q_shift) & 1, giving_up)) break;
                const int4 seg = segments[slot];  // first row, rows, block of vectors, kv head
                if (seg.y < 0) break;
                const int v_first = seg.z * a.tiles * 16, n_here = min(seg.y * a.G - v_first, a.tiles * 16);
                unsigned char *dst = queries + slot * a.tiles * F::QTILE;
#pragma unroll 4
                for (int i = tid - (PT_WARPS + 1) * 32; i < n_here * (HD / 8); i += PT_Q_WARPS * 32) {
                    const int v = i / (HD / 8), c = i % (HD / 8), r = pt_row_of(a, v_first + v);
                    const uint16_t *src = reinterpret_cast<const uint16_t *>(a.q) + (seg.x + r) * a.q_row_stride +
                                          (seg.w * a.G + v_first + v - r * a.G) * a.q_head_stride + c * 8;
                    unsigned char *to_q = dst + F::at_q(v, c);
                    if (a.q_wide) cp_async16(to_q, src, 16);
                    else {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; k++) w[k] = (uint32_t)src[2 * k] | ((uint32_t)src[2 * k + 1] << 16);
                        *reinterpret_cast<uint4 *>(to_q) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
                if (a.q_wide) asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&q_full[slot])) : "memory");
                else mbar_arrive(&q_full[slot]);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            pt_left();
            return;
        }
        // ---------------------------------------------------------------- the warp that brings the boxes
        long long upto = lane < PT_THREADS / 32 ? plan[lane * 32 + 31] : 0;
#pragma unroll
        for (int o = 1; o < PT_THREADS / 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        const long long total = __shfl_sync(0xffffffffu, upto, PT_THREADS / 32 - 1);
        const long long share = pt_share(total);
        const long long beg = share * blockIdx.x, end = min(beg + share, total);
        int seq = 0, base = 0, it = 0, issued = 0, flags = 0, segs = 0;
        long long at = 0, x = beg;
        PtSeq now{}, ahead{};  // `ahead`: of sequence base + lane
        if (beg < end) {
            // the sequence in which it begins: its warp, its thread, and of a thread's sequences which
            const int w = __ffs(__ballot_sync(0xffffffffu, beg < upto && lane < PT_THREADS / 32)) - 1;
            const long long before = w > 0 ? __shfl_sync(0xffffffffu, upto, w - 1) : 0, in_warp = plan[w * 32 + lane];
            const int l = __ffs(__ballot_sync(0xffffffffu, beg < before + in_warp)) - 1;
            const long long before_lane = __shfl_sync(0xffffffffu, in_warp, max(l - 1, 0));
            at = before + (l > 0 ? before_lane : 0);
            seq = base = (w * 32 + l) * per;
            if (per == 1) {
                if (seq + lane < a.n_seqs) ahead = plan_seq[seq + lane];
            } else if (seq + lane < a.n_seqs) ahead = pt_seq(a, seq + lane);
            now.row0 = __shfl_sync(0xffffffffu, ahead.row0, 0);
            now.rows = __shfl_sync(0xffffffffu, ahead.rows, 0);
            now.len = __shfl_sync(0xffffffffu, ahead.len, 0);
            __syncwarp();
        }
        PtRecord rec{};
        bool ok = true;
        const auto next_stage = [&]() {
            const int s = it % NS;
            if (it >= NS) ok = pt_wait(&empty[s], ((it / NS) - 1) & 1, giving_up);
            it++;
            return s;
        };
        const int page_boxes = a.page_size / PT_BOX;
        const auto page_of = [&](int box) { return a.page_shift >= 0 ? box >> a.page_shift : box / page_boxes; };
        while (ok && x < end) {
            const int cost = cost_of(now), boxes = boxes_of(now), each = box_cost(now);
            const long long all = (long long)pt_segments(a, now.rows) * cost;
            if (x >= at + all) {
                at += all;
                seq++;
                if (seq - base >= 32) {
                    base = seq;
                    if (seq + lane < a.n_seqs) ahead = pt_seq(a, seq + lane);
                }
                now.row0 = __shfl_sync(0xffffffffu, ahead.row0, seq - base);
                now.rows = __shfl_sync(0xffffffffu, ahead.rows, seq - base);
                now.len = __shfl_sync(0xffffffffu, ahead.len, seq - base);
                continue;
            }
            const long long seg = pt_div(x - at, cost);
            const int from = (int)(x - at - seg * cost);
            int to = (int)min((long long)cost, from + (end - x));
            x += to - from;
            if (boxes <= a.whole_boxes) {
                if (from > 0) continue;  // the share before this one has it
                to = cost;
            }
            // a box is the share's in which its cost begins
            constexpr uint32_t INV2 = (uint32_t)(((1ull << 32) + F::PT_C2 - 1) / F::PT_C2), INV4 = (uint32_t)(((1ull << 32) + F::PT_C4 - 1) / F::PT_C4);
            const uint32_t inverse = each == 2 ? 0x80000000u : each == F::PT_C2 ? INV2 : INV4;  // (exact below 2^30)
            const int b0 = min((int)__umulhi(from + each - 1, inverse), boxes), b1 = min((int)__umulhi(to + each - 1, inverse), boxes);
            if (b0 >= b1 && !(boxes == 0 && from == 0)) continue;
            const int qblk = (int)pt_div(seg, a.Hk), head = (int)(seg - (long long)qblk * a.Hk);
            int part = 0;
            if (b0 > 0) {
                part = PT_HEAD_PART;
                flags |= b1 == boxes ? 4 : 2;
            } else if (b1 < boxes) {
                part = PT_TAIL_PART;
                flags |= 1;
                rec.row0 = now.row0;
                rec.rows = now.rows;
                rec.qblk = qblk;
                rec.head = head;
            }
            {
                const int slot = segs & (q_slots - 1);
                if (segs >= q_slots) ok = ok && pt_wait(&q_empty[slot], ((segs >> q_shift) - 1) & 1, giving_up);
                if (!ok) break;
                segs++;
                if (lane == 0) {
                    segments[slot] = make_int4(now.row0, now.rows, qblk, head);
                    mbar_arrive(&q_told[slot]);
                }
            }
            const int pos_end = min(min(now.len, cap), b1 * PT_BOX);
            int page = -1;
            for (int b = b0; ok && (b < b1 || b == b0); b += 4) {
                const int chunk = (b - b0) & 31;
                if (chunk == 0) {  // the pages of the next 32 boxes
                    const int mine_b = b + lane;
                    page = mine_b < b1 ? __ldcg(a.block_table + seq * a.table_stride + page_of(mine_b)) : -1;
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
                    d.row0 = now.row0;
                    d.rows = now.rows;
                    d.len = now.len;
                    d.qblk = qblk;
                    d.head = head;
                    mbar_expect_tx(&full[st], (uint32_t)__popc(have) * 2u * PT_BOX * RB + (a.short_copy == (int)blockIdx.x + 1 ? 16u : 0u));
                }
                __syncwarp();
                if (copy) {
                    const int box = b + j, y = (box - page_of(box) * page_boxes) * PT_BOX;
                    const uint32_t dst = smem_u32(ring + st * F::STAGE + (lane & 1) * (PT_STAGE * RB) + j * (PT_BOX * RB));
                    tma_load_5d(dst, (lane & 1) ? &mv : &mk, &full[st], y, head, my_page);
                }
                issued = it;
            }
        }
        if (ok && segs >= q_slots) ok = pt_wait(&q_empty[segs & (q_slots - 1)], ((segs >> q_shift) - 1) & 1, giving_up);
        if (ok && lane == 0) {
            segments[segs & (q_slots - 1)].y = -1;
            mbar_arrive(&q_told[segs & (q_slots - 1)]);
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
            for (int k = max(0, issued - NS); k < issued; k++) pt_wait(&full[k % NS], (k / NS) & 1, giving_up + 1);
        pt_left();
        return;
    }

    // -------------------------------------------------------------------- the warps that compute
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(PT_REGS));
    const int t4 = lane & 3;
    int mt = 0, pg = 0, PG = 1;  // this warp's tile of 16 vectors, its place among the PG warps of the tile
    uint32_t qa[KS][4];
    // of a vector: its maximum, what its weights are taken relative to, the middle of the maxima that a box may have without
    // scaling, and how far they may lie from it
    float o[NT][4], m_run[2], m_use[2], m_mid[2], m_far[2], l_run[2], c_log2 = 0.f;
    // where this lane reads its rows of a box: the chunk's low bit is the lane's, even steps turn the others
    const int k_at = F::at((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1), v_at = F::at((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);
    int limit[2], lim_min = 0, meetings = 0, segs = 0;
    // all four warps; like every wait here it ends by itself when another warp has given up
    const auto meet_here = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(meeting);
        return pt_wait(meeting, meetings++ & 1, giving_up);
    };
    for (int it = 0;; it++) {
        const int st = it % NS;
        if (!pt_wait(&full[st], (it / NS) & 1, giving_up)) break;
        const PtStage d = stages[st];
        if (d.flags & PT_STOP) break;
        const int n_vec = d.rows * a.G;  // of the sequence
        if (d.flags & PT_FIRST) {
            const int n_here = min(n_vec - d.qblk * a.tiles * 16, a.tiles * 16), shift = n_here <= 16 ? 0 : n_here <= 32 ? 1 : 2;
            mt = warp & ((1 << shift) - 1);
            pg = warp >> shift;
            PG = PT_WARPS >> shift;
        }
        const int v0 = (d.qblk * a.tiles + mt) * 16;  // this warp's query vectors: v0 .. v0 + 15, as far as there are
        if (d.flags & PT_FIRST) {
            c_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[d.head] : 1.f);
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
                for (int e = 0; e < 4; e++) o[nt][e] = 0.f;
            lim_min = d.len - d.rows + pt_row_of(a, v0);
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                const int v = v0 + (lane >> 2) + hf * 8;
                const bool have = v < n_vec;
                m_run[hf] = m_mid[hf] = -INFINITY;
                m_use[hf] = l_run[hf] = 0.f;
                m_far[hf] = !have ? INFINITY : F::UP > 0.f ? (PT_LAG + PT_DEEP) / 2 : PT_LAG;
                limit[hf] = have ? d.len - d.rows + pt_row_of(a, v) : -1;  // the last position that this vector sees
            }
            // (the rows of vectors that a tile does not have hold anything, and nobody reads what comes of them)
            const int slot = segs & (q_slots - 1);
            if (!pt_wait(&q_full[slot], (segs >> q_shift) & 1, giving_up)) break;
            segs++;
            const unsigned char *Q = queries + (slot * a.tiles + mt) * F::QTILE;
#pragma unroll
            for (int ks = 0; ks < KS; ks++) {
                if constexpr (F::ES == 1) {
                    // 8-bit keys come four dimensions to a lane
                    const uint2 x = *reinterpret_cast<const uint2 *>(Q + F::at_q(lane >> 2, ks * 2 + (t4 >> 1)) + (t4 & 1) * 8);
                    const uint2 y = *reinterpret_cast<const uint2 *>(Q + F::at_q((lane >> 2) + 8, ks * 2 + (t4 >> 1)) + (t4 & 1) * 8);
                    qa[ks][0] = x.x; qa[ks][1] = y.x; qa[ks][2] = x.y; qa[ks][3] = y.y;
                } else ldsm_x4(qa[ks], Q + F::at_q(lane & 15, ks * 2 + (lane >> 4)));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_empty[slot]);
#pragma unroll
            for (int ks = 0; ks < KS; ks++)
#pragma unroll
                for (int i = 0; i < 4; i++) qa[ks][i] = pt_query2<CT>(qa[ks][i], a.q_type);
        }
        bool wrote = false;
#pragma unroll 1
        for (int b = v0 < n_vec ? pg : 4; b < 4; b += PG) {  // (a tile without vectors has nothing to do)
            const int p0 = d.p0 + b * PT_BOX;
            if (!(d.flags >> (8 + b) & 1)) continue;
            const unsigned char *K = ring + st * F::STAGE + b * (PT_BOX * RB), *V = K + PT_STAGE * RB;
            // S = Q K^T for 16 positions, two chains
            float s[2][2][4];
#pragma unroll
            for (int i = 0; i < 16; i++) s[i >> 3][i >> 2 & 1][i & 3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ks += 2) {
                uint32_t kb[4];
                if constexpr (F::ES == 2) {
                    uint32_t kb2[4];
                    ldsm_x4(kb, K + F::turn(k_at, ks * 2));
                    ldsm_x4(kb2, K + F::turn(k_at, ks * 2 + 2));
                    pt_mma<CT>(s[0][0], qa[ks], kb[0], kb[1]);
                    pt_mma<CT>(s[0][1], qa[ks], kb[2], kb[3]);
                    pt_mma<CT>(s[1][0], qa[ks + 1], kb2[0], kb2[1]);
                    pt_mma<CT>(s[1][1], qa[ks + 1], kb2[2], kb2[3]);
                } else {
                    ldsm_x4(kb, K + F::turn(k_at, ks));
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 4; i++) pt_widen4(kb[i], w[2 * i], w[2 * i + 1]);
                    pt_mma<CT>(s[0][0], qa[ks], w[0], w[1]);
                    pt_mma<CT>(s[0][1], qa[ks], w[4], w[5]);
                    pt_mma<CT>(s[1][0], qa[ks + 1], w[2], w[3]);
                    pt_mma<CT>(s[1][1], qa[ks + 1], w[6], w[7]);
                }
            }
            // a box that every vector sees whole needs no mask
            const bool whole = p0 + PT_BOX <= d.end && p0 + PT_BOX - 1 <= lim_min;
            float v[2][4], top[2];
#pragma unroll
            for (int hf = 0; hf < 2; hf++)
#pragma unroll
                for (int i = 0; i < 4; i++) v[hf][i] = (s[0][i >> 1][hf * 2 + (i & 1)] + s[1][i >> 1][hf * 2 + (i & 1)]) * c_log2;
            if (!whole) {
#pragma unroll
                for (int hf = 0; hf < 2; hf++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int p = p0 + (i >> 1) * 8 + t4 * 2 + (i & 1);
                        if (p >= d.end || p > limit[hf]) v[hf][i] = -INFINITY;
                    }
            }
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                top[hf] = fmaxf(fmaxf(v[hf][0], v[hf][1]), fmaxf(v[hf][2], v[hf][3]));
                top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xffffffffu, top[hf], 1));
                top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xffffffffu, top[hf], 2));
            }
            // Weights are taken relative to a maximum that follows the true one only when that has grown by more than
            // 2^PT_LAG: up to there they fit fp16 as well, and what was summed before needs no rescaling (which almost every box
            // would ask for otherwise: it is enough that one of sixteen vectors meets a larger score).
            // fp16 ends at 2^-24 and has all its bits from 2^-14 on, and many light positions can outweigh a heavy one whose values
            // are near zero.  So weights are 2^UP times what they are, and those of a box that holds none above 2^-PT_DEEP (of
            // the maximum) are raised by a power of two of their own, for which the sums are raised before the products and
            // let down after them (exactly): a weight is right to its rounding and 2^-20 of the largest of its box.  (Left as they
            // were, 32,768 positions e^-17 below one of zero values came out 44 % too large.)
            float m_box[2] = {m_use[0], m_use[1]};
            int lift[2] = {0, 0};
            bool lifted = false;
            const auto stays = [&](int hf) {  // (true where there is nothing yet and nothing comes: a difference of infinities)
                const float off = top[hf] - m_mid[hf];
                return !((F::UP > 0.f ? fabsf(off) : off) > m_far[hf]);
            };
            if (!__all_sync(0xffffffffu, stays(0) && stays(1))) {
#pragma unroll
                for (int hf = 0; hf < 2; hf++) {
                    float alpha = 1.f;
                    if (top[hf] > m_run[hf] + PT_LAG) {  // (each vector by its own scores alone)
                        alpha = exp2f(m_run[hf] - top[hf]);  // 2^-inf = 0 at first
                        m_run[hf] = top[hf];
                        m_box[hf] = m_use[hf] = top[hf] - F::UP;
                        m_mid[hf] = top[hf] - (F::UP > 0.f ? (PT_DEEP - PT_LAG) / 2 : 0.f);
                    } else if (!stays(hf) && top[hf] != -INFINITY) {
                        lift[hf] = (int)fminf(m_run[hf] - top[hf], PT_LIFT);
                        alpha = pt_power(lift[hf]);
                        m_box[hf] = m_use[hf] - (float)lift[hf];
                    }
                    l_run[hf] *= alpha;
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        o[nt][hf * 2] *= alpha;
                        o[nt][hf * 2 + 1] *= alpha;
                    }
                }
                if (F::UP > 0.f) lifted = __any_sync(0xffffffffu, (lift[0] | lift[1]) != 0);
            }
            uint32_t pa[4], pr[4];
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                float w[4];
#pragma unroll
                for (int i = 0; i < 4; i++) w[i] = exp2f(v[hf][i] - m_box[hf]);  // (nothing seen yet: 2^-inf = 0)
                l_run[hf] += (w[0] + w[1]) + (w[2] + w[3]);  // a lane's own positions; lanes are summed at the end
                pa[hf] = pt_pack2<CT>(w[0], w[1]);
                pa[2 + hf] = pt_pack2<CT>(w[2], w[3]);
                if (P2) {
                    pr[hf] = pt_rest2<CT>(w[0], w[1], pa[hf]);
                    pr[2 + hf] = pt_rest2<CT>(w[2], w[3], pa[2 + hf]);
                }
            }
            // O += P V
            bool odd = false;
            if (!whole) odd = pt_clean<HD, CT>(const_cast<unsigned char *>(V), p0, d.end, lim_min, lane, wrote);
            if (__builtin_expect(odd, 0)) pt_values<HD, CT, P2, true>(o, pa, pr, V, v_at, lane, p0, d.end, limit);
            else pt_values<HD, CT, P2, false>(o, pa, pr, V, v_at, lane, p0, d.end, limit);
            if (F::UP > 0.f && lifted) {
#pragma unroll
                for (int hf = 0; hf < 2; hf++) {
                    const float down = pt_power(-lift[hf]);
                    l_run[hf] *= down;
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        o[nt][hf * 2] *= down;
                        o[nt][hf * 2 + 1] *= down;
                    }
                }
            }
        }
        const auto release = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);
        };
        if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (!(d.flags & PT_LAST)) {
            release();
            continue;
        }

        // ---------------------------------------------------------------- the piece's end
        const auto finish = [&](auto warps) {
            constexpr int W = decltype(warps)::value;  // of the tile
            const bool part = d.flags & (PT_HEAD_PART | PT_TAIL_PART);
            const size_t cell = ((size_t)blockIdx.x * 2 + (d.flags & PT_TAIL_PART ? 1 : 0)) * a.tiles + mt;
            const float vs = a.v_scale ? a.v_scale[d.head] : 1.f;
            float l[2], m[2] = {m_run[0], m_run[1]}, inv[2];
            long long to[2];
            bool have[2];
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                l[hf] = l_run[hf];
                l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 1);
                l[hf] += __shfl_xor_sync(0xffffffffu, l[hf], 2);
                if (W > 1 && t4 == 0) meet_ml[warp * 16 + (lane >> 2) + hf * 8] = make_float2(m[hf], l[hf]);
                const int v = v0 + (lane >> 2) + hf * 8, r = pt_row_of(a, v), h = d.head * a.G + v - r * a.G;
                have[hf] = v < n_vec;
                to[hf] = (d.row0 + r) * a.out_row_stride + h * a.out_head_stride;
            }
            if (W > 1) {
                // to a common maximum (and everybody has read the stage)
                if (!meet_here()) return false;
                float2 ml[2][W];
#pragma unroll
                for (int hf = 0; hf < 2; hf++)
#pragma unroll
                    for (int g = 0; g < W; g++) ml[hf][g] = meet_ml[(mt + g * (PT_WARPS / W)) * 16 + (lane >> 2) + hf * 8];
#pragma unroll
                for (int hf = 0; hf < 2; hf++) {
                    float top = ml[hf][0].x, sum = 0.f;
#pragma unroll
                    for (int g = 1; g < W; g++) top = fmaxf(top, ml[hf][g].x);
                    const float use = top == -INFINITY ? 0.f : top;
#pragma unroll
                    for (int g = 0; g < W; g++) sum += ml[hf][g].y * exp2f(ml[hf][g].x - use);
                    const float f = exp2f(m[hf] - use);
#pragma unroll
                    for (int nt = 0; nt < NT; nt++) {
                        o[nt][hf * 2] *= f;
                        o[nt][hf * 2 + 1] *= f;
                    }
                    m[hf] = top;
                    l[hf] = sum;
                }
            }
            // the tile's warps add their sums up in the stage that they have just read (and held back)
            const auto sums = [&](int w, int nt) {
                const int i = (w * NT + nt) * 32 + lane;
                return F::MEET && i >= F::STAGE / 16 ? meet + (i - F::STAGE / 16) : reinterpret_cast<float4 *>(ring + st * F::STAGE) + i;
            };
            if (W > 1) {
#pragma unroll
                for (int nt = 0; nt < NT; nt++) *sums(warp, nt) = make_float4(o[nt][0], o[nt][1], o[nt][2], o[nt][3]);
            } else release();
#pragma unroll
            for (int hf = 0; hf < 2; hf++) {
                inv[hf] = l[hf] == 0.f ? 0.f : __fdividef(vs, l[hf]);
                if (t4 == 0 && pg == 0) {
                    if (part) a.part_ml[cell * 16 + (lane >> 2) + hf * 8] = make_float2(m[hf], l[hf]);
                    else if (a.lse && have[hf]) {
                        const int v = v0 + (lane >> 2) + hf * 8, r = pt_row_of(a, v);
                        a.lse[(long long)(d.row0 + r) * a.Hk * a.G + d.head * a.G + v - r * a.G] = l[hf] == 0.f ? -INFINITY : (m[hf] + (log2f(l[hf]) - F::UP)) * LN2;
                    }
                }
            }
            if (W > 1 && !meet_here()) return false;
            // every warp its share of the dimensions, two neighbouring products at a time
#pragma unroll
            for (int j = 0; j < NT / 2 / W; j++) {
                const int nt = (j * W + pg) * 2;
                float4 x[2];
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    if (W == 1) x[k] = make_float4(o[j * 2 + k][0], o[j * 2 + k][1], o[j * 2 + k][2], o[j * 2 + k][3]);
                    else x[k] = *sums(mt, nt + k);
#pragma unroll
                    for (int g = 1; g < W; g++) {
                        const float4 y = *sums(mt + g * (PT_WARPS / W), nt + k);
                        x[k].x += y.x; x[k].y += y.y; x[k].z += y.z; x[k].w += y.w;
                    }
                }
                if (part) {
                    a.part_o[(cell * NT + nt) * 32 + lane] = x[0];
                    a.part_o[(cell * NT + nt + 1) * 32 + lane] = x[1];
                } else {
                    if (have[0]) pt_put<F::ES>(a, to[0], nt, t4, x[0].x * inv[0], x[0].y * inv[0], x[1].x * inv[0], x[1].y * inv[0]);
                    if (have[1]) pt_put<F::ES>(a, to[1], nt, t4, x[0].z * inv[1], x[0].w * inv[1], x[1].z * inv[1], x[1].w * inv[1]);
                }
            }
            if (W > 1) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                release();
            }
            return true;
        };
        if (PG == 4) {
            if (!finish(std::integral_constant<int, 4>{})) break;
        } else if (PG == 2) {
            if (!finish(std::integral_constant<int, 2>{})) break;
        } else finish(std::integral_constant<int, 1>{});
    }
    asm volatile("barrier.sync 1, %0;" ::"n"(PT_THREADS) : "memory");
    if (giving_up[0] == 0) return;

    // -------------------------------------------------------------------- given up
    // Every segment that this share has a part of becomes NaN: here, and through NaN partials in what the join makes of it.  (The
    // records may lack what the share had not come to, so that the join takes partials of other segments along, or is not called for
    // a segment that begins here: either way it writes NaN or nothing.)
    if (tid == 0 && a.status) atomicOr(a.status, SPARSK_PAGED_TIMEOUT);
    if (tid < 2 * a.tiles * 16) a.part_ml[(size_t)blockIdx.x * 2 * a.tiles * 16 + tid] = make_float2(-INFINITY, __int_as_float(0x7fffffff));
    long long total = 0, at = 0;
#pragma unroll 1
    for (int i = 0; i < a.n_seqs; i++) {
        const PtSeq s = pt_seq(a, i);
        total += (long long)pt_segments(a, s.rows) * cost_of(s);
    }
    const long long share = pt_share(total), beg = share * blockIdx.x, end = min(beg + share, total);
#pragma unroll 1
    for (int i = 0; i < a.n_seqs && at < end; i++) {
        const PtSeq s = pt_seq(a, i);
        const int cost = cost_of(s), boxes = boxes_of(s), each = box_cost(s), n_segs = pt_segments(a, s.rows);
#pragma unroll 1
        for (long long g = at < beg ? min(pt_div(beg - at, cost), (long long)n_segs) : 0; g < n_segs && at + g * cost < end; g++) {
            const long long first = at + g * cost;
            const int from = (int)max(beg - first, 0ll), to = (int)min(end - first, (long long)cost);
            const int b0 = min((from + each - 1) / each, boxes), b1 = min((to + each - 1) / each, boxes);
            if (boxes <= a.whole_boxes ? from > 0 : b0 >= b1 && !(boxes == 0 && from == 0)) continue;
            const int qblk = (int)(g / a.Hk), head = (int)(g % a.Hk), v0 = qblk * a.tiles * 16, n = min(s.rows * a.G - v0, a.tiles * 16);
#pragma unroll 1
            for (int k = tid; k < n * HD; k += PT_WARPS * 32) {
                const int v = v0 + k / HD, r = v / a.G, h = head * a.G + v % a.G;
                reinterpret_cast<uint16_t *>(a.out)[(s.row0 + r) * a.out_row_stride + h * a.out_head_stride + k % HD] = 0x7fff;  // (bf16 and fp16)
                if (a.lse && k % HD == 0) a.lse[(long long)(s.row0 + r) * a.Hk * a.G + h] = __int_as_float(0x7fffffff);
            }
        }
        at += (long long)n_segs * cost;
    }
}

// ------------------------------------------------------------------ the join
// Share `blockIdx.x` ends in the middle of a segment: its last partial and the first ones of the shares behind it, up to
// the one in which the segment ends.  blockIdx.y: which tile of 16 vectors, and which of PARTS parts of its accumulators: one where
// segments are many and a segment's partials two or three (blocks that start and end are then what the join costs), four
// where a few segments lie in tens of shares each.
template <int HD, int ES, int PARTS>
static __global__ void __launch_bounds__(PJ_THREADS) paged_join_kernel(const PtArgs a, int shares)
{
    // a block takes a tile's accumulators or a quarter of them: QP pairs of products, GROUPS partials side by side
    constexpr int NT = HD / 8, QP = NT / 2 / PARTS, COLS = QP * 32, GROUPS = PJ_THREADS / COLS, PER = PJ_THREADS / 16;
    constexpr float LN2 = 0.6931471805599453f;
    constexpr int FIRST = 4;  // partials a thread asks for before it knows their weights
    __shared__ float weight[PT_MAX_SHARES][16], red[PER][16], sums[PER][16];
    __shared__ float4 acc[GROUPS > 1 ? GROUPS : 1][COLS][2];
    const int w0 = blockIdx.x, mt = blockIdx.y / PARTS, quarter = blockIdx.y % PARTS, tid = threadIdx.x, lane = tid & 31;
    griddep_wait();
    // the record, and where the segment ends: every warp for itself
    const int4 rec = __ldcg(reinterpret_cast<const int4 *>(&a.records[w0]));
    const int head = __ldcg(&a.records[w0].head);
    int ends[2];
#pragma unroll
    for (int k = 0; k < 2; k++) ends[k] = w0 + 1 + k * 32 + lane < shares ? __ldcg(&a.records[w0 + 1 + k * 32 + lane].flags) & 4 : 0;
    if (!(rec.x & 1)) return;
    const int row0 = rec.y, v0 = (rec.w * a.tiles + mt) * 16, n_vec = rec.z * a.G;
    if (v0 >= n_vec) return;
    int n = 1;
    for (int w = w0 + 1;;) {
        const uint32_t b0 = __ballot_sync(0xffffffffu, ends[0]), b1 = __ballot_sync(0xffffffffu, ends[1]);
        n += b0 ? __ffs(b0) : b1 ? 32 + __ffs(b1) : min(64, shares - w);
        w += 64;
        if (b0 || b1 || w >= shares) break;
#pragma unroll
        for (int k = 0; k < 2; k++) ends[k] = w + k * 32 + lane < shares ? __ldcg(&a.records[w + k * 32 + lane].flags) & 4 : 0;
    }
    const auto cell = [&](int i) { return ((size_t)(w0 + i) * 2 + (i == 0 ? 1 : 0)) * a.tiles + mt; };
    const int col = tid % COLS, grp = tid / COLS, nt = (quarter * QP + col / 32) * 2;
    const auto partial = [&](int i, float4 (&y)[2]) {
#pragma unroll
        for (int k = 0; k < 2; k++) y[k] = __ldcg(&a.part_o[(cell(i) * NT + nt + k) * 32 + lane]);
    };
    float4 early[FIRST][2];
#pragma unroll
    for (int k = 0; k < FIRST; k++)
        if (grp + k * GROUPS < n) partial(grp + k * GROUPS, early[k]);
    // weights of the partials for each vector
    const int v = tid & 15, i0 = tid >> 4;
    float top = -INFINITY, sum = 0.f;  // (of a thread's own partials, the sum relative to their largest)
    for (int i = i0; i < n; i += PER) {
        const float2 ml = __ldcg(&a.part_ml[cell(i) * 16 + v]);
        weight[i][v] = ml.x;
        const float m = fmaxf(top, ml.x), use = m == -INFINITY ? 0.f : m;
        sum = sum * exp2f(top - use) + ml.y * exp2f(ml.x - use);
        top = m;
    }
    const float mine = top;
    red[i0][v] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; i++) top = fmaxf(top, red[i][v]);
    const float use = top == -INFINITY ? 0.f : top;
    for (int i = i0; i < n; i += PER) weight[i][v] = exp2f(weight[i][v] - use);
    sums[i0][v] = sum * exp2f(mine - use);
    __syncthreads();
    float4 x[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    const auto add = [&](int i, const float4 (&y)[2]) {
        const float f0 = weight[i][lane >> 2], f1 = weight[i][(lane >> 2) + 8];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            x[k].x += f0 * y[k].x; x[k].y += f0 * y[k].y; x[k].z += f1 * y[k].z; x[k].w += f1 * y[k].w;
        }
    };
#pragma unroll
    for (int k = 0; k < FIRST; k++)
        if (grp + k * GROUPS < n) add(grp + k * GROUPS, early[k]);
#pragma unroll 4
    for (int i = grp + FIRST * GROUPS; i < n; i += GROUPS) {
        float4 y[2];
        partial(i, y);
        add(i, y);
    }
    acc[grp][col][0] = x[0];
    acc[grp][col][1] = x[1];
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < GROUPS; g++)
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const float4 y = acc[g][col][k];
            x[k].x += y.x; x[k].y += y.y; x[k].z += y.z; x[k].w += y.w;
        }
    const float vs = a.v_scale ? a.v_scale[head] : 1.f;
#pragma unroll
    for (int hf = 0; hf < 2; hf++) {
        const int vec = (lane >> 2) + hf * 8;
        if (v0 + vec >= n_vec) continue;
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < PER; i++) l += sums[i][vec];
        const int r = pt_row_of(a, v0 + vec), h = head * a.G + v0 + vec - r * a.G;
        const float inv = l == 0.f ? 0.f : __fdividef(vs, l);
        const long long to = (row0 + r) * a.out_row_stride + h * a.out_head_stride;
        if (hf == 0) pt_put<ES>(a, to, nt, lane & 3, x[0].x * inv, x[0].y * inv, x[1].x * inv, x[1].y * inv);
        else pt_put<ES>(a, to, nt, lane & 3, x[0].z * inv, x[0].w * inv, x[1].z * inv, x[1].w * inv);
        if (a.lse && nt == 0 && (lane & 3) == 0) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; i++) m = fmaxf(m, red[i][vec]);
            a.lse[(long long)(row0 + r) * a.Hk * a.G + h] = l == 0.f ? -INFINITY : (m + (log2f(l) - a.up)) * LN2;
        }
    }
}

}  // namespace sparsk
