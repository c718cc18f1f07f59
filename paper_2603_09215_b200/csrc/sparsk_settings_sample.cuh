// A token for each row of logits by the row's own temperature, top-k, top-p and min-p.
//
// With w = exp((z - max) / T), the ids in the order of falling z (equal z: lower id first): every cut, and the draw, is the
// question up to which id of that order a count or a mass reaches a target, and no sort is needed to answer it.
//   1. Bins of equal width in (max - z) / T, as many as the row's range asks for (40 at most: beyond that even a
//      quarter of a million ids weigh less than 2^-40 of the whole).  A bin adds up how many ids it holds and what they weigh; the sums of
//      bins, in order, say in which bin a target lies.
//   2. The bin's ids (a few hundred at the most, nearly always) are gathered, put in order and added up one by one.  A bin of more ids is
//      divided again, by the bits of its logits, until few are left or all are equal.
// Sums do not depend on the order of the additions: all masses are whole numbers of 2^-44, and within a bin the weights
// are added as whole numbers too.  With x = s (max - z) / T, bin
// b = floor(x) and f = x - b, an id weighs e^(-b/s) (1 - h / s), h = s (1 - e^(-f/s)) < 1, and h is added as a number of 32 bits behind
// the point (s is 51 or more: 2^-38 of the id's weight).  x is worked out in 64 bits, h by four terms of its series
// (the next one is 2^-35 of the id's weight): a draw is decided at the border between two ids, and of a flat row of 150,000 ids each weighs 2^-17, so
// that 24 bits would draw a neighbour once in a hundred times.  The FP64 units run at half the FP32 rate here.
//
// A row is read from memory once, into the shared memory of a cluster of up to eight CTAs.  Counts of a bin and the carries of its
// h are the halves of one word, so an id costs two shared-memory atomics and seven FP64 operations.  Of the 65,000 cycles of a row with top-p
// 7,000 are its loads, 13,000 the bins (some forty instructions an id; without the atomics of h, or without its series, all is 3 % faster);
// the rest are five cluster barriers (about 900 cycles each) and short passes between them, which wait for one another.
// One row of 6,561 ids 14.6 us, of 151,936 (top-p) 28.5, 16 of 151,552 in bf16 with settings of every kind 37.7, 64 of 151,936 60 without and 76 with
// top-p (all of them fp32); 64 rows of both lengths with settings of every kind 73 (82 with min-p's border found by bisection and each
// row's ids above it added up where the bins already say that it cuts nothing).  What was tried: clusters of sixteen 60 for 38 us
// and 34 for 31; 512 threads a CTA 52 for 46; 64 registers a thread and twice the warps 96 for 80; rows read anew from the L2 in each
// pass, without the shared memory for them, in clusters of four: 100,000 cycles a CTA for 60,000, a pass waits for 32 KB in flight an SM.
#pragma once

#include <cooperative_groups.h>

#include "../../include/sparsk.h"
#include "sparsk_common.cuh"

namespace sparsk {

namespace cg = cooperative_groups;

// A logit as an unsigned number of the same order; 0 for what can never be drawn (minus infinity, NaN).
__device__ __forceinline__ uint32_t st_key(uint32_t bits)
{
    if ((bits << 1) > 0xff000000u || bits == 0xff800000u) return 0u;
    return (bits & 0x80000000u) ? ~bits : (bits | 0x80000000u);
}
__device__ __forceinline__ uint32_t st_bits(uint32_t key) { return (key & 0x80000000u) ? (key & 0x7fffffffu) : ~key; }
// The bits of a 16-bit number as those of an fp32 number
template <int TYPE>
__device__ __forceinline__ uint32_t st_widen(uint32_t h)
{
    return TYPE == SPARSK_BF16 ? h << 16 : __float_as_uint(__half2float(__ushort_as_half((unsigned short)h)));
}
template <int TYPE>
__device__ __forceinline__ uint32_t st_load(const void *p, long long at)
{
    if (TYPE == SPARSK_FP32) return reinterpret_cast<const uint32_t *>(p)[at];
    return st_widen<TYPE>(reinterpret_cast<const uint16_t *>(p)[at]);
}
// The number as a double, by its bits (the conversion instruction runs at a quarter of the rate): infinity becomes 2^128,
// zero 2^-127, which is all the same to the weights.
__device__ __forceinline__ double st_double(uint32_t bits)
{
    return __hiloint2double((int)((bits & 0x80000000u) | (((bits & 0x7fffffffu) >> 3) + 0x38000000u)), (int)(bits << 29));
}

constexpr int ST_MAX_WARPS = 16;
constexpr int ST_BINS = 2048;   // the last one holds what lies beyond the range
constexpr int ST_FEW_LOG = 9;
constexpr int ST_FEW = 1 << ST_FEW_LOG;  // ids that are put in order
// Up to so many by comparing each with all, more by counting them into parts, whose barriers take what 130 comparisons a thread take.  64 rows of
// 151,936 fp32 ids with top-p: 84 us by comparing alone, 76 like this (81 from 256 ids on); rows with settings of every kind, mostly few
// ids: 73 like this, 79 by parts alone.
constexpr int ST_COMPARED = 128;
constexpr double ST_RANGE = 40;
constexpr double ST_UNIT = 17592186044416.0;  // 2^44 units of mass are the largest weight (2^18 ids of it fit 64 bits)
constexpr uint32_t ST_DEAD = 0xffffffffu;
constexpr double ST_POINT = 1048576.0;  // 2^20: a double from there on has 32 bits behind the point in its lower word
constexpr uint32_t ST_POINT_HI = 0x41300000u;

enum { ST_BY_COUNT = 0, ST_BY_MASS = 1, ST_BEYOND = 2 };  // the first id at which the count, the mass reaches the target; the mass exceeds it

struct StShared {
    unsigned long long list[2][ST_FEW];  // gathered ids of this CTA, two lists in turn (the cluster reads them)
    int list_n[2];
    uint32_t pub_max[2], pub_min[2];     // this CTA's, for the cluster
    unsigned long long pub_mass[2];
    int pub_count[2];
    // this CTA's own
    unsigned long long all_mass[9];      // sums before each CTA of the cluster
    int all_count[9];
    unsigned long long wsum[ST_MAX_WARPS];
    int wcnt[ST_MAX_WARPS];
    uint32_t wmax[ST_MAX_WARPS], wmin[ST_MAX_WARPS];
    int found, found_cnt, found_n;       // a search's answer: which, ids before it, ids in it
    unsigned long long found_mass;       // mass before it
    int taken;
    unsigned long long taken_mass;
};

template <int C>
struct StCluster {
    __device__ __forceinline__ static int rank() { return C > 1 ? (int)cluster_rank() : 0; }
    __device__ __forceinline__ static void sync()
    {
        if (C > 1) cluster_barrier();
        else __syncthreads();
    }
    template <class T>
    __device__ __forceinline__ static T *of(T *p, int r)
    {
        if (C > 1) return cg::this_cluster().map_shared_rank(p, r);
        return p;
    }
};

template <int TYPE, int C, int T>
static __global__ void __launch_bounds__(T, 512 / T) settings_sample_kernel(sparsk_sample_args a)
{
    typedef StCluster<C> Cl;
    constexpr int WARPS = T / 32, OWN = ST_BINS / C, PER = OWN > T ? OWN / T : 1;  // bins a CTA, a thread adds up
    constexpr int EACH = ST_FEW / T;  // ids to put in order, a thread
    constexpr int GRAIN = TYPE == SPARSK_BF16 ? 16 : TYPE == SPARSK_FP16 ? 13 : 0;  // different keys are 2^GRAIN apart at least
    extern __shared__ __align__(16) unsigned char st_smem[];
    uint32_t *bin_lo = reinterpret_cast<uint32_t *>(st_smem), *bin_hi = bin_lo + ST_BINS;
    // ranked ids and their masses take the bins' place when these have been added up
    unsigned long long *ranked = reinterpret_cast<unsigned long long *>(st_smem);
    unsigned long long *ranked_mass = reinterpret_cast<unsigned long long *>(st_smem + ST_FEW * 8);
    unsigned long long *staged = reinterpret_cast<unsigned long long *>(st_smem + ST_FEW * 16);
    int *part_n = reinterpret_cast<int *>(st_smem + ST_FEW * 24), *part_at = part_n + ST_FEW;
    static_assert(ST_FEW * 32 <= ST_BINS * 8, "all of them in the bins' place");
    unsigned long long *own_mass = reinterpret_cast<unsigned long long *>(st_smem + ST_BINS * 8);  // before each of this CTA's bins
    int *own_count = reinterpret_cast<int *>(own_mass + OWN);
    uint32_t *slice = reinterpret_cast<uint32_t *>(own_count + OWN);
    __shared__ StShared sh;
    const int row = blockIdx.x / C, rank = Cl::rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lo = a.id_lo ? min(max(a.id_lo[row], 0), a.n_ids) : 0, hi = a.id_hi ? min(max(a.id_hi[row], 0), a.n_ids) : a.n_ids;
    const int n = max(hi - lo, 0), per_cta = (n + C - 1) / C, beg = min(rank * per_cta, n), mine = min(per_cta, n - beg),
              mine4 = (mine + 3) & ~3;  // (filled up with ids that nobody draws)

    // (asked for before anything waits)
    const float temp = a.temperature ? a.temperature[row] : 1.f, u = a.uniforms[row];
    const float top_p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f;
    const int row_k = a.top_k ? a.top_k[row] : 0;

    // ---- the row, its largest and smallest logit
    for (int b = tid; b < 2 * ST_BINS; b += T) bin_lo[b] = 0u;
    if (tid == 0) {  // (a search finds its bin in every case; where it did not, this or an earlier answer would stay inside the arrays)
        sh.found = sh.found_cnt = sh.found_n = 0;
        sh.found_mass = 0;
    }
    uint32_t kmax = 0u, kmin = ~0u;
    {
        constexpr int ES = TYPE == SPARSK_FP32 ? 4 : 2, WIDE = 16 / ES;
        const long long at = row * a.row_stride + lo + beg;
        const auto take = [&](int i, uint32_t bits) {
            bits = (bits << 1) == 0u ? 0u : bits;  // the two zeros are one number
            const uint32_t k = st_key(bits);
            slice[i] = k ? bits : ST_DEAD;
            kmax = max(kmax, k);
            kmin = min(kmin, k ? k : ~0u);
        };
        // single ids up to a 16-byte boundary and behind the last one
        const unsigned char *src = reinterpret_cast<const unsigned char *>(a.logits) + at * ES;
        const int ahead = min(mine, (int)((16 - ((uintptr_t)src & 15)) & 15) / ES), wide = (mine - ahead) / WIDE;
        if (tid < ahead) take(tid, st_load<TYPE>(a.logits, at + tid));
        for (int i = ahead + wide * WIDE + tid; i < mine; i += T) take(i, st_load<TYPE>(a.logits, at + i));
        const uint4 *body = reinterpret_cast<const uint4 *>(src + ahead * ES);
        constexpr int BATCH = 6;  // (all asked for at once, the last ones too)
        for (int i0 = tid; i0 < wide; i0 += T * BATCH) {
            uint4 x[BATCH];
#pragma unroll
            for (int q = 0; q < BATCH; q++)
                if (i0 + q * T < wide) x[q] = body[i0 + q * T];
#pragma unroll
            for (int q = 0; q < BATCH; q++) {
                const int i = i0 + q * T;
                if (i >= wide) break;
                const uint32_t w[4] = {x[q].x, x[q].y, x[q].z, x[q].w};
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    if (TYPE == SPARSK_FP32) take(ahead + i * 4 + k, w[k]);
                    else {
                        take(ahead + i * 8 + k * 2, st_widen<TYPE>(w[k] & 0xffffu));
                        take(ahead + i * 8 + k * 2 + 1, st_widen<TYPE>(w[k] >> 16));
                    }
                }
            }
        }
        for (int i = mine + tid; i < mine4; i += T) slice[i] = ST_DEAD;
    }
    int turn = 0;  // of what the cluster reads: written anew two turns later, when everybody has passed the barrier between
    const auto max_min = [&]() {
        kmax = __reduce_max_sync(0xffffffffu, kmax);
        kmin = __reduce_min_sync(0xffffffffu, kmin);
        if (lane == 0) {
            sh.wmax[warp] = kmax;
            sh.wmin[warp] = kmin;
        }
        __syncthreads();
        if (warp == 0) {
            kmax = __reduce_max_sync(0xffffffffu, lane < WARPS ? sh.wmax[lane] : 0u);
            kmin = __reduce_min_sync(0xffffffffu, lane < WARPS ? sh.wmin[lane] : ~0u);
            if (lane == 0) {
                sh.pub_max[turn] = kmax;
                sh.pub_min[turn] = kmin;
            }
        }
        Cl::sync();
        kmax = __reduce_max_sync(0xffffffffu, *Cl::of(&sh.pub_max[turn], lane % C));
        kmin = __reduce_min_sync(0xffffffffu, *Cl::of(&sh.pub_min[turn], lane % C));
        turn ^= 1;
    };
    max_min();
    const uint32_t top = kmax;
    if (top == 0u) {
        if (rank == 0 && tid == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        Cl::sync();  // nobody leaves while its shared memory may be read
        return;
    }
    const bool greedy = !(temp > 0.f);
    const double z0 = st_double(st_bits(top)), inv_t = greedy ? 1.0 : 1.0 / (double)temp;
    const double range = fmin((z0 - st_double(st_bits(kmin))) * inv_t, ST_RANGE);
    const double s = range > 0 ? (ST_BINS - 1.001) / range : 1.0, scale = s * inv_t;
    const double c1 = 0.5 / s, c2 = c1 / (3 * s), c3 = c2 / (4 * s);

    // x of a logit, in ST_POINT's form
    const auto place = [&](uint32_t bits) { return fma(z0 - st_double(bits), scale, ST_POINT); };
    const auto bin_of = [&](double y) { return (int)min((uint32_t)__double2hiint(y) - ST_POINT_HI, (uint32_t)ST_BINS - 1u); };
    const auto h_of = [&](double y) {
        const double f = y - __hiloint2double(__double2hiint(y), 0);
        return (uint32_t)__double2loint(fma(f, fma(-f, fma(-f, fma(-f, c3, c2), c1), 1.0), ST_POINT));
    };
    const auto log_weight = [&](uint32_t key) { return key == top ? 0.0 : (st_double(st_bits(key)) - z0) * inv_t; };
    const auto mass_of = [&](uint32_t key) { return __double2ull_rn(exp(log_weight(key)) * ST_UNIT); };

    // ---- the bins
    // Adds the ids for which `which` names a bin into them: h in one word, ids (upper half) and carries of h (lower half) in the
    // other.  Warps whose ids all fall into one bin add up first; what lies beyond a whole row's range (ids that a program has ruled
    // out by the type's lowest value, say) is only counted, by every thread for itself.
    const auto fill = [&](auto which, bool whole_row) {
        int beyond = 0;
        const auto at = [&](int i) { return i < mine4 ? *reinterpret_cast<const uint4 *>(slice + i) : make_uint4(ST_DEAD, ST_DEAD, ST_DEAD, ST_DEAD); };
        uint4 after = at(tid * 4);
        for (int i0 = warp * 128; i0 < mine4; i0 += T * 4) {
            const uint4 four = after;
            after = at(i0 + lane * 4 + T * 4);  // (ahead of this round's atomics)
            const uint32_t word[4] = {four.x, four.y, four.z, four.w};
            int b[4];
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const double y = place(word[k]);
                b[k] = word[k] == ST_DEAD ? -1 : which(word[k], y);
                h[k] = h_of(y);
                if (whole_row && b[k] == ST_BINS - 1) {
                    beyond++;
                    b[k] = -1;
                }
            }
            const int b0 = __shfl_sync(0xffffffffu, b[0], 0);
            if (b0 >= 0 && __all_sync(0xffffffffu, b[0] == b0 && b[1] == b0 && b[2] == b0 && b[3] == b0)) {
                uint32_t h_lo = 0, h_hi = 0;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    h_lo += h[k] & 0xffffu;
                    h_hi += h[k] >> 16;
                }
                h_lo = __reduce_add_sync(0xffffffffu, h_lo);
                h_hi = __reduce_add_sync(0xffffffffu, h_hi);
                if (lane == 0) {
                    const unsigned long long all = ((unsigned long long)h_hi << 16) + h_lo;
                    const uint32_t part = (uint32_t)all, old = atomicAdd(bin_lo + b0, part);
                    atomicAdd(bin_hi + b0, (128u << 16) + (uint32_t)(all >> 32) + (old + part < old ? 1u : 0u));
                }
            } else {
                uint32_t old[4];
#pragma unroll
                for (int k = 0; k < 4; k++)
                    if (b[k] >= 0) old[k] = atomicAdd(bin_lo + b[k], h[k]);
#pragma unroll
                for (int k = 0; k < 4; k++)
                    if (b[k] >= 0) atomicAdd(bin_hi + b[k], 0x10000u + (old[k] + h[k] < old[k] ? 1u : 0u));
            }
        }
        beyond = __reduce_add_sync(0xffffffffu, beyond);
        if (lane == 0 && beyond) atomicAdd(bin_hi + ST_BINS - 1, (uint32_t)beyond << 16);
    };
    // The largest key below the top for which `holds`, which no larger one may follow; 0 if none does.  Five bits at a time.
    const auto last_key = [&](auto holds) {
        uint32_t at = 0;
        for (int shift = 27;; shift = max(shift - 5, 0)) {
            const uint32_t k = at + ((uint32_t)lane << shift);
            const bool yes = k > at && k < top && holds(k);
            at += (uint32_t)(31 - __clz(__ballot_sync(0xffffffffu, yes) | 1u)) << shift;
            if (shift == 0) return at;
        }
    };
    // The keys of bin `bin`'s logits, the smallest and the largest.  The places rise and fall with the keys, so that they are
    // a stretch; its ends are a rounding or two from where the bin's borders lie, and 32 lanes look at 32 keys there.
    const auto keys_of = [&](int bin, uint32_t &k_lo, uint32_t &k_hi) {
        const auto edge = [&](double x) {  // the smallest key whose place is below x, for a whole number x
            const float z = (float)(z0 - x / scale);
            const auto below = [&](uint32_t k) { return place(st_bits(k)) < ST_POINT + x; };
            const uint32_t k = max(st_key(__float_as_uint(z)), 17u) - 16u;
            const uint32_t b = __ballot_sync(0xffffffffu, below(min(k + lane, top)));
            if (b && !(b & 1u)) return min(k + __ffs(b) - 1, top);
            return last_key([&](uint32_t i) { return !below(i); }) + 1u;  // (numbers around zero are much finer than the places)
        };
        k_lo = bin == ST_BINS - 1 || !(scale > 0) ? 1u : edge(bin + 1);
        k_hi = bin == 0 || !(scale > 0) ? top : edge(bin) - 1u;
    };
    // Calls f(key, place in the slice) for the ids with keys from k_lo to k_hi.
    const auto each_of = [&](uint32_t k_lo, uint32_t k_hi, auto f) {
        const auto key_of = [](uint32_t word) { return word ^ ((uint32_t)((int)word >> 31) | 0x80000000u); };  // (0 for what is never drawn)
        const auto all = [&](auto hit) {
            for (int i = tid * 4; i < mine4; i += T * 16) {
                // sixteen ids at a time, so that their loads do not wait for what f writes
                uint4 four[4];
#pragma unroll
                for (int q = 0; q < 4; q++)
                    four[q] = i + q * T * 4 < mine4 ? *reinterpret_cast<const uint4 *>(slice + i + q * T * 4) : make_uint4(ST_DEAD, ST_DEAD, ST_DEAD, ST_DEAD);
                uint32_t hits = 0;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const uint32_t word[4] = {four[q].x, four[q].y, four[q].z, four[q].w};
#pragma unroll
                    for (int k = 0; k < 4; k++) if (hit(word[k])) hits |= 1u << (q * 4 + k);
                }
                for (; hits; hits &= hits - 1) {
                    const int k = __ffs(hits) - 1, at = i + (k >> 2) * T * 4 + (k & 3);
                    f(key_of(slice[at]), at);
                }
            }
        };
        const uint32_t base = (k_lo & 0x80000000u) ? st_bits(k_lo) : st_bits(k_hi), span = k_hi - k_lo;
        // (numbers of one sign are a stretch of words, too)
        if ((int)(k_lo ^ k_hi) < 0) all([&](uint32_t word) { return key_of(word) - k_lo <= span; });
        else all([&](uint32_t word) { return word - base <= span; });
    };
    // The cluster's bins added up, this CTA's share of them: ids and mass before each; `e` of a bin is what its ids weigh less h / s, `next` of a
    // bin by that of the one before.  What lies beyond a whole row's range weighs nothing.
    const auto add_up = [&](auto e, double next, bool whole_row) {
        Cl::sync();
        double weigh = tid * PER < OWN ? e(rank * OWN + tid * PER) : 0.0;
        int cnt[PER], c_sum = 0;
        unsigned long long mass[PER], m_sum = 0;
#pragma unroll
        for (int k = 0; k < PER; k++) {
            const int own = tid * PER + k, b = rank * OWN + own;
            cnt[k] = 0;
            mass[k] = 0;
            if (own < OWN) {
                unsigned long long h = 0;
#pragma unroll
                for (int r = 0; r < C; r++) {
                    const uint32_t w = *Cl::of(bin_hi + b, r);
                    cnt[k] += (int)(w >> 16);
                    h += ((unsigned long long)(w & 0xffffu) << 32) + *Cl::of(bin_lo + b, r);
                }
                if (cnt[k] && (b < ST_BINS - 1 || !whole_row)) mass[k] = __double2ull_rn(weigh * ST_UNIT * ((double)cnt[k] - (double)h * (1.0 / 4294967296.0) / s));
            }
            c_sum += cnt[k];
            m_sum += mass[k];
            weigh *= next;
        }
        int c_in = c_sum;
        unsigned long long m_in = m_sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int c = __shfl_up_sync(0xffffffffu, c_in, o);
            const unsigned long long m = __shfl_up_sync(0xffffffffu, m_in, o);
            if (lane >= o) {
                c_in += c;
                m_in += m;
            }
        }
        if (lane == 31) {
            sh.wcnt[warp] = c_in;
            sh.wsum[warp] = m_in;
        }
        __syncthreads();
        int c_at = 0, c_all = 0;
        unsigned long long m_at = 0, m_all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; w++) {
            if (w == warp) {
                c_at = c_all;
                m_at = m_all;
            }
            c_all += sh.wcnt[w];
            m_all += sh.wsum[w];
        }
        c_at += c_in - c_sum;
        m_at += m_in - m_sum;
#pragma unroll
        for (int k = 0; k < PER; k++) {
            if (tid * PER + k < OWN) {
                own_count[tid * PER + k] = c_at;
                own_mass[tid * PER + k] = m_at;
            }
            c_at += cnt[k];
            m_at += mass[k];
        }
        if (tid == 0) {
            sh.pub_count[turn] = c_all;
            sh.pub_mass[turn] = m_all;
        }
        Cl::sync();
        if (warp == 0) {
            int c = *Cl::of(&sh.pub_count[turn], lane % C);
            unsigned long long m = *Cl::of(&sh.pub_mass[turn], lane % C);
#pragma unroll
            for (int o = 1; o < C; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, c, o);
                const unsigned long long y = __shfl_up_sync(0xffffffffu, m, o);
                if (lane >= o) {
                    c += x;
                    m += y;
                }
            }
            if (lane < C) {
                sh.all_count[lane + 1] = c;
                sh.all_mass[lane + 1] = m;
            }
            if (lane == 0) {
                sh.all_count[0] = 0;
                sh.all_mass[0] = 0;
            }
        }
        turn ^= 1;
        __syncthreads();
    };
    // One count and one mass of every CTA, added up.
    const auto sum_up = [&](int &c, unsigned long long &m) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            c += __shfl_xor_sync(0xffffffffu, c, o);
            m += __shfl_xor_sync(0xffffffffu, m, o);
        }
        __syncthreads();
        if (lane == 0) {
            sh.wcnt[warp] = c;
            sh.wsum[warp] = m;
        }
        __syncthreads();
        if (warp == 0) {
            c = lane < WARPS ? sh.wcnt[lane] : 0;
            m = lane < WARPS ? sh.wsum[lane] : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                c += __shfl_xor_sync(0xffffffffu, c, o);
                m += __shfl_xor_sync(0xffffffffu, m, o);
            }
            if (lane == 0) {
                sh.pub_count[turn] = c;
                sh.pub_mass[turn] = m;
            }
        }
        Cl::sync();
        c = lane < C ? *Cl::of(&sh.pub_count[turn], lane % C) : 0;
        m = lane < C ? *Cl::of(&sh.pub_mass[turn], lane % C) : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            c += __shfl_xor_sync(0xffffffffu, c, o);
            m += __shfl_xor_sync(0xffffffffu, m, o);
        }
        turn ^= 1;
    };
    // The bin in which the target lies (`found`), ids and mass before it, ids in it.  Every CTA finds out for itself.
    const auto meets = [](int by, double target, int count, unsigned long long mass) {
        return by == ST_BY_COUNT ? count >= target : by == ST_BY_MASS ? (double)mass >= target : (double)mass > target;
    };
    const auto locate = [&](int by, double target) {
        const int l = lane % C;
        const uint32_t met = __ballot_sync(0xffffffffu, meets(by, target, sh.all_count[l + 1], sh.all_mass[l + 1])) & ((1u << C) - 1u),
                       any = __ballot_sync(0xffffffffu, sh.all_count[l + 1] > sh.all_count[l]) & ((1u << C) - 1u);
        const bool none = met == 0u;  // (no bin's end meets it, for a rounding's sake: it is the last id's bin)
        const int r = none ? 31 - __clz(any | 1u) : __ffs(met) - 1;
        const unsigned long long *masses = Cl::of(own_mass, r), m_here = sh.all_mass[r], m_all = sh.all_mass[r + 1];
        const int *counts = Cl::of(own_count, r), c_here = sh.all_count[r], c_all = sh.all_count[r + 1];
        for (int b = tid; b < OWN; b += T) {
            const int c0 = c_here + counts[b], c1 = b + 1 < OWN ? c_here + counts[b + 1] : c_all;
            const unsigned long long m0 = m_here + masses[b], m1 = b + 1 < OWN ? m_here + masses[b + 1] : m_all;
            if (none ? c1 > c0 && c1 == c_all : meets(by, target, c1, m1) && !meets(by, target, c0, m0)) {
                sh.found = r * OWN + b;
                sh.found_cnt = c0;
                sh.found_mass = m0;
                sh.found_n = c1 - c0;
            }
        }
        __syncthreads();
    };
    fill([&](uint32_t, double y) { return bin_of(y); }, true);
    add_up([&](int b) { return exp(-(double)b / s); }, PER > 1 ? exp(-1.0 / s) : 1.0, true);
    const unsigned long long total = sh.all_mass[C];
    const auto logprob = [&](uint32_t key) { return (float)(log_weight(key) - log((double)total / ST_UNIT)); };
    const int n_live = sh.all_count[C];

    // ---- cuts and the draw
    int keep = n_live, gathered = -1, gathered_n = 0, g_cnt = 0;
    unsigned long long kept = total, g_mass = 0;
    bool divided = false;  // the bins are those of a bin that has been divided
    const int want_k = greedy ? 1 : row_k;
    const auto clear_bins = [&]() {
        __syncthreads();
        for (int b = tid; b < 2 * ST_BINS; b += T) bin_lo[b] = 0u;
        __syncthreads();
    };
    for (int step = 0; step < 4; step++) {
        int by;
        double target;
        if (step == 0) {
            if (want_k <= 0 || want_k >= keep) continue;
            by = ST_BY_COUNT;
            target = want_k;
        } else if (step == 1) {
            if (greedy || !(top_p < 1.f)) continue;
            by = ST_BY_MASS;
            target = (double)top_p * (double)kept;
            if (!(top_p > 0.f)) {
                by = ST_BY_COUNT;
                target = 1;
            }
        } else if (step == 2) {
            if (greedy || !(min_p > 0.f)) continue;
            if (min_p > 1.f) {
                keep = 1;
                continue;
            }
            // The largest logit that is too light: a rounding or two from where the logarithm says, where 32 lanes look at 32 keys
            const auto heavy = [&](uint32_t k) { return !(exp(log_weight(k)) < (double)min_p); };
            const uint32_t k0 = max(st_key(__float_as_uint((float)(z0 + log((double)min_p) / inv_t))), 17u) - 16u;
            const uint32_t heavies = __ballot_sync(0xffffffffu, heavy(min(k0 + lane, top)));
            const uint32_t light = heavies && !(heavies & 1u) ? min(k0 + __ffs(heavies) - 1, top) - 1u : last_key([&](uint32_t k) { return !heavy(k); });
            // (nothing to cut where the bins before its own hold all that is left)
            const int lb = bin_of(place(st_bits(light)));
            if (!divided && light && sh.all_count[lb / OWN] + *Cl::of(own_count + lb % OWN, lb / OWN) >= keep) continue;
            // ids and mass above it, added up in a fixed order
            int c = 0;
            unsigned long long m = 0;
            each_of(light + 1u, top, [&](uint32_t k, int) {
                c++;
                m += mass_of(k);
            });
            sum_up(c, m);
            if (c < keep) {
                keep = c;
                kept = m;
            }
            continue;
        } else {
            by = ST_BEYOND;
            target = (u > 0.f ? fmin((double)u, 1.0 - 1.0 / 16777216) : 0.0) * (double)kept;
            if (keep == 1) {
                by = ST_BY_COUNT;
                target = 1;
            }
        }
        if (divided) {  // back to the bins of the whole row
            clear_bins();
            fill([&](uint32_t, double y) { return bin_of(y); }, true);
            add_up([&](int b) { return exp(-(double)b / s); }, PER > 1 ? exp(-1.0 / s) : 1.0, true);
            divided = false;
            gathered = -1;
        }
        locate(by, target);
        if (step == 3 && sh.found_cnt >= keep) {  // a rounding beyond the kept ids: the last of them
            __syncthreads();
            by = ST_BY_COUNT;
            target = keep;
            locate(by, target);
        }
        const int bin = sh.found;
        int before = sh.found_cnt, in = sh.found_n;
        unsigned long long mass_before = sh.found_mass;
        uint32_t k_lo, k_hi;  // the ids in question are those with keys from here to there
        keys_of(bin, k_lo, k_hi);
        __syncthreads();
        if (!(bin == gathered && !divided)) {
            while (in > ST_FEW && k_lo != k_hi) {
                // too many to rank: divided by the bits of their logits
                gathered = -1;
                if (!divided) {
                    kmax = 0u;
                    kmin = ~0u;
                    each_of(k_lo, k_hi, [&](uint32_t k, int) {
                        kmax = max(kmax, k);
                        kmin = min(kmin, k);
                    });
                    __syncthreads();
                    max_min();
                    k_lo = kmin;
                    k_hi = kmax;
                    if (k_lo == k_hi) break;
                }
                divided = true;
                const int shift = max(0, 32 - __clz(k_hi - k_lo) - 11);  // 2,048 bins cover k_hi - k_lo < 2^(shift + 11)
                clear_bins();
                const double e_bin = bin == ST_BINS - 1 ? 0.0 : exp(-(double)bin / s);
                fill([&](uint32_t bits, double) { return st_key(bits) - k_lo <= k_hi - k_lo ? (int)((k_hi - st_key(bits)) >> shift) : -1; }, false);
                add_up([&](int) { return e_bin; }, 1.0, false);
                const int b_all = before;
                const unsigned long long m_all = mass_before;
                locate(by, target - (by == ST_BY_COUNT ? (double)b_all : (double)m_all));
                before = b_all + sh.found_cnt;
                mass_before = m_all + sh.found_mass;
                in = sh.found_n;
                k_hi = k_hi - ((uint32_t)sh.found << shift);
                k_lo = max(k_lo, k_hi - ((1u << shift) - 1u));
                __syncthreads();
            }
            if (in <= ST_FEW) {
                // gathered, put in order, and added up
                if (tid == 0) sh.list_n[turn] = 0;
                for (int b = tid; b < ST_FEW; b += T) part_n[b] = 0;
                __syncthreads();
                each_of(k_lo, k_hi, [&](uint32_t k, int i) {
                    const int at = atomicAdd(&sh.list_n[turn], 1);
                    if (at < ST_FEW) sh.list[turn][at] = ((unsigned long long)(~k) << 32) | (uint32_t)(beg + i);
                });
                Cl::sync();
                const int from = min(*Cl::of(&sh.list_n[turn], lane % C), ST_FEW);
                int have = 0;
                unsigned long long me[EACH];
#pragma unroll
                for (int q = 0; q < EACH; q++) me[q] = ~0ull;
#pragma unroll
                for (int r = 0; r < C; r++) {
                    const int m = __shfl_sync(0xffffffffu, from, r);
#pragma unroll
                    for (int q = 0; q < EACH; q++) {
                        const int at = tid + q * T - have;
                        if (at >= 0 && at < m) me[q] = *Cl::of(&sh.list[turn][at], r);
                    }
                    have += m;
                }
                turn ^= 1;
                have = min(have, ST_FEW);
                if (have <= ST_COMPARED) {
                    // each compared with all
#pragma unroll
                    for (int q = 0; q < EACH; q++) ranked[tid + q * T] = me[q];
                    __syncthreads();
                    int place_of = 0;
                    if (warp * 32 < have) {
#pragma unroll 8
                        for (int j = 0; j < have; j++) place_of += ranked[j] < me[0] ? 1 : 0;
                    }
                    __syncthreads();
                    if (tid < have) ranked[place_of] = me[0];
                    __syncthreads();
                } else {
                    // ST_FEW parts of the keys' stretch (a part a key, or several parts by ids where it has few keys, as with
                    // logits of 16 bits), counted, and each put in order by itself
                    const uint32_t span = k_hi - k_lo, values = (span >> GRAIN) + 1u;
                    const int per_value = values <= ST_FEW ? ST_FEW / (int)values : 0, shift = max(0, 32 - __clz(span) - ST_FEW_LOG);
                    const float by_id = (float)per_value / (float)n;
                    const auto part_of = [&](unsigned long long it) {
                        const uint32_t off = k_hi - ~(uint32_t)(it >> 32);
                        if (per_value) return (int)(off >> GRAIN) * per_value + min((int)((float)(uint32_t)it * by_id), per_value - 1);
                        return (int)(off >> shift);
                    };
                    int part[EACH], at_part[EACH];
#pragma unroll
                    for (int q = 0; q < EACH; q++)
                        if (tid + q * T < have) {
                            part[q] = part_of(me[q]);
                            at_part[q] = atomicAdd(part_n + part[q], 1);
                        }
                    __syncthreads();
                    int p_n[EACH], p_all = 0;
#pragma unroll
                    for (int q = 0; q < EACH; q++) p_all += p_n[q] = part_n[tid * EACH + q];
                    int p_at = p_all;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xffffffffu, p_at, o);
                        if (lane >= o) p_at += x;
                    }
                    if (lane == 31) sh.wcnt[warp] = p_at;
                    __syncthreads();
                    p_at -= p_all;
                    for (int w = 0; w < warp; w++) p_at += sh.wcnt[w];
#pragma unroll
                    for (int q = 0; q < EACH; q++) {
                        part_at[tid * EACH + q] = p_at;
                        p_at += p_n[q];
                    }
                    __syncthreads();
#pragma unroll
                    for (int q = 0; q < EACH; q++)
                        if (tid + q * T < have) staged[part_at[part[q]] + at_part[q]] = me[q];
                    __syncthreads();
#pragma unroll
                    for (int q = 0; q < EACH; q++)
                        if (tid + q * T < have) {
                            const int first = part_at[part[q]], end = first + part_n[part[q]];
                            int place_of = first;
                            for (int j = first; j < end; j++) place_of += staged[j] < me[q] ? 1 : 0;
                            ranked[place_of] = me[q];
                        }
                    __syncthreads();
                }
                unsigned long long m[EACH], all = 0;
#pragma unroll
                for (int q = 0; q < EACH; q++) {
                    const int at = tid * EACH + q;
                    all += at < have ? mass_of(~(uint32_t)(ranked[at] >> 32)) : 0;
                    m[q] = all;
                }
                unsigned long long in_warp = all;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const unsigned long long x = __shfl_up_sync(0xffffffffu, in_warp, o);
                    if (lane >= o) in_warp += x;
                }
                if (lane == 31) sh.wsum[warp] = in_warp;
                __syncthreads();
                unsigned long long off = in_warp - all;
                for (int w = 0; w < warp; w++) off += sh.wsum[w];
#pragma unroll
                for (int q = 0; q < EACH; q++) ranked_mass[tid * EACH + q] = off + m[q];
                gathered = bin;
                gathered_n = have;
                g_cnt = before;
                g_mass = mass_before;
                __syncthreads();
            }
        }
        if (gathered == bin) {
            before = g_cnt;
            mass_before = g_mass;
            // the first of them that meets the target
            if (tid == 0) {
                sh.taken = gathered_n;
                sh.taken_mass = gathered_n ? ranked_mass[gathered_n - 1] : 0;
            }
            __syncthreads();
            for (int j = tid; j < gathered_n; j += T)
                if (meets(by, target, before + j + 1, mass_before + ranked_mass[j]) &&
                    (j == 0 || !meets(by, target, before + j, mass_before + ranked_mass[j - 1]))) {
                    sh.taken = j + 1;
                    sh.taken_mass = ranked_mass[j];
                }
            __syncthreads();
            int taken = sh.taken;
            if (step < 3) {
                if (before + taken < keep) {
                    keep = before + taken;
                    kept = mass_before + sh.taken_mass;
                }
            } else if (rank == 0 && tid == 0) {
                taken = max(1, min(min(taken, keep - before), gathered_n));
                const unsigned long long it = ranked[taken - 1];
                const uint32_t key = ~(uint32_t)(it >> 32);
                a.token[row] = lo + (int)(uint32_t)it;
                if (a.logprob) a.logprob[row] = logprob(key);
            }
            __syncthreads();
        } else {
            // all of them are equal: so many of the same weight
            const unsigned long long w = mass_of(k_lo);
            const double need = by == ST_BY_COUNT ? target - before : w ? (target - (double)mass_before) / (double)w : (double)in;
            int taken = (int)fmin(fmax(need, 0.0), (double)in);
            while (taken > 0 && meets(by, target, before + taken, mass_before + taken * w)) taken--;
            while (taken < in && !meets(by, target, before + taken, mass_before + taken * w)) taken++;
            if (step < 3) {
                if (before + taken < keep) {
                    keep = before + taken;
                    kept = mass_before + taken * w;
                }
                continue;
            }
            taken = max(1, min(taken, keep - before));
            // the id of the one numbered `taken`: a thread's ids side by side, threads and CTAs in order
            const int chunk = (mine + T - 1) / T, i0 = min(tid * chunk, mine), i1 = min(i0 + chunk, mine);
            const uint32_t bits = st_bits(k_lo);
            int c = 0;
            for (int i = i0; i < i1; i++) c += slice[i] == bits ? 1 : 0;
            int in_warp = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, in_warp, o);
                if (lane >= o) in_warp += x;
            }
            if (lane == 31) sh.wcnt[warp] = in_warp;
            __syncthreads();
            int at = in_warp - c, all = 0;
            for (int x = 0; x < WARPS; x++) {
                if (x < warp) at += sh.wcnt[x];
                all += sh.wcnt[x];
            }
            if (tid == 0) sh.pub_count[turn] = all;
            Cl::sync();
            at += __reduce_add_sync(0xffffffffu, lane < rank ? *Cl::of(&sh.pub_count[turn], lane % C) : 0);
            turn ^= 1;
            for (int i = i0; i < i1; i++)
                if (slice[i] == bits && ++at == taken) {
                    a.token[row] = lo + beg + i;
                    if (a.logprob) a.logprob[row] = logprob(k_lo);
                }
        }
    }
    Cl::sync();  // nobody leaves while its shared memory may be read
}

template <int TYPE, int C, int T>
static cudaError_t launch_settings_form(const sparsk_sample_args &a, cudaStream_t st)
{
    static PerDevice<bool> ready_dev;
    const auto bytes = [](int ids) { return ST_BINS * 8 + ST_BINS / C * 12 + ((ids + C - 1) / C + 3) / 4 * 16; };
    bool &ready = ready_dev.here();
    if (!ready) {
        const cudaError_t e = cudaFuncSetAttribute(settings_sample_kernel<TYPE, C, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes(C * 32768));
        if (e != cudaSuccess) return e;
        ready = true;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.n_rows * C);
    cfg.blockDim = dim3(T);
    cfg.dynamicSmemBytes = bytes(a.n_ids);
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = C;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, settings_sample_kernel<TYPE, C, T>, a);
}
// CTAs of a row, by its ids: what is fastest for few rows.  us with top-p in one / four / eight CTAs, fp32:
//              8,192               12,288              32,768              65,536              131,072 ids
//   1 row      14.9  16.2  16.1    17.3  16.8  16.8    25.4  18.4  18.0       -  22.7  21.1       -  29.1  25.9
//   64 rows    15.4  32.6  37.8    17.6  33.4  38.5    26.2  37.7  42.8       -  45.4  50.2       -  60.2  65.4
// (Many rows would take fewer CTAs each up to 32,768 ids; the choice does not look at the rows.)
inline int settings_ctas(int n_ids) { return n_ids <= 8192 ? 1 : n_ids <= 32768 ? 4 : 8; }
template <int TYPE>
static cudaError_t launch_settings_type(const sparsk_sample_args &a, cudaStream_t st)
{
    static_assert(SPARSK_MAX_SAMPLE_IDS <= 8 * 32768, "a CTA counts up to 65,535 ids a bin and holds 32,768");
    const int ctas = settings_ctas(a.n_ids);
    if (ctas == 1) return launch_settings_form<TYPE, 1, 512>(a, st);
    if (ctas == 4) return launch_settings_form<TYPE, 4, 512>(a, st);
    return launch_settings_form<TYPE, 8, 256>(a, st);
}
inline cudaError_t launch_settings_sample(const sparsk_sample_args &a, cudaStream_t st)
{
    if (a.type == SPARSK_FP32) return launch_settings_type<SPARSK_FP32>(a, st);
    if (a.type == SPARSK_BF16) return launch_settings_type<SPARSK_BF16>(a, st);
    return launch_settings_type<SPARSK_FP16>(a, st);
}

}  // namespace sparsk
