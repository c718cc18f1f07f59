// A token for each row of logits by the row's own temperature, top-k, top-p and min-p.
#pragma once

#include "../../include/sparsk.h"
#include "sparsk_common.cuh"

namespace sparsk {

// A logit as an unsigned number of the same order; 0 for what can never be drawn (minus infinity, NaN).  The
// two zeros are one number.
__device__ __forceinline__ uint32_t st_key(uint32_t bits)
{
    if ((bits << 1) == 0u) return 0x80000000u;
    if ((bits << 1) > 0xff000000u || bits == 0xff800000u) return 0u;
    return (bits & 0x80000000u) ? ~bits : (bits | 0x80000000u);
}
__device__ __forceinline__ uint32_t st_bits(uint32_t key) { return (key & 0x80000000u) ? (key & 0x7fffffffu) : ~key; }
template <int TYPE>
__device__ __forceinline__ uint32_t st_load(const void *p, long long at)
{
    if (TYPE == SPARSK_FP32) return reinterpret_cast<const uint32_t *>(p)[at];
    const uint16_t h = reinterpret_cast<const uint16_t *>(p)[at];
    if (TYPE == SPARSK_BF16) return (uint32_t)h << 16;
    return __float_as_uint(__half2float(__ushort_as_half(h)));
}

constexpr int ST_SIMPLE_THREADS = 1024;

// One block a row; every question ("how many ids, and what mass, lie at or above this key") is a pass over the row.
template <int TYPE>
static __global__ void __launch_bounds__(ST_SIMPLE_THREADS) sample_simple_kernel(sparsk_sample_args a)
{
    __shared__ double wd[32];
    __shared__ int wi[32];
    __shared__ uint32_t wu[32];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int lo = a.id_lo ? max(a.id_lo[row], 0) : 0, hi = a.id_hi ? min(a.id_hi[row], a.n_ids) : a.n_ids;
    const long long base = row * a.row_stride;
    uint32_t top = 0;
    for (int i = lo + tid; i < hi; i += ST_SIMPLE_THREADS) top = max(top, st_key(st_load<TYPE>(a.logits, base + i)));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) wu[warp] = top;
    __syncthreads();
    for (int w = 0; w < 32; w++) top = max(top, wu[w]);
    if (top == 0) {
        if (tid == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    const float temp = a.temperature ? a.temperature[row] : 1.f;
    const bool greedy = !(temp > 0.f);
    const double inv_t = greedy ? 1.0 : 1.0 / (double)temp, z0 = (double)__uint_as_float(st_bits(top));
    const auto weight = [&](uint32_t key) { return key == top ? 1.0 : exp(((double)__uint_as_float(st_bits(key)) - z0) * inv_t); };
    const auto ask = [&](uint32_t t, int &count, double &mass) {
        int c = 0;
        double m = 0;
        for (int i = lo + tid; i < hi; i += ST_SIMPLE_THREADS) {
            const uint32_t k = st_key(st_load<TYPE>(a.logits, base + i));
            if (k != 0 && k >= t) {
                c++;
                m += weight(k);
            }
        }
        for (int o = 16; o > 0; o >>= 1) {
            c += __shfl_xor_sync(0xffffffffu, c, o);
            m += __shfl_xor_sync(0xffffffffu, m, o);
        }
        __syncthreads();
        if (lane == 0) {
            wi[warp] = c;
            wd[warp] = m;
        }
        __syncthreads();
        count = 0;
        mass = 0;
        for (int w = 0; w < 32; w++) {
            count += wi[w];
            mass += wd[w];
        }
    };
    int n_all;
    double total;
    ask(1u, n_all, total);
    // Largest key t such that the ids at or above it reach a count (by_count) or a mass (strictly: go beyond it); how many of
    // the ids at t it takes, and the mass up to them.
    struct Cut {
        uint32_t t;
        int above, take;
        double mass;
    };
    const auto search = [&](bool by_count, bool strict, double target) {
        uint32_t t = 0;
        int c;
        double m;
        for (int bit = 31; bit >= 0; bit--) {
            ask(t | (1u << bit), c, m);
            if (by_count ? c >= target : strict ? m > target : m >= target) t |= 1u << bit;
        }
        if (t == 0) t = 1;
        int c0, c1;
        double m0 = 0, m1;
        if (t == 0xffffffffu) c0 = 0;
        else ask(t + 1, c0, m0);
        ask(t, c1, m1);
        Cut r;
        const double w = weight(t);
        r.t = t;
        r.above = c0;
        const double need = by_count ? target - c0 : (target - m0) / w;
        r.take = (int)fmin(fmax(strict ? floor(need) + 1 : ceil(need), 1.0), (double)(c1 - c0));
        r.mass = m0 + r.take * w;
        return r;
    };
    uint32_t v = top;
    int nth = 0;  // the drawn id is this one, in the order of ids, of those at v
    if (!greedy) {
        int keep = n_all;
        double kept = total;
        const int k = a.top_k ? a.top_k[row] : 0;
        if (k > 0 && k < keep) {
            const Cut c = search(true, false, k);
            keep = k;
            kept = c.mass;
        }
        const float top_p = a.top_p ? a.top_p[row] : 1.f, min_p = a.min_p ? a.min_p[row] : 0.f;
        if (top_p <= 0.f) {
            keep = 1;
            kept = 1;
        } else if (top_p < 1.f) {
            const Cut c = search(false, false, (double)top_p * kept);
            if (c.above + c.take < keep) {
                keep = c.above + c.take;
                kept = c.mass;
            }
        }
        if (min_p > 0.f) {
            uint32_t t = 0;  // the largest key that is too light
            for (int bit = 31; bit >= 0; bit--)
                if ((t | (1u << bit)) < top && weight(t | (1u << bit)) < (double)min_p) t |= 1u << bit;
            int c;
            double m;
            ask(t + 1, c, m);
            if (c < keep) {
                keep = c;
                kept = m;
            }
        }
        const float u = a.uniforms[row];
        const double uu = u > 0.f ? fmin((double)u, 1.0 - 1.0 / 16777216) : 0.0;
        const Cut c = search(false, true, uu * kept);
        v = c.t;
        nth = min(c.take, keep - c.above) - 1;
        nth = max(nth, 0);
    }
    // the nth id at v
    int before = 0;
    for (int i0 = lo; i0 < hi; i0 += ST_SIMPLE_THREADS) {
        const int i = i0 + tid;
        const bool is = i < hi && st_key(st_load<TYPE>(a.logits, base + i)) == v;
        const uint32_t b = __ballot_sync(0xffffffffu, is);
        __syncthreads();
        if (lane == 0) wi[warp] = __popc(b);
        __syncthreads();
        int mine = before + __popc(b & ((1u << lane) - 1u));
        for (int w = 0; w < 32; w++) {
            if (w < warp) mine += wi[w];
            before += wi[w];
        }
        if (is && mine == nth) {
            a.token[row] = i;
            if (a.logprob) a.logprob[row] = (float)((v == top ? 0.0 : ((double)__uint_as_float(st_bits(v)) - z0) * inv_t) - log(total));
        }
    }
}

inline cudaError_t launch_settings_sample(const sparsk_sample_args &a, cudaStream_t st)
{
    if (a.type == SPARSK_FP32) sample_simple_kernel<SPARSK_FP32><<<a.n_rows, ST_SIMPLE_THREADS, 0, st>>>(a);
    else if (a.type == SPARSK_BF16) sample_simple_kernel<SPARSK_BF16><<<a.n_rows, ST_SIMPLE_THREADS, 0, st>>>(a);
    else sample_simple_kernel<SPARSK_FP16><<<a.n_rows, ST_SIMPLE_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace sparsk
