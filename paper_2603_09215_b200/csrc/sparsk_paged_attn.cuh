// Attention of a step's new rows over a paged cache.
#pragma once

#include "sparsk_paged.cuh"

namespace sparsk {

// One warp per (row, query head): a lane holds head_dim / 32 dimensions of the query and of the output, the
// positions come one after another.
template <int HD>
static __global__ void __launch_bounds__(128) paged_attn_simple_kernel(sparsk_paged_attn_args a, float scale)
{
    constexpr int D = HD / 32;
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int row = (int)(w / a.n_q_heads), head = (int)(w % a.n_q_heads), Hk = a.pool.n_kv_heads, hk = head / (a.n_q_heads / Hk);
    if (row >= a.n_rows) return;
    int seq = -1, rows = 1, j = 0;
    if (a.row_start) {
        for (int i = 0; i < a.n_seqs; i++)
            if (row >= a.row_start[i] && row < a.row_start[i + 1]) {
                seq = i;
                rows = a.row_start[i + 1] - a.row_start[i];
                j = row - a.row_start[i];
                break;
            }
    } else seq = row < a.n_seqs ? row : -1;
    if (seq < 0) return;
    const long long room = (long long)a.max_blocks * a.pool.page_size;
    const long long len = min((long long)a.seq_len[seq], room), seen = min(len, (long long)a.seq_len[seq] - rows + 1 + j);
    const auto get = [&](const void *p, int type, long long at) -> float {
        if (type == SPARSK_E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(((const uint8_t *)p)[at], __NV_E4M3)));
        return type == SPARSK_BF16 ? __bfloat162float(((const bf16 *)p)[at]) : __half2float(((const __half *)p)[at]);
    };
    float q[D], o[D], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < D; d++) {
        q[d] = get(a.q, a.q_type, row * a.q_row_stride + head * a.q_head_stride + lane * D + d);
        o[d] = 0.f;
    }
    const float ks = (a.pool.k_scale ? a.pool.k_scale[hk] : 1.f) * scale, vs = a.pool.v_scale ? a.pool.v_scale[hk] : 1.f;
    for (int p = 0; p < seen; p++) {
        const int page = a.block_table[seq * a.table_stride + p / a.pool.page_size];
        if (page < 0 || page >= a.pool.n_pages) continue;
        const long long at = page * a.pool.page_stride + hk * a.pool.head_stride + (p % a.pool.page_size) * a.pool.pos_stride + lane * D;
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < D; d++) s += q[d] * get(a.pool.k, a.pool.type, at + d);
        s = warp_sum(s) * ks;
        const float m2 = fmaxf(m, s);
        const float f = m2 == -INFINITY ? 1.f : expf(m - m2), e = m2 == -INFINITY ? 0.f : expf(s - m2);
        l = l * f + e;
        m = m2;
#pragma unroll
        for (int d = 0; d < D; d++) o[d] = o[d] * f + e * get(a.pool.v, a.pool.type, at + d);
    }
#pragma unroll
    for (int d = 0; d < D; d++) {
        const float x = l > 0.f ? o[d] / l * vs : (l == 0.f ? 0.f : l);
        const long long at = row * a.out_row_stride + head * a.out_head_stride + lane * D + d;
        if (a.q_type == SPARSK_BF16) ((bf16 *)a.out)[at] = __float2bfloat16(x);
        else ((__half *)a.out)[at] = __float2half(x);
    }
    if (a.lse && lane == 0) a.lse[(long long)row * a.n_q_heads + head] = l > 0.f ? m + logf(l) : (l == 0.f ? -INFINITY : l);
}

}  // namespace sparsk
