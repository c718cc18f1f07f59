// Entry points of the paged cache (C ABI in include/sparsk.h): page map, rows into pages.
#include <algorithm>
#include <climits>
#include <cstdint>

#include "../../include/sparsk.h"
#include "sparsk_paged.cuh"
#include "sparsk_paged_host.h"

using namespace sparsk;


// ------------------------------------------------------------------ page map
extern "C" int sparsk_page_map(const sparsk_page_map_args *a, void *cuda_stream)
{
    if (!a || !a->seq_len || !a->seq_rows || !a->block_table || !a->ring || !a->queue || !a->seq_len_out || !a->queue_out ||
        !a->row_start || !a->status)
        return SPARSK_EINVAL;
    if (a->max_rows < 0 || (a->max_rows > 0 && (!a->row_seq || !a->row_pos || !a->slot_map))) return SPARSK_EINVAL;
    if (a->n_seqs < 1 || a->max_blocks < 1 || a->page_size < 1 || a->ring_size < 1) return SPARSK_EINVAL;
    if (a->table_stride < a->max_blocks || a->table_stride > INT_MAX) return SPARSK_EINVAL;
    for (const void *p : {(const void *)a->seq_len, (const void *)a->seq_rows, (const void *)a->block_table, (const void *)a->ring,
                          (const void *)a->queue, (const void *)a->seq_len_out, (const void *)a->queue_out, (const void *)a->row_start,
                          (const void *)a->row_seq, (const void *)a->row_pos, (const void *)a->status})
        if (!aligned(p, 4)) return SPARSK_EINVAL;
    if (!aligned(a->slot_map, 8)) return SPARSK_EINVAL;
    if (a->n_seqs > SPARSK_MAX_MAP_SEQS) return SPARSK_ECAPACITY;
    // blocks read the old lengths and the old queue while another writes the new ones
    const size_t n = (size_t)a->n_seqs * 4;
    for (const void *out : {(const void *)a->seq_len_out, (const void *)a->queue_out}) {
        const size_t m = out == a->queue_out ? 8 : n;
        if (overlap(out, m, a->seq_len, n) || overlap(out, m, a->seq_rows, n) || overlap(out, m, a->queue, 8)) return SPARSK_EINVAL;
    }
    const int smem = 4 * a->n_seqs * (int)sizeof(int);
    static PerDevice<bool> ready;
    if (!ready.here()) {
        if (cudaFuncSetAttribute(page_map_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 4 * SPARSK_MAX_MAP_SEQS * (int)sizeof(int)) != cudaSuccess)
            return SPARSK_ECUDA;
        ready.here() = true;
    }
    PageMapArgs p{*a, -1};
    for (int i = 0; i < 31; i++)
        if (a->page_size == 1 << i) p.shift = i;
    const int grid = std::max(1, std::min(256, (a->max_rows + PM_THREADS - 1) / PM_THREADS));  // a row a thread
    page_map_kernel<<<grid, PM_THREADS, smem, (cudaStream_t)cuda_stream>>>(p);
    return cudaGetLastError() == cudaSuccess ? SPARSK_OK : SPARSK_ECUDA;
}

// ------------------------------------------------------------------ rows into pages
template <int XT>
static void append_launch(const sparsk_paged_append_args &a, int row0, unsigned items, int vec, cudaStream_t st)
{
    const unsigned grid = (items + PA_THREADS - 1) / PA_THREADS;
    if (a.pool.type == SPARSK_FP16) paged_append_kernel<XT, SPARSK_FP16><<<grid, PA_THREADS, 0, st>>>(a, row0, items, vec);
    else if (a.pool.type == SPARSK_BF16) paged_append_kernel<XT, SPARSK_BF16><<<grid, PA_THREADS, 0, st>>>(a, row0, items, vec);
    else paged_append_kernel<XT, SPARSK_E4M3><<<grid, PA_THREADS, 0, st>>>(a, row0, items, vec);
}

extern "C" int sparsk_paged_append(const sparsk_paged_append_args *a, void *cuda_stream)
{
    if (!a || !pool_ok(a->pool) || !a->k || !a->v || !a->slot_map || !aligned(a->slot_map, 8)) return SPARSK_EINVAL;
    if (a->x_type != SPARSK_FP32 && a->x_type != SPARSK_BF16 && a->x_type != SPARSK_FP16) return SPARSK_EINVAL;
    if (a->n_rows < 0 || !strides_ok(a->k_row_stride, a->k_head_stride) || !strides_ok(a->v_row_stride, a->v_head_stride)) return SPARSK_EINVAL;
    const size_t es = type_bytes(a->x_type);
    if (!aligned(a->k, es) || !aligned(a->v, es)) return SPARSK_EINVAL;
    if (a->q) {
        if (!a->q_out || a->n_q_heads < 1 || !strides_ok(a->q_row_stride, a->q_head_stride) || !strides_ok(a->q_out_row_stride, a->q_out_head_stride))
            return SPARSK_EINVAL;
        if ((a->q_out_type != SPARSK_BF16 && a->q_out_type != SPARSK_FP16) || !aligned(a->q, es) || !aligned(a->q_out, 2)) return SPARSK_EINVAL;
    }
    if (a->rope && (!a->row_pos || a->rope_len < 1 || !aligned(a->rope, 4) || !aligned(a->row_pos, 4))) return SPARSK_EINVAL;
    int vec = 0;
    if (wide(a->k, es, a->k_row_stride, a->k_head_stride)) vec |= 1;
    if (wide(a->v, es, a->v_row_stride, a->v_head_stride)) vec |= 2;
    if (a->q && wide(a->q, es, a->q_row_stride, a->q_head_stride)) vec |= 4;
    if (a->q && wide(a->q_out, 2, a->q_out_row_stride, a->q_out_head_stride)) vec |= 8;
    if (aligned(a->rope, 16)) vec |= 16;
    const int64_t per_row = ((a->q ? (int64_t)a->n_q_heads : 0) + 2ll * a->pool.n_kv_heads) * (a->pool.head_dim / 16);
    if (per_row > (1ll << 30)) return SPARSK_EINVAL;
    const int most = (int)std::max<int64_t>(1, (1ll << 30) / per_row);  // rows whose items a launch can number
    for (int row0 = 0; row0 < a->n_rows; row0 += std::min(most, a->n_rows - row0)) {
        const unsigned items = (unsigned)(std::min(most, a->n_rows - row0) * per_row);
        if (a->x_type == SPARSK_FP32) append_launch<SPARSK_FP32>(*a, row0, items, vec, (cudaStream_t)cuda_stream);
        else if (a->x_type == SPARSK_BF16) append_launch<SPARSK_BF16>(*a, row0, items, vec, (cudaStream_t)cuda_stream);
        else append_launch<SPARSK_FP16>(*a, row0, items, vec, (cudaStream_t)cuda_stream);
        if (cudaGetLastError() != cudaSuccess) return SPARSK_ECUDA;
    }
    return SPARSK_OK;
}
