// Entry point of attention over a paged cache (C ABI in include/sparsk.h).
#include <algorithm>
#include <climits>
#include <cstdint>

#include "../../include/sparsk.h"
#include "sparsk_paged_attn.cuh"
#include "sparsk_paged_host.h"

using namespace sparsk;

namespace {
int sm_count()
{
    static PerDevice<int> sms;
    int &n = sms.here();
    if (n == 0) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 0;
    }
    return n;
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                             const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn()
{
    static EncodeFn fn = nullptr;
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult qr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qr) == cudaSuccess && qr == cudaDriverEntryPointSuccess)
            fn = (EncodeFn)p;
    }
    return fn;
}

// A pool as [pages][heads][parts of 128 bytes][positions][numbers], boxes of 16 positions of one head.
bool encode_pool(CUtensorMap *m, const void *base, const sparsk_page_pool &p)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t es = type_bytes(p.type), inner = std::min<cuuint64_t>(p.head_dim, 128 / es), parts = p.head_dim / inner;
    const cuuint64_t dims[5] = {inner, (cuuint64_t)p.page_size, parts, (cuuint64_t)p.n_kv_heads, (cuuint64_t)p.n_pages};
    // (the stride of a dimension of one element says nothing and may be anything)
    const cuuint64_t pos = (cuuint64_t)p.pos_stride * es;
    const cuuint64_t strides[4] = {pos, inner * es, p.n_kv_heads > 1 ? (cuuint64_t)p.head_stride * es : pos,
                                   p.n_pages > 1 ? (cuuint64_t)p.page_stride * es : pos};
    const cuuint32_t box[5] = {(cuuint32_t)inner, PT_BOX, (cuuint32_t)parts, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
    const CUtensorMapDataType type = p.type == SPARSK_E4M3   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                     : p.type == SPARSK_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                             : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(m, type, 5, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
              inner * es == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

bool paged_attn_ok(const sparsk_paged_attn_args *a)
{
    if (!a || !pool_ok(a->pool) || a->pool.page_size % 16) return false;
    if (a->q_type != SPARSK_BF16 && !(a->q_type == SPARSK_FP16 && a->pool.type != SPARSK_BF16)) return false;
    if (a->n_rows < 0 || a->n_seqs < 1 || a->max_blocks < 1 || a->n_q_heads < 1 || a->n_q_heads % a->pool.n_kv_heads) return false;
    if (a->max_rows < 0 || a->max_len < 0 || a->inject_short_copy < 0 || (!a->row_start && a->n_rows != a->n_seqs)) return false;
    if (!(a->scale >= 0.f) || !(a->scale < INFINITY)) return false;
    if (a->table_stride < a->max_blocks || a->table_stride > INT_MAX) return false;
    if ((int64_t)a->max_blocks * a->pool.page_size > INT_MAX - 64 || (int64_t)a->n_rows * a->n_q_heads > INT_MAX / 2) return false;
    return strides_ok(a->q_row_stride, a->q_head_stride) && strides_ok(a->out_row_stride, a->out_head_stride);
}

// Tiles of 16 query vectors that a segment may have, for one read of a head's keys and values: as many as the most rows of a
// sequence fill, four at most.
int tiles_of(const sparsk_paged_attn_args *a)
{
    const int64_t rows = !a->row_start ? 1 : a->max_rows > 0 ? a->max_rows : ((int64_t)a->n_rows + a->n_seqs - 1) / a->n_seqs;
    const int64_t vectors = rows * (a->n_q_heads / a->pool.n_kv_heads);
    return vectors <= 16 ? 1 : vectors <= 32 ? 2 : 4;
}

struct Scratch {
    size_t ml, o, bytes;
};
Scratch scratch_of(const sparsk_paged_attn_args *a)
{
    const size_t cells = (size_t)PT_MAX_SHARES * 2 * tiles_of(a);
    Scratch s;
    s.ml = up256(PT_MAX_SHARES * sizeof(PtRecord));
    s.o = s.ml + up256(cells * 16 * sizeof(float2));
    s.bytes = s.o + cells * (a->pool.head_dim / 8) * 32 * sizeof(float4);
    return s;
}

template <int HD, int CT, bool P2>
cudaError_t launch(const PtArgs &p, const CUtensorMap &mk, const CUtensorMap &mv, int shares, int join, cudaStream_t st)
{
    static PerDevice<bool> ready;
    constexpr int smem = PtForm<HD, CT>::SMEM;
    if (!ready.here()) {
        const cudaError_t e = cudaFuncSetAttribute(paged_attn_kernel<HD, CT, P2>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        ready.here() = true;
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(shares);
    cfg.blockDim = dim3(PT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, paged_attn_kernel<HD, CT, P2>, p, mk, mv);
    if (e != cudaSuccess || !join) return e;
    cfg.gridDim = dim3(shares, join * p.tiles);
    cfg.blockDim = dim3(PJ_THREADS);
    cfg.dynamicSmemBytes = 0;
    constexpr int ES = PtForm<HD, CT>::ES;
    return join == 1 ? cudaLaunchKernelEx(&cfg, paged_join_kernel<HD, ES, 1>, p, shares) : cudaLaunchKernelEx(&cfg, paged_join_kernel<HD, ES, 4>, p, shares);
}
// A softmax weight is rounded to 16 bits where it meets the values; where that is no finer than the output's own
// rounding, a second term carries the rest.
template <int HD, class... A>
cudaError_t launch_types(int pool_type, int q_type, A... x)
{
    if (pool_type == SPARSK_BF16) return launch<HD, SPARSK_BF16, true>(x...);
    if (pool_type == SPARSK_FP16) return q_type == SPARSK_FP16 ? launch<HD, SPARSK_FP16, true>(x...) : launch<HD, SPARSK_FP16, false>(x...);
    return q_type == SPARSK_FP16 ? launch<HD, SPARSK_E4M3, true>(x...) : launch<HD, SPARSK_E4M3, false>(x...);
}
}  // namespace

extern "C" size_t sparsk_paged_attention_scratch_bytes(const sparsk_paged_attn_args *a)
{
    return paged_attn_ok(a) ? scratch_of(a).bytes : 0;
}

extern "C" int sparsk_paged_attention(const sparsk_paged_attn_args *a, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    if (!paged_attn_ok(a) || !a->q || !a->out || !a->block_table || !a->seq_len || !scratch || !aligned(scratch, 256)) return SPARSK_EINVAL;
    if (!aligned(a->q, 2) || !aligned(a->out, 2) || !aligned(a->lse, 4) || !aligned(a->block_table, 4) || !aligned(a->seq_len, 4) ||
        !aligned(a->row_start, 4) || !aligned(a->status, 4))
        return SPARSK_EINVAL;
    const Scratch sc = scratch_of(a);
    if (scratch_bytes < sc.bytes) return SPARSK_EINVAL;
    if (a->n_rows == 0) return SPARSK_OK;
    const int n_sm = sm_count();
    if (n_sm == 0) return SPARSK_ECUDA;
    CUtensorMap mk, mv;
    if (!encode_pool(&mk, a->pool.k, a->pool) || !encode_pool(&mv, a->pool.v, a->pool)) return SPARSK_EINVAL;
    PtArgs p{};
    p.q = a->q; p.out = a->out; p.lse = a->lse;
    p.block_table = a->block_table; p.seq_len = a->seq_len; p.row_start = a->row_start;
    p.k_scale = a->pool.k_scale; p.v_scale = a->pool.v_scale;
    p.records = (PtRecord *)scratch;
    p.status = a->status; p.short_copy = a->inject_short_copy;
    p.part_ml = (float2 *)((char *)scratch + sc.ml);
    p.part_o = (float4 *)((char *)scratch + sc.o);
    p.table_stride = a->table_stride;
    p.q_row_stride = a->q_row_stride; p.q_head_stride = a->q_head_stride;
    p.out_row_stride = a->out_row_stride; p.out_head_stride = a->out_head_stride;
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)a->pool.head_dim)) * 1.4426950408889634f;
    p.up = a->pool.type == SPARSK_BF16 ? 0.f : PT_UP;
    p.q_type = a->q_type; p.n_rows = a->n_rows; p.n_seqs = a->n_seqs; p.max_blocks = a->max_blocks;
    p.page_size = a->pool.page_size; p.n_pages = a->pool.n_pages;
    p.Hk = a->pool.n_kv_heads; p.G = a->n_q_heads / a->pool.n_kv_heads;
    p.tiles = tiles_of(a);
    p.g_inverse = (uint32_t)(((1ull << 32) + p.G - 1) / p.G);
    p.g_limit = p.G == 1 ? 0 : (uint32_t)((1ull << 32) / p.G);  // (by 1 the plain division does)
    p.whole_boxes = PT_WHOLE;
    p.page_shift = -1;
    for (int i = 0; i < 28; i++)
        if (p.page_size == PT_BOX << i) p.page_shift = i;
    p.q_wide = wide(a->q, 2, a->q_row_stride, a->q_head_stride);
    p.out_words = aligned(a->out, 4) && a->out_row_stride % 2 == 0 && a->out_head_stride % 2 == 0;
    int shares = std::min(PT_CTAS * n_sm, PT_MAX_SHARES);
    const int64_t segs = ((int64_t)a->n_rows * p.G / (16 * p.tiles) + a->n_seqs) * p.Hk;  // no more than so many
    // parts of a tile that the join deals out (0: no join); one of 8,191 positions 14.5 us in four, 64 ragged sequences 35.7 in one
    // and 37.2 in four
    int join = segs * 8 <= shares ? 4 : 1;
    if (a->max_len > 0) {
        // no more CTAs than there can be shares, and no join where no segment is long enough to be cut (if one is all
        // the same, its share takes the whole of it)
        const int64_t boxes = ((int64_t)a->max_len + PT_BOX - 1) / PT_BOX;
        shares = (int)std::max<int64_t>(1, std::min<int64_t>(shares, segs * (boxes * PtForm<64, SPARSK_FP16>::PT_C4 + PT_END_COST) / PT_MIN_SHARE + 1));
        if (boxes <= PT_WHOLE) {
            p.whole_boxes = INT_MAX;
            join = 0;
        }
    }
    const cudaError_t e = a->pool.head_dim == 64 ? launch_types<64>(a->pool.type, a->q_type, p, mk, mv, shares, join, (cudaStream_t)cuda_stream)
                                                 : launch_types<128>(a->pool.type, a->q_type, p, mk, mv, shares, join, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? SPARSK_OK : SPARSK_ECUDA;
}
