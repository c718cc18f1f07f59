// Host-side checks that the paged entry points share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/sparsk.h"

namespace sparsk {

// [a, a + na) and [b, b + nb) share a byte
inline bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}
inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p % n) == 0; }
inline size_t type_bytes(int type) { return type == SPARSK_FP32 ? 4 : type == SPARSK_E4M3 ? 1 : 2; }

inline bool pool_ok(const sparsk_page_pool &p)
{
    if (!p.k || !p.v || !aligned(p.k, 16) || !aligned(p.v, 16) || !aligned(p.k_scale, 4) || !aligned(p.v_scale, 4)) return false;
    if (p.type != SPARSK_FP16 && p.type != SPARSK_BF16 && p.type != SPARSK_E4M3) return false;
    if (p.head_dim != 64 && p.head_dim != 128) return false;
    if (p.n_pages < 1 || p.n_kv_heads < 1 || p.page_size < 1) return false;
    const int64_t es = (int64_t)type_bytes(p.type);
    for (int64_t s : {p.page_stride, p.head_stride, p.pos_stride})
        if (s < 0 || s > (1ll << 30) || s * es % 16) return false;
    return p.pos_stride >= p.head_dim;
}
// strides of [rows][heads][head_dim] numbers: any, as long as no address can overflow
inline bool strides_ok(int64_t row, int64_t head) { return row >= 0 && head >= 0 && row < (1ll << 30) && head < (1ll << 30); }
inline bool wide(const void *p, size_t es, int64_t row, int64_t head) { return aligned(p, 16) && row * es % 16 == 0 && head * es % 16 == 0; }

}  // namespace sparsk
