// What the host decides about a call with trees: whether its arguments are in range, dense strides for those left out.  Plain C++, no GPU.
#pragma once

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "specsteer_tree.h"

namespace {

struct Strides3 {
    long a, b, c;
};

// Strides of [n, m, heads, dim] rows; false for those that are negative, off 16 bytes or whose last offset in bytes is no number.  Strides
// of dimensions of one element mean nothing.  Outputs may not overlap themselves: heads, rows and sequences each behind the last.
inline bool tree_strides(const int64_t (&given)[3], long n, long m, long heads, long dim, bool written, Strides3& out) {
    for (int i = 0; i < 3; ++i)
        if (given[i] < 0 || (given[i] & 7)) return false;
    long row = 0, all = 0;
    out.c = given[2] ? given[2] : dim;
    if (__builtin_mul_overflow(heads, out.c, &row)) return false;
    // a head-major array (pages of [heads, slots, dim]) has its slots inside of its heads: only what is dense is derived
    out.b = given[1] ? given[1] : row;
    if (__builtin_mul_overflow(m, out.b > row ? out.b : row, &all)) return false;
    out.a = given[0] ? given[0] : all;
    long end = 0, part = 0;
    const long counts[3] = {n, m, heads}, steps[3] = {out.a, out.b, out.c};
    for (int i = 0; i < 3; ++i) {
        if (counts[i] < 1) return true;
        if (__builtin_mul_overflow(counts[i] - 1, steps[i], &part) || __builtin_add_overflow(end, part, &end)) return false;
    }
    if (__builtin_add_overflow(end, dim, &end) || __builtin_mul_overflow(end, 2L, &end)) return false;
    if (!written) return true;
    // written elements are written once: sorted by stride, each dimension steps over all that is inside of it
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (steps[order[j]] < steps[order[i]]) {
                const int t = order[i];
                order[i] = order[j];
                order[j] = t;
            }
    long inside = dim;
    for (int i = 0; i < 3; ++i) {
        const int d = order[i];
        if (counts[d] == 1) continue;
        if (steps[d] < inside) return false;
        inside += (counts[d] - 1) * steps[d];
    }
    return true;
}

struct TreeShape {
    Strides3 q, k, out, cache;
    long table;
};

inline ss_status tree_shape(const ss_tree_params* p, bool attention, TreeShape& s) {
    if (!p) return SS_ERR_NULL;
    if (p->dtype != SS_BF16 && p->dtype != SS_TREE_F16) return SS_ERR_DTYPE;
    if (p->batch < 0 || p->nodes < 0 || p->nodes > SS_MAX_K || p->kv_heads < 1 || p->kv_heads > SS_TREE_MAX_HEADS) return SS_ERR_SHAPE;
    if (p->pages < 0 || p->page_size < 1 || p->table_width < 0) return SS_ERR_SHAPE;
    if ((long)p->batch * (p->nodes + 1) > SS_TREE_MAX_ROWS) return SS_ERR_SHAPE;
    if ((long)p->table_width * p->page_size > INT32_MAX) return SS_ERR_SHAPE;  // lengths are of 32 bits
    if (attention) {
        if (p->heads < 1 || p->heads > SS_TREE_MAX_HEADS || p->heads % p->kv_heads || (p->head_dim != 64 && p->head_dim != 128)) return SS_ERR_SHAPE;
        if (!std::isfinite(p->scale)) return SS_ERR_PARAM;
    } else if (p->head_dim < 8 || p->head_dim > 1024 || (p->head_dim & 7)) {
        return SS_ERR_SHAPE;
    }
    const long rows = p->nodes + 1;
    if (!tree_strides(p->k_stride, p->batch, rows, p->kv_heads, p->head_dim, false, s.k)) return SS_ERR_STRIDE;
    if (!tree_strides(p->cache_stride, p->pages, p->page_size, p->kv_heads, p->head_dim, !attention, s.cache)) return SS_ERR_STRIDE;
    if (attention && ((p->pages > 1 && s.cache.a >= 1l << 31) || (p->page_size > 1 && s.cache.b >= 1l << 31))) return SS_ERR_STRIDE;
    if (attention && (!tree_strides(p->q_stride, p->batch, rows, p->heads, p->head_dim, false, s.q) ||
                      !tree_strides(p->out_stride, p->batch, rows, p->heads, p->head_dim, true, s.out)))
        return SS_ERR_STRIDE;
    if (p->table_stride < 0) return SS_ERR_STRIDE;
    s.table = p->table_stride ? p->table_stride : p->table_width;
    long end = 0;
    if (p->batch > 1 && (__builtin_mul_overflow((long)(p->batch - 1), s.table, &end) || end > (1L << 60))) return SS_ERR_STRIDE;
    return SS_OK;
}

// Params of the walk: those of the block, greedy or not.
inline ss_status verify_shape(const ss_params* p, long& st, long& sb) {
    if (!p) return SS_ERR_NULL;
    if (p->batch < 0 || p->k_max < 0 || p->k_max > SS_MAX_K || p->vocab < 1 || p->vocab > SS_MAX_VOCAB) return SS_ERR_SHAPE;
    if ((long)p->batch * (p->k_max + 1) > SS_TREE_MAX_ROWS) return SS_ERR_SHAPE;
    if (p->dtype != SS_F32 && p->dtype != SS_BF16) return SS_ERR_DTYPE;
    if (!(p->lambda > 0.f) || !std::isfinite(p->lambda) || !std::isfinite(p->beta) || !(p->temperature > 0.f) || !std::isfinite(p->temperature) ||
        !(1.4426950408889634 / (double)p->temperature < 3e38) || (p->flags & ~SS_FLAG_GREEDY))
        return SS_ERR_PARAM;
    if (p->stride_b < 0 || p->stride_t < 0) return SS_ERR_STRIDE;
    st = p->stride_t ? p->stride_t : p->vocab;
    long span = 0, end = 0;
    if (p->k_max > 0 && st < p->vocab) return SS_ERR_STRIDE;
    if (__builtin_mul_overflow((long)p->k_max, st, &span) || __builtin_add_overflow(span, (long)p->vocab, &span)) return SS_ERR_STRIDE;
    sb = p->stride_b;
    if (!sb && __builtin_mul_overflow((long)p->k_max + 1, st, &sb)) return SS_ERR_STRIDE;
    if (p->batch > 1 && (sb < span || __builtin_mul_overflow((long)(p->batch - 1), sb, &end))) return SS_ERR_STRIDE;
    if (__builtin_add_overflow(end, span, &end) || __builtin_mul_overflow(end, 4L, &end)) return SS_ERR_STRIDE;
    return SS_OK;
}

}  // namespace
