// Attention of a tree's rows over a paged cache and their ancestors, for MI355X (gfx950); include/specsteer_tree.h says what it computes.
//
// A wave a row and query head: it goes over the keys with a running maximum m and sum l of the weights 2^(s - m), s = scale log2(e) q.k, and
// holds the weighted sum of the values, two elements a lane (one of head_dim 64).
#include "tree_common.h"

namespace {

struct AttnArgs {
    const char *q, *k, *v, *kc, *vc;
    const int32_t *table, *cache_len, *parents, *tree_len;
    char* out;
    Strides3 qs, ks, os, cs;
    long ts;
    int B, N, heads, group, pages, page_size, width;
    float scale;  // times log2(e)
};

template <int DT>
__device__ __forceinline__ float ld_half(const char* p) {
    if (DT == SS_BF16) return __uint_as_float((unsigned)*reinterpret_cast<const unsigned short*>(p) << 16);
    return (float)*reinterpret_cast<const _Float16*>(p);
}
template <int DT>
__device__ __forceinline__ void st_half(char* p, float x) {
    if (DT == SS_BF16) *reinterpret_cast<unsigned short*>(p) = __builtin_bit_cast(unsigned short, (__bf16)x);
    else *reinterpret_cast<_Float16*>(p) = (_Float16)x;
}

template <int DT, int D>
__global__ __launch_bounds__(kWave) void attention_kernel(const AttnArgs a) {
    constexpr int E = D / kWave;
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y, b = blockIdx.z, kv = head / a.group;
    const int L = a.cache_len[b], N = a.tree_len ? a.tree_len[b] : a.N;
    char* const out = a.out + 2 * (b * a.os.a + row * a.os.b + head * a.os.c + lane * E);
    bool bad = L < 0 || L > (long)a.width * a.page_size || N < 0 || N > a.N;
    if (!bad && a.parents)
        for (int i = lane; i < N; i += kWave) {
            const int p = a.parents[(long)b * a.N + i];
            bad = bad || p < -1 || p >= i;
        }
    if (!bad)
        for (int i = lane; i < (L + a.page_size - 1) / a.page_size; i += kWave) {
            const int p = a.table[b * a.ts + i];
            bad = bad || p < 0 || p >= a.pages;
        }
    const bool mine = row <= N;
    if (__ballot(bad) || !mine) {
        for (int e = 0; e < E; ++e) st_half<DT>(out + 2 * e, __ballot(bad) ? __builtin_nanf("") : 0.f);
        return;
    }
    float q[E], o[E], m = -__builtin_huge_valf(), l = 0.f;
    for (int e = 0; e < E; ++e) {
        q[e] = ld_half<DT>(a.q + 2 * (b * a.qs.a + row * a.qs.b + head * a.qs.c + lane * E + e));
        o[e] = 0.f;
    }
    const auto take = [&](const char* k, const char* v) {
        float s = 0.f;
        for (int e = 0; e < E; ++e) s = fmaf(q[e], ld_half<DT>(k + 2 * e), s);
        s = wave_sum_f32(s) * a.scale;
        const float top = fmaxf(m, s), by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), p = __builtin_amdgcn_exp2f(s - top);
        l = fmaf(l, by, p);
        for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], by, p * ld_half<DT>(v + 2 * e));
        m = top;
    };
    for (int t = 0; t < L; ++t) {
        const long at = 2 * (a.table[b * a.ts + t / a.page_size] * a.cs.a + t % a.page_size * a.cs.b + kv * a.cs.c + lane * E);
        take(a.kc + at, a.vc + at);
    }
    for (int j = row;;) {
        const long at = 2 * (b * a.ks.a + j * a.ks.b + kv * a.ks.c + lane * E);
        take(a.k + at, a.v + at);
        if (j == 0) break;
        j = a.parents ? a.parents[(long)b * a.N + j - 1] + 1 : j - 1;
    }
    for (int e = 0; e < E; ++e) st_half<DT>(out + 2 * e, o[e] / l);
}

}  // namespace

extern "C" {

size_t specsteer_tree_attention_workspace_bytes(const ss_tree_params* params) {
    TreeShape s;
    return tree_shape(params, true, s) == SS_OK ? 256 : 0;
}

ss_status specsteer_tree_attention(const void* q, const void* k, const void* v, const void* k_cache, const void* v_cache, const int32_t* block_table,
                                   const int32_t* cache_len, const int32_t* parents, const int32_t* tree_len, const ss_tree_params* params, void* out,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    TreeShape s;
    const ss_status chk = tree_shape(params, true, s);
    if (chk != SS_OK) return chk;
    if (params->batch == 0) return SS_OK;
    const bool cached = params->pages > 0 && params->table_width > 0;
    if (!q || !k || !v || !cache_len || !out || (cached && (!k_cache || !v_cache || !block_table))) return SS_ERR_NULL;
    if (off_16(q) || off_16(k) || off_16(v) || off_16(out) || (cached && (off_16(k_cache) || off_16(v_cache)))) return SS_ERR_STRIDE;
    if (bad_workspace(workspace, workspace_bytes, 256)) return SS_ERR_WORKSPACE;
    const auto in = [](const void* p) { return static_cast<const char*>(p); };
    AttnArgs a{in(q), in(k), in(v), in(k_cache), in(v_cache), block_table, cache_len, params->nodes ? parents : nullptr, tree_len, static_cast<char*>(out),
               s.q, s.k, s.out, s.cache, s.table, params->batch, params->nodes, params->heads, params->heads / params->kv_heads, params->pages,
               params->page_size, params->table_width, params->scale * 1.4426950408889634f};
    if (!cached) a.width = 0;
    const dim3 grid((unsigned)(params->nodes + 1), (unsigned)params->heads, (unsigned)params->batch);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (params->dtype == SS_BF16) launch(params->head_dim == 64 ? attention_kernel<SS_BF16, 64> : attention_kernel<SS_BF16, 128>, grid, dim3(kWave), 0, st, (const AttnArgs)a);
    else launch(params->head_dim == 64 ? attention_kernel<SS_TREE_F16, 64> : attention_kernel<SS_TREE_F16, 128>, grid, dim3(kWave), 0, st, (const AttnArgs)a);
    return tree_launched();
}

const char* specsteer_tree_status_string(int status) {
    switch (status) {
        case SS_OK: return "ok";
        case SS_ERR_NULL: return "a required pointer is NULL";
        case SS_ERR_SHAPE: return "batch, nodes, heads, head_dim, pages or vocab out of range";
        case SS_ERR_DTYPE: return "unknown dtype";
        case SS_ERR_PARAM: return "scale, lambda, beta, temperature or flags out of range";
        case SS_ERR_STRIDE: return "strides negative, off 16 bytes or overlapping, or a pointer off its alignment";
        case SS_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case SS_ERR_DEVICE: return "HIP launch failed";
        default: return "unknown status";
    }
}

}  // extern "C"
