// Keys and values of the accepted path into the paged cache, for MI355X (gfx950); include/specsteer_tree.h says what it computes.
//
// A copy of a few rows: bound by a launch and its round trips (length, path and page, then the row).  A workgroup takes up to kRowsEach rows of one
// sequence, each of its threads 16 bytes at a time; every workgroup looks the whole path over first, since nothing is written of a bad one.  One path of
// one sequence takes 5 us, a launch's least; 256 paths in trees of 24 nodes, 8 heads of 128 in bf16 (6.4 MB read and written) 6.8.
#include "tree_common.h"
#include "tree_schedule.h"

namespace {

constexpr int kCommitThreads = 256, kRowsEach = 8;

struct CommitArgs {
    const char *k, *v;
    char *kc, *vc;
    const int32_t *table, *cache_len, *accepted, *path;
    int32_t* new_len;
    Strides3 ks, cs;
    long ts;
    int N, heads, pieces, pages, page_size, width;  // pieces: of 16 bytes a head
};

__global__ __launch_bounds__(kCommitThreads) void commit_kernel(const CommitArgs a) {
    __shared__ int wrong;
    const int b = blockIdx.y, tid = threadIdx.x;
    const int L = a.cache_len[b], n = a.accepted[b];
    const long room = (long)a.width * a.page_size;
    const bool in_range = n >= 0 && n <= a.N && L >= 0 && (long)L + n + 1 <= room;
    const int first = blockIdx.x * kRowsEach;
    if (first > 0 && (!in_range || first > n)) return;
    if (tid == 0) wrong = in_range ? 0 : 1;
    __syncthreads();
    if (in_range) {
        bool bad = false;
        if (a.path)
            for (int i = tid; i < n; i += kCommitThreads) {
                const int r = a.path[(long)b * a.N + i];
                bad = bad || r < 0 || r >= a.N;
            }
        const PageRange pages = pages_written(L, n, a.page_size);
        for (int i = tid; i <= pages.more; i += kCommitThreads) {
            const int p = a.table[b * a.ts + pages.first + i];
            bad = bad || p < 0 || p >= a.pages;
        }
        if (bad) wrong = 1;
    }
    __syncthreads();
    const bool none = wrong != 0;
    if (first == 0 && tid == 0) a.new_len[b] = none ? -1 : L + n + 1;
    if (none) return;
    const int row_pieces = a.heads * a.pieces, rows = min(kRowsEach, n + 1 - first), all = rows * row_pieces;
    for (int i = tid; i < all; i += kCommitThreads) {
        const int j = first + i / row_pieces, rest = i % row_pieces, head = rest / a.pieces, piece = rest % a.pieces;
        const int row = j == 0 ? 0 : a.path ? a.path[(long)b * a.N + j - 1] + 1 : j, t = L + j;
        const long from = 2 * (b * a.ks.a + row * a.ks.b + head * a.ks.c) + 16 * piece;
        const long to = 2 * (a.table[b * a.ts + t / a.page_size] * a.cs.a + t % a.page_size * a.cs.b + head * a.cs.c) + 16 * piece;
        const uint4 kk = *reinterpret_cast<const uint4*>(a.k + from), vv = *reinterpret_cast<const uint4*>(a.v + from);
        *reinterpret_cast<uint4*>(a.kc + to) = kk;
        *reinterpret_cast<uint4*>(a.vc + to) = vv;
    }
}

}  // namespace

extern "C" ss_status specsteer_tree_commit(const void* k, const void* v, void* k_cache, void* v_cache, const int32_t* block_table,
                                           const int32_t* cache_len, const int32_t* accepted_len, const int32_t* path, const ss_tree_params* params,
                                           int32_t* new_len, void* stream) {
    TreeShape s;
    const ss_status chk = tree_shape(params, false, s);
    if (chk != SS_OK) return chk;
    if (params->batch == 0) return SS_OK;
    const bool cached = params->pages > 0 && params->table_width > 0;
    if (!k || !v || !cache_len || !accepted_len || !new_len || (cached && (!k_cache || !v_cache || !block_table))) return SS_ERR_NULL;
    if (shared({new_len}, {cache_len, accepted_len, path, block_table})) return SS_ERR_PARAM;
    if (off_16(k) || off_16(v) || (cached && (off_16(k_cache) || off_16(v_cache)))) return SS_ERR_STRIDE;
    if (cached && k_cache == v_cache) return SS_ERR_PARAM;  // keys and values would race for their places
    const CommitArgs a{static_cast<const char*>(k), static_cast<const char*>(v), static_cast<char*>(k_cache), static_cast<char*>(v_cache), block_table,
                       cache_len, accepted_len, params->nodes ? path : nullptr, new_len, s.k, s.cache, s.table, params->nodes, params->kv_heads,
                       params->head_dim / 8, params->pages, params->page_size, cached ? params->table_width : 0};
    // a grid's second dimension holds 65535 sequences
    for (int b = 0; b < params->batch; b += 65535) {
        CommitArgs c = a;
        c.k += 2 * b * s.k.a;
        c.v += 2 * b * s.k.a;
        if (c.table) c.table += b * s.table;
        c.cache_len += b;
        c.accepted += b;
        if (c.path) c.path += (long)b * params->nodes;
        c.new_len += b;
        const int left = params->batch - b;
        launch(commit_kernel, dim3((unsigned)(params->nodes / kRowsEach + 1), (unsigned)(left < 65535 ? left : 65535)), dim3(kCommitThreads), 0,
               static_cast<hipStream_t>(stream), (const CommitArgs)c);
    }
    return tree_launched();
}
