// The verify-and-recover step down a tree of drafts, for MI355X (gfx950); include/specsteer_tree.h says what it computes.
//
// The rows that the walk comes through are known only as it goes, and a row is read by many workgroups.  A tree is therefore taken in stages
// (verify_plan.h), two at most: one sums some rows at and below the cursor, of G and S_noctx, whichever way the walk may take there; the next one's workgroups
// each walk over those sums for themselves, from what lies in LDS by then, and sum the rows that follow.  The last launch walks to the
// end, forms the recovery row's masses a chunk of 4 vectors a lane at a time, and the workgroup of a sequence that comes last draws the token.
//
// A walk: with d_r = log2 sum of G's row - log2 sum of S_noctx's, node i at row r = parent + 1 is accepted if
//     u_i <= 2^((G_y - S_y) c - d_r) / lambda;
// every row's first accepted child is found at once, and the walk follows them.
//
// What bounds it are the launches' beginnings, a chain of loads and two logarithms that each has to walk before it can load a row, and rows that the walk does
// not come through in the end.  64 trees of up to 31 nodes, V = 128256 bf16: 62 to 75 us, of which the stages of rows take 17 and 25 and the draw 23; one tree of 12
// nodes, V = 32000 fp32, 17.5, of which the draw 13.
#include "../loss/loss_rows.h"
#include "tree_common.h"
#include "verify_plan.h"

#include <type_traits>

namespace {

struct Cursor {
    int cur, n, done, pad;  // done: 1 at the walk's end, 2 of a sequence that is marked
};
struct Mass {
    float E, s;  // s 2^E; with kByLogit for E relative to a logit that stands in `tops`
};
constexpr float kByLogit = __builtin_huge_valf();
struct Best {
    double h;
    int id, pad;
};

struct VerifyArgs {
    const void *G, *Sp, *Sm;
    const int32_t *tokens, *parents, *tree_len;
    const float* uniforms;
    int32_t *accepted_len, *path, *next_token;
    float* next_logprob;
    Cursor* cursors;      // [stages + 1][B]
    char* arrive;         // [B] counters, kArriveBytes apart
    Total<Sum>* sums;     // [B][N + 1][2][slices]
    float2* logits;       // [B][N]: of the nodes' tokens at their rows
    Mass* masses;         // [B][chunks]
    double* tops;         // [B][chunks]
    Best* best;           // [B][parts]
    long sb, st;
    int B, N, V;
    Factor c;
    double c64, lambda, beta;
    float steer_hi, steer_lo;  // beta c in two parts
    float steer_size, steer_most;  // |beta c|, and the difference whose product with it is kFar
    int far, greedy, plain;    // plain: beta is 0
    int by_logit;              // all masses are
    int slices, slice_vecs, chunks, parts, part_chunks;
};

constexpr int kNever = 0x7FFFFFFF, kUnsummed = -2;
struct WalkShared {
    short parent[SS_MAX_K], above[SS_MAX_K];  // above: an ancestor, not over the cursor
    unsigned char inner[SS_MAX_K + 4];        // rows with children
    short rows[SS_MAX_K + 1];                 // of the stage
    int first[SS_MAX_K + 1];                  // every row's first accepted child
    double diff[SS_MAX_K + 1];
    Total<Sum> part[kVerifyGroup / kWave];
    int scan[kVerifyGroup / kWave];
    int count, flag;
    Cursor at;
};

// the steering term's difference: a token that both of the specialist's rows mask has none
__device__ __forceinline__ double steer(float sp, float sm) { return sp == sm ? 0.0 : (double)sp - (double)sm; }
__device__ __forceinline__ int nodes_of(const VerifyArgs& a, int b) { return a.tree_len ? a.tree_len[b] : a.N; }

// A sequence's tree into LDS, N nodes of it.
__device__ __forceinline__ void load_tree(const VerifyArgs& a, int b, int N, WalkShared& w) {
    for (int r = threadIdx.x; r <= N; r += kVerifyGroup) {
        w.inner[r] = 0;
        w.first[r] = kUnsummed;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < N; i += kVerifyGroup) {
        const int p = a.parents ? a.parents[(long)b * a.N + i] : i - 1;
        w.parent[i] = (short)p;
        w.inner[p + 1] = 1;
    }
    __syncthreads();
}

// The first `most` rows with children at and below the cursor into w.rows, their number into w.count.
__device__ __forceinline__ void pick_rows(const VerifyArgs& a, int N, int cur, int most, WalkShared& w) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kWaves = kVerifyGroup / kWave;
    const bool all = cur < 0 || !a.parents;  // whatever lies behind the cursor is below it
    if (!all) {
        for (int i = tid; i < N; i += kVerifyGroup) w.above[i] = w.parent[i];
        // steps up, doubled each time, that end at the cursor or over it; an entry that another lane has moved on already is an ancestor too
        for (int step = 1; step < N; step *= 2) {
            __syncthreads();
            bool moved = false;
            for (int i = tid; i < N; i += kVerifyGroup) {
                const int p = w.above[i];
                if (p > cur) {
                    w.above[i] = w.above[p];
                    moved = true;
                }
            }
            if (!__syncthreads_or(moved)) break;
        }
    }
    __syncthreads();
    int count = 0;
    for (int r0 = cur + 1; r0 <= N && count < most; r0 += kVerifyGroup) {
        const int r = r0 + tid;
        const bool in = r <= N && w.inner[r] && (all || r == cur + 1 || w.above[r - 1] == cur);
        const unsigned long long mask = __ballot(in);
        __syncthreads();
        if (lane == 0) w.scan[wave] = __popcll(mask);
        __syncthreads();
        int at = count + __popcll(mask & ((1ull << lane) - 1));
        for (int v = 0; v < kWaves; ++v) {
            at += v < wave ? w.scan[v] : 0;
            count += w.scan[v];
        }
        if (in && at < most) w.rows[at] = (short)r;
    }
    if (tid == 0) w.count = count < most ? count : most;
    __syncthreads();
}

// What is taken from the difference of a node's logits in its test: `ref`, in logits, before its product with c, and d_r less that behind it.  Of rows far
// from zero ref is the difference of the largest logits, both of which may be beyond what h c has bits for; of others it is 0.
struct RowDiff {
    double ref, diff;
};
// The row far from zero, or one of whose tensors' is, by the whole workgroup.
template <int DT>
__device__ __forceinline__ RowDiff far_diff(const VerifyArgs& a, int b, int r, Total<Sum>* part) {
    Total<Sum> s[2];
    for (int x = 0; x < 2; ++x) {
        const void* const h = row_ptr<DT>(x ? a.Sm : a.G, b * a.sb + r * a.st);
        __syncthreads();
        s[x] = far_sum<DT, Sum>(h, nullptr, a.V, a.c64, kVerifyGroup, part);
    }
    return RowDiff{(double)s[0].E - (double)s[1].E, log2(s[0].s) - log2(s[1].s)};
}
// Whether a node with logits h of G and S_noctx is accepted: masked by G never, by S_noctx alone always
__device__ __forceinline__ bool accepts(const VerifyArgs& a, float2 h, double u, RowDiff d) {
    const double alpha = h.x == -__builtin_huge_valf() ? -1.0 : exp2((((double)h.x - (double)h.y) - d.ref) * a.c64 - d.diff) / a.lambda;
    return u <= 1.0 && !(u > alpha);
}

// On from w.at over the rows of w.rows, whose sums are there.
template <int DT>
__device__ __forceinline__ void walk(const VerifyArgs& a, int b, int N, bool leader, WalkShared& w) {
    const int tid = threadIdx.x;
    constexpr int kLanes = 16, kAtOnce = kVerifyGroup / kLanes;  // lanes a row and tensor
    const int n = w.count;
    bool far = false;
    for (int k0 = 0; k0 < 2 * n; k0 += kAtOnce) {
        const int k = k0 + tid / kLanes, l = tid % kLanes;
        Total<Sum> s;
        clear_total(s);
        if (k < 2 * n && l < a.slices) s = a.sums[(((long)b * (a.N + 1) + w.rows[k >> 1]) * 2 + (k & 1)) * a.slices + l];
        s = join_group(s, kLanes);
        const bool is = a.far || is_far(s);
        far = far || (k < 2 * n && is);
        const double lse = (double)s.E + log2(s.s), other = __shfl_xor(lse, kLanes, kWave);
        if (k < 2 * n && l == 0 && !(k & 1)) {
            w.diff[w.rows[k >> 1]] = lse - other;
            w.first[w.rows[k >> 1]] = kNever;
        }
    }
    const auto test = [&](int i, int r, RowDiff d) {
        const float2 h = a.logits[(long)b * a.N + i];
        const double u = a.uniforms[(long)b * (a.N + 1) + i];
        if (accepts(a, h, u, d)) atomicMin(&w.first[r], i);
    };
    constexpr double kTested = __builtin_huge_val();
    if (__syncthreads_or(far))
        for (int k = 0; k < n; ++k) {
            const int r = w.rows[k];
            bool of_row = a.far;
            for (int x = 0; x < 2; ++x) {
                Total<Sum> s;
                clear_total(s);
                for (int l = 0; l < a.slices; ++l) {
                    const Total<Sum> o = a.sums[(((long)b * (a.N + 1) + r) * 2 + x) * a.slices + l];
                    const float E = fmaxf(s.E, o.E);
                    s.s = moved(s.s, s.E, E) + moved(o.s, o.E, E);
                    s.E = E;
                }
                of_row = of_row || is_far(s);
            }
            if (!of_row) continue;
            const RowDiff d = far_diff<DT>(a, b, r, w.part);
            for (int i = r + tid; i < N; i += kVerifyGroup)  // children lie behind their parent
                if (w.parent[i] == r - 1) test(i, r, d);
            if (tid == 0) w.diff[r] = kTested;
        }
    __syncthreads();
    for (int i = tid; i < N; i += kVerifyGroup) {
        const int r = w.parent[i] + 1;
        if (w.first[r] >= 0 && w.diff[r] != kTested) test(i, r, RowDiff{0.0, w.diff[r]});
    }
    __syncthreads();
    if (tid == 0) {
        Cursor c = w.at;
        for (;;) {
            const int r = c.cur + 1;
            const int next = w.inner[r] ? w.first[r] : kNever;
            if (next == kUnsummed) break;
            if (next == kNever) {
                c.done = 1;
                break;
            }
            c.cur = next;
            if (leader) a.path[(long)b * a.N + c.n] = next;
            ++c.n;
        }
        w.at = c;
    }
    __syncthreads();
}

// The cursor from which stage `stage` goes on, in w.at, with the tree in LDS if it goes on at all.
template <int DT>
__device__ __forceinline__ int reach(const VerifyArgs& a, int b, int stage, int rows_before, bool leader, WalkShared& w) {
    int N = nodes_of(a, b);
    if (stage == 0) {
        bool bad = N < 0 || N > a.N;
        if (!bad)
            for (int i = threadIdx.x; i < N; i += kVerifyGroup) {
                const int p = a.parents ? a.parents[(long)b * a.N + i] : i - 1, y = a.tokens[(long)b * a.N + i];
                bad = bad || p < -1 || p >= i || y < 0 || y >= a.V;
            }
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) w.at = Cursor{-1, 0, bad ? 2 : N == 0 ? 1 : 0, 0};
        __syncthreads();
        if (w.at.done) return 0;
        load_tree(a, b, N, w);
    } else {
        if (threadIdx.x == 0) w.at = a.cursors[(long)(stage - 1) * a.B + b];
        __syncthreads();
        if (w.at.done) return 0;
        load_tree(a, b, N, w);
        pick_rows(a, N, w.at.cur, rows_before, w);
        walk<DT>(a, b, N, leader, w);
    }
    return N;
}

// ------------------------------------------------------------------ trees of up to 63 nodes

// The same for a tree whose rows are the bits of a word: a lane a node, children and descendants by ballots.  Everything that memory holds of the walk
// so far, the sums of rows that were not summed among it, is on its way at once; what bounds a stage's beginning is that one round trip and the
// two logarithms of a row.  By the general walk, whose loads wait for one another and whose steps for barriers, the rows' launches of 64 trees of up to 31 nodes
// took 12 to 28 us and the draw 27.
constexpr int kSmall = 63;
struct SmallShared {
    double diff[kSmall + 1], ref[kSmall + 1];
    unsigned long long far[kVerifyGroup / kWave], inner, set, rows;
    signed char parent[kSmall + 1];
    Total<Sum> part[kVerifyGroup / kWave];
    int scan[kVerifyGroup / kWave];
    double table[SS_MAX_K + 1];
    Cursor at;
};

__device__ __forceinline__ unsigned long long lowest_bits(unsigned long long m, int n) {
    while (__popcll(m) > n) m &= ~(1ull << (63 - __clzll((long long)m)));
    return m;
}
// Rows at and below the cursor, by a wave whose lane i has node i's parent (or one that no row is).
__device__ __forceinline__ unsigned long long rows_below(int cur, int parent) {
    unsigned long long m = 1ull << (cur + 1);
    for (;;) {
        const unsigned long long more = m | __ballot(parent >= -1 && (m >> (parent + 1) & 1)) << 1;
        if (more == m) return m;
        m = more;
    }
}

template <int DT>
__device__ __forceinline__ int reach(const VerifyArgs& a, int b, int stage, int rows_before, int rows, bool leader, SmallShared& w) {
    constexpr int kLanes = 4, kMine = 16 / kLanes;  // lanes a row
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = tid / kLanes, l = tid % kLanes;
    Total<Sum> s[2][kMine];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            clear_total(s[x][k]);
            const int i = k * kLanes + l;
            if (stage > 0 && r <= a.N && i < a.slices) s[x][k] = a.sums[(((long)b * (a.N + 1) + r) * 2 + x) * a.slices + i];
        }
    Cursor c{-1, 0, 0, 0};
    if (stage > 0) c = a.cursors[(long)(stage - 1) * a.B + b];
    int N = nodes_of(a, b), parent = -5, token = 0;
    float2 h = make_float2(0.f, 0.f);
    double u = 0.0;
    if (wave == 0 && lane < a.N) {
        parent = a.parents ? a.parents[(long)b * a.N + lane] : lane - 1;
        if (stage == 0) token = a.tokens[(long)b * a.N + lane];
        else {
            h = a.logits[(long)b * a.N + lane];
            u = a.uniforms[(long)b * (a.N + 1) + lane];
        }
    }
    if (tid == 0) w.inner = 0;
    if (stage > 0) {
        double lse[2];
        bool far = false;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            Total<Sum> t;
            t.E = fmaxf(fmaxf(s[x][0].E, s[x][1].E), fmaxf(s[x][2].E, s[x][3].E));
            t.s = 0.0;
#pragma unroll
            for (int k = 0; k < kMine; ++k) t.s += moved(s[x][k].s, s[x][k].E, t.E);
            t = join_group(t, kLanes);
            far = far || a.far || is_far(t);
            lse[x] = (double)t.E + log2(t.s);
        }
        if (l == 0) {
            w.diff[r] = lse[0] - lse[1];
            w.ref[r] = 0.0;
        }
        unsigned long long mask = 0;
        const unsigned long long ballot = __ballot(far && l == 0 && r <= a.N);
        for (int k = 0; k < kWave / kLanes; ++k) mask |= (ballot >> (kLanes * k) & 1) << (wave * (kWave / kLanes) + k);
        if (lane == 0) w.far[wave] = mask;
    }
    __syncthreads();
    unsigned long long set = 0, inner = 0;
    if (wave == 0) {
        if (stage == 0) {
            const bool bad = N < 0 || N > a.N || (lane < N && (parent < -1 || parent >= lane || token < 0 || token >= a.V));
            c.done = __ballot(bad) ? 2 : N == 0 ? 1 : 0;
        }
        if (c.done || lane >= N) parent = -5;
        if (parent >= -1) atomicOr(&w.inner, 1ull << (parent + 1));
        w.parent[lane] = (signed char)parent;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        inner = *const_cast<volatile unsigned long long*>(&w.inner);
        if (stage > 0 && !c.done) set = lowest_bits(rows_below(c.cur, parent) & inner, rows_before);
        if (lane == 0) {
            w.at = c;
            w.set = set;
        }
    }
    if (stage > 0) {
        __syncthreads();
        const unsigned long long all = w.set, far = all & (w.far[0] | w.far[1] | w.far[2] | w.far[3]);
        if (far) {  // rows far from zero, by the whole workgroup
            for (unsigned long long m = far; m; m &= m - 1) {
                const int fr = first_lane(m);
                const RowDiff d = far_diff<DT>(a, b, fr, w.part);
                if (tid == 0) {
                    w.diff[fr] = d.diff;
                    w.ref[fr] = d.ref;
                }
            }
            __syncthreads();
        }
    }
    if (wave == 0) {
        if (stage > 0 && !c.done) {
            bool accept = false;
            if (parent >= -1 && (set >> (parent + 1) & 1)) accept = accepts(a, h, u, RowDiff{w.ref[parent + 1], w.diff[parent + 1]});
            for (;;) {
                const int row = c.cur + 1;
                if (!(inner >> row & 1)) c.done = 1;
                else if (!(set >> row & 1)) break;
                const unsigned long long taken = c.done ? 0 : __ballot(accept && parent == c.cur);
                if (!taken) {
                    c.done = 1;
                    break;
                }
                c.cur = first_lane(taken);
                if (leader && lane == 0) a.path[(long)b * a.N + c.n] = c.cur;
                ++c.n;
            }
        }
        const unsigned long long next = c.done ? 0 : lowest_bits(rows_below(c.cur, parent) & inner, rows);
        if (lane == 0) {
            w.at = c;
            w.rows = next;
        }
    }
    __syncthreads();
    return N;
}

// The same by the general walk.
template <int DT>
__device__ __forceinline__ int reach(const VerifyArgs& a, int b, int stage, int rows_before, int rows, bool leader, WalkShared& w) {
    const int N = reach<DT>(a, b, stage, rows_before, leader, w);
    if (!w.at.done && rows) pick_rows(a, N, w.at.cur, rows, w);
    return N;
}
__device__ __forceinline__ int row_count(const WalkShared& w) { return w.count; }
__device__ __forceinline__ int row_count(const SmallShared& w) { return __popcll(w.rows); }
__device__ __forceinline__ int nth_row(const WalkShared& w, int k) { return w.rows[k]; }
__device__ __forceinline__ int nth_row(const SmallShared& w, int k) {
    unsigned long long m = w.rows;
    for (; k > 0; --k) m &= m - 1;
    return first_lane(m);
}
__device__ __forceinline__ double* space_of(WalkShared& w) { return w.diff; }
__device__ __forceinline__ double* space_of(SmallShared& w) { return w.table; }

// One lane's share of a slice, some sixteen vectors: eight on their way at a time, the last ones too.  By four, and the last ones one by one, 64 trees of up to
// 31 nodes took 67 us and not 63, 16 of 60 50 and not 46, 256 of 8 (four times the vectors a lane) 120 and not 124; four with the next four behind them 67, 47 and
// 127, sixteen 66, 54 and 125.
template <int DT>
__device__ __forceinline__ Sum slice_sum(const void* h, const Layout<DT>& lay, int begin, int end, bool extra, Factor c) {
    constexpr int kVec = Row<DT>::kVec, kUnroll = 8, kElem = DT == SS_BF16 ? 2 : 4;
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
    Sum a;
    clear(a);
    typename Row<DT>::Raw r[kUnroll];
    const auto load = [&](int from, typename Row<DT>::Raw (&to)[kUnroll]) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int v = from + u * kVerifyGroup + (int)threadIdx.x;
            to[u] = neg_inf_raw<DT, kVec>();
            if (v < end) to[u] = ld_once<DT>(hv, v);
        }
    };
    for (int i = begin; i < end; i += kUnroll * kVerifyGroup) {
        load(i, r);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float x[kVec];
            unpack(r[u], x);
            add<2>(a, x, c);
        }
    }
    if (extra && lay.extra >= 0) {
        const float x[1] = {ld_elem<DT>(h, lay.extra)};
        add<2>(a, x, c);
    }
    return a;
}

// Stage `stage`: the sums of one slice of some of its rows.
template <int DT, typename W>
__global__ __launch_bounds__(kVerifyGroup) void rows_kernel(const VerifyArgs a, const int stage, const int rows_before, const int rows, const int groups) {
    __shared__ W w;
    const int per = groups * 2 * a.slices, b = (int)(blockIdx.x / (unsigned)per), id = (int)(blockIdx.x - (unsigned)(b * per));
    const int slice = id % a.slices, x = id / a.slices & 1, group = id / (2 * a.slices);
    const bool leader = id == 0;
    // a small tree's tokens, a lane each, beside the walk's loads, and their logits beside the row's: behind the sums both took two round trips more
    constexpr bool kSmallTree = std::is_same<W, SmallShared>::value;
    const int i_mine = threadIdx.x;
    const int token = kSmallTree && slice == 0 && i_mine < a.N ? a.tokens[(long)b * a.N + i_mine] : 0;
    const int N = reach<DT>(a, b, stage, rows_before, rows, leader, w);
    if (leader && threadIdx.x == 0) {
        a.cursors[(long)stage * a.B + b] = w.at;
        if (stage == 0 && a.parts > 1) *reinterpret_cast<int*>(a.arrive + (long)b * kArriveBytes) = 0;
    }
    if (w.at.done) return;
    const int count = row_count(w);
    for (int k = group; k < count; k += groups) {
        const int r = nth_row(w, k);
        const void* const h = row_ptr<DT>(x ? a.Sm : a.G, b * a.sb + r * a.st);
        const Layout<DT> lay(h, a.V, threadIdx.x);
        const int begin = min(lay.vecs, slice * a.slice_vecs), end = slice + 1 == a.slices ? lay.vecs : min(lay.vecs, begin + a.slice_vecs);
        const bool child = kSmallTree && slice == 0 && i_mine < N && w.parent[i_mine] == r - 1;
        float child_logit = 0.f;
        if (child) child_logit = ld_elem<DT>(h, token);
        const Sum mine = slice_sum<DT>(h, lay, begin, end, slice == 0, a.c);
        asm volatile("" : "+v"(child_logit));  // not loaded later
        if (child) reinterpret_cast<float*>(a.logits + (long)b * a.N + i_mine)[x] = child_logit;
        if (!kSmallTree && slice == 0)
            for (int i = r + threadIdx.x; i < N; i += kVerifyGroup)  // children lie behind their parent, node r - 1
                if (w.parent[i] == r - 1)
                    reinterpret_cast<float*>(a.logits + (long)b * a.N + i)[x] = ld_elem<DT>(h, a.tokens[(long)b * a.N + i]);
        const Total<Sum> s = block_total(mine, kVerifyGroup, w.part);
        if (threadIdx.x == 0) a.sums[(((long)b * (a.N + 1) + r) * 2 + x) * a.slices + slice] = s;
        __syncthreads();
    }
}

// ------------------------------------------------------------------ the draw

template <int DT>
struct RecoveryRow {
    const void *g, *sp, *sm;
};
// Eq. 8's exponent less E, in fp32: g c first, whose upper part is exact for bf16 (loss_rows.h), so that what is rounded is of the difference's size.
// In double the masses of 64 rows of V = 128256 took 14 us, most of it arithmetic.  A term near E is off by up to 3 half steps of its steering term's
// size, 2^-24 of it each: the sum's share of that, sum p |d beta c| / sum p, is formed beside the sum, and a chunk where it passes kSteerMean, or whose
// exponents are far from zero, is summed again in double, by its logits' differences to their largest, which hold at any temperature: 64 trees 65 us,
// with all chunks so 88.
__device__ __forceinline__ float rec_exponent(const VerifyArgs& a, float g, float d, float E) {
    const float t = exponent<2>(g, E, a.c);
    return a.plain ? t : fmaf(d, a.steer_lo, fmaf(d, a.steer_hi, t));
}
constexpr double kSteerMean = 16.0;
// and in double, for the token drawn
__device__ __forceinline__ double rec_exponent64(const VerifyArgs& a, float g, float sp, float sm) { return fma((double)g, a.c64, a.plain ? 0.0 : steer(sp, sm) * (a.beta * a.c64)); }
// Eq. 8's logit, the operations in this order
__device__ __forceinline__ double rec_logit(const VerifyArgs& a, float g, float sp, float sm) {
    return a.plain ? (double)g : __dadd_rn((double)g, __dmul_rn(a.beta, steer(sp, sm)));
}
__device__ __forceinline__ float logit_term(double h, double top, double c) { return exp2_hw((float)((h - top) * c)); }

// A step of chunk `c` of a row by a wave: each lane's logits of G, -inf where there are none, and the steering term's differences; returns the
// first one's id.  The last chunk has the elements behind the last vector, one a lane.
template <int DT>
struct Chunk {
    typename Row<DT>::Raw g, sp, sm;
    int id;
};
template <int DT>
__device__ __forceinline__ Chunk<DT> load_chunk(const VerifyArgs& a, const RecoveryRow<DT>& row, int c, int step) {
    constexpr int kVec = Row<DT>::kVec;
    const int lane = threadIdx.x & 63, vecs = a.V / kVec;
    Chunk<DT> k;
    k.g = neg_inf_raw<DT, kVec>();
    k.sp = k.sm = typename Row<DT>::Raw{};
    if (c + 1 < a.chunks) {
        const int v = c * kMassVecs + step * kWave + lane;
        if (v < vecs) {
            k.g = ld_raw<DT, kVec>(row.g, v);
            if (!a.plain) {
                k.sp = ld_raw<DT, kVec>(row.sp, v);
                k.sm = ld_raw<DT, kVec>(row.sm, v);
            }
        }
        k.id = v * kVec;
        return k;
    }
    k.id = vecs * kVec + lane;
    if (step == 0 && k.id < a.V) {
        const auto first = [&](typename Row<DT>::Raw& r, const void* p) {
            if constexpr (DT == SS_BF16) r.x = (r.x & 0xFFFF0000u) | reinterpret_cast<const unsigned short*>(p)[k.id];
            else r.x = reinterpret_cast<const float*>(p)[k.id];
        };
        first(k.g, row.g);
        if (!a.plain) {
            first(k.sp, row.sp);
            first(k.sm, row.sm);
        }
    }
    return k;
}
// a token that both of the specialist's rows mask has no steering term
template <int DT>
__device__ __forceinline__ void unpack_chunk(const Chunk<DT>& k, float (&g)[Row<DT>::kVec], float (&d)[Row<DT>::kVec]) {
    constexpr int kVec = Row<DT>::kVec;
    float sp[kVec], sm[kVec];
    unpack(k.g, g);
    unpack(k.sp, sp);
    unpack(k.sm, sm);
#pragma unroll
    for (int i = 0; i < kVec; ++i) d[i] = sp[i] == sm[i] ? 0.f : sp[i] - sm[i];
}
template <typename T>
__device__ __forceinline__ T either(bool first, const T& a, const T& b) {  // of registers
    typedef unsigned u32v4 __attribute__((ext_vector_type(4)));
    const u32v4 x = __builtin_bit_cast(u32v4, a), y = __builtin_bit_cast(u32v4, b);
    u32v4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = first ? x[i] : y[i];
    return __builtin_bit_cast(T, r);
}
constexpr int kMassSteps = kMassVecs / kWave;

// What workgroups hand over inside a launch goes past the caches of one die with stores and loads at device scope; a wave has delivered when its
// stores are acknowledged.  Fences, which write a die's whole cache back, took 100 us of a launch of 512 workgroups.
__device__ __forceinline__ void put(unsigned long long* p, unsigned long long v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ unsigned long long get(const unsigned long long* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(Mass* p, Mass m) { put(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, m)); }
__device__ __forceinline__ void put(double* p, double v) { put(reinterpret_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, v)); }
__device__ __forceinline__ double get(const double* p) { return __builtin_bit_cast(double, get(reinterpret_cast<const unsigned long long*>(p))); }
__device__ __forceinline__ Mass get(const Mass* p) { return __builtin_bit_cast(Mass, get(reinterpret_cast<const unsigned long long*>(p))); }
__device__ __forceinline__ void put(Best* p, Best v) {
    unsigned long long* const q = reinterpret_cast<unsigned long long*>(p);
    put(q, __builtin_bit_cast(unsigned long long, v.h));
    put(q + 1, (unsigned long long)(unsigned)v.id);
}
__device__ __forceinline__ Best get(const Best* p) {
    const unsigned long long* const q = reinterpret_cast<const unsigned long long*>(p);
    return Best{__builtin_bit_cast(double, get(q)), (int)(unsigned)get(q + 1), 0};
}
__device__ __forceinline__ void delivered() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
}

// Chunks by their logits: seldom, so that each step is loaded again where it is needed and no registers are held for it.
template <int DT>
__device__ __forceinline__ void chunk_logits(const VerifyArgs& a, const Chunk<DT>& k, double (&h)[Row<DT>::kVec]) {
    constexpr int kVec = Row<DT>::kVec;
    float g[kVec], sp[kVec], sm[kVec];
    unpack(k.g, g);
    unpack(k.sp, sp);
    unpack(k.sm, sm);
#pragma unroll
    for (int i = 0; i < kVec; ++i) h[i] = rec_logit(a, g[i], sp[i], sm[i]);
}
// A chunk's largest logit of Eq. 8, -inf of masked tokens alone, and the sum of its terms relative to that, by a wave.
template <int DT>
__device__ __forceinline__ double chunk_by_logit(const VerifyArgs& a, const RecoveryRow<DT>& row, int c, double& sum) {
    constexpr int kVec = Row<DT>::kVec;
    double top = -__builtin_huge_val(), h[kVec];
#pragma unroll 1
    for (int s = 0; s < kMassSteps; ++s) {
        chunk_logits<DT>(a, load_chunk<DT>(a, row, c, s), h);
#pragma unroll
        for (int i = 0; i < kVec; ++i) top = fmax(top, h[i]);
    }
    for (int d = 1; d < kWave; d <<= 1) top = fmax(top, __shfl_xor(top, d, kWave));
    sum = 0.0;
    if (!(top > -__builtin_huge_val())) return top;
#pragma unroll 1
    for (int s = 0; s < kMassSteps; ++s) {
        chunk_logits<DT>(a, load_chunk<DT>(a, row, c, s), h);
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum += (double)logit_term(h[i], top, a.c64);
    }
    sum = wave_sum_f64(sum);
    return top;
}
// The token of such a chunk, by a wave: the first that brings the sum from `cum` on past the target, or the last one with any mass; and its logit.
template <int DT>
__device__ __forceinline__ int token_by_logit(const VerifyArgs& a, const RecoveryRow<DT>& row, int c, double top, double scale, double cum, double target, bool last,
                                              double& logit) {
    constexpr int kVec = Row<DT>::kVec;
    int token = -1;
    logit = top;
#pragma unroll 1
    for (int s = 0; s < kMassSteps; ++s) {
        const Chunk<DT> k = load_chunk<DT>(a, row, c, s);
        double h[kVec], own = 0.0, mine = 0.0, tail = 0.0;
        float e[kVec];
        int hit = -1, end = -1;
        chunk_logits<DT>(a, k, h);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            e[i] = logit_term(h[i], top, a.c64);
            own += (double)e[i];
        }
        const double incl = wave_incl_scan_f64(own * scale);
        double at = cum + wave_shift_up_f64(incl);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            at += (double)e[i] * scale;
            if (e[i] > 0.f) {
                end = k.id + i;
                tail = h[i];
                if (!last && hit < 0 && at > target) {
                    hit = k.id + i;
                    mine = h[i];
                }
            }
        }
        const unsigned long long hits = __ballot(hit >= 0), ends = __ballot(end >= 0);
        if (hits) {
            logit = __shfl(mine, first_lane(hits), kWave);
            return __shfl(hit, first_lane(hits), kWave);
        }
        if (ends) {
            const int L = 63 - __clzll((long long)ends);
            token = __shfl(end, L, kWave);
            logit = __shfl(tail, L, kWave);
        }
        cum += wave_last_f64(incl);
    }
    return token;
}

template <int DT, typename W>
__global__ __launch_bounds__(kVerifyGroup) void draw_kernel(const VerifyArgs a, const int stages, const int rows_before) {
    constexpr int kVec = Row<DT>::kVec, kWaves = kVerifyGroup / kWave;
    __shared__ W w;
    __shared__ Best best[kWaves];
    __shared__ double sum[kWaves];
    __shared__ int before_us, last_of[kWaves];
    const int b = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)(b * a.parts));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool leader = part == 0;
    reach<DT>(a, b, stages, rows_before, 0, leader, w);
    const Cursor at = w.at;
    const bool marked = at.done == 2;
    if (leader) {
        if (tid == 0) a.accepted_len[b] = marked ? -1 : at.n;
        for (int i = at.n + tid; i < a.N; i += kVerifyGroup) a.path[(long)b * a.N + i] = -1;
        if (marked && tid == 0) {
            a.next_token[b] = -1;
            if (a.next_logprob) a.next_logprob[b] = __builtin_nanf("");
        }
    }
    if (marked) return;
    const long off = b * a.sb + (at.cur + 1) * a.st;
    const RecoveryRow<DT> row{row_ptr<DT>(a.G, off), row_ptr<DT>(a.Sp, off), row_ptr<DT>(a.Sm, off)};
    Mass* const masses = a.masses + (long)b * a.chunks;
    double* const tops = a.tops + (long)b * a.chunks;
    Best top{-__builtin_huge_val(), kNever, 0};
    const int c1 = min(a.chunks, (part + 1) * a.part_chunks);
    for (int c = part * a.part_chunks + wave; c < c1; c += kWaves) {
        Chunk<DT> k[kMassSteps];
#pragma unroll
        for (int s = 0; s < kMassSteps; ++s) k[s] = load_chunk<DT>(a, row, c, s);
        float most = -__builtin_huge_valf(), apart = 0.f;
#pragma unroll
        for (int s = 0; s < kMassSteps; ++s) {
            float g[kVec], d[kVec];
            unpack_chunk<DT>(k[s], g, d);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                most = fmaxf(most, rec_exponent(a, g[i], d[i], 0.f));
                apart = fmaxf(apart, fabsf(d[i]));
            }
            if (a.greedy) {
                float sp[kVec], sm[kVec];
                unpack(k[s].sp, sp);
                unpack(k[s].sm, sm);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const double h = rec_logit(a, g[i], sp[i], sm[i]);
                    if (h > top.h) top = Best{h, k[s].id + i, 0};
                }
            }
        }
        for (int d = 1; d < kWave; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, kWave));
        // a reference near the largest exponent; a chunk of masked tokens has any
        const float E = fmaxf(fminf(ceilf(most), 3e38f), -3e38f);
        float s = 0.f, steered = 0.f;
#pragma unroll
        for (int u = 0; u < kMassSteps; ++u) {
            float g[kVec], d[kVec], e[kVec];
            unpack_chunk<DT>(k[u], g, d);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                e[i] = exp2_hw(rec_exponent(a, g[i], d[i], E));
                steered = fmaf(e[i], fabsf(d[i]), steered);
            }
            s += tree_sum(e);
        }
        const double all = wave_sum_f64((double)s), share = (double)wave_sum_f32(steered) * (double)a.steer_size;
        // the largest term is at least a half and no sum infinite, or the exponents are not what they are taken for
        const bool holds = !a.by_logit && fabsf(E) <= kFar && all >= 0.25 && all < 1e6 && share <= kSteerMean * all && !__ballot(!(apart <= a.steer_most));
        Mass m{E, (float)all};
        bool none = false;
        if (__builtin_expect(!holds && most == -__builtin_huge_valf(), 0)) {  // masked tokens alone, or none, as behind the last vector; or logits beyond what fp32 holds
            float g_most = most;
#pragma unroll
            for (int u = 0; u < kMassSteps; ++u) {
                float g[kVec];
                unpack(k[u].g, g);
                g_most = fmaxf(g_most, largest(g));
            }
            none = !__ballot(g_most > most);
        }
        if (none) {
            m = Mass{0.f, 0.f};
        } else if (__builtin_expect(!holds, 0)) {
            double sum;
            const double h = chunk_by_logit<DT>(a, row, c, sum);
            m = h > -__builtin_huge_val() ? Mass{kByLogit, (float)sum} : Mass{0.f, 0.f};
            if (lane == 0) put(tops + c, h);
        }
        if (lane == 0) put(masses + c, m);
    }
    if (a.greedy) {
        for (int d = 1; d < kWave; d <<= 1) {
            const double h = __shfl_xor(top.h, d, kWave);
            const int id = __shfl_xor(top.id, d, kWave);
            if (h > top.h || (h == top.h && id < top.id)) top = Best{h, id, 0};
        }
        if (lane == 0) best[wave] = top;
        __syncthreads();
        if (tid == 0) {
            for (int v = 1; v < kWaves; ++v)
                if (best[v].h > top.h || (best[v].h == top.h && best[v].id < top.id)) top = best[v];
            put(a.best + (long)b * a.parts + part, top);
        }
    }
    delivered();
    __syncthreads();
    if (a.parts > 1) {  // the last of the sequence's workgroups goes on
        if (tid == 0) before_us = atomicAdd(reinterpret_cast<int*>(a.arrive + (long)b * kArriveBytes), 1);
        __syncthreads();
        if (before_us + 1 < a.parts) return;
    }
    // all masses at the largest reference
    static_assert(sizeof(Mass) <= sizeof(double) && SS_MAX_VOCAB / 4 / kMassVecs + 1 <= SS_MAX_K + 1, "space for a row's masses");
    Mass* const table = reinterpret_cast<Mass*>(space_of(w));
    float E = -__builtin_huge_valf();
    for (int c = tid; c < a.chunks; c += kVerifyGroup) {
        const Mass m = get(masses + c);
        table[c] = m;
        if (m.s > 0.f) E = fmaxf(E, m.E);
    }
    for (int d = 1; d < kWave; d <<= 1) E = fmaxf(E, __shfl_xor(E, d, kWave));
    if (lane == 0) sum[wave] = (double)E;
    __syncthreads();
    for (int v = 0; v < kWaves; ++v) E = fmaxf(E, (float)sum[v]);
    // Of a row some of whose chunks are relative to logits all of them are moved to the largest logit, in double.
    const bool by_logit = E == kByLogit;
    double high = -__builtin_huge_val();
    const auto logit_of = [&](Mass m, int c) { return m.E == kByLogit ? get(tops + c) : (double)m.E / a.c64; };
    if (__builtin_expect(by_logit, 0)) {
        for (int c = tid; c < a.chunks; c += kVerifyGroup)
            if (table[c].s > 0.f) high = fmax(high, logit_of(table[c], c));
        for (int d = 1; d < kWave; d <<= 1) high = fmax(high, __shfl_xor(high, d, kWave));
        __syncthreads();
        if (lane == 0) sum[wave] = high;
        __syncthreads();
        for (int v = 0; v < kWaves; ++v) high = fmax(high, sum[v]);
        for (int c = tid; c < a.chunks; c += kVerifyGroup) {
            const Mass m = table[c];
            table[c] = __builtin_bit_cast(Mass, m.s > 0.f ? (double)m.s * exp2((logit_of(m, c) - high) * a.c64) : 0.0);
        }
        __syncthreads();
    }
    const auto mass = [&](Mass m) { return by_logit ? __builtin_bit_cast(double, m) : m.s > 0.f ? moved((double)m.s, m.E, E) : 0.0; };
    // a lane's chunks lie next to each other, so that the lanes' sums are in order
    const int each = (a.chunks + kVerifyGroup - 1) / kVerifyGroup, lo = min(a.chunks, tid * each), hi = min(a.chunks, lo + each);
    double mine = 0.0;
    for (int c = lo; c < hi; ++c) mine += mass(table[c]);
    const double incl = wave_incl_scan_f64(mine);
    __syncthreads();
    if (lane == 63) sum[wave] = incl;
    __syncthreads();
    double Z = 0.0, before = incl - mine;
    for (int v = 0; v < kWaves; ++v) {
        if (v < wave) before += sum[v];
        Z += sum[v];
    }
    const double log2Z = (by_logit ? 0.0 : (double)E) + log2(Z);  // relative to `high`, or whole
    if (a.greedy) {
        if (tid == 0) {
            Best t = get(a.best + (long)b * a.parts);
            for (int v = 1; v < a.parts; ++v) {
                const Best o = get(a.best + (long)b * a.parts + v);
                if (o.h > t.h || (o.h == t.h && o.id < t.id)) t = o;
            }
            a.next_token[b] = min(t.id, a.V - 1);
            if (a.next_logprob) a.next_logprob[b] = (float)(((by_logit ? t.h - high : t.h) * a.c64 - log2Z) * kLn2);
        }
        return;
    }
    const double target = (double)a.uniforms[(long)b * (a.N + 1) + a.N] * Z;
    // the chunk whose masses pass the target, or the last with any
    {
        double cum = before;
        int found = kNever, last = -1;
        double start = 0.0;
        for (int c = lo; c < hi; ++c) {
            const double m = mass(table[c]);
            if (m > 0.0) last = c;
            if (found == kNever && m > 0.0 && cum + m > target) {
                found = c;
                start = cum;
            }
            cum += m;
        }
        for (int d = 1; d < kWave; d <<= 1) last = max(last, __shfl_xor(last, d, kWave));
        const unsigned long long any = __ballot(found != kNever);
        const int L = any ? first_lane(any) : 0;
        found = __shfl(found, L, kWave);
        start = __shfl(start, L, kWave);
        __syncthreads();
        if (lane == 0) {
            w.scan[wave] = found;
            sum[wave] = start;
            last_of[wave] = last;
        }
        __syncthreads();
    }
    int chunk = kNever, last_chunk = 0;
    double start = 0.0;
    for (int v = kWaves - 1; v >= 0; --v)
        if (w.scan[v] != kNever) {
            chunk = w.scan[v];
            start = sum[v];
        }
    for (int v = 0; v < kWaves; ++v) last_chunk = max(last_chunk, last_of[v]);
    const bool take_last = chunk == kNever;
    if (take_last) chunk = last_chunk;
    if (wave != 0) return;
    // wave 0 goes over the chunk again, in the order of its tokens
    const Mass of_chunk = by_logit ? get(masses + chunk) : table[chunk];
    const float cE = of_chunk.E;
    const double c_top = by_logit ? logit_of(of_chunk, chunk) : 0.0, scale = by_logit ? exp2((c_top - high) * a.c64) : moved(1.0, cE, E);
    if (__builtin_expect(cE == kByLogit, 0)) {
        double h;
        const int token = token_by_logit<DT>(a, row, chunk, c_top, scale, start, target, take_last, h);
        if (lane == 0) {
            a.next_token[b] = min(max(token, 0), a.V - 1);
            if (a.next_logprob) a.next_logprob[b] = (float)(((h - high) * a.c64 - log2Z) * kLn2);
        }
        return;
    }
    Chunk<DT> k[kMassSteps];
#pragma unroll
    for (int s = 0; s < kMassSteps; ++s) k[s] = load_chunk<DT>(a, row, chunk, s);
    // all its steps' sums at once, the token in the step that passes the target
    double in[kMassSteps], from[kMassSteps + 1];
    from[0] = start;
#pragma unroll
    for (int s = 0; s < kMassSteps; ++s) {
        float g[kVec], d[kVec];
        double own = 0.0;
        unpack_chunk<DT>(k[s], g, d);
#pragma unroll
        for (int i = 0; i < kVec; ++i) own += (double)exp2_hw(rec_exponent(a, g[i], d[i], cE));
        in[s] = wave_incl_scan_f64(own * scale);
    }
#pragma unroll
    for (int s = 0; s < kMassSteps; ++s) from[s + 1] = from[s] + wave_last_f64(in[s]);
    int first = kMassSteps;
#pragma unroll
    for (int s = kMassSteps - 1; s >= 0; --s)
        if (!take_last && from[s + 1] > target) first = s;
    int token = -1;
    double y_token = 0.0;
    // of step s the first token that passes the target, or the last one with any mass
    const auto look = [&](int s, bool last) {
        Chunk<DT> now = k[0];
        double cum = from[0], incl = in[0];
#pragma unroll
        for (int v = 1; v < kMassSteps; ++v)
            {
                now.g = either(s == v, k[v].g, now.g);
                now.sp = either(s == v, k[v].sp, now.sp);
                now.sm = either(s == v, k[v].sm, now.sm);
                now.id = s == v ? k[v].id : now.id;
                cum = s == v ? from[v] : cum;
                incl = s == v ? in[v] : incl;
            }
        cum += wave_shift_up_f64(incl);
        float g[kVec], d[kVec], sp[kVec], sm[kVec], g_hit = 0.f, sp_hit = 0.f, sm_hit = 0.f;
        int hit = -1;
        unpack_chunk<DT>(now, g, d);
        unpack(now.sp, sp);
        unpack(now.sm, sm);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float e = exp2_hw(rec_exponent(a, g[i], d[i], cE));
            cum += (double)e * scale;
            if (e > 0.f && (last || (hit < 0 && cum > target))) {
                hit = now.id + i;
                g_hit = g[i];
                sp_hit = sp[i];
                sm_hit = sm[i];
            }
        }
        const unsigned long long hits = __ballot(hit >= 0);
        if (!hits) return;
        const int L = last ? 63 - __clzll((long long)hits) : first_lane(hits);
        token = __shfl(hit, L, kWave);
        y_token = __shfl(by_logit ? (rec_logit(a, g_hit, sp_hit, sm_hit) - high) * a.c64 : rec_exponent64(a, g_hit, sp_hit, sm_hit), L, kWave);
    };
    for (int s = first; s < kMassSteps && token < 0; ++s) look(s, false);
    for (int s = kMassSteps - 1; s >= 0 && token < 0; --s) look(s, true);
    token = max(token, 0);
    if (lane == 0) {
        a.next_token[b] = min(token, a.V - 1);
        if (a.next_logprob) a.next_logprob[b] = (float)((y_token - log2Z) * kLn2);
    }
}

__global__ void clear_kernel(char* arrive, int B) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) *reinterpret_cast<int*>(arrive + (long)b * kArriveBytes) = 0;
}

}  // namespace

extern "C" {

size_t specsteer_tree_verify_workspace_bytes(const ss_params* params) {
    long st, sb;
    return verify_shape(params, st, sb) == SS_OK ? verify_plan(*params, device_cu_count()).bytes : 0;
}

ss_status specsteer_tree_verify(const void* G, const void* S_ctx, const void* S_noctx, const int32_t* tokens, const int32_t* parents,
                                const int32_t* tree_len, const float* uniforms, const ss_params* params, int32_t* accepted_len, int32_t* path,
                                int32_t* next_token, float* next_token_logprob, void* workspace, size_t workspace_bytes, void* stream) {
    long st, sb;
    const ss_status chk = verify_shape(params, st, sb);
    if (chk != SS_OK) return chk;
    if (params->batch == 0) return SS_OK;
    const bool nodes = params->k_max > 0;
    if (!G || !S_ctx || !S_noctx || !uniforms || !accepted_len || !next_token || (nodes && (!tokens || !path))) return SS_ERR_NULL;
    if (shared({accepted_len, next_token, next_token_logprob, nodes ? path : nullptr}, {tree_len, uniforms, nodes ? tokens : nullptr, nodes ? parents : nullptr})) return SS_ERR_PARAM;
    const uintptr_t elem = params->dtype == SS_BF16 ? 1 : 3;
    if ((reinterpret_cast<uintptr_t>(G) | reinterpret_cast<uintptr_t>(S_ctx) | reinterpret_cast<uintptr_t>(S_noctx)) & elem) return SS_ERR_STRIDE;
    const VerifyPlan p = verify_plan(*params, device_cu_count());
    if (bad_workspace(workspace, workspace_bytes, p.bytes)) return SS_ERR_WORKSPACE;
    ss_loss_params lp{params->batch, params->k_max + 1, params->vocab, params->dtype, 0, 0, 0, 0, params->temperature, 1.f};
    const Rows r = make_rows(G, nullptr, nullptr, tokens, nullptr, lp, LossShape{});
    char* const ws = static_cast<char*>(workspace);
    VerifyArgs a{};
    a.G = G;
    a.Sp = S_ctx;
    a.Sm = S_noctx;
    a.tokens = tokens;
    a.parents = nodes ? parents : nullptr;
    a.tree_len = tree_len;
    a.uniforms = uniforms;
    a.accepted_len = accepted_len;
    a.path = path;
    a.next_token = next_token;
    a.next_logprob = next_token_logprob;
    a.cursors = reinterpret_cast<Cursor*>(ws);
    a.arrive = ws + p.off_arrive;
    a.sums = reinterpret_cast<Total<Sum>*>(ws + p.off_sums);
    a.logits = reinterpret_cast<float2*>(ws + p.off_logits);
    a.masses = reinterpret_cast<Mass*>(ws + p.off_masses);
    a.tops = reinterpret_cast<double*>(ws + p.off_masses) + (long)params->batch * p.chunks;
    a.best = reinterpret_cast<Best*>(ws + p.off_best);
    a.sb = sb;
    a.st = st;
    a.B = params->batch;
    a.N = params->k_max;
    a.V = params->vocab;
    a.c = r.c;
    a.c64 = r.c64;
    a.lambda = (double)params->lambda;
    a.beta = (double)params->beta;
    a.steer_hi = (float)(a.beta * a.c64);
    a.steer_lo = (float)(a.beta * a.c64 - (double)a.steer_hi);
    const double steer_size = std::fabs(a.beta * a.c64);
    a.steer_size = (float)steer_size;
    a.steer_most = params->beta == 0.f ? __builtin_huge_valf() : (float)std::fmin((double)kFar / steer_size, 3e38);
    a.far = r.far;
    // factors that fp32 does not hold
    a.by_logit = r.far || (params->beta != 0.f && !(steer_size > 1e-30 && steer_size < 1e30));
    a.greedy = (params->flags & SS_FLAG_GREEDY) ? 1 : 0;
    a.plain = params->beta == 0.f ? 1 : 0;
    a.slices = p.slices;
    a.slice_vecs = p.slice_vecs;
    a.chunks = p.chunks;
    a.parts = p.parts;
    a.part_chunks = p.part_chunks;
    hipStream_t q = static_cast<hipStream_t>(stream);
    if (p.stages == 0 && p.parts > 1) launch(clear_kernel, dim3((unsigned)((a.B + 255) / 256)), dim3(256), 0, q, a.arrive, a.B);
    const bool bf = params->dtype == SS_BF16, small = params->k_max <= kSmall;
    const auto rows = bf ? small ? rows_kernel<SS_BF16, SmallShared> : rows_kernel<SS_BF16, WalkShared> : small ? rows_kernel<SS_F32, SmallShared> : rows_kernel<SS_F32, WalkShared>;
    const auto draw = bf ? small ? draw_kernel<SS_BF16, SmallShared> : draw_kernel<SS_BF16, WalkShared> : small ? draw_kernel<SS_F32, SmallShared> : draw_kernel<SS_F32, WalkShared>;
    for (int k = 0; k < p.stages; ++k)
        launch(rows, dim3((unsigned)a.B * (unsigned)(p.groups[k] * 2 * p.slices)), dim3(kVerifyGroup), 0, q, (const VerifyArgs)a, (const int)k,
               (const int)(k ? p.rows[k - 1] : 0), (const int)p.rows[k], (const int)p.groups[k]);
    launch(draw, dim3((unsigned)a.B * (unsigned)p.parts), dim3(kVerifyGroup), 0, q, (const VerifyArgs)a, (const int)p.stages,
           (const int)(p.stages ? p.rows[p.stages - 1] : 0));
    return tree_launched();
}

}  // extern "C"
