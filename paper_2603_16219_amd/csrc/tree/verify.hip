// The verify-and-recover step down a tree of drafts, for MI355X (gfx950); include/specsteer_tree.h says what it computes.
//
// The rows that the walk comes through are known only as it goes, and a row is read by many workgroups.  A tree is therefore taken in stages
// (verify_plan.h): one sums some rows at and below the cursor, of G and S_noctx, whichever way the walk may take there; the next one's workgroups
// each walk over those sums for themselves, from what lies in LDS by then, and sum the rows that follow.  The last launch walks to the
// end, forms the recovery row's masses a chunk of 4 vectors a lane at a time, and the workgroup of a sequence that comes last draws the token.
//
// A walk: with d_r = log2 sum of G's row - log2 sum of S_noctx's, node i at row r = parent + 1 is accepted if
//     u_i <= 2^((G_y - S_y) c - d_r) / lambda;
// every row's first accepted child is found at once, and the walk follows them.
#include "../loss/loss_rows.h"
#include "tree_common.h"
#include "verify_plan.h"

namespace {

struct Cursor {
    int cur, n, done, pad;  // done: 1 at the walk's end, 2 of a sequence that is marked
};
struct Mass {
    float E, s;
};
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
    Best* best;           // [B][parts]
    long sb, st;
    int B, N, V;
    Factor c;
    double c64, inv_tau, lambda, beta;
    int far, greedy, plain;  // plain: beta is 0
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

template <int DT>
__device__ __forceinline__ double log2_sum(const VerifyArgs& a, int b, int r, int x, Total<Sum> s, WalkShared& w) {
    const bool far = a.far || is_far(s);
    if (far) {
        const void* const h = row_ptr<DT>(x ? a.Sm : a.G, b * a.sb + r * a.st);
        __syncthreads();
        s = far_sum<DT, Sum>(h, nullptr, a.V, a.c64, kVerifyGroup, w.part);
    }
    return (far ? (double)s.E * a.c64 : (double)s.E) + log2(s.s);
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
    if (__syncthreads_or(far))
        for (int k = 0; k < n; ++k) {  // rows far from zero, by the whole workgroup
            const int r = w.rows[k];
            double lse[2];
            for (int x = 0; x < 2; ++x) {
                Total<Sum> s;
                clear_total(s);
                for (int l = 0; l < a.slices; ++l) {
                    const Total<Sum> o = a.sums[(((long)b * (a.N + 1) + r) * 2 + x) * a.slices + l];
                    const float E = fmaxf(s.E, o.E);
                    s.s = moved(s.s, s.E, E) + moved(o.s, o.E, E);
                    s.E = E;
                }
                lse[x] = log2_sum<DT>(a, b, r, x, s, w);
            }
            if (tid == 0) w.diff[r] = lse[0] - lse[1];
        }
    __syncthreads();
    for (int i = tid; i < N; i += kVerifyGroup) {
        const int r = w.parent[i] + 1;
        if (w.first[r] < 0) continue;
        const float2 h = a.logits[(long)b * a.N + i];
        const double u = a.uniforms[(long)b * (a.N + 1) + i];
        // masked by G: never accepted; by S_noctx alone: always
        const double alpha = h.x == -__builtin_huge_valf() ? -1.0 : exp2(((double)h.x - (double)h.y) * a.c64 - w.diff[r]) / a.lambda;
        if (u <= 1.0 && !(u > alpha)) atomicMin(&w.first[r], i);
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

// Stage `stage`: the sums of one slice of some of its rows.
template <int DT>
__global__ __launch_bounds__(kVerifyGroup) void rows_kernel(const VerifyArgs a, const int stage, const int rows_before, const int rows, const int groups) {
    __shared__ WalkShared w;
    const int per = groups * 2 * a.slices, b = (int)(blockIdx.x / (unsigned)per), id = (int)(blockIdx.x - (unsigned)(b * per));
    const int slice = id % a.slices, x = id / a.slices & 1, group = id / (2 * a.slices);
    const bool leader = id == 0;
    const int N = reach<DT>(a, b, stage, rows_before, leader, w);
    if (leader && threadIdx.x == 0) {
        a.cursors[(long)stage * a.B + b] = w.at;
        if (stage == 0 && a.parts > 1) *reinterpret_cast<int*>(a.arrive + (long)b * kArriveBytes) = 0;
    }
    if (w.at.done) return;
    pick_rows(a, N, w.at.cur, rows, w);
    for (int k = group; k < w.count; k += groups) {
        const int r = w.rows[k];
        const void* const h = row_ptr<DT>(x ? a.Sm : a.G, b * a.sb + r * a.st);
        const Layout<DT> lay(h, a.V, threadIdx.x);
        const int begin = min(lay.vecs, slice * a.slice_vecs), end = slice + 1 == a.slices ? lay.vecs : min(lay.vecs, begin + a.slice_vecs);
        const Sum mine = lane_sum<DT, Sum, 2, true>(h, nullptr, lay, begin + threadIdx.x, end, kVerifyGroup, slice == 0, a.c);
        if (slice == 0)
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
// Eq. 8's exponent, in double
__device__ __forceinline__ double rec_exponent(const VerifyArgs& a, float g, float sp, float sm) {
    return a.plain ? (double)g * a.c64 : fma((double)g, a.c64, steer(sp, sm) * (a.beta * a.c64));
}

// Chunk `c` of a row by a wave: each lane's logits, -inf where there are none, and the first one's id.  The last chunk has the elements behind the
// last vector, one a lane.
template <int DT>
__device__ __forceinline__ int load_chunk(const VerifyArgs& a, const RecoveryRow<DT>& row, int c, int step, float (&g)[Row<DT>::kVec],
                                          float (&sp)[Row<DT>::kVec], float (&sm)[Row<DT>::kVec]) {
    constexpr int kVec = Row<DT>::kVec;
    const int lane = threadIdx.x & 63, vecs = a.V / kVec;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        g[i] = -__builtin_huge_valf();
        sp[i] = sm[i] = 0.f;
    }
    if (c + 1 < a.chunks) {
        const int v = c * kMassVecs + step * kWave + lane;
        if (v < vecs) {
            unpack(ld_raw<DT, kVec>(row.g, v), g);
            if (!a.plain) {
                unpack(ld_raw<DT, kVec>(row.sp, v), sp);
                unpack(ld_raw<DT, kVec>(row.sm, v), sm);
            }
        }
        return v * kVec;
    }
    const int at = vecs * kVec + lane;
    if (step == 0 && at < a.V) {
        g[0] = ld_elem<DT>(row.g, at);
        if (!a.plain) {
            sp[0] = ld_elem<DT>(row.sp, at);
            sm[0] = ld_elem<DT>(row.sm, at);
        }
    }
    return at;
}
constexpr int kMassSteps = kMassVecs / kWave;

template <int DT>
__global__ __launch_bounds__(kVerifyGroup) void draw_kernel(const VerifyArgs a, const int stages, const int rows_before) {
    constexpr int kVec = Row<DT>::kVec, kWaves = kVerifyGroup / kWave;
    __shared__ WalkShared w;
    __shared__ Best best[kWaves];
    __shared__ double sum[kWaves];
    __shared__ int pick[4];
    __shared__ Mass held[kVerifyGroup];
    const int b = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)(b * a.parts));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool leader = part == 0;
    reach<DT>(a, b, stages, rows_before, leader, w);
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
    Best top{-__builtin_huge_val(), kNever, 0};
    const int c1 = min(a.chunks, (part + 1) * a.part_chunks);
    for (int c = part * a.part_chunks + wave; c < c1; c += kWaves) {
        double y[kMassSteps][kVec];
        float most = -__builtin_huge_valf();
#pragma unroll
        for (int s = 0; s < kMassSteps; ++s) {
            float g[kVec], sp[kVec], sm[kVec];
            const int id = load_chunk<DT>(a, row, c, s, g, sp, sm);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                y[s][i] = rec_exponent(a, g[i], sp[i], sm[i]);
                most = fmaxf(most, (float)y[s][i]);
            }
            if (a.greedy)
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const double h = a.plain ? (double)g[i] : __dadd_rn((double)g[i], __dmul_rn(a.beta, steer(sp[i], sm[i])));
                    if (h > top.h) top = Best{h, id + i, 0};
                }
        }
        for (int d = 1; d < kWave; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, kWave));
        // a reference near the largest exponent; a chunk of masked tokens has any
        const float E = fmaxf(fminf(ceilf(most), 3e38f), -3e38f);
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kMassSteps; ++k) {
            float e[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) e[i] = exp2_hw((float)(y[k][i] - (double)E));
            s += tree_sum(e);
        }
        const double all = wave_sum_f64((double)s);
        if (lane == 0) masses[c] = Mass{E, (float)all};
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
            a.best[(long)b * a.parts + part] = top;
        }
    }
    __threadfence();
    __syncthreads();
    if (a.parts > 1) {  // the last of the sequence's workgroups goes on
        if (tid == 0) pick[0] = atomicAdd(reinterpret_cast<int*>(a.arrive + (long)b * kArriveBytes), 1);
        __syncthreads();
        if (pick[0] + 1 < a.parts) return;
        __threadfence();
    }
    // all masses at the largest reference
    float E = -__builtin_huge_valf();
    for (int c = tid; c < a.chunks; c += kVerifyGroup) {
        const Mass m = masses[c];
        if (m.s > 0.f) E = fmaxf(E, m.E);
    }
    for (int d = 1; d < kWave; d <<= 1) E = fmaxf(E, __shfl_xor(E, d, kWave));
    if (lane == 0) sum[wave] = (double)E;
    __syncthreads();
    for (int v = 0; v < kWaves; ++v) E = fmaxf(E, (float)sum[v]);
    const auto mass = [&](Mass m) { return m.s > 0.f ? (double)m.s * exp2((double)m.E - (double)E) : 0.0; };
    // a lane's chunks lie next to each other, so that the lanes' sums are in order
    const int each = (a.chunks + kVerifyGroup - 1) / kVerifyGroup, lo = min(a.chunks, tid * each), hi = min(a.chunks, lo + each);
    double mine = 0.0;
    for (int c = lo; c < hi; ++c) mine += mass(masses[c]);
    const double incl = wave_incl_scan_f64(mine);
    __syncthreads();
    if (lane == 63) sum[wave] = incl;
    if (tid == 0) pick[1] = pick[2] = -1;
    __syncthreads();
    double Z = 0.0, before = incl - mine;
    for (int v = 0; v < kWaves; ++v) {
        if (v < wave) before += sum[v];
        Z += sum[v];
    }
    const double log2Z = (double)E + log2(Z);
    if (a.greedy) {
        if (tid == 0) {
            Best t = a.best[(long)b * a.parts];
            for (int v = 1; v < a.parts; ++v) {
                const Best o = a.best[(long)b * a.parts + v];
                if (o.h > t.h || (o.h == t.h && o.id < t.id)) t = o;
            }
            a.next_token[b] = min(t.id, a.V - 1);
            if (a.next_logprob) a.next_logprob[b] = (float)((t.h * a.c64 - log2Z) * kLn2);
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
            const double m = mass(masses[c]);
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
            held[wave] = Mass{0.f, __int_as_float(last)};
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
    for (int v = 0; v < kWaves; ++v) last_chunk = max(last_chunk, __float_as_int(held[v].s));
    const bool take_last = chunk == kNever;
    if (take_last) chunk = last_chunk;
    if (wave != 0) return;
    // wave 0 goes over the chunk again, a vector a lane at a time
    const double cE = (double)masses[chunk].E, scale = exp2(cE - (double)E);
    int token = -1, last = 0;
    double y_token = 0.0, y_last = 0.0;
    for (int s = 0; s < kMassSteps && token < 0; ++s) {
        float g[kVec], sp[kVec], sm[kVec];
        const int id = load_chunk<DT>(a, row, chunk, s, g, sp, sm);
        double y[kVec], e[kVec], own = 0.0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            y[i] = rec_exponent(a, g[i], sp[i], sm[i]);
            e[i] = (double)exp2_hw((float)(y[i] - cE)) * scale;
            own += e[i];
        }
        const double in = wave_incl_scan_f64(own);
        double cum = start + (in - own);
        int hit = -1, some = -1;
        double y_hit = 0.0, y_some = 0.0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            cum += e[i];
            if (e[i] > 0.0) {
                some = id + i;
                y_some = y[i];
                if (hit < 0 && !take_last && cum > target) {
                    hit = id + i;
                    y_hit = y[i];
                }
            }
        }
        const unsigned long long hits = __ballot(hit >= 0), somes = __ballot(some >= 0);
        if (hits) {
            const int L = first_lane(hits);
            token = __shfl(hit, L, kWave);
            y_token = __shfl(y_hit, L, kWave);
        }
        if (somes) {
            const int L = 63 - __clzll((long long)somes);
            last = __shfl(some, L, kWave);
            y_last = __shfl(y_some, L, kWave);
        }
        start += wave_last_f64(in);
    }
    if (token < 0) {
        token = last;
        y_token = y_last;
    }
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
    a.best = reinterpret_cast<Best*>(ws + p.off_best);
    a.sb = sb;
    a.st = st;
    a.B = params->batch;
    a.N = params->k_max;
    a.V = params->vocab;
    a.c = r.c;
    a.c64 = r.c64;
    a.inv_tau = r.inv_tau;
    a.lambda = (double)params->lambda;
    a.beta = (double)params->beta;
    a.far = r.far;
    a.greedy = (params->flags & SS_FLAG_GREEDY) ? 1 : 0;
    a.plain = params->beta == 0.f ? 1 : 0;
    a.slices = p.slices;
    a.slice_vecs = p.slice_vecs;
    a.chunks = p.chunks;
    a.parts = p.parts;
    a.part_chunks = p.part_chunks;
    hipStream_t q = static_cast<hipStream_t>(stream);
    const bool bf = params->dtype == SS_BF16;
    if (p.stages == 0 && p.parts > 1)
        launch(clear_kernel, dim3((unsigned)((a.B + 255) / 256)), dim3(256), 0, q, a.arrive, a.B);
    for (int k = 0; k < p.stages; ++k)
        launch(bf ? rows_kernel<SS_BF16> : rows_kernel<SS_F32>, dim3((unsigned)a.B * (unsigned)(p.groups[k] * 2 * p.slices)), dim3(kVerifyGroup), 0, q, (const VerifyArgs)a, (const int)k,
               (const int)(k ? p.rows[k - 1] : 0), (const int)p.rows[k], (const int)p.groups[k]);
    launch(bf ? draw_kernel<SS_BF16> : draw_kernel<SS_F32>, dim3((unsigned)a.B * (unsigned)p.parts), dim3(kVerifyGroup), 0, q, (const VerifyArgs)a, (const int)p.stages,
           (const int)(p.stages ? p.rows[p.stages - 1] : 0));
    return tree_launched();
}

}  // extern "C"
