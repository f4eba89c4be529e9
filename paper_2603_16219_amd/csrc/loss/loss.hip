// The losses over full-vocabulary logits for MI355X (gfx950); include/specsteer_loss.h says what they compute.
// loss_rows.h has the arithmetic of a row.
#include "loss_rows.h"

namespace {

// ------------------------------------------------------------------ token log-probs

// Threads of a workgroup that sums a row, and of one for a row of up to kShortVecs vectors, where half as many waves start for nothing at rows
// that do not count (8192 of 16384 rows of V = 32000 bf16 104 us in 512, 98 in 256; 1024 rows of V = 151936 50 in either).
constexpr int kRowThreads = 512, kShortThreads = 256, kShortVecs = 4096;
constexpr int kMaxThreads = kWave * kUnitWaves;

struct ScoreArgs {
    Rows r;
    float* logprobs;    // or NULL
    float* stats;       // or NULL
    double* logprob64;  // or NULL
    long keep_from;     // rows from here on are read through the caches, for a gradient that reads them again soon,
    int if_sparse;      // if few enough of them count
};

// Whether few enough of the rows from keep_from on count, by 64 of them at multiples of the golden ratio, which fall anywhere in sequences of any
// length and are the same for all workgroups.
__device__ __forceinline__ bool sparse(const ScoreArgs& a) {
    const unsigned long of = (unsigned)((threadIdx.x & 63) + 1) * 2654435769u;
    const uint8_t m = a.r.mask[a.keep_from + (long)((unsigned long)(a.r.rows - a.keep_from) * of >> 32)];
    return __popcll(__ballot(m != 0)) <= kSparse;
}

__device__ __forceinline__ void write_score(const ScoreArgs& a, long row, double lp, float E, double s) {
    if (a.logprobs) a.logprobs[row] = (float)lp;
    if (a.logprob64) a.logprob64[row] = lp;
    if (a.stats) {
        a.stats[2 * row] = E;
        a.stats[2 * row + 1] = (float)s;
    }
}
// A row far from zero, which has the negative of its sum in the statistics, by the whole workgroup.
template <int DT>
__device__ __forceinline__ void score_far_row(const ScoreArgs& a, long row, int threads, Total<Sum>* part) {
    long at, grad_at;
    place(a.r, row, at, grad_at);
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const Total<Sum> s = far_sum<DT, Sum>(h, nullptr, a.r.V, a.r.c64, threads, part);
    if (threadIdx.x == 0) {
        const int y = a.r.tokens[row];
        write_score(a, row, token_logprob<2>(a.r, true, y, y >= 0 && y < a.r.V ? ld_elem<DT>(h, y) : 0.f, s.E, s.s), s.E, -s.s);
    }
}

// One workgroup a row, past the caches: 1024 rows of V = 151936 bf16 50 us (6.2 TB/s), 56 through them; fp32 6.6 TB/s.  Bound by the memory:
// the exponentials of bf16 rows take half the arithmetic units' time.
template <int DT>
__global__ __launch_bounds__(kMaxThreads) void score_kernel(const ScoreArgs a) {
    __shared__ Total<Sum> part[kUnitWaves];
    const int threads = blockDim.x;
    const long row = this_row();
    if (row >= a.r.rows) return;
    if (!counts(a.r, row)) {
        if (threadIdx.x == 0) write_score(a, row, 0.0, 0.f, 1.0);
        return;
    }
    long at, grad_at;
    place(a.r, row, at, grad_at);
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const Layout<DT> lay(h, a.r.V, threadIdx.x);
    const bool keep = row >= a.keep_from && (!a.if_sparse || sparse(a));
    const Sum mine = keep ? lane_sum<DT, Sum, 2, false>(h, nullptr, lay, threadIdx.x, lay.vecs, threads, true, a.r.c)
                          : lane_sum<DT, Sum, 2, true>(h, nullptr, lay, threadIdx.x, lay.vecs, threads, true, a.r.c);
    const Total<Sum> s = block_total(mine, threads, part);
    if (a.r.far || is_far(s)) {
        score_far_row<DT>(a, row, threads, part);
    } else if (threadIdx.x == 0) {
        const int y = a.r.tokens[row];
        write_score(a, row, token_logprob<2>(a.r, false, y, y >= 0 && y < a.r.V ? ld_elem<DT>(h, y) : 0.f, s.E, s.s), s.E, s.s);
    }
}

// ------------------------------------------------------------------ few rows: several workgroups each

constexpr int kSliceThreads = 256;

struct Slices {
    void* parts;          // the sums of every row's slices, Total<S> each
    float* token_logits;  // of every row: the gradient may replace the logits before all workgroups have read them
    int n, vecs;          // slices a row, vectors a slice
};
template <typename S>
__device__ __forceinline__ Total<S>* parts_of(const Slices& p, long row) { return static_cast<Total<S>*>(p.parts) + row * p.n; }

template <int DT, typename S>
__global__ __launch_bounds__(kSliceThreads) void slice_kernel(const Rows r, const Slices p) {
    static_assert(sizeof(Total<S>) <= kPartBytes, "space for a slice's sums");
    __shared__ Total<S> part[kSliceThreads / kWave];
    const long row = blockIdx.x / (unsigned)p.n;
    const int slice = (int)(blockIdx.x - row * p.n);
    if (!counts(r, row)) return;
    long at, grad_at;
    place(r, row, at, grad_at);
    const void* const h = row_ptr<DT>(r.logits, at);
    const void* const z = std::is_same<S, SumRef>::value ? row_ptr<DT>(r.ref, at) : nullptr;
    const Layout<DT> lay(h, r.V, threadIdx.x);
    const int end = slice + 1 == p.n ? lay.vecs : min(lay.vecs, (slice + 1) * p.vecs);
    const S mine = lane_sum<DT, S, 2>(h, z, lay, slice * p.vecs + threadIdx.x, end, kSliceThreads, slice == 0, r.c);
    const Total<S> s = block_total(mine, kSliceThreads, part);
    if (threadIdx.x == 0) {
        parts_of<S>(p, row)[slice] = s;
        if (slice == 0) {
            const int y = r.tokens[row];
            p.token_logits[row] = y >= 0 && y < r.V ? ld_elem<DT>(h, y) : 0.f;
        }
    }
}

template <typename S>
__device__ __forceinline__ Total<S> join_slices(const Slices& p, long row) {
    const int lane = threadIdx.x & 63;
    return join(parts_of<S>(p, row)[lane < p.n ? lane : 0], p.n);
}

// The log-prob of a row in slices, by one wave; true if the row is far from zero, and has none yet then.
template <int DT>
__device__ __forceinline__ bool score_joined(const ScoreArgs& a, const Slices& p, long row) {
    const bool first = (threadIdx.x & 63) == 0;
    if (!counts(a.r, row)) {
        if (first) write_score(a, row, 0.0, 0.f, 1.0);
        return false;
    }
    const Total<Sum> s = join_slices<Sum>(p, row);
    if (a.r.far || is_far(s)) return true;
    if (first) write_score(a, row, token_logprob<2>(a.r, false, a.r.tokens[row], p.token_logits[row], s.E, s.s), s.E, s.s);
    return false;
}

template <int DT>
__global__ __launch_bounds__(kSliceThreads) void score_slices_kernel(const ScoreArgs a, const Slices p) {
    constexpr int kWaves = kSliceThreads / kWave;
    __shared__ Total<Sum> part[kWaves];
    __shared__ int far_rows[kWaves];
    const long first = (long)blockIdx.x * kWaves;
    const int wave = threadIdx.x >> 6;
    const bool far = first + wave < a.r.rows && score_joined<DT>(a, p, first + wave);
    if ((threadIdx.x & 63) == 0) far_rows[wave] = far ? 1 : 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        if (far_rows[w]) score_far_row<DT>(a, first + w, kSliceThreads, part);
}

// ------------------------------------------------------------------ gradient from known statistics

struct GradArgs {
    Rows r;
    const float* stats;
    const float* weight;      // of every row's log-prob, or NULL:
    const double* seq_weight; // of the first P sequences' log-probs, the other P have the negative
    int pairs;
    int slices;               // workgroups a row
};
// A workgroup takes this much of a row, four vectors a lane, all in flight at once, and is gone: stores of one workgroup and loads of the next
// overlap better than in longer ones.  2048 rows of V = 128256 bf16 169 us in these (6.2 TB/s), 178 in halves, 181 in twice as much, 203 a
// workgroup of 512 a row; of V = 50257 fp32, 4096 rows, 281, 281, 320, 361.
constexpr int kGradThreads = 256, kGradVecs = kGradThreads * 4;

template <int DT>
__global__ __launch_bounds__(kGradThreads) void grad_kernel(const GradArgs a) {
    // from the last row on: what the sums' sweep read last may be in the caches still
    const long id = a.r.rows * a.slices - 1 - this_row();
    if (id < 0) return;
    const long row = (unsigned)id / (unsigned)a.slices;
    const int slice = (int)(id - row * a.slices);
    long at, grad_at;
    place(a.r, row, at, grad_at);
    void* const g = const_cast<void*>(row_ptr<DT>(a.r.grad, grad_at));
    const Layout<DT> lay(g, a.r.V, threadIdx.x);
    const int first = slice * kGradVecs + threadIdx.x, end = slice + 1 == a.slices ? lay.vecs : min(lay.vecs, (slice + 1) * kGradVecs);
    if (!counts(a.r, row)) {
        zero_slice<DT>(g, lay, first, end, kGradThreads, slice == 0);
        return;
    }
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const int y = a.r.tokens[row], b = (int)((unsigned)row / (unsigned)a.r.T);
    double w = a.weight ? (double)a.weight[row] : b < a.pairs ? a.seq_weight[b] : -a.seq_weight[b - a.pairs];
    w *= a.r.scale;
    if (y < 0 || y >= a.r.V) w = nan64();
    const float s = a.stats[2 * row + 1];
    const bool far = s < 0.f;
    const RowGrad rg = row_grad<DT, false, 2>(a.r, far, a.stats[2 * row], fabsf(s), w, 0.0, 0.0);
    if (far) {
        if (slice == 0) far_grad<DT, false>(h, nullptr, g, a.r, rg, y, kGradThreads);
        return;
    }
    write_grad<DT, false, true>(h, nullptr, g, lay, rg, y, first, end, kGradThreads, slice == 0, a.r.c);
}

// ------------------------------------------------------------------ policy loss

struct PolicyArgs {
    Rows r;
    const float* old_logprobs;
    const float* ref_logprobs;  // or NULL
    const float* advantages;
    const double* norm;  // what a token of each sequence counts, or NULL: norm_all, or one over the tokens that count
    double norm_all;
    int count;  // the rows form their number themselves
    double clip_lo, clip_hi, kl_coef;
    int seq_advantages;
    float* logprobs;  // or NULL
    float* kl;        // or NULL
    double* terms;    // every row's share of the loss
    float* loss;
};

struct RowLoss {
    double lp, kl, term, g, k, mean;
};

// What a token of the row counts, by any one wave.
__device__ __forceinline__ double row_norm(const PolicyArgs& a, long row) { return a.norm ? a.norm[(unsigned)row / (unsigned)a.r.T] : a.norm_all; }
__device__ __forceinline__ double token_norm(const PolicyArgs& a, long row) {
    return a.count ? 1.0 / (double)wave_count(a.r.mask, a.r.rows) : row_norm(a, row);  // the row itself counts
}

// A row's log-prob, KL and share of the loss, and their gradients, from its sums; hy is its token's logit.
template <bool REF, int PARTS, typename S>
__device__ __forceinline__ RowLoss row_loss(const PolicyArgs& a, bool far, long row, int y, float hy, float old, float advantage, double n,
                                               const Total<S>& s) {
    RowLoss o;
    const double adv = advantage;
    o.lp = token_logprob<PARTS>(a.r, far, y, hy, s.E, s.s);
    o.kl = o.k = o.mean = 0.0;
    const double ratio = exp(o.lp - (double)old);
    const double plain = ratio * adv, bound = fmin(fmax(ratio, a.clip_lo), a.clip_hi) * adv;
    const bool clipped = plain > bound;  // NaN: not clipped, and NaN below
    o.term = clipped ? -bound : -plain;
    o.g = clipped ? 0.0 : -plain;
    if constexpr (REF) {
        divergence<PARTS>(a.r, far, s, o.mean, o.kl);
        o.k = a.kl_coef;
    } else if (a.ref_logprobs) {
        const double d = (double)a.ref_logprobs[row] - o.lp, e = expm1(d);
        o.kl = d == __builtin_huge_val() ? d : e - d;  // a token of probability zero: e^d outgrows d
        if (a.kl_coef != 0.0) o.g -= a.kl_coef * e;
    }
    if (a.kl_coef != 0.0) o.term += a.kl_coef * o.kl;
    o.term *= n;
    o.g *= n * a.r.scale;
    o.k *= n * a.r.scale;
    return o;
}

__device__ __forceinline__ float advantage_of(const PolicyArgs& a, long row) {
    return a.advantages[a.seq_advantages ? (unsigned)row / (unsigned)a.r.T : row];
}
__device__ __forceinline__ void write_policy(const PolicyArgs& a, long row, double lp, double kl) {
    if (a.logprobs) a.logprobs[row] = (float)lp;
    if (a.kl) a.kl[row] = (float)kl;
}
// The same written down, and what the gradient needs.
template <int DT, bool REF, typename S>
__device__ __forceinline__ RowGrad finish_row(const PolicyArgs& a, bool far, long row, int y, float hy, float old, float advantage, double n,
                                             const Total<S>& s) {
    const RowLoss o = row_loss<REF, 1>(a, far, row, y, hy, old, advantage, n, s);
    write_policy(a, row, o.lp, o.kl);
    a.terms[row] = o.term;
    return row_grad<DT, REF, 1>(a.r, far, s.E, s.s, o.g, o.k, o.mean);
}

// The compiler is not to keep anything it has formed of a held vector (its logits widened, twice the registers) for the next use.
__device__ __forceinline__ void forget(uint4& r) { asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w)); }
__device__ __forceinline__ void forget(float4& r) { asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w)); }

struct RowShared {
    RowGrad grad;
    int far;
};

// One workgroup a row, which it reads once: its lanes keep their first NV vectors in registers from the sums to the gradient.  Of longer
// rows the rest is read again, first in the gradient since it was read last in the sums.  The last wave has no part of the row: it forms what
// is formed once a row, whose double arithmetic beside the held vectors would not fit the registers.
// Bound by the memory's bandwidth; what a workgroup stores and what another loads overlap, so that holding as much as a compute unit can is
// worth more than reading less again.  4096 rows of V = 128256 bf16 394 us a call (5.3 TB/s, a large copy reaches 4.8 to 5.3; swept
// twice 498), of V = 32000 95 (147).  8, 12, 16 and 20 vectors a lane were measured: 20 gains 3 % at V = 256000 and loses 4 at 151936.
template <int DT, bool REF, int NV>
__global__ __launch_bounds__(kMaxThreads) void policy_kernel(const PolicyArgs a) {
    using S = typename std::conditional<REF, SumRef, Sum>::type;
    using Raw = typename Row<DT>::Raw;
    constexpr int kVec = Row<DT>::kVec, kElem = DT == SS_BF16 ? 2 : 4, kHeldRef = REF ? NV : 1;
    __shared__ Total<S> part[kUnitWaves];
    __shared__ RowShared shared;
    const int tid = threadIdx.x, threads = (int)blockDim.x - kWave;  // of those that hold the row
    const bool helper = __builtin_amdgcn_readfirstlane(tid >= threads ? 1 : 0) != 0;
    const long row = this_row();
    if (row >= a.r.rows) return;
    long at, grad_at;
    place(a.r, row, at, grad_at);
    void* const g = a.r.grad ? const_cast<void*>(row_ptr<DT>(a.r.grad, grad_at)) : nullptr;
    if (!counts(a.r, row)) {
        if (g) {
            const Layout<DT> lay(g, a.r.V, tid);
            zero_slice<DT>(g, lay, tid, lay.vecs, blockDim.x, true);
        }
        if (tid == 0) {
            write_policy(a, row, 0.0, 0.0);
            a.terms[row] = 0.0;
        }
        return;
    }
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const void* const z = REF ? row_ptr<DT>(a.r.ref, at) : nullptr;
    const int y = a.r.tokens[row];
    const bool valid = y >= 0 && y < a.r.V;
    if (helper) {
        const float hy = valid ? ld_elem<DT>(h, y) : 0.f;
        const float old = a.old_logprobs[row], adv = advantage_of(a, row);
        const double n = token_norm(a, row);
        __syncthreads();
        const int lane = tid & 63, waves = threads / kWave;
        const Total<S> s = join(part[lane < waves ? lane : 0], waves);
        const bool far = a.r.far || is_far(s);
        if (lane == 0) {
            if (!far) shared.grad = finish_row<DT, REF>(a, false, row, y, hy, old, adv, n, s);
            shared.far = far ? 1 : 0;
        }
        __syncthreads();
    } else {
        const Layout<DT> lay(g ? g : h, a.r.V, tid);
        const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
        const char* const zv = REF ? static_cast<const char*>(z) + (long)lay.head * kElem : nullptr;
        // past the row's end the last vector again, which is masked below
        Raw r[NV], rz[kHeldRef];
        if (lay.vecs > 0) {
#pragma unroll
            for (int u = 0; u < NV; ++u) {
                const int first = min(u * threads, lay.vecs - 1);  // the same in all lanes: a scalar base and one offset a lane
                const unsigned off = (unsigned)min(tid, lay.vecs - 1 - first) * 16u;
                r[u] = ld_once_at<DT>(hv + (long)first * 16, off);
                if constexpr (REF) rz[u] = ld_once_at<DT>(zv + (long)first * 16, off);
            }
        }
        S sums;
        clear(sums);
#pragma unroll
        for (int u = 0; u < NV; u += 2) {  // one look at the reference for two vectors
            if (u * threads >= lay.vecs) break;
            float x[2][kVec], w[2][kVec];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                if ((u + v + 1) * threads > lay.vecs && tid >= lay.vecs - (u + v) * threads) {
                    r[u + v] = neg_inf_raw<DT, kVec>();
                    if constexpr (REF) rz[u + v] = r[u + v];
                }
                unpack(r[u + v], x[v]);
                if constexpr (REF) unpack(rz[u + v], w[v]);
            }
            if constexpr (REF) {
                raise(sums, fmaxf(largest(x[0]), largest(x[1])), fmaxf(largest(w[0]), largest(w[1])), a.r.c);
                add_under<1>(sums, x[0], w[0], a.r.c);
                add_under<1>(sums, x[1], w[1], a.r.c);
            } else {
                raise(sums, fmaxf(largest(x[0]), largest(x[1])), a.r.c);
                add_under<1>(sums, x[0], a.r.c);
                add_under<1>(sums, x[1], a.r.c);
            }
        }
        const S rest = lane_sum<DT, S, 1>(h, z, lay, tid + NV * threads, lay.vecs, threads, true, a.r.c);
        merge(sums, rest);
        const Total<S> mine = wave_total(sums);
        if ((tid & 63) == 0) part[tid >> 6] = mine;
        __syncthreads();
        __syncthreads();
        if (g && !shared.far) {
            const RowGrad rg = shared.grad;
            write_grad<DT, REF>(h, z, g, lay, rg, y, tid + NV * threads, lay.vecs, threads, true, a.r.c);
            char* const gv = static_cast<char*>(g) + (long)lay.head * kElem;
            // the token's element of a held vector is written again, by the lane that writes the vector
            const int e = y - lay.head, vec = e / kVec;
            const bool mine = valid && e >= 0 && vec < min(lay.vecs, NV * threads) && vec % threads == tid;
            const float hy = mine ? ld_elem<DT>(h, y) : 0.f, zy = REF && mine ? ld_elem<DT>(z, y) : 0.f;
            const auto write_held = [&](const Raw& raw, const Raw& rawz, int u) {
                float x[kVec], w[kVec];
                unpack(raw, x);
                if constexpr (REF) unpack(rawz, w);
#pragma unroll
                for (int j = 0; j < kVec; ++j) x[j] = grad_of<DT, REF>(rg, x[j], REF ? w[j] : 0.f, a.r.c);
                st_vec<DT>(gv + (long)(u * threads) * 16 + (unsigned)tid * 16u, 0, x);
            };
#pragma unroll
            for (int u = 0; u < NV; ++u) {
                if (u * threads >= lay.vecs) break;
                if (tid < lay.vecs - u * threads) {
                    forget(r[u]);
                    if constexpr (REF) forget(rz[u]);
                    write_held(r[u], rz[REF ? u : 0], u);
                }
            }
            if (mine) {
                asm volatile("" ::: "memory");
                st_elem<DT>(g, y, rg.at_token + grad_of<DT, REF>(rg, hy, zy, a.r.c));
            }
        }
    }
    if (shared.far) {
        const Total<S> s = far_sum<DT, S>(h, z, a.r.V, a.r.c64, blockDim.x, part);
        const double n = token_norm(a, row);
        if (tid == 0)
            shared.grad = finish_row<DT, REF>(a, true, row, y, valid ? ld_elem<DT>(h, y) : 0.f, a.old_logprobs[row],
                                              advantage_of(a, row), n, s);
        __syncthreads();
        const RowGrad rg = shared.grad;
        if (g) far_grad<DT, REF>(h, z, g, a.r, rg, y, blockDim.x);
    }
}

// The loss of rows in slices, and what each has once, by one workgroup: a group of lanes a row, a lane a slice.  Rows far from zero it does alone,
// their gradients among them, one after the other.
template <int DT, bool REF>
__device__ __forceinline__ void policy_slices_loss(const PolicyArgs& a, const Slices& p) {
    using S = typename std::conditional<REF, SumRef, Sum>::type;
    __shared__ Total<S> part[kSliceThreads / kWave];
    __shared__ double sums[kSliceThreads / kWave];
    __shared__ RowGrad shared_grad;
    __shared__ Total<S> joined[kSliceRows];
    __shared__ unsigned char far_rows[kSliceRows];
    static_assert(kSliceRows <= kSliceThreads, "a lane a row");
    const int tid = threadIdx.x, group = p.n <= 2 ? 2 : 1 << (32 - __clz(p.n - 1)), slice = tid & (group - 1);
    const double counted = a.count ? 1.0 / (double)wave_count(a.r.mask, a.r.rows) : 0.0;
#pragma unroll 2
    for (long first = 0; first < a.r.rows; first += kSliceThreads / group) {
        const long row = first + tid / group;
        Total<S> s;
        clear_total(s);
        if (row < a.r.rows && slice < p.n && counts(a.r, row)) s = parts_of<S>(p, row)[slice];
        s = join_group(s, group);
        if (row < a.r.rows && slice == 0) joined[row] = s;
    }
    __syncthreads();
    double loss = 0.0;
    bool any_far = false;
    if (tid < a.r.rows) {
        const bool kept = counts(a.r, tid);
        const Total<S> s = joined[tid];
        any_far = kept && (a.r.far || is_far(s));
        far_rows[tid] = any_far ? 1 : 0;
        if (!kept) {
            write_policy(a, tid, 0.0, 0.0);
        } else if (!any_far) {
            const RowLoss o = row_loss<REF, 2>(a, false, tid, a.r.tokens[tid], p.token_logits[tid], a.old_logprobs[tid], advantage_of(a, tid),
                                            a.count ? counted : row_norm(a, tid), s);
            write_policy(a, tid, o.lp, o.kl);
            loss = o.term;
        }
    }
    if (__syncthreads_or(any_far ? 1 : 0)) {
        for (long row = 0; row < a.r.rows; ++row) {
            if (!far_rows[row]) continue;
            long at, grad_at;
            place(a.r, row, at, grad_at);
            const void* const h = row_ptr<DT>(a.r.logits, at);
            const void* const z = REF ? row_ptr<DT>(a.r.ref, at) : nullptr;
            const int y = a.r.tokens[row];
            const Total<S> s = far_sum<DT, S>(h, z, a.r.V, a.r.c64, kSliceThreads, part);
            if (tid == 0) {
                const RowLoss o = row_loss<REF, 2>(a, true, row, y, p.token_logits[row], a.old_logprobs[row], advantage_of(a, row),
                                                a.count ? counted : row_norm(a, row), s);
                write_policy(a, row, o.lp, o.kl);
                loss += o.term;
                shared_grad = row_grad<DT, REF, 2>(a.r, true, s.E, s.s, o.g, o.k, o.mean);
            }
            __syncthreads();
            const RowGrad rg = shared_grad;
            if (a.r.grad) far_grad<DT, REF>(h, z, const_cast<void*>(row_ptr<DT>(a.r.grad, grad_at)), a.r, rg, y, kSliceThreads);
            __syncthreads();
        }
    }
    loss = block_sum(loss, sums);
    if (tid == 0) *a.loss = (float)loss;
}

// Rows in slices: the first workgroup forms the loss, the others, each with what its row has once formed for itself, a slice of the gradient.
template <int DT, bool REF>
__global__ __launch_bounds__(kSliceThreads) void policy_slices_kernel(const PolicyArgs a, const Slices p) {
    using S = typename std::conditional<REF, SumRef, Sum>::type;
    if (blockIdx.x == 0) {
        policy_slices_loss<DT, REF>(a, p);
        return;
    }
    const long row = (blockIdx.x - 1) / (unsigned)p.n;
    const int slice = (int)(blockIdx.x - 1 - row * p.n);
    long at, grad_at;
    place(a.r, row, at, grad_at);
    void* const g = const_cast<void*>(row_ptr<DT>(a.r.grad, grad_at));
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const void* const z = REF ? row_ptr<DT>(a.r.ref, at) : nullptr;
    const Layout<DT> lay(g, a.r.V, threadIdx.x);
    const int first = slice * p.vecs + threadIdx.x, end = slice + 1 == p.n ? lay.vecs : min(lay.vecs, (slice + 1) * p.vecs);
    if (!counts(a.r, row)) {
        zero_slice<DT>(g, lay, first, end, kSliceThreads, slice == 0);
        return;
    }
    // the first vectors are on their way while the row's sums are joined
    constexpr int kAhead = REF ? 2 : 4;
    typename Row<DT>::Raw r[kAhead], rz[kAhead];
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * (DT == SS_BF16 ? 2 : 4);
    const char* const zv = REF ? static_cast<const char*>(z) + (long)lay.head * (DT == SS_BF16 ? 2 : 4) : nullptr;
    if (lay.vecs > 0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = min(first + u * kSliceThreads, lay.vecs - 1);
            r[u] = ld_vec<DT>(hv, i);
            if constexpr (REF) rz[u] = ld_vec<DT>(zv, i);
        }
    }
    const Total<S> s = join_slices<S>(p, row);
    if (a.r.far || is_far(s)) return;
    const int y = a.r.tokens[row];
    const RowLoss o = row_loss<REF, 2>(a, false, row, y, p.token_logits[row], a.old_logprobs[row], advantage_of(a, row), token_norm(a, row), s);
    const RowGrad rg = row_grad<DT, REF, 2>(a.r, false, s.E, s.s, o.g, o.k, o.mean);
    write_grad<DT, REF>(h, z, g, lay, rg, y, first, end, kSliceThreads, slice == 0, a.r.c, kAhead, r, rz);
}

// ------------------------------------------------------------------ what is formed once a call

constexpr int kOneThreads = 1024;

// What a token of each sequence counts for the mean over tokens or over sequences: one workgroup, a wave a sequence or a lane a short one.
__global__ __launch_bounds__(kOneThreads) void norm_kernel(const uint8_t* mask, int B, int T, int seq_mean, double* norm) {
    __shared__ double part[kOneThreads / kWave];
    const bool short_ones = T <= kWave;
    const int lane = threadIdx.x & 63, step = short_ones ? kOneThreads : kOneThreads / kWave;
    double all = 0.0;  // tokens, or sequences that have any
    for (int b = short_ones ? threadIdx.x : threadIdx.x >> 6; b < B; b += step) {
        const uint8_t* const m = mask + (long)b * T;
        int n = 0;
        if (short_ones) {
            for (int t = 0; t < T; ++t) n += m[t] != 0 ? 1 : 0;
        } else {
            n = wave_count(m, T);
        }
        if (short_ones || lane == 0) {
            norm[b] = (double)n;
            all += seq_mean ? (n > 0 ? 1.0 : 0.0) : (double)n;
        }
    }
    all = block_sum(all, part);
    for (int b = threadIdx.x; b < B; b += kOneThreads) {
        const double n = norm[b];
        norm[b] = n == 0.0 ? 0.0 : seq_mean ? 1.0 / (n * all) : 1.0 / all;
    }
}

__global__ __launch_bounds__(kOneThreads) void sum_kernel(const double* terms, long n, double factor, float* loss) {
    __shared__ double part[kOneThreads / kWave];
    double x = 0.0;
    for (long i = threadIdx.x; i < n; i += kOneThreads) x += terms[i];
    x = block_sum(x, part);
    if (threadIdx.x == 0) *loss = (float)(x * factor);
}

struct PairArgs {
    const double* logprob64;
    const float* ref_logprobs;  // or NULL
    const uint8_t* mask;        // or NULL
    int pairs, T;
    double beta, smoothing, factor;  // factor: what a pair counts
    double* weight;  // [P] out: of the preferred sequence's log-probs
    double* loss64;  // [P] out
    float* loss;     // [P] out, or NULL
    float* margin;   // [P] out, or NULL
};

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

constexpr int kPairThreads = 256;

// One lane's share of what a sequence of a pair adds to their difference.
__device__ __forceinline__ double pair_side(const PairArgs& a, long p, int side, int first, int step) {
    const long at = (p + (side ? a.pairs : 0)) * (long)a.T;
    double x = 0.0;
#pragma unroll 4
    for (int t = first; t < a.T; t += step) {
        if (a.mask && a.mask[at + t] == 0) continue;
        const double d = a.logprob64[at + t] - (a.ref_logprobs ? (double)a.ref_logprobs[at + t] : 0.0);
        x += side ? -d : d;
    }
    return x;
}
// A pair's loss from the difference of its sequences' log ratios.
__device__ __forceinline__ double finish_pair(const PairArgs& a, long p, double x, bool write) {
    const double h = a.beta * x, e = a.smoothing;
    const double loss = (1.0 - e) * softplus(-h) + (e > 0.0 ? e * softplus(h) : 0.0);  // a margin of +inf costs nothing without smoothing
    const double dh = (e - 1.0) / (1.0 + exp(h)) + e / (1.0 + exp(-h));
    if (write) {
        a.weight[p] = a.beta * a.factor * dh;
        a.loss64[p] = loss;
        if (a.loss) a.loss[p] = (float)loss;
        if (a.margin) a.margin[p] = (float)h;
    }
    return loss;
}

__global__ __launch_bounds__(kPairThreads) void pair_kernel(const PairArgs a) {
    __shared__ double part[kPairThreads / kWave];
    const long p = blockIdx.x;
    double x = 0.0;
    for (int side = 0; side < 2; ++side) x += pair_side(a, p, side, threadIdx.x, kPairThreads);
    x = block_sum(x, part);
    if (threadIdx.x < kWave) finish_pair(a, p, x, threadIdx.x == 0);
}

// One workgroup for all pairs, a wave each, and the loss; rows in slices it joins first.
template <int DT>
__global__ __launch_bounds__(kOneThreads) void pairs_kernel(const ScoreArgs r, const Slices c, const PairArgs a, float* total) {
    constexpr int kWaves = kOneThreads / kWave;
    __shared__ Total<Sum> far_part[kWaves];
    __shared__ double part[kWaves];
    __shared__ int far_rows[kJoinRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (c.n > 1) {
        for (int row = wave; row < (int)r.r.rows; row += kWaves) {
            const bool far = score_joined<DT>(r, c, row);
            if (lane == 0) far_rows[row] = far ? 1 : 0;
        }
        __syncthreads();
        for (int row = 0; row < (int)r.r.rows; ++row)
            if (far_rows[row]) score_far_row<DT>(r, row, kOneThreads, far_part);
        __syncthreads();
    }
    double loss = 0.0;
    for (int p = wave; p < a.pairs; p += kWaves) {
        double x = 0.0;
        for (int side = 0; side < 2; ++side) x += pair_side(a, p, side, lane, kWave);
        x = wave_sum_f64(x);
        const double one = finish_pair(a, p, x, lane == 0);
        if (lane == 0) loss += one;
    }
    loss = block_sum(loss, part);
    if (threadIdx.x == 0) *total = (float)(loss * a.factor);
}

__global__ void zero_loss_kernel(float* loss) { *loss = 0.f; }

// ------------------------------------------------------------------ launches

// The sums of the rows' slices; false if there is one a row.
template <typename S>
bool launch_slices(const ss_loss_params& p, const Rows& r, const LossScratch& w, void* workspace, int slices, Slices& out, hipStream_t q) {
    const int vecs = row_vecs(p);
    out.n = slices;
    if (slices < 2) return false;
    out.vecs = (vecs + out.n - 1) / out.n;
    out.parts = static_cast<char*>(workspace) + w.parts;
    out.token_logits = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.token_logits);
    launch(p.dtype == SS_BF16 ? slice_kernel<SS_BF16, S> : slice_kernel<SS_F32, S>, dim3((unsigned)(r.rows * out.n)), dim3(kSliceThreads), 0, q, r, out);
    return true;
}

void launch_score(const ss_loss_params& p, const ScoreArgs& a, const LossScratch& w, void* workspace, hipStream_t q) {
    Slices c;
    if (launch_slices<Sum>(p, a.r, w, workspace, score_slices(a.r.rows, row_vecs(p)), c, q)) {
        constexpr long kRowsEach = kSliceThreads / kWave;
        launch(p.dtype == SS_BF16 ? score_slices_kernel<SS_BF16> : score_slices_kernel<SS_F32>, dim3((unsigned)((a.r.rows + kRowsEach - 1) / kRowsEach)),
               dim3(kSliceThreads), 0, q, a, c);
        return;
    }
    launch(p.dtype == SS_BF16 ? score_kernel<SS_BF16> : score_kernel<SS_F32>, row_grid(a.r.rows), dim3(a.r.rows <= device_cu_count() ? kMaxThreads : row_vecs(p) <= kShortVecs ? kShortThreads : kRowThreads), 0, q, a);
}

void launch_grad(const ss_loss_params& p, GradArgs& a, hipStream_t q) {
    const int vecs = row_vecs(p);
    a.slices = vecs > kGradVecs ? (vecs + kGradVecs - 1) / kGradVecs : 1;
    launch(p.dtype == SS_BF16 ? grad_kernel<SS_BF16> : grad_kernel<SS_F32>, row_grid(a.r.rows * a.slices), dim3(kGradThreads), 0, q, a);
}

// The loss is left to the caller to sum unless true comes back.
template <bool REF>
bool launch_policy(const ss_loss_params& p, const PolicyArgs& a, const LossScratch& w, void* workspace, hipStream_t q) {
    constexpr int kHeld = REF ? kHeldPairs : kHeldVecs;
    Slices c;
    const int vecs = row_vecs(p);
    if (launch_slices<typename std::conditional<REF, SumRef, Sum>::type>(p, a.r, w, workspace, row_slices(a.r.rows, vecs), c, q)) {
        const unsigned groups = 1 + (a.r.grad ? (unsigned)(a.r.rows * c.n) : 0u);
        launch(p.dtype == SS_BF16 ? policy_slices_kernel<SS_BF16, REF> : policy_slices_kernel<SS_F32, REF>, dim3(groups), dim3(kSliceThreads), 0, q, a, c);
        return true;
    }
    launch(p.dtype == SS_BF16 ? policy_kernel<SS_BF16, REF, kHeld> : policy_kernel<SS_F32, REF, kHeld>, row_grid(a.r.rows),
           dim3((unsigned)(kWave * call_waves(a.r.rows, device_cu_count(), vecs, kHeld))), 0, q, a);
    return false;
}

}  // namespace

extern "C" {

size_t specsteer_loss_workspace_bytes(const ss_loss_params* params) {
    LossShape s;
    return loss_shape(params, s) == SS_OK ? loss_scratch(*params).bytes : 0;
}

ss_status specsteer_token_logprobs(const void* logits, const int32_t* tokens, const uint8_t* mask, const ss_loss_params* params,
                                   float* logprobs, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    LossShape s;
    const ss_status chk = loss_shape(params, s);
    if (chk != SS_OK) return chk;
    if (s.rows == 0) return SS_OK;
    if (!logits || !tokens || !logprobs) return SS_ERR_NULL;
    if (off_element(logits, *params)) return SS_ERR_STRIDE;
    const LossScratch w = loss_scratch(*params);
    if (check_workspace(workspace, workspace_bytes, w.bytes) != SS_OK) return SS_ERR_WORKSPACE;
    const long kept = stats ? cached_rows(*params, s.rows, false).n : 0;
    const ScoreArgs a{make_rows(logits, nullptr, nullptr, tokens, mask, *params, s), logprobs, stats, nullptr, s.rows - kept, 0};
    launch_score(*params, a, w, workspace, static_cast<hipStream_t>(stream));
    return launched();
}

ss_status specsteer_token_logprobs_grad(const void* logits, const int32_t* tokens, const uint8_t* mask, const float* stats,
                                        const float* grad_logprobs, const ss_loss_params* params, void* grad_logits, void* stream) {
    LossShape s;
    const ss_status chk = loss_shape(params, s);
    if (chk != SS_OK) return chk;
    if (s.rows == 0) return SS_OK;
    if (!logits || !tokens || !stats || !grad_logprobs || !grad_logits) return SS_ERR_NULL;
    if (off_element(logits, *params) || off_element(grad_logits, *params)) return SS_ERR_STRIDE;
    GradArgs a{make_rows(logits, nullptr, grad_logits, tokens, mask, *params, s), stats, grad_logprobs, nullptr, 0, 0};
    launch_grad(*params, a, static_cast<hipStream_t>(stream));
    return launched();
}

ss_status specsteer_policy_loss(const void* logits, const void* ref_logits, const int32_t* tokens, const uint8_t* mask,
                                const float* old_logprobs, const float* ref_logprobs, const float* advantages,
                                const ss_loss_params* params, const ss_policy_params* policy, float* loss, float* logprobs, float* kl,
                                void* grad_logits, void* workspace, size_t workspace_bytes, void* stream) {
    LossShape s;
    ss_status chk = loss_shape(params, s);
    if (chk == SS_OK) chk = check_policy(policy);
    if (chk != SS_OK) return chk;
    if (!loss || (s.rows > 0 && (!logits || !tokens || !old_logprobs || !advantages))) return SS_ERR_NULL;
    if (ref_logits && ref_logprobs) return SS_ERR_PARAM;
    if (s.rows > 0 && (policy->kl_coef > 0.f || kl) && !ref_logits && !ref_logprobs) return SS_ERR_NULL;
    if (off_element(logits, *params) || off_element(ref_logits, *params) || off_element(grad_logits, *params)) return SS_ERR_STRIDE;
    const LossScratch w = loss_scratch(*params);
    if (check_workspace(workspace, workspace_bytes, w.bytes) != SS_OK) return SS_ERR_WORKSPACE;
    hipStream_t q = static_cast<hipStream_t>(stream);
    if (s.rows == 0) {
        launch(zero_loss_kernel, dim3(1), dim3(1), 0, q, loss);
        return launched();
    }
    PolicyArgs a;
    a.r = make_rows(logits, ref_logits, grad_logits, tokens, mask, *params, s);
    a.old_logprobs = old_logprobs;
    a.ref_logprobs = ref_logprobs;
    a.advantages = advantages;
    a.norm = nullptr;
    a.norm_all = (policy->flags & SS_LOSS_SUM) ? 1.0 : 1.0 / (double)s.rows;  // without a mask both means are this one
    a.clip_lo = 1.0 - (double)policy->clip_low;
    a.clip_hi = 1.0 + (double)policy->clip_high;
    a.kl_coef = (double)policy->kl_coef;
    a.seq_advantages = (policy->flags & SS_LOSS_SEQ_ADVANTAGES) ? 1 : 0;
    a.logprobs = logprobs;
    a.kl = kl;
    char* const base = static_cast<char*>(workspace);
    a.terms = reinterpret_cast<double*>(base + w.row_value);
    // the mean over tokens: each row counts them itself, beside its loads, up to 16 bytes of the mask 16 times a lane (a launch of its own 5 us)
    a.count = mask && !(policy->flags & (SS_LOSS_SUM | SS_LOSS_SEQ_MEAN)) && s.rows <= 16384 ? 1 : 0;
    if (mask && !(policy->flags & SS_LOSS_SUM) && !a.count) {
        double* const norm = reinterpret_cast<double*>(base + w.seq);
        launch(norm_kernel, dim3(1), dim3(kOneThreads), 0, q, mask, (int)params->batch, (int)params->length,
               (policy->flags & SS_LOSS_SEQ_MEAN) ? 1 : 0, norm);
        a.norm = norm;
    }
    a.loss = loss;
    const bool summed = ref_logits ? launch_policy<true>(*params, a, w, workspace, q) : launch_policy<false>(*params, a, w, workspace, q);
    if (!summed) launch(sum_kernel, dim3(1), dim3(kOneThreads), 0, q, static_cast<const double*>(a.terms), s.rows, 1.0, loss);
    return launched();
}

ss_status specsteer_preference_loss(const void* logits, const int32_t* tokens, const uint8_t* mask, const float* ref_logprobs,
                                    const ss_loss_params* params, const ss_preference_params* preference, float* loss, float* pair_loss,
                                    float* margin, float* logprobs, void* grad_logits, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    LossShape s;
    ss_status chk = loss_shape(params, s);
    if (chk == SS_OK) chk = check_preference(preference);
    if (chk != SS_OK) return chk;
    if (params->batch & 1) return SS_ERR_SHAPE;
    if (!loss || (s.rows > 0 && (!logits || !tokens))) return SS_ERR_NULL;
    if (off_element(logits, *params) || off_element(grad_logits, *params)) return SS_ERR_STRIDE;
    const LossScratch w = loss_scratch(*params);
    if (check_workspace(workspace, workspace_bytes, w.bytes) != SS_OK) return SS_ERR_WORKSPACE;
    hipStream_t q = static_cast<hipStream_t>(stream);
    const int pairs = params->batch / 2;
    if (pairs == 0) {
        launch(zero_loss_kernel, dim3(1), dim3(1), 0, q, loss);
        return launched();
    }
    char* const base = static_cast<char*>(workspace);
    double* const lp64 = reinterpret_cast<double*>(base + w.row_value);
    float* const stats = reinterpret_cast<float*>(base + w.stats);
    double *const weight = reinterpret_cast<double*>(base + w.seq), *const loss64 = weight + pairs;
    const Rows r = make_rows(logits, nullptr, grad_logits, tokens, mask, *params, s);
    const CachedRows kept = grad_logits ? cached_rows(*params, s.rows, mask != nullptr) : CachedRows{0, false};
    const ScoreArgs sa{r, logprobs, stats, lp64, s.rows - kept.n, kept.if_sparse ? 1 : 0};
    Slices c{nullptr, nullptr, 1, 0};
    const bool one = pairs_in_one(pairs, params->length), join = one && s.rows > 0 && s.rows <= kJoinRows && score_slices(s.rows, row_vecs(*params)) > 1;
    if (join) launch_slices<Sum>(*params, r, w, workspace, score_slices(s.rows, row_vecs(*params)), c, q);
    else if (s.rows > 0) launch_score(*params, sa, w, workspace, q);
    const double factor = (preference->flags & SS_LOSS_SUM) ? 1.0 : 1.0 / (double)pairs;
    PairArgs pa{lp64, ref_logprobs, mask, pairs, params->length, (double)preference->beta, (double)preference->label_smoothing, factor,
                weight, loss64, pair_loss, margin};
    if (one) launch(params->dtype == SS_BF16 ? pairs_kernel<SS_BF16> : pairs_kernel<SS_F32>, dim3(1), dim3(kOneThreads), 0, q, sa, c, pa, loss);
    else launch(pair_kernel, dim3((unsigned)pairs), dim3(kPairThreads), 0, q, pa);
    if (grad_logits && s.rows > 0) {
        GradArgs a{r, stats, nullptr, weight, pairs, 0};
        launch_grad(*params, a, q);
    }
    if (!one) launch(sum_kernel, dim3(1), dim3(kOneThreads), 0, q, static_cast<const double*>(loss64), (long)pairs, factor, loss);
    return launched();
}

const char* specsteer_loss_status_string(int status) {
    switch (status) {
        case SS_OK: return "ok";
        case SS_ERR_NULL: return "a required pointer is NULL";
        case SS_ERR_SHAPE: return "batch, length or vocab out of range, or an odd batch of pairs";
        case SS_ERR_DTYPE: return "unknown logits dtype";
        case SS_ERR_PARAM: return "temperature, coefficients or flags out of range, or two references";
        case SS_ERR_STRIDE: return "strides negative, rows that overlap, sequences that interleave, or a pointer off its element";
        case SS_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case SS_ERR_DEVICE: return "HIP launch failed";
        default: return "unknown status";
    }
}

}  // extern "C"
