// Entropies and top alternatives of rows of logits, and the gradient of the entropy, for MI355X (gfx950);
// include/specsteer_alternatives.h says what they compute, loss_rows.h has the arithmetic of a row.
//
// With t_v = h_v c - E, one pass forms beside the sum s = sum 2^t the cross term x = sum 2^t t:
//     H = (log2 s - x / s) ln 2,      dH/dh_v = -(P(v) / tau) (log P(v) + H),  log P(v) = (t_v - log2 s) ln 2.
// c is one fp32 number here; what it leaves out is made up for at the reference, as in the policy loss.
//
// The n likeliest tokens come from the same pass.  The lanes of a workgroup form n groups or more, each with the largest logit that it has
// met: the least of these is a lower bound of the n-th largest of the row, since n tokens reach it.  What reaches the bound goes to a list in
// LDS.  The bound rises as the pass goes on; about n ln n (1 + ln(rounds)) of a row's tokens ever reach it, half as many more where it is formed
// after rounds that double (1000 of 128256 for n = 64), and n ln n reach the last one, which are ranked against each other.  Waves read the others'
// bounds without waiting: an old one is lower, and
// holds.  A row with more ties than the lists hold is searched for its n-th largest logit a digit at a time.
#include "alternatives_plan.h"
#include "loss_rows.h"

namespace {

struct SumX {
    float E, s, x;
};
template <> struct Total<SumX> {
    float E;
    double s, x;
};
static_assert(sizeof(Total<SumX>) <= kAltPartBytes, "space for a slice's sums");

__device__ __forceinline__ void clear(SumX& a) { a.E = -kFar; a.s = a.x = 0.f; }
// The reference as high as logits up to `top` take.  A term moved by d has t - d in the cross term.
__device__ __forceinline__ void raise(SumX& a, float top, Factor c) {
    top = fmaf(top, c.hi, -kBelow);
    if (top > a.E) {
        const float to = fminf(ceilf(top), 2.f * kFar);
        a.s = moved(a.s, a.E, to);
        a.x = a.s > 0.f ? fmaf(a.s, a.E - to, moved(a.x, a.E, to)) : 0.f;
        a.E = to;
    }
}
template <int N>
__device__ __forceinline__ void add_under(SumX& a, const float (&h)[N], Factor c) {
    float e[N], x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = exponent<1>(h[i], a.E, c);
        e[i] = exp2_hw(t);
        x[i] = mul_or_zero(e[i], t);
    }
    a.s += tree_sum(e);
    a.x += tree_sum(x);
}
__device__ __forceinline__ bool is_far(const Total<SumX>& a) { return a.s == a.s && is_far(a.E); }
__device__ __forceinline__ double crossed_x(double x, double s, float by) { return s > 0.0 ? x - s * (double)by : 0.0; }
__device__ __forceinline__ Total<SumX> wave_total(const SumX& a) {
    Total<SumX> r;
    r.E = (float)wave_max_i32((int)a.E);
    const double s = (double)moved(a.s, a.E, r.E);
    r.s = wave_sum_f64(s);
    r.x = wave_sum_f64(crossed_x((double)moved(a.x, a.E, r.E), s, r.E - a.E));
    return r;
}
__device__ __forceinline__ Total<SumX> join(const Total<SumX>& a, int n) {
    const bool has = (int)(threadIdx.x & 63) < n;
    Total<SumX> r;
    r.E = (float)wave_max_i32((int)a.E);
    const double s = moved(a.s, a.E, r.E);
    r.s = wave_sum_f64(has ? s : 0.0);
    r.x = wave_sum_f64(has ? crossed_x(moved(a.x, a.E, r.E), s, r.E - a.E) : 0.0);
    return r;
}
// A row far from zero: E = m its largest logit, s = sum 2^((h - m) c), x = sum 2^((h - m) c) (h - m), by a workgroup.
template <int DT>
__device__ __forceinline__ Total<SumX> far_sum_x(const void* h, int V, double c, int threads, Total<SumX>* part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = threads / kWave;
    float m = -__builtin_huge_valf();
    for (int i = threadIdx.x; i < V; i += threads) m = fmaxf(m, ld_elem<DT>(h, i));
    for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
    __syncthreads();
    if (lane == 0) part[wave].E = m;
    __syncthreads();
    m = part[lane < waves ? lane : 0].E;
    for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
    double s = 0.0, x = 0.0;
    for (int i = threadIdx.x; i < V; i += threads) {
        const float v = ld_elem<DT>(h, i), e = far_term(v, m, c);
        s += (double)e;
        if (e > 0.f) x += (double)e * ((double)v - (double)m);
    }
    s = wave_sum_f64(s);
    x = wave_sum_f64(x);
    __syncthreads();
    if (lane == 0) {
        part[wave].s = s;
        part[wave].x = x;
    }
    __syncthreads();
    Total<SumX> r;
    r.E = m;
    r.s = wave_sum_f64(lane < waves ? part[lane].s : 0.0);
    r.x = wave_sum_f64(lane < waves ? part[lane].x : 0.0);
    __syncthreads();
    return r;
}
__device__ __forceinline__ double entropy_of(const Rows& r, bool far, const Total<SumX>& s) {
    const double h = far ? log(s.s) - s.x / s.s * r.inv_tau : (log2(s.s) - s.x / s.s * (1.0 + r.rest)) * kLn2;
    return h < 0.0 ? 0.0 : h;  // by rounding only
}

// ------------------------------------------------------------------ the likeliest tokens

// A token as one number: by increasing logit (the order of their bits, turned round for negative ones), then by decreasing id.  0 is no token's.
__device__ __forceinline__ unsigned ordered(float h) {
    const unsigned b = __float_as_uint(h + 0.f);  // -0 becomes 0
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ unsigned long long key_of(float h, int id) { return (unsigned long long)ordered(h) << 32 | (0xFFFFFFFFu - (unsigned)id); }
__device__ __forceinline__ float key_logit(unsigned long long k) { return unordered((unsigned)(k >> 32)); }
__device__ __forceinline__ int key_id(unsigned long long k) { return (int)(0xFFFFFFFFu - (unsigned)k); }

constexpr int kHits = 4096, kRanked = 1024;  // tokens that reached a bound, and the last one
constexpr int kRankedAtOnce = 8;
struct Finder {
    alignas(16) unsigned long long ranked[kRanked + kRankedAtOnce];
    int hits[kHits];  // ids
    float bound[kUnitWaves];  // of every wave
    int hit_count, ranked_count, digit, above;
};

// Only the id, which the shortlist reads the logit of again: to pick it out of the lane's vectors here took 50 us more for
// 1024 rows of 151936 in bf16 with n = 16.
__device__ __forceinline__ void push(Finder& f, int id) {
    const int at = atomicAdd(&f.hit_count, 1);
    if (at < kHits) f.hits[at] = id;
}
// The least of the groups' largest logits, over the wave.
__device__ __forceinline__ float wave_bound(float top, int group) {
    for (int d = 1; d < kWave; d <<= 1) {
        const float o = __shfl_xor(top, d, kWave);
        top = d < group ? fmaxf(top, o) : fminf(top, o);
    }
    return top;
}
__device__ __forceinline__ float block_bound(const Finder& f, int waves) {
    const volatile float* const b = f.bound;
    float v = b[0];
    for (int w = 1; w < waves; ++w) v = fminf(v, b[w]);
    return v;
}

// The elements of a row that a search goes over, by increasing id: [begin, hole) and what lies `gap` behind it, `end` - `begin` in all.
struct Span {
    int begin, end, hole, gap;
    __device__ __forceinline__ int id(int i) const { return i + (i < hole ? 0 : gap); }
};
// The n likeliest of a span into f.ranked, in no order, by a workgroup: the n-th largest logit a digit of 8 bits at a
// time, then those above it and the first ones equal to it.  For rows with more ties than the lists hold (all logits the same, say): up to five
// sweeps, a row of V = 128256 bf16 in about 0.1 ms.
template <int DT>
__device__ __forceinline__ void find_slowly(Finder& f, const void* h, Span span, int n, int threads) {
    int* const count = f.hits;
    const float lowest = -__builtin_huge_valf();
    unsigned prefix = 0, fixed = 0;  // digits of the n-th largest known so far
    int above = 0;                   // tokens above all that share them
    bool all = false;                // fewer than n tokens in all
    for (int shift = 24; shift >= (DT == SS_BF16 ? 16 : 0); shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += threads) count[i] = 0;
        __syncthreads();
        for (int i = span.begin + (int)threadIdx.x; i < span.end; i += threads) {
            const float v = ld_elem<DT>(h, span.id(i));
            const unsigned o = ordered(v);
            if (v > lowest && (o & fixed) == prefix) atomicAdd(&count[o >> shift & 255u], 1);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int d = 255, sum = above;
            while (d >= 0 && sum + count[d] < n) sum += count[d--];
            f.digit = d;
            f.above = sum;
        }
        __syncthreads();
        above = f.above;
        if (f.digit < 0) {  // in the first round only
            all = true;
            break;
        }
        prefix |= (unsigned)f.digit << shift;
        fixed |= 255u << shift;
    }
    if (DT == SS_BF16) prefix |= prefix >> 31 ? 0u : 0xFFFFu;  // a negative one's lower bits are turned round
    __syncthreads();
    if (threadIdx.x == 0) f.ranked_count = 0;
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = threads / kWave;
    int equal = 0;  // tokens equal to the n-th largest so far, the same in all lanes
    for (int first = span.begin; first < span.end; first += threads) {
        const int at = first + (int)threadIdx.x, i = span.id(at);
        const float v = at < span.end ? ld_elem<DT>(h, i) : lowest;
        const unsigned o = ordered(v);
        const bool over = v > lowest && (all || o > prefix), same = !all && v > lowest && o == prefix;
        if (over) f.ranked[atomicAdd(&f.ranked_count, 1)] = key_of(v, i);
        const unsigned long long ballot = __ballot(same);
        __syncthreads();
        if (lane == 0) count[wave] = __popcll(ballot);
        __syncthreads();
        int before = equal;
        for (int w = 0; w < waves; ++w) {
            before += w < wave ? count[w] : 0;
            equal += count[w];
        }
        before += __popcll(ballot & ((1ull << lane) - 1));
        if (same && above + before < n) f.ranked[atomicAdd(&f.ranked_count, 1)] = key_of(v, i);
    }
    __syncthreads();
}

// ------------------------------------------------------------------ the pass

struct AltArgs {
    Rows r;
    int topk, group;      // group: lanes of a group
    float* logprobs;      // or NULL
    float* entropy;       // or NULL
    int32_t* top_tokens;
    float* top_logprobs;
    float* stats;         // or NULL
    Total<SumX>* parts;   // of every row's slices
    unsigned long long* keys;
    int slices, slice_vecs;
    int keep;             // rows are read through the caches, for a gradient that reads them again soon
};

// A workgroup's share of a row: vectors [begin, end), and the elements outside of vectors if `extra`.  What may be among the n likeliest is in
// f.hits behind the next barrier.
template <int DT, bool TOP, bool ONCE>
__device__ __forceinline__ SumX scan(const AltArgs& a, const void* h, const Layout<DT>& lay, int begin, int end, bool extra, int threads, Finder* f) {
    constexpr int kVec = Row<DT>::kVec, kElem = DT == SS_BF16 ? 2 : 4, kUnroll = 4;
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
    const int waves = threads / kWave, wave = threadIdx.x >> 6;
    SumX sum;
    clear(sum);
    float top = -__builtin_huge_valf(), bound = top;
    if (TOP) {
        if (threadIdx.x == 0) f->hit_count = f->ranked_count = 0;
    }
    for (int i = begin, round = 0; i < end || round == 0; i += kUnroll * threads, ++round) {
        typename Row<DT>::Raw r[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int v = i + u * threads + (int)threadIdx.x;
            r[u] = neg_inf_raw<DT, kVec>();
            if (v < end) r[u] = ONCE ? ld_once<DT>(hv, v) : ld_vec<DT>(hv, v);
        }
        float x[kUnroll][kVec], m[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            unpack(r[u], x[u]);
            m[u] = largest(x[u]);
        }
        const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
        raise(sum, most, a.r.c);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) add_under(sum, x[u], a.r.c);
        if (TOP) {
            top = fmaxf(top, most);
            if ((round & (round - 1)) == 0) {  // it rises less and less; every round, 3 us more
                const float b = wave_bound(top, a.group);
                if ((threadIdx.x & 63) == 0) reinterpret_cast<volatile float*>(f->bound)[wave] = b;
                if (round == 0) __syncthreads();  // without the others' first bounds there is none
            }
            bound = fmaxf(block_bound(*f, waves), -3.402823466e38f);  // what is masked is none
            unsigned hit = 0;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (m[u] >= bound)
#pragma unroll
                    for (int j = 0; j < kVec; ++j) hit |= (x[u][j] >= bound ? 1u : 0u) << (u * kVec + j);
            for (; hit; hit &= hit - 1) {
                const int k = __ffs((int)hit) - 1;
                push(*f, lay.head + (i + k / kVec * threads + (int)threadIdx.x) * kVec + k % kVec);
            }
        }
    }
    if (TOP) {  // the last bound is that of all rounds: by one of five eighths of a row, one row in 300 had more tokens than the list holds, n = 64
        const float b = wave_bound(top, a.group);
        if ((threadIdx.x & 63) == 0) reinterpret_cast<volatile float*>(f->bound)[wave] = b;
    }
    if (extra && lay.extra >= 0) {
        const float x[1] = {ld_elem<DT>(h, lay.extra)};
        raise(sum, x[0], a.r.c);
        add_under(sum, x, a.r.c);
        if (TOP && x[0] >= bound) push(*f, lay.extra);
    }
    return sum;
}

// The hits that reach `least` into f.ranked; false if there are too many of either.
template <int DT>
__device__ __forceinline__ bool shortlist(Finder& f, const void* h, float least, int threads) {
    const int n = f.hit_count;
    if (n > kHits) return false;
    for (int i = threadIdx.x; i < n; i += threads) {
        const int id = f.hits[i];
        const float v = ld_elem<DT>(h, id);
        if (v >= least) {
            const int at = atomicAdd(&f.ranked_count, 1);
            if (at < kRanked) f.ranked[at] = key_of(v, id);
        }
    }
    __syncthreads();
    return f.ranked_count <= kRanked;
}
// out(rank, key) for the n first of f.ranked, or with the key 0 where there are fewer.  Each thread compares its key with all others, eight at a time: one by
// one, each waited for, the some 300 of a row with n = 64 took 8 us.
template <typename F>
__device__ __forceinline__ void rank(Finder& f, int n, int threads, F out) {
    const int count = f.ranked_count;
    if (threadIdx.x < kRankedAtOnce) f.ranked[count + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += threads) {
        const unsigned long long k = f.ranked[i];
        int before = 0;
        for (int j = 0; j < count; j += kRankedAtOnce) {
            unsigned long long o[kRankedAtOnce];
            __builtin_memcpy(o, __builtin_assume_aligned(f.ranked + j, 16), sizeof(o));
#pragma unroll
            for (int x = 0; x < kRankedAtOnce; ++x) before += o[x] > k ? 1 : 0;
        }
        if (before < n) out(before, k);
    }
    for (int i = count + threadIdx.x; i < n; i += threads) out(i, 0ull);
}

__device__ __forceinline__ void write_row(const AltArgs& a, long row, double lp, double H, float E, double s) {
    if (a.logprobs) a.logprobs[row] = (float)lp;
    if (a.entropy) a.entropy[row] = (float)H;
    if (a.stats) {
        a.stats[2 * row] = E;
        a.stats[2 * row + 1] = (float)s;
    }
}
__device__ __forceinline__ void write_none(const AltArgs& a, long row, int threads) {
    if (threadIdx.x == 0) write_row(a, row, 0.0, 0.0, 0.f, 1.0);
    for (int i = threadIdx.x; i < a.topk; i += threads) {
        a.top_tokens[row * a.topk + i] = -1;
        a.top_logprobs[row * a.topk + i] = -__builtin_huge_valf();
    }
}
// The given token and its logit, for the first thread, asked for beside other loads: behind the sums they are two round trips.
__device__ __forceinline__ int given_token(const AltArgs& a, long row) { return a.logprobs && threadIdx.x == 0 ? a.r.tokens[row] : -1; }
template <int DT>
__device__ __forceinline__ float given_logit(const AltArgs& a, const void* h, int y) { return y >= 0 && y < a.r.V ? ld_elem<DT>(h, y) : 0.f; }

// What is written of a row whose sums and, in f.ranked, likeliest tokens are known.
template <int DT, bool TOP>
__device__ __forceinline__ void finish(const AltArgs& a, long row, int y, float hy, bool far, const Total<SumX>& s, int threads, Finder* f) {
    if (threadIdx.x == 0) {
        const double lp = a.logprobs ? token_logprob<1>(a.r, far, y, hy, s.E, s.s) : 0.0;
        // the statistics are those of the whole c
        write_row(a, row, lp, entropy_of(a.r, far, s), s.E, far ? -s.s : s.s * exp2((double)s.E * a.r.rest));
    }
    if (TOP) {
        const float lowest = DT == SS_BF16 ? __uint_as_float(0xFF7F0000u) : -3.402823466e38f;
        const bool only_lowest = far && s.E <= lowest;
        rank(*f, a.topk, threads, [&](int at, unsigned long long k) {
            const float v = k ? key_logit(k) : -__builtin_huge_valf();
            const bool some = k && (v > lowest || only_lowest);
            a.top_tokens[row * a.topk + at] = some ? key_id(k) : -1;
            a.top_logprobs[row * a.topk + at] = some ? (float)token_logprob<1>(a.r, far, 0, v, s.E, s.s) : -__builtin_huge_valf();
        });
    }
}

// Bytes bound it: 1024 rows of 151936 in bf16 take 56 us without likeliest tokens, 5.6 TB/s, and 73 with 16 of them, 4.25 TB/s; 104 with 64.  Registers
// for four waves a SIMD hold two workgroups a unit, one of which computes while the other waits: with one it was 113 us.
constexpr int kAltThreads = 512;
template <int DT, bool TOP>
__global__ __launch_bounds__(kAltThreads) __attribute__((amdgpu_waves_per_eu(4))) void alternatives_kernel(const AltArgs a) {
    __shared__ Total<SumX> part[kAltThreads / kWave];
    __shared__ typename std::conditional<TOP, Finder, int>::type finder;
    Finder* const f = TOP ? reinterpret_cast<Finder*>(&finder) : nullptr;
    const long row = this_row();
    if (row >= a.r.rows) return;
    if (!counts(a.r, row)) {
        write_none(a, row, kAltThreads);
        return;
    }
    long at, grad_at;
    place(a.r, row, at, grad_at);
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const Layout<DT> lay(h, a.r.V, threadIdx.x);
    const int y = given_token(a, row);
    const SumX mine = a.keep ? scan<DT, TOP, false>(a, h, lay, 0, lay.vecs, true, kAltThreads, f) : scan<DT, TOP, true>(a, h, lay, 0, lay.vecs, true, kAltThreads, f);
    const float hy = given_logit<DT>(a, h, y);
    Total<SumX> s = block_total(mine, kAltThreads, part);
    const bool far = a.r.far || is_far(s);
    if (far) s = far_sum_x<DT>(h, a.r.V, a.r.c64, kAltThreads, part);
    if (TOP) {
        if (!shortlist<DT>(*f, h, block_bound(*f, kAltThreads / kWave), kAltThreads)) find_slowly<DT>(*f, h, Span{0, a.r.V, a.r.V, 0}, a.topk, kAltThreads);
    }
    finish<DT, TOP>(a, row, y, hy, far, s, kAltThreads, f);
}

// Few rows: several workgroups each, whose sums and likeliest tokens a second launch joins.
template <int DT, bool TOP>
__global__ __launch_bounds__(256) void alternatives_slice_kernel(const AltArgs a) {
    constexpr int kThreads = 256;
    __shared__ Total<SumX> part[kThreads / kWave];
    __shared__ typename std::conditional<TOP, Finder, int>::type finder;
    Finder* const f = TOP ? reinterpret_cast<Finder*>(&finder) : nullptr;
    const long row = blockIdx.x / (unsigned)a.slices;
    const int slice = (int)(blockIdx.x - row * a.slices);
    if (!counts(a.r, row)) return;
    long at, grad_at;
    place(a.r, row, at, grad_at);
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const Layout<DT> lay(h, a.r.V, threadIdx.x);
    const int begin = min(lay.vecs, slice * a.slice_vecs), end = slice + 1 == a.slices ? lay.vecs : min(lay.vecs, begin + a.slice_vecs);
    const SumX mine = scan<DT, TOP, false>(a, h, lay, begin, end, slice == 0, kThreads, f);
    const Total<SumX> s = block_total(mine, kThreads, part);
    if (threadIdx.x == 0) a.parts[row * a.slices + slice] = s;
    if (TOP) {
        unsigned long long* const keys = a.keys + (row * a.slices + slice) * a.topk;
        if (!shortlist<DT>(*f, h, block_bound(*f, kThreads / kWave), kThreads)) {
            // the first slice has the elements before and behind the vectors, as in the pass: whichever way the others go, each element is looked at once
            constexpr int kVec = Row<DT>::kVec;
            const int lo = lay.head + begin * kVec, hi = lay.head + end * kVec, tail = lay.head + lay.vecs * kVec;
            find_slowly<DT>(*f, h, slice == 0 ? Span{0, hi + a.r.V - tail, hi, tail - hi} : Span{lo, hi, hi, 0}, a.topk, kThreads);
        }
        rank(*f, a.topk, kThreads, [&](int i, unsigned long long k) { keys[i] = k; });
    }
}

template <int DT, bool TOP>
__global__ __launch_bounds__(256) void alternatives_join_kernel(const AltArgs a) {
    constexpr int kThreads = 256;
    __shared__ Total<SumX> part[kThreads / kWave];
    __shared__ typename std::conditional<TOP, Finder, int>::type finder;
    __shared__ unsigned least;
    Finder* const f = TOP ? reinterpret_cast<Finder*>(&finder) : nullptr;
    const long row = blockIdx.x;
    if (!counts(a.r, row)) {
        write_none(a, row, kThreads);
        return;
    }
    long at, grad_at;
    place(a.r, row, at, grad_at);
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const int lane = threadIdx.x & 63;
    // all that does not wait for anything is asked for at once
    const int y = given_token(a, row), count = a.slices * a.topk;
    const Total<SumX> sums = a.parts[row * a.slices + (lane < a.slices ? lane : 0)];
    if (TOP) {
        // each slice's q-th, q slices' worth of n: the least of them is reached by n tokens at least
        const unsigned long long* const keys = a.keys + row * a.slices * a.topk;
        const int q = (a.topk + a.slices - 1) / a.slices;
        const unsigned long long ahead = (int)threadIdx.x < count ? keys[threadIdx.x] : 0;
        unsigned o = lane < a.slices ? (unsigned)(keys[lane * a.topk + q - 1] >> 32) : 0xFFFFFFFFu;
        for (int d = 1; d < kWave; d <<= 1) o = min(o, (unsigned)__shfl_xor((int)o, d, kWave));
        if (threadIdx.x == 0) {
            least = o;
            f->ranked_count = 0;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < count; i += kThreads) {
            const unsigned long long k = i == (int)threadIdx.x ? ahead : keys[i];
            if (k && (unsigned)(k >> 32) >= least) {
                const int to = atomicAdd(&f->ranked_count, 1);
                if (to < kRanked) f->ranked[to] = k;
            }
        }
    }
    const float hy = given_logit<DT>(a, h, y);
    __syncthreads();
    Total<SumX> s = join(sums, a.slices);
    const bool far = a.r.far || is_far(s);
    if (far) s = far_sum_x<DT>(h, a.r.V, a.r.c64, kThreads, part);
    if (TOP && f->ranked_count > kRanked) find_slowly<DT>(*f, h, Span{0, a.r.V, a.r.V, 0}, a.topk, kThreads);
    finish<DT, TOP>(a, row, y, hy, far, s, kThreads, f);
}

// ------------------------------------------------------------------ gradient

struct AltGradArgs {
    Rows r;
    const float* stats;
    const float* entropy;        // or NULL without grad_entropy
    const float* grad_logprobs;  // or NULL
    const float* grad_entropy;   // or NULL
    int slices;                  // workgroups a row
};

// dL/dh_v = e_v (slope t_v + scale) + at_token 1[v = y],  e = 2^t, t = h c - E.  For a row far from zero t = (h - E) / tau in nats, in double.
struct AltRowGrad {
    float E, slope, scale, at_token;
};
__device__ __forceinline__ float alt_grad_of(const AltRowGrad& g, float h, Factor c) {
    const float t = exponent<1>(h, g.E, c);
    return mul_or_zero(exp2_hw(t), fmaf(t, g.slope, g.scale));
}

// As grad_kernel: a workgroup takes four vectors a lane, all in flight, and is gone; the last rows first.  Bound by bytes: 2048 rows of
// 128256 in bf16, 1281 of which count, 329 MB read and 525 written in 151 us, 5.7 TB/s.
template <int DT>
__global__ __launch_bounds__(256) void alternatives_grad_kernel(const AltGradArgs a) {
    constexpr int kThreads = 256, kUnroll = 4, kVec = Row<DT>::kVec, kElem = DT == SS_BF16 ? 2 : 4;
    const long id = a.r.rows * a.slices - 1 - this_row();
    if (id < 0) return;
    const long row = (unsigned)id / (unsigned)a.slices;
    const int slice = (int)(id - row * a.slices);
    long at, grad_at;
    place(a.r, row, at, grad_at);
    void* const out = const_cast<void*>(row_ptr<DT>(a.r.grad, grad_at));
    const Layout<DT> lay(out, a.r.V, threadIdx.x);
    const int begin = slice * kThreads * kUnroll + (int)threadIdx.x, end = slice + 1 == a.slices ? lay.vecs : min(lay.vecs, (slice + 1) * kThreads * kUnroll);
    if (!counts(a.r, row)) {
        zero_slice<DT>(out, lay, begin, end, kThreads, slice == 0);
        return;
    }
    const void* const h = row_ptr<DT>(a.r.logits, at);
    const int y = a.grad_logprobs ? a.r.tokens[row] : -1;
    double g = a.grad_logprobs ? (double)a.grad_logprobs[row] * a.r.scale : 0.0;
    const double k = a.grad_entropy ? (double)a.grad_entropy[row] * a.r.scale : 0.0;
    if (a.grad_logprobs && (y < 0 || y >= a.r.V)) g = nan64();
    const float stat = a.stats[2 * row + 1], E = a.stats[2 * row];
    const bool far = stat < 0.f;
    double s = fabsf(stat);
    if (!far) s *= exp2(-(double)E * a.r.rest);  // of terms with c as one number
    const double H = a.grad_entropy ? (double)a.entropy[row] : 0.0, f = a.r.inv_tau / s;
    AltRowGrad w;
    w.E = E;
    w.at_token = (float)(g * a.r.inv_tau);
    if (far) {
        w.slope = (float)(-k * f);
        w.scale = (float)(-(g + (k != 0.0 ? k * (H - log(s)) : 0.0)) * f);
        if (slice == 0)
            for (int i = threadIdx.x; i < a.r.V; i += kThreads) {
                const float v = ld_elem<DT>(h, i), e = far_term(v, E, a.r.c64);
                const float t = e > 0.f ? (float)(((double)v - (double)E) * a.r.inv_tau) : 0.f;
                st_elem<DT>(out, i, e * fmaf(t, w.slope, w.scale) + (i == y ? w.at_token : 0.f));
            }
        return;
    }
    w.slope = (float)(-k * f * kLn2 * (1.0 + a.r.rest));
    w.scale = (float)(-(g + (k != 0.0 ? k * (H - log2(s) * kLn2) : 0.0)) * f);
    // the lane that owns the token's element writes it again: its logit is read before anything of the row is overwritten
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
    char* const gv = static_cast<char*>(out) + (long)lay.head * kElem;
    const int of = y - lay.head, vec = of >= 0 && of < lay.vecs * kVec ? of / kVec : -1;
    const bool mine = vec >= 0 ? vec >= begin && vec < end && (vec - begin) % kThreads == 0 : slice == 0 && y >= 0 && lay.extra == y;
    const float mine_h = mine ? ld_elem<DT>(h, y) : 0.f;
    typename Row<DT>::Raw raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (begin + u * kThreads < end) raw[u] = ld_once<DT>(hv, begin + u * kThreads);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
        if (begin + u * kThreads < end) {
            float x[kVec];
            unpack(raw[u], x);
#pragma unroll
            for (int j = 0; j < kVec; ++j) x[j] = alt_grad_of(w, x[j], a.r.c);
            st_vec<DT>(gv, begin + u * kThreads, x);
        }
    if (slice == 0 && lay.extra >= 0) st_elem<DT>(out, lay.extra, alt_grad_of(w, ld_elem<DT>(h, lay.extra), a.r.c));
    if (mine) {
        asm volatile("" ::: "memory");  // behind the stores above, which cover this element too
        st_elem<DT>(out, y, w.at_token + alt_grad_of(w, mine_h, a.r.c));
    }
}

template <int DT, bool TOP>
void launch_alternatives(const ss_loss_params& p, AltArgs& a, const AltScratch& w, void* workspace, hipStream_t q) {
    const int vecs = row_vecs(p);
    a.slices = row_slices(a.r.rows, vecs);
    if (a.slices < 2) {
        a.group = group_lanes(kAltThreads, a.topk);
        launch(alternatives_kernel<DT, TOP>, row_grid(a.r.rows), dim3(kAltThreads), 0, q, (const AltArgs)a);
        return;
    }
    a.group = group_lanes(256, a.topk);
    a.slice_vecs = (vecs + a.slices - 1) / a.slices;
    a.parts = reinterpret_cast<Total<SumX>*>(static_cast<char*>(workspace) + w.parts);
    a.keys = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + w.keys);
    launch(alternatives_slice_kernel<DT, TOP>, dim3((unsigned)(a.r.rows * a.slices)), dim3(256), 0, q, (const AltArgs)a);
    launch(alternatives_join_kernel<DT, TOP>, dim3((unsigned)a.r.rows), dim3(256), 0, q, (const AltArgs)a);
}

}  // namespace

extern "C" {

size_t specsteer_token_alternatives_workspace_bytes(const ss_loss_params* params, int32_t topk) {
    LossShape s;
    return loss_shape(params, s) == SS_OK && topk >= 0 && topk <= SS_MAX_TOPK ? alt_scratch(*params, topk).bytes : 0;
}

ss_status specsteer_token_alternatives(const void* logits, const int32_t* tokens, const uint8_t* mask, const ss_loss_params* params, int32_t topk,
                                       float* logprobs, float* entropy, int32_t* top_tokens, float* top_logprobs, float* stats,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    LossShape s;
    const ss_status chk = loss_shape(params, s);
    if (chk != SS_OK) return chk;
    if (topk < 0 || topk > SS_MAX_TOPK) return SS_ERR_PARAM;
    if (s.rows == 0) return SS_OK;
    if (!logits || (logprobs && !tokens) || (topk > 0 && (!top_tokens || !top_logprobs))) return SS_ERR_NULL;
    if (off_element(logits, *params)) return SS_ERR_STRIDE;
    const AltScratch w = alt_scratch(*params, topk);
    if (check_workspace(workspace, workspace_bytes, w.bytes) != SS_OK) return SS_ERR_WORKSPACE;
    AltArgs a{};
    a.r = make_rows(logits, nullptr, nullptr, tokens, mask, *params, s);
    a.topk = topk;
    a.logprobs = logprobs;
    a.entropy = entropy;
    a.top_tokens = top_tokens;
    a.top_logprobs = top_logprobs;
    a.stats = stats;
    a.keep = stats && cached_rows(*params, s.rows, false).n == s.rows ? 1 : 0;
    hipStream_t q = static_cast<hipStream_t>(stream);
    if (params->dtype == SS_BF16) topk ? launch_alternatives<SS_BF16, true>(*params, a, w, workspace, q) : launch_alternatives<SS_BF16, false>(*params, a, w, workspace, q);
    else topk ? launch_alternatives<SS_F32, true>(*params, a, w, workspace, q) : launch_alternatives<SS_F32, false>(*params, a, w, workspace, q);
    return launched();
}

ss_status specsteer_token_alternatives_grad(const void* logits, const int32_t* tokens, const uint8_t* mask, const float* stats, const float* entropy,
                                            const float* grad_logprobs, const float* grad_entropy, const ss_loss_params* params, void* grad_logits,
                                            void* stream) {
    LossShape s;
    const ss_status chk = loss_shape(params, s);
    if (chk != SS_OK) return chk;
    if (s.rows == 0) return SS_OK;
    if (!logits || !stats || !grad_logits || (!grad_logprobs && !grad_entropy) || (grad_logprobs && !tokens) || (grad_entropy && !entropy)) return SS_ERR_NULL;
    if (off_element(logits, *params) || off_element(grad_logits, *params)) return SS_ERR_STRIDE;
    AltGradArgs a{make_rows(logits, nullptr, grad_logits, tokens, mask, *params, s), stats, entropy, grad_logprobs, grad_entropy, 1};
    const int vecs = row_vecs(*params), each = 256 * 4;
    a.slices = vecs > each ? (vecs + each - 1) / each : 1;
    launch(params->dtype == SS_BF16 ? alternatives_grad_kernel<SS_BF16> : alternatives_grad_kernel<SS_F32>, row_grid(a.r.rows * a.slices), dim3(256), 0,
           static_cast<hipStream_t>(stream), (const AltGradArgs)a);
    return launched();
}

}  // extern "C"
