// What the kernels over rows of logits have in common: a row's sums, its gradient from them, the rows of a call.  Included by each .hip file
// of this folder; nothing here has external linkage.
//
// Every loss is passes over rows of V logits.  With c = log2(e) / tau, a whole number E near the largest h_v c, and
//     s = sum_v 2^(h_v c - E),
// a token's log-prob is (h_y c - E - log2 s) ln 2 and every gradient of a loss of log-probs is, in the row's logits,
//     dL/dh_v = (g / tau) (1[v = y] - 2^(h_v c - E) / s),    g = dL/dlp.
// A whole-vocabulary KL to a reference with logits z takes, in the same pass, the reference's own (E', s') and
//     x = sum_v 2^(h_v c - E) ((h_v c - E) - (z_v c - E')):     KL = (x / s - log2 s + log2 s') ln 2,
// of exponents that are there anyway: what is common to a row's logits, by which policy and reference may differ, is in E and E'.  With the
// mean M = E[h - z] / tau, from x / s + E - E', it adds
//     (k / tau) P(v) ((h_v - z_v) / tau - M)     to the gradient.
// A whole E makes moving a sum to another reference exact.  Terms and a lane's sums are fp32; what is formed once a row (log-probs, KL,
// weights, losses) is double.  Sums of hundreds of log-probs with either sign are small beside their terms, so an error that all rows
// share counts: c goes into the sums' exponents in two parts, rounded to one it left 6e-8 a token, 1e-5 of a margin over 16 pairs of 1024.
//
// Rows whose largest |h c| is beyond 2^20, rows of the type's lowest value among them, and all rows at temperatures beyond 10^+-12 take a
// sweep of their own that subtracts the maximum first (far_sum).
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "../device_common.h"
#include "loss_plan.h"
#include "specsteer_loss.h"

namespace {

// E lies this far under the largest h c, rounded up: an exponent is rounded to 2^-24 of itself, and the terms that carry a sum, mostly within 8 of
// the largest, have small ones then.
constexpr float kBelow = 4.f;
constexpr float kFar = 1048576.f;  // |E| up to which a row is summed by exponents
constexpr double kLn2 = 0.6931471805599453;

template <int DT> struct Row;
template <> struct Row<SS_BF16> { static constexpr int kVec = 8; using Raw = uint4; };
template <> struct Row<SS_F32> { static constexpr int kVec = 4; using Raw = float4; };

// A row as whole vectors between the elements before the first 16-byte boundary and those behind the last: vectors are
// aligned in `aligned_to` (the gradient's row where there is one, since stores pay more for it than loads), and a lane has at most one
// of the other elements.
template <int DT>
struct Layout {
    int head, vecs, extra;  // extra: the lane's element outside of the vectors, or -1
    __device__ __forceinline__ Layout(const void* aligned_to, int V, int tid) {
        constexpr int kVec = Row<DT>::kVec, kElem = DT == SS_BF16 ? 2 : 4;
        const int off = (int)(reinterpret_cast<uintptr_t>(aligned_to) & 15);
        head = min(V, ((16 - off) & 15) / kElem);
        vecs = (V - head) / kVec;
        const int tail = V - head - vecs * kVec;
        extra = tid < head ? tid : tid >= 8 && tid < 8 + tail ? V - tail + tid - 8 : -1;
    }
};

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <int DT>
__device__ __forceinline__ typename Row<DT>::Raw ld_vec(const void* p, long vec) {
    if constexpr (DT == SS_BF16) {
        const u32x4 t = reinterpret_cast<const u32x4*>(p)[vec];
        return make_uint4(t.x, t.y, t.z, t.w);
    } else {
        const f32x4 t = reinterpret_cast<const f32x4*>(p)[vec];
        return make_float4(t.x, t.y, t.z, t.w);
    }
}

// A vector that this launch reads once: past the caches, like the gradient's stores.  Both together are 3 to 8 % of a policy loss (2048 rows of
// V = 256000 bf16 443 us with loads and stores through the caches, 437 with the stores, 414); the zeros of rows that do not count gain most (4
// pairs of 512 tokens, V = 128256, 391 us, 421 with those through the caches, 450 with all stores).
template <int DT>
__device__ __forceinline__ typename Row<DT>::Raw ld_once(const void* p, long vec) { return ld_raw<DT, Row<DT>::kVec>(p, vec); }
template <int DT>
__device__ __forceinline__ typename Row<DT>::Raw ld_once_at(const char* base, unsigned off) { return ld_once<DT>(base + off, 0); }

__device__ __forceinline__ unsigned bf16_bits(float x) {
    const __bf16 b = (__bf16)x;  // to nearest, ties to even
    return __builtin_bit_cast(unsigned short, b);
}
template <int DT>
__device__ __forceinline__ void st_elem(void* row, long e, float x) {
    if constexpr (DT == SS_BF16) reinterpret_cast<unsigned short*>(row)[e] = (unsigned short)bf16_bits(x);
    else reinterpret_cast<float*>(row)[e] = x;
}
template <int DT>
__device__ __forceinline__ void st_vec(void* p, long vec, const float (&h)[Row<DT>::kVec]) {
    if constexpr (DT == SS_BF16) {
        typedef unsigned int out_t __attribute__((ext_vector_type(4)));
        out_t r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = bf16_bits(h[2 * i]) | bf16_bits(h[2 * i + 1]) << 16;
        __builtin_nontemporal_store(r, reinterpret_cast<out_t*>(p) + vec);
    } else {
        typedef float out_t __attribute__((ext_vector_type(4)));
        out_t r = {h[0], h[1], h[2], h[3]};
        __builtin_nontemporal_store(r, reinterpret_cast<out_t*>(p) + vec);
    }
}

// ------------------------------------------------------------------ statistics of a row

// c = log2(e) / tau in two fp32 parts, the first of 16 bits, so that a bf16 logit's product with it is exact; and as one fp32 number.
struct Factor {
    float hi, lo, whole;
};
// h c - E, c in two parts or as one number
template <int PARTS>
__device__ __forceinline__ float exponent(float h, float E, Factor c) { return PARTS == 2 ? fmaf(h, c.lo, fmaf(h, c.hi, -E)) : fmaf(h, c.whole, -E); }
template <int PARTS>
__device__ __forceinline__ float term(float h, float E, Factor c) { return exp2_hw(exponent<PARTS>(h, E, c)); }

// A product that is 0 if a factor is, whatever the other: the term of a token that the policy masks, or gives no probability in fp32, times the difference
// of its exponents, which is infinite or NaN (-inf - -inf) then.  +inf remains where the reference alone masks a token.
extern "C" __device__ float mul_or_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");  // v_mul_legacy_f32, which has no builtin

// A running sum: the reference E and sum 2^(h c - E).
struct Sum {
    float E, s;
};
// The same with the cross term sum 2^(h c - E) ((h c - E) - (z c - Ez)) and the reference's own sum.
struct SumRef {
    float E, s, x, Ez, sz;
};
__device__ __forceinline__ void clear(Sum& a) { a.E = -kFar; a.s = 0.f; }
__device__ __forceinline__ void clear(SumRef& a) { a.E = a.Ez = -kFar; a.s = a.x = a.sz = 0.f; }
__device__ __forceinline__ float moved(float s, float from, float to) { return __builtin_ldexpf(s, (int)(from - to)); }
// A cross term at other references, by and byz higher, from what it is with only its terms moved to them, and their sum.  Where that has become nothing, so
// has the cross term, which stays infinite by itself if the reference masks one of the tokens (padding that the policy only holds far down).
__device__ __forceinline__ float crossed(float x, float s, float by, float byz) { return s > 0.f ? fmaf(s, byz - by, x) : 0.f; }
__device__ __forceinline__ double crossed(double x, double s, float by, float byz) { return s > 0.0 ? x + s * (double)(byz - by) : 0.0; }

__device__ __forceinline__ void merge(Sum& a, const Sum& b) {
    const float E = fmaxf(a.E, b.E);
    a.s = moved(a.s, a.E, E) + moved(b.s, b.E, E);
    a.E = E;
}
__device__ __forceinline__ void merge(SumRef& a, const SumRef& b) {
    const float E = fmaxf(a.E, b.E), Ez = fmaxf(a.Ez, b.Ez), sa = moved(a.s, a.E, E), sb = moved(b.s, b.E, E);
    a.s = sa + sb;
    a.x = crossed(moved(a.x, a.E, E), sa, E - a.E, Ez - a.Ez) + crossed(moved(b.x, b.E, E), sb, E - b.E, Ez - b.Ez);
    a.sz = moved(a.sz, a.Ez, Ez) + moved(b.sz, b.Ez, Ez);
    a.E = E;
    a.Ez = Ez;
}

template <int N>
__device__ __forceinline__ float largest(const float (&h)[N]) {
    float top = h[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, h[i]);
    return top;
}
// The references as high as logits up to `top` (and the reference's up to `topz`) take.
__device__ __forceinline__ void raise(Sum& a, float top, Factor c) {
    top = fmaf(top, c.hi, -kBelow);
    if (top > a.E) {
        const float to = fminf(ceilf(top), 2.f * kFar);
        a.s = moved(a.s, a.E, to);
        a.E = to;
    }
}
__device__ __forceinline__ void raise(SumRef& a, float top, float topz, Factor c) {
    top = fmaf(top, c.hi, -kBelow);
    topz = fmaf(topz, c.hi, -kBelow);
    if (top > a.E) {
        const float to = fminf(ceilf(top), 2.f * kFar);
        a.s = moved(a.s, a.E, to);
        a.x = crossed(moved(a.x, a.E, to), a.s, to - a.E, 0.f);
        a.E = to;
    }
    if (topz > a.Ez) {
        const float to = fminf(ceilf(topz), 2.f * kFar);
        a.sz = moved(a.sz, a.Ez, to);
        a.x = crossed(a.x, a.s, 0.f, to - a.Ez);
        a.Ez = to;
    }
}
template <int N>
__device__ __forceinline__ float tree_sum(float (&e)[N]) {
#pragma unroll
    for (int w = N / 2; w > 0; w /= 2)
#pragma unroll
        for (int i = 0; i < w; ++i) e[i] += e[i + w];
    return e[0];
}
template <int PARTS, int N>
__device__ __forceinline__ void add_under(Sum& a, const float (&h)[N], Factor c);
template <int PARTS, int N>
__device__ __forceinline__ void add(Sum& a, const float (&h)[N], Factor c) {
    raise(a, largest(h), c);
    add_under<PARTS>(a, h, c);
}
// The same where the reference is as high as it has to be.
template <int PARTS, int N>
__device__ __forceinline__ void add_under(Sum& a, const float (&h)[N], Factor c) {
    float e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = term<PARTS>(h[i], a.E, c);
    a.s += tree_sum(e);
}
template <int PARTS, int N>
__device__ __forceinline__ void add_under(SumRef& a, const float (&h)[N], const float (&z)[N], Factor c);
template <int PARTS, int N>
__device__ __forceinline__ void add(SumRef& a, const float (&h)[N], const float (&z)[N], Factor c) {
    raise(a, largest(h), largest(z), c);
    add_under<PARTS>(a, h, z, c);
}
template <int PARTS, int N>
__device__ __forceinline__ void add_under(SumRef& a, const float (&h)[N], const float (&z)[N], Factor c) {
    float e[N], ez[N], x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = exponent<PARTS>(h[i], a.E, c), tz = exponent<PARTS>(z[i], a.Ez, c);
        e[i] = exp2_hw(t);
        x[i] = mul_or_zero(e[i], t - tz);
        ez[i] = exp2_hw(tz);
    }
    a.s += tree_sum(e);
    a.x += tree_sum(x);
    a.sz += tree_sum(ez);
}

// The sums of a whole row.  Lanes' sums are added in double: their last few additions are not averaged over many, and were most of the
// error of a log-sum (5e-8 by fp32 to the end).
template <typename S> struct Total;
template <> struct Total<Sum> {
    float E;
    double s;
};
template <> struct Total<SumRef> {
    float E, Ez;
    double s, x, sz;
};
// Whether sums by exponents do not hold for a row.  Lanes whose logits all lie further down (masked ones) have nothing in their sums.  A sum is
// NaN only by a logit that is, and so is whatever depends on it: 100 rows of NaN of V = 128256, a diverged model's, 23 ms swept again, 20 us so.
__device__ __forceinline__ bool is_far(float E) { return !(E > 256.f - kFar && E < kFar); }
__device__ __forceinline__ bool is_far(const Total<Sum>& a) { return a.s == a.s && is_far(a.E); }
__device__ __forceinline__ bool is_far(const Total<SumRef>& a) { return a.s == a.s && (is_far(a.E) || (a.sz == a.sz && is_far(a.Ez))); }

__device__ __forceinline__ double wave_sum_f64(double x) { return wave_last_f64(wave_incl_scan_f64(x)); }
__device__ __forceinline__ double moved(double s, float from, float to) { return ldexp(s, (int)(from - to)); }

__device__ __forceinline__ Total<Sum> wave_total(const Sum& a) {
    Total<Sum> r;
    r.E = (float)wave_max_i32((int)a.E);
    r.s = wave_sum_f64((double)moved(a.s, a.E, r.E));
    return r;
}
__device__ __forceinline__ Total<SumRef> wave_total(const SumRef& a) {
    Total<SumRef> r;
    r.E = (float)wave_max_i32((int)a.E);
    r.Ez = (float)wave_max_i32((int)a.Ez);
    const double s = (double)moved(a.s, a.E, r.E);
    r.s = wave_sum_f64(s);
    r.x = wave_sum_f64(crossed((double)moved(a.x, a.E, r.E), s, r.E - a.E, r.Ez - a.Ez));
    r.sz = wave_sum_f64((double)moved(a.sz, a.Ez, r.Ez));
    return r;
}
// n totals to one: lane i has the i-th if i < n (and any of them otherwise), n <= 64.  Every lane has the result.
__device__ __forceinline__ Total<Sum> join(const Total<Sum>& a, int n) {
    const bool has = (int)(threadIdx.x & 63) < n;
    Total<Sum> r;
    r.E = (float)wave_max_i32((int)a.E);
    r.s = wave_sum_f64(has ? moved(a.s, a.E, r.E) : 0.0);
    return r;
}
__device__ __forceinline__ Total<SumRef> join(const Total<SumRef>& a, int n) {
    const bool has = (int)(threadIdx.x & 63) < n;
    Total<SumRef> r;
    r.E = (float)wave_max_i32((int)a.E);
    r.Ez = (float)wave_max_i32((int)a.Ez);
    const double s = moved(a.s, a.E, r.E);
    r.s = wave_sum_f64(has ? s : 0.0);
    r.x = wave_sum_f64(has ? crossed(moved(a.x, a.E, r.E), s, r.E - a.E, r.Ez - a.Ez) : 0.0);
    r.sz = wave_sum_f64(has ? moved(a.sz, a.Ez, r.Ez) : 0.0);
    return r;
}
// Totals of aligned groups of lanes, 2 to 64 of them, each its group's.  Cleared ones add nothing.
__device__ __forceinline__ void clear_total(Total<Sum>& a) { a.E = -kFar; a.s = 0.0; }
__device__ __forceinline__ void clear_total(Total<SumRef>& a) { a.E = a.Ez = -kFar; a.s = a.x = a.sz = 0.0; }
__device__ __forceinline__ float group_max(float v, int group) {
    for (int d = 1; d < group; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, kWave));
    return v;
}
__device__ __forceinline__ double group_sum(double v, int group) {
    for (int d = 1; d < group; d <<= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
__device__ __forceinline__ Total<Sum> join_group(const Total<Sum>& a, int group) {
    Total<Sum> r;
    r.E = group_max(a.E, group);
    r.s = group_sum(moved(a.s, a.E, r.E), group);
    return r;
}
__device__ __forceinline__ Total<SumRef> join_group(const Total<SumRef>& a, int group) {
    Total<SumRef> r;
    r.E = group_max(a.E, group);
    r.Ez = group_max(a.Ez, group);
    const double s = moved(a.s, a.E, r.E);
    r.s = group_sum(s, group);
    r.x = group_sum(crossed(moved(a.x, a.E, r.E), s, r.E - a.E, r.Ez - a.Ez), group);
    r.sz = group_sum(moved(a.sz, a.Ez, r.Ez), group);
    return r;
}
// Over a workgroup; `part` is free again behind the next barrier.
template <typename S>
__device__ __forceinline__ Total<S> block_total(const S& a, int threads, Total<S>* part) {
    const int lane = threadIdx.x & 63, waves = threads / kWave;
    const Total<S> mine = wave_total(a);
    if (lane == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    return join(part[lane < waves ? lane : 0], waves);
}

// ------------------------------------------------------------------ rows of a call

struct Rows {
    const void* logits;
    const void* ref;       // or NULL
    void* grad;            // or NULL
    const int32_t* tokens;
    const uint8_t* mask;   // or NULL
    long rows, sb, st, gsb, gst;
    int T, V;
    Factor c;              // log2(e) / tau
    int far;               // all rows take the sweeps for those far from zero
    double c64;
    double tau, inv_tau;
    double scale;          // the gradient's factor
    double rest;           // what c as one fp32 number leaves out, in shares of it
};

// The row of a workgroup.  Rows of a call are spread over two dimensions, in either of which a launch holds less than 2^32 lanes.
constexpr long kGridWidth = 1 << 16;
__device__ __forceinline__ long this_row() { return (long)blockIdx.y * kGridWidth + blockIdx.x; }

__device__ __forceinline__ bool counts(const Rows& a, long row) { return !a.mask || a.mask[row] != 0; }
__device__ __forceinline__ void place(const Rows& a, long row, long& at, long& grad_at) {
    const long b = (unsigned)row / (unsigned)a.T, t = row - b * a.T;
    at = b * a.sb + t * a.st;
    grad_at = b * a.gsb + t * a.gst;
}

// The gradient of a row that does not count, the part that write_grad takes of another.
template <int DT>
__device__ __forceinline__ void zero_slice(void* g, const Layout<DT>& lay, int first, int end, int step, bool extra) {
    const float none[Row<DT>::kVec] = {};
    char* const base = static_cast<char*>(g) + (long)lay.head * (DT == SS_BF16 ? 2 : 4);
    for (int i = first; i < end; i += step) st_vec<DT>(base, i, none);
    if (extra && lay.extra >= 0) st_elem<DT>(g, lay.extra, 0.f);
}

// One lane's share of a row: vectors [first, end) by step, and its extra element if `extra`.
template <int DT, typename S, int PARTS, bool ONCE = false>
__device__ __forceinline__ S lane_sum(const void* h, const void* z, const Layout<DT>& lay, int first, int end, int step, bool extra, Factor c) {
    constexpr int kVec = Row<DT>::kVec, kUnroll = 4, kElem = DT == SS_BF16 ? 2 : 4;
    constexpr bool kRef = std::is_same<S, SumRef>::value;
    S a;
    clear(a);
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
    const char* const zv = kRef ? static_cast<const char*>(z) + (long)lay.head * kElem : nullptr;
    const auto one = [&](const typename Row<DT>::Raw& r, const typename Row<DT>::Raw& rz) {
        float x[kVec];
        unpack(r, x);
        if constexpr (kRef) {
            float y[kVec];
            unpack(rz, y);
            add<PARTS>(a, x, y, c);
        } else {
            add<PARTS>(a, x, c);
        }
    };
    int i = first;
    for (; i + (kUnroll - 1) * step < end; i += kUnroll * step) {
        typename Row<DT>::Raw r[kUnroll], rz[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            r[u] = ONCE ? ld_once<DT>(hv, i + u * step) : ld_vec<DT>(hv, i + u * step);
            if constexpr (kRef) rz[u] = ld_vec<DT>(zv, i + u * step);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) one(r[u], rz[u]);
    }
    for (; i < end; i += step) {
        typename Row<DT>::Raw r = ONCE ? ld_once<DT>(hv, i) : ld_vec<DT>(hv, i), rz = r;
        if constexpr (kRef) rz = ld_vec<DT>(zv, i);
        one(r, rz);
    }
    if (extra && lay.extra >= 0) {
        const float x[1] = {ld_elem<DT>(h, lay.extra)};
        if constexpr (kRef) {
            const float y[1] = {ld_elem<DT>(z, lay.extra)};
            add<PARTS>(a, x, y, c);
        } else {
            add<PARTS>(a, x, c);
        }
    }
    return a;
}

// ------------------------------------------------------------------ rows far from zero

// 2^((h - m) c), in double but for the exponential: at temperatures near the type's largest value the difference may not be a number in fp32,
// and c have few bits.
__device__ __forceinline__ float far_term(float h, double m, double c) { return exp2_hw((float)(((double)h - m) * c)); }

// The sums of a row with its largest logit m for a reference: E = m and s = sum 2^((h - m) c), x = sum 2^((h - m) c) (h - z), element by element
// over a workgroup.
// Differences are exact where they matter, so that this holds for any finite row (of lowest values only: a uniform one).
template <int DT, typename S>
__device__ __forceinline__ Total<S> far_sum(const void* h, const void* z, int V, double c, int threads, Total<S>* part) {
    constexpr bool kRef = std::is_same<S, SumRef>::value;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = threads / kWave;
    float m = -__builtin_huge_valf(), mz = m;
    for (int i = threadIdx.x; i < V; i += threads) {
        m = fmaxf(m, ld_elem<DT>(h, i));
        if constexpr (kRef) mz = fmaxf(mz, ld_elem<DT>(z, i));
    }
    const auto all_max = [&](float v) {
        for (int d = 1; d < kWave; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, kWave));
        __syncthreads();
        if (lane == 0) part[wave].E = v;
        __syncthreads();
        v = part[lane < waves ? lane : 0].E;
        for (int d = 1; d < kWave; d <<= 1) v = fmaxf(v, __shfl_xor(v, d, kWave));
        return v;
    };
    Total<S> a;
    a.E = m = all_max(m);
    if constexpr (kRef) a.Ez = mz = all_max(mz);
    double s = 0.0, x = 0.0, sz = 0.0;
    for (int i = threadIdx.x; i < V; i += threads) {
        const float hv = ld_elem<DT>(h, i), e = far_term(hv, m, c);
        s += (double)e;
        if constexpr (kRef) {
            const float zv = ld_elem<DT>(z, i);
            x += e > 0.f ? (double)e * ((double)hv - (double)zv) : 0.0;
            sz += (double)far_term(zv, mz, c);
        }
    }
    const auto all_sum = [&](double v) {
        v = wave_sum_f64(v);
        __syncthreads();
        if (lane == 0) part[wave].s = v;
        __syncthreads();
        return wave_sum_f64(lane < waves ? part[lane].s : 0.0);
    };
    a.s = all_sum(s);
    if constexpr (kRef) {
        a.x = all_sum(x);
        a.sz = all_sum(sz);
    }
    __syncthreads();
    return a;
}

// What the gradient of a row needs: dL/dh_v = e (scale + cross (h_v - z_v)) + at_token 1[v = y], e = 2^(h_v c - E).  For a row far from zero
// e = 2^((h_v - m) c) with the maximum m in E, and cross is to be divided by tau still.  Differences of logits count up to +-limit, which times
// cross is a number: that of a token which either side masks is infinite or the type's largest, and its e = 0 has to come out as 0.  For an fp32
// gradient they are taken less their mean, `shift`, which leaves nothing for `scale` to cancel.  A bf16 one is rounded by far more than the
// cancelling loses (2^-24 of the mean against 2^-9 of the difference to it), and the subtraction is 1 to 2 % of the policy loss.
struct RowGrad {
    float E, scale, cross, at_token, shift, limit;
};

// g = weight of the row's log-prob, k that of its KL, both with the call's factor; mean = E[h - z] / tau.
// Gradients are formed with c as one number: where the sums are not, what its rest adds at the reference goes into the factor here, and what is
// left is 2^-24 of |h c - E| of a term.
template <int DT, bool REF, int PARTS>
__device__ __forceinline__ RowGrad row_grad(const Rows& a, bool far, float E, double s, double g, double k, double mean) {
    RowGrad r;
    double f = a.inv_tau / s;
    if (PARTS == 2 && !far) f *= (double)exp2_hw(E * (float)a.rest);
    r.E = E;
    r.shift = REF && DT == SS_F32 ? (float)(mean * a.tau) : 0.f;
    if (!(fabsf(r.shift) < 3e38f)) r.shift = 0.f;
    r.scale = (float)((REF && k != 0.0 ? -g - k * (mean - (double)r.shift * a.inv_tau) : -g) * f);
    r.cross = REF ? (float)(k * (far ? 1.0 : a.inv_tau) * f) : 0.f;
    const int e = __builtin_amdgcn_frexp_expf(r.cross);  // |cross| < 2^e
    r.limit = __builtin_ldexpf(1.f, 126 - (e > 0 ? e : 0));
    r.at_token = (float)(g * a.inv_tau);
    return r;
}

template <int DT, bool REF>
__device__ __forceinline__ float grad_of_term(const RowGrad& r, float e, float h, float z) {
    // bounded above as well: without a weight of the KL a token that the reference alone masks takes nothing from it
    if constexpr (REF) {
        const float d = DT == SS_F32 ? h - z - r.shift : h - z;
        return e * fmaf(r.cross, __builtin_amdgcn_fmed3f(d, -r.limit, r.limit), r.scale);
    }
    return e * r.scale;
}
template <int DT, bool REF>
__device__ __forceinline__ float grad_of(const RowGrad& r, float h, float z, Factor c) {
    return grad_of_term<DT, REF>(r, term<1>(h, r.E, c), h, z);
}

// The gradient of a row far from zero, element by element over a workgroup.
template <int DT, bool REF>
__device__ __forceinline__ void far_grad(const void* h, const void* z, void* g, const Rows& a, const RowGrad& r, int token, int threads) {
    for (int i = threadIdx.x; i < a.V; i += threads) {
        const float hv = ld_elem<DT>(h, i), zv = REF ? ld_elem<DT>(z, i) : 0.f, e = far_term(hv, r.E, a.c64);
        // a token that the policy masks counts nothing, whatever the reference says of it
        const float by = REF && e > 0.f && r.cross != 0.f ? fmaf(r.cross, (float)(((double)hv - (double)zv - (double)r.shift) * a.inv_tau), r.scale) : r.scale;
        st_elem<DT>(g, i, e * by + (i == token ? r.at_token : 0.f));
    }
}

// Vectors [first, end) by step, and the lane's extra element if `extra`, of a row's gradient.  The lane that owns the token's element
// writes it again: its logit is read before anything of the row is overwritten.
template <int DT, bool REF, bool ONCE = false>
__device__ __forceinline__ void write_grad(const void* h, const void* z, void* g, const Layout<DT>& lay, const RowGrad& r, int token, int first,
                                           int end, int step, bool extra, Factor c, const int ahead = 0, const typename Row<DT>::Raw* r_ahead = nullptr,
                                           const typename Row<DT>::Raw* rz_ahead = nullptr) {
    constexpr int kVec = Row<DT>::kVec, kElem = DT == SS_BF16 ? 2 : 4, kUnroll = 4;
    const char* const hv = static_cast<const char*>(h) + (long)lay.head * kElem;
    const char* const zv = REF ? static_cast<const char*>(z) + (long)lay.head * kElem : nullptr;
    char* const gv = static_cast<char*>(g) + (long)lay.head * kElem;
    const int at = token - lay.head, vec = at >= 0 && at < lay.vecs * kVec ? at / kVec : -1;
    // lanes without an extra element have -1 there, which a token outside of the vocabulary may be too
    const bool mine = vec >= 0 ? vec >= first && vec < end && (vec - first) % step == 0 : extra && token >= 0 && lay.extra == token;
    float mine_h = 0.f, mine_z = 0.f;
    if (mine) {
        mine_h = ld_elem<DT>(h, token);
        if constexpr (REF) mine_z = ld_elem<DT>(z, token);
    }
    const auto one = [&](const typename Row<DT>::Raw& raw, const typename Row<DT>::Raw& rawz, int i) {
        float x[kVec], y[kVec];
        unpack(raw, x);
        if constexpr (REF) unpack(rawz, y);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] = grad_of<DT, REF>(r, x[j], REF ? y[j] : 0.f, c);
        st_vec<DT>(gv, i, x);
    };
    int i = first;
#pragma unroll
    for (int u = 0; u < ahead; ++u, i += step)
        if (i < end) one(r_ahead[u], rz_ahead[u], i);
    for (; i + (kUnroll - 1) * step < end; i += kUnroll * step) {
        typename Row<DT>::Raw raw[kUnroll], rawz[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            raw[u] = ONCE ? ld_once<DT>(hv, i + u * step) : ld_vec<DT>(hv, i + u * step);
            if constexpr (REF) rawz[u] = ld_vec<DT>(zv, i + u * step);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) one(raw[u], rawz[u], i + u * step);
    }
    for (; i < end; i += step) {
        const typename Row<DT>::Raw raw = ONCE ? ld_once<DT>(hv, i) : ld_vec<DT>(hv, i);
        if constexpr (REF) one(raw, ld_vec<DT>(zv, i), i);
        else one(raw, raw, i);
    }
    if (extra && lay.extra >= 0)
        st_elem<DT>(g, lay.extra, grad_of<DT, REF>(r, ld_elem<DT>(h, lay.extra), REF ? ld_elem<DT>(z, lay.extra) : 0.f, c));
    if (mine) {
        asm volatile("" ::: "memory");  // behind the stores above, which cover this element too
        st_elem<DT>(g, token, r.at_token + grad_of<DT, REF>(r, mine_h, mine_z, c));
    }
}

__device__ __forceinline__ double nan64() { return __longlong_as_double(0x7FF8000000000000ll); }
// What a sum's reference is worth.  In sums with c as one number the terms that carry them lie near the reference, where c's rest moves all of them
// alike; what is left out then is 2^-24 of their distances to it.
template <int PARTS>
__device__ __forceinline__ double reference(const Rows& a, float E) { return PARTS == 2 ? (double)E : (double)E * (1.0 + a.rest); }

// log P(y) of a row's token with logit h, from the row's sums
template <int PARTS>
__device__ __forceinline__ double token_logprob(const Rows& a, bool far, int token, float h, float E, double s) {
    if (token < 0 || token >= a.V) return nan64();
    if (far) return ((double)h - (double)E) * a.inv_tau - log(s);
    return ((double)h * a.c64 - reference<PARTS>(a, E) - log2(s)) * kLn2;
}
// mean: E[h - z] / tau of a row; kl: that less the difference of the log-sum-exps
template <int PARTS>
__device__ __forceinline__ void divergence(const Rows& a, bool far, const Total<SumRef>& s, double& mean, double& kl) {
    const double sums = log2(s.s) - log2(s.sz);
    if (far) {
        mean = s.x / s.s * a.inv_tau;
        kl = mean - (((double)s.E - (double)s.Ez) * a.inv_tau + sums * kLn2);
    } else {
        const double x = s.x / s.s * (PARTS == 2 ? 1.0 : 1.0 + a.rest);  // c's rest counts in differences of exponents too
        mean = (x + (reference<PARTS>(a, s.E) - reference<PARTS>(a, s.Ez))) * kLn2;
        kl = (x - sums) * kLn2;
    }
    if (kl < 0.0) kl = 0.0;  // by rounding only
}

// The sum of x over the workgroup, in every lane of wave 0.  The order is fixed.
__device__ __forceinline__ double block_sum(double x, double* part) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) part[wave] = x;
    __syncthreads();
    x = lane < (int)blockDim.x / kWave ? part[lane] : 0.0;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
    __syncthreads();
    return x;
}

// Bytes of m that are not 0, over one wave.
__device__ __forceinline__ int wave_count(const uint8_t* m, long n) {
    const int lane = threadIdx.x & 63;
    const long head = min(n, (long)((16 - (reinterpret_cast<uintptr_t>(m) & 15)) & 15)), vecs = (n - head) / 16, tail = head + vecs * 16;
    int k = lane < head && m[lane] != 0 ? 1 : 0;
    if (tail + lane < n && m[tail + lane] != 0) ++k;
    const auto bytes = [](unsigned w) { return __popc((((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) & 0x80808080u); };
#pragma unroll 4
    for (long i = lane; i < vecs; i += kWave) {
        const uint4 w = reinterpret_cast<const uint4*>(m + head)[i];
        k += bytes(w.x) + bytes(w.y) + bytes(w.z) + bytes(w.w);
    }
    return wave_sum_i32(k);
}

// ------------------------------------------------------------------ launches

inline dim3 row_grid(long rows) {
    return rows <= kGridWidth ? dim3((unsigned)rows) : dim3((unsigned)kGridWidth, (unsigned)((rows + kGridWidth - 1) / kGridWidth));
}

inline Rows make_rows(const void* logits, const void* ref, void* grad, const int32_t* tokens, const uint8_t* mask, const ss_loss_params& p,
               const LossShape& s) {
    Rows r;
    r.logits = logits;
    r.ref = ref;
    r.grad = grad;
    r.tokens = tokens;
    r.mask = mask;
    r.rows = s.rows;
    r.sb = s.sb;
    r.st = s.st;
    r.gsb = s.gsb;
    r.gst = s.gst;
    r.T = p.length;
    r.V = p.vocab;
    r.c64 = 1.4426950408889634 / (double)p.temperature;
    int e;
    const double frac = std::frexp(r.c64, &e);  // 0.5 .. 1
    // rounded down, so that the lower part is positive: a logit of -inf stays -inf under both
    r.c.hi = (float)std::ldexp(std::floor(std::ldexp(frac, 16)), e - 16);
    r.c.lo = std::fmax((float)(r.c64 - (double)r.c.hi), 1.1754944e-38f);
    r.c.whole = (float)r.c64;
    // 1 / tau^2 is a factor otherwise, which fp32 may not hold, nor c's lower part
    r.far = !(p.temperature > 1e-12f && p.temperature < 1e12f);
    r.tau = (double)p.temperature;
    r.inv_tau = 1.0 / r.tau;
    r.scale = (double)p.grad_scale;
    r.rest = (r.c64 - (double)r.c.whole) / (double)r.c.whole;
    return r;
}

inline bool off_element(const void* p, const ss_loss_params& q) { return (reinterpret_cast<uintptr_t>(p) & (q.dtype == SS_BF16 ? 1 : 3)) != 0; }

inline ss_status check_workspace(const void* workspace, size_t bytes, size_t need) {
    return workspace && (reinterpret_cast<uintptr_t>(workspace) & 255) == 0 && bytes >= need ? SS_OK : SS_ERR_WORKSPACE;
}

inline ss_status launched() { return hipGetLastError() == hipSuccess ? SS_OK : SS_ERR_DEVICE; }

}  // namespace
