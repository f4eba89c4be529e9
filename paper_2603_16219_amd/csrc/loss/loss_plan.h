// What the host decides about a call of the losses: whether its arguments are in range and where its scratch lies.
// Plain C++, no GPU.
#pragma once

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "specsteer_loss.h"

namespace {

struct LossShape {
    long rows;      // B * T
    long sb, st;    // element strides of the logits
    long gsb, gst;  // of their gradient
};

// Dense strides for those that are 0; false for rows that overlap and for sequences that interleave.
inline bool loss_strides(int64_t sb, int64_t st, const ss_loss_params& p, long& out_sb, long& out_st) {
    if (sb < 0 || st < 0) return false;
    out_st = st ? st : (long)p.vocab;
    long span = 0;
    if (out_st < p.vocab || __builtin_mul_overflow((long)(p.length > 0 ? p.length - 1 : 0), out_st, &span) ||
        __builtin_add_overflow(span, (long)p.vocab, &span))
        return false;
    out_sb = sb;
    if (!sb && __builtin_mul_overflow((long)p.length, out_st, &out_sb)) return false;
    // the last element's offset in bytes has to be a number too
    long end = 0;
    if (p.batch > 1 && __builtin_mul_overflow((long)(p.batch - 1), out_sb, &end)) return false;
    if (__builtin_add_overflow(end, span, &end) || __builtin_mul_overflow(end, 4L, &end)) return false;
    return p.batch <= 1 || p.length == 0 || out_sb >= span;
}

inline ss_status loss_shape(const ss_loss_params* p, LossShape& s) {
    if (!p) return SS_ERR_NULL;
    if (p->dtype != SS_F32 && p->dtype != SS_BF16) return SS_ERR_DTYPE;
    if (p->batch < 0 || p->length < 0 || p->length > SS_LOSS_MAX_LENGTH || p->vocab < 1 || p->vocab > SS_MAX_VOCAB) return SS_ERR_SHAPE;
    s.rows = (long)p->batch * p->length;
    if (p->batch > SS_LOSS_MAX_ROWS || s.rows > SS_LOSS_MAX_ROWS) return SS_ERR_SHAPE;
    // log2(e) / tau is the factor of every exponent: it has to be a number in fp32, rounded up as well
    if (!(p->temperature > 0.f) || !std::isfinite(p->temperature) || !(1.4426950408889634 / (double)p->temperature < 3e38))
        return SS_ERR_PARAM;
    if (!std::isfinite(p->grad_scale)) return SS_ERR_PARAM;
    if (!loss_strides(p->stride_b, p->stride_t, *p, s.sb, s.st) || !loss_strides(p->grad_stride_b, p->grad_stride_t, *p, s.gsb, s.gst))
        return SS_ERR_STRIDE;
    return SS_OK;
}

inline ss_status check_policy(const ss_policy_params* q) {
    if (!q) return SS_ERR_NULL;
    if (!(q->clip_low >= 0.f && q->clip_low <= 1.f) || !(q->clip_high >= 0.f) || !std::isfinite(q->clip_high)) return SS_ERR_PARAM;
    if (!(q->kl_coef >= 0.f) || !std::isfinite(q->kl_coef)) return SS_ERR_PARAM;
    const uint32_t means = SS_LOSS_SUM | SS_LOSS_SEQ_MEAN;
    if ((q->flags & ~(means | SS_LOSS_SEQ_ADVANTAGES)) != 0 || (q->flags & means) == means) return SS_ERR_PARAM;
    return SS_OK;
}

inline ss_status check_preference(const ss_preference_params* q) {
    if (!q) return SS_ERR_NULL;
    if (!std::isfinite(q->beta) || !(q->label_smoothing >= 0.f && q->label_smoothing <= 0.5f)) return SS_ERR_PARAM;
    return (q->flags & ~SS_LOSS_SUM) == 0 ? SS_OK : SS_ERR_PARAM;
}

// The scratch: a double a row (its share of the policy loss, or its log-prob for the preference loss), its statistics, and two
// doubles a sequence (what a token of it counts; a pair's weight and loss).
//
// Calls of few rows give each to several workgroups, whose sums over their slices lie behind that.
struct LossScratch {
    size_t row_value, stats, seq, parts, token_logits, bytes;
};

// Workgroups that a row of so many vectors takes: about 1024 in all, 512 vectors each at least.  In a third of the compute units and less one
// workgroup a row leaves most of them idle: the policy loss of one row of V = 128256 bf16 20 us in one workgroup, 6.7 in slices, of 16 20.9 and
// 9.3, of 64 21.2 and 15.1, of 100 21.4 and 19.4, of 128 21.6 and 23.3; of 4 rows of V = 32000 10.4 and 6.4, of 32 11 and 7.9.
// Log-probs alone gain less: of rows up to 8192 vectors, 8 a lane of a workgroup, they are faster in one (4 of V = 32000 fp32 4.5 and 5.2 us; of
// V = 50257 6.5 and 5.2).
constexpr int kMaxRowSlices = 64, kPartBytes = 32;
constexpr long kSliceRows = 100, kSliceGroups = 1024, kSliceVecs = 512;
constexpr int kScoreVecs = 8192;
inline int row_slices(long rows, int vecs) {
    if (rows < 1 || rows > kSliceRows) return 1;
    const long want = (kSliceGroups + rows - 1) / rows, most = vecs / kSliceVecs;
    const long n = want < most ? want : most;
    return (int)(n > kMaxRowSlices ? kMaxRowSlices : n < 1 ? 1 : n);
}
inline int score_slices(long rows, int vecs) { return vecs > kScoreVecs ? row_slices(rows, vecs) : 1; }
// Pairs that one workgroup of 16 waves forms with their loss, a wave a pair: 14 rows 4.1 us, a launch of its own for the loss 2 more.
inline bool pairs_in_one(int pairs, int length) { return pairs <= 16 && length <= 512; }
// Rows in slices that the same workgroup joins first.
constexpr long kJoinRows = 64;
inline int row_vecs(const ss_loss_params& p) { return p.vocab / (p.dtype == SS_BF16 ? 8 : 4); }

// How many of a call's last rows are read through the caches for a gradient behind it.  All where 256 MiB of last-level cache may hold them (2048
// rows of V = 50257 bf16 scored and their gradient 108 us past the caches, 101 through them).  In larger calls the gradient, which begins
// at the end, finds little, and reading past the caches is faster (4096 rows of V = 128256 515 us a preference loss, 531 with 300 MB through them) -- but
// for a preference loss whose mask leaves out enough: of 600 MB of rows those that count are about what the caches hold then.  Only the GPU knows
// what a mask keeps, so that its rows ask (kSparse of 64 of them).  Past the caches and through them, us, by the share of rows kept:
//   16 x 1024 of V = 32000 bf16   a quarter 326, 289   half 423, 401   three quarters 466, 467   19 of 20 519, 536
//   8 x 512 of V = 128256 bf16    a quarter 330, 294   half 380, 352   three quarters 461, 467   19 of 20 504, 531
//   8 x 512 of V = 50257 fp32                          half 321, 301   five eighths 353, 339     19 of 20 414, 442
struct CachedRows {
    long n;
    bool if_sparse;  // only if few enough of them count
};
constexpr int kSparse = 45;
inline CachedRows cached_rows(const ss_loss_params& p, long rows, bool masked) {
    const double row = (double)p.vocab * (p.dtype == SS_BF16 ? 2 : 4);
    if (rows * row <= 268435456.0) return {rows, false};
    const long n = masked ? (long)(600e6 / row) : 0;
    return {n < rows ? n : rows, masked};
}

inline LossScratch loss_scratch(const ss_loss_params& p) {
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t rows = (size_t)p.batch * (size_t)p.length;
    LossScratch w;
    w.row_value = 0;
    w.stats = up(rows * sizeof(double));
    w.seq = w.stats + up(rows * 2 * sizeof(float));
    w.parts = w.seq + up((size_t)p.batch * 2 * sizeof(double)) + 256;
    const int slices = row_slices((long)rows, row_vecs(p));
    w.token_logits = w.parts + (slices > 1 ? up(rows * slices * kPartBytes) : 0);
    w.bytes = w.token_logits + (slices > 1 ? up(rows * sizeof(float)) : 0);
    return w;
}

// Waves of a workgroup that holds a row of so many vectors with `held` of them a lane, one wave of it for what is formed once a row.  16
// waves share a compute unit at the registers that takes (128 a lane): as many as hold the most there, over all workgroups.  A pair of
// rows of 4000 vectors, 8 a lane, in 9 waves leaves 7 waves' registers unused: 225 us for 4096 of them, 164 in 8, before the arithmetic was
// cut down to 158.
constexpr int kUnitWaves = 16;
constexpr int kHeldVecs = 16, kHeldPairs = 8;  // of a row, and of a row and its reference
inline int row_waves(int vecs, int held) {
    int best = 2;
    long most = -1;
    for (int w = 2; w <= kUnitWaves; ++w) {
        const long one = (long)(w - 1) * 64 * held;
        const long all = (kUnitWaves / w) * (one < vecs ? one : (long)vecs);
        if (all > most || (all == most && one < vecs)) {
            most = all;
            best = w;
        }
    }
    return best;
}
// The same for a call of so many rows on so many compute units: where all of them run at once with more waves each, with as many.
inline int call_waves(long rows, int units, int vecs, int held) {
    const int most = (int)(kUnitWaves / ((rows + units - 1) / units)), useful = (vecs + 63) / 64 + 1, w = row_waves(vecs, held);
    const int wide = most < useful ? most : useful;
    return wide > w ? wide : w;
}

}  // namespace
