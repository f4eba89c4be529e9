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

// Dense strides for those that are 0; false for rows that overlap.
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
    if (p.batch > 1 && (__builtin_mul_overflow((long)(p.batch - 1), out_sb, &end) || __builtin_add_overflow(end, span, &end) ||
                        __builtin_mul_overflow(end, 4L, &end)))
        return false;
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
struct LossScratch {
    size_t row_value, stats, seq, bytes;
};

inline LossScratch loss_scratch(const ss_loss_params& p) {
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t rows = (size_t)p.batch * (size_t)p.length;
    LossScratch w;
    w.row_value = 0;
    w.stats = up(rows * sizeof(double));
    w.seq = w.stats + up(rows * 2 * sizeof(float));
    w.bytes = w.seq + up((size_t)p.batch * 2 * sizeof(double)) + 256;
    return w;
}

// Waves of a workgroup that holds a row of so many vectors with `held` of them a lane, one wave of it for what is formed once a row.  16
// waves share a compute unit at the registers that takes (128 a lane): as many as hold the most there, over all workgroups.  A pair of
// rows of 4000 vectors, 8 a lane, in 9 waves leaves 7 waves' registers unused: 225 us for 4096 of them, 164 in 8.
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

}  // namespace
