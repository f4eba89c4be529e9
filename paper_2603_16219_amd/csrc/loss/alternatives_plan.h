// What the host decides about a call of the alternatives: where its scratch lies, how many workgroups take a row.  Plain C++, no GPU.
#pragma once

#include "loss_plan.h"
#include "specsteer_alternatives.h"

namespace {

// A slice's sums (Total<SumX>) and its alternatives, a word of 64 bits each, behind those of all slices.
constexpr int kAltPartBytes = 24;
struct AltScratch {
    size_t parts, keys, bytes;
};
inline AltScratch alt_scratch(const ss_loss_params& p, int topk) {
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t rows = (size_t)p.batch * (size_t)p.length;
    const int slices = row_slices((long)rows, row_vecs(p));
    AltScratch w;
    w.parts = 0;
    w.keys = slices > 1 ? up(rows * slices * kAltPartBytes) : 0;
    w.bytes = w.keys + (slices > 1 ? up(rows * slices * (size_t)topk * 8) : 0) + 256;
    return w;
}

// Lanes of a group whose largest logit is one of the n that bound the n-th largest of a row from below: n groups at least.
inline int group_lanes(int threads, int topk) {
    int lanes = 64;
    while (lanes > 1 && threads / lanes < topk) lanes /= 2;
    return lanes;
}

}  // namespace
