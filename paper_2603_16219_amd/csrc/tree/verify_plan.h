// What the host decides about a walk: in how many stages a tree's rows are summed, the slices of rows, the scratch.  Plain C++, no GPU.
#pragma once

#include "tree_plan.h"

namespace {

// A stage sums the first `rows` rows with children at and below the cursor, in the order of the nodes; the next one walks on over them, and
// goes on from there.  The last one takes all that are left.
constexpr int kMaxStages = 5;
struct VerifyPlan {
    int stages;
    int rows[kMaxStages];
    int slices, slice_vecs;  // of a row, vectors each
    int groups[kMaxStages];  // workgroups a slice of a sequence's rows of a stage
    int parts, part_chunks;  // workgroups that share the row a token is drawn from, chunks each
    int chunks;
    size_t off_arrive, off_sums, off_logits, off_masses, off_best, bytes;
};

constexpr int kVerifyGroup = 256;                      // threads
constexpr int kMassVecs = 4 * 64;                     // of a wave
constexpr long kStageBytes = 24l << 20;                // about what a launch costs by itself
constexpr int kArriveBytes = 256;                      // between the counters of two sequences
inline VerifyPlan verify_plan(const ss_params& p, int units) {
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    VerifyPlan r{};
    const long B = p.batch > 0 ? p.batch : 1, N = p.k_max, esz = p.dtype == SS_BF16 ? 2 : 4, vec = 16 / esz, vecs = p.vocab / vec;
    const double pair = 2.0 * B * p.vocab * esz;  // a row of every sequence
    // about half of a tree's rows have children
    if (N == 0) {
        r.stages = 0;
    } else if (pair * (N + 1) * 0.5 <= 2.0 * kStageBytes) {
        r.stages = 1;
        r.rows[0] = (int)N + 1;
    } else {
        const int first = pair < kStageBytes ? (int)(kStageBytes / pair) : 1;
        int left = (int)N + 1, w = first;
        while (left > 0 && r.stages < kMaxStages - 1 && left > w) {
            r.rows[r.stages++] = w;
            left -= w;
            w = r.stages == 1 ? 2 * first : 2 * w;
            if (pair < kStageBytes && r.stages == 2) break;
        }
        r.rows[r.stages++] = (int)N + 1;
    }
    // slices: two workgroups a unit or more from the first stage's rows, 512 vectors each at least
    const long tasks = 2 * B * (r.stages ? r.rows[0] > 1 && r.stages == 1 ? (r.rows[0] + 1) / 2 : r.rows[0] : 1);
    long want = (4l * units + tasks - 1) / tasks;
    const long most = vecs / 512 > 0 ? vecs / 512 : 1;
    r.slices = (int)(want < 1 ? 1 : want > most ? most : want > 16 ? 16 : want);
    r.slice_vecs = (int)((vecs + r.slices - 1) / r.slices);
    for (int k = 0; k < r.stages; ++k) {
        const int rows = r.rows[k] < N + 1 ? r.rows[k] : (int)N + 1;
        // a stage of any number of rows: as many as fill the chip, the others behind them
        long g = rows;
        if (k + 1 == r.stages) {
            const long fill = (8l * units + 2 * B * r.slices - 1) / (2 * B * r.slices);
            g = g < fill ? g : fill;
        }
        r.groups[k] = (int)(g < 1 ? 1 : g);
    }
    r.chunks = (int)((vecs + kMassVecs - 1) / kMassVecs) + 1;  // the last one's are the elements behind the last vector
    long parts = (2l * units + B - 1) / B;
    if (B > 4096) parts = 1;  // no counters
    parts = parts > 32 ? 32 : parts;
    const long rounds = (r.chunks + 3) / 4;  // of a workgroup's four waves
    if (parts > rounds) parts = rounds;
    r.parts = (int)(parts < 1 ? 1 : parts);
    r.part_chunks = (r.chunks + r.parts - 1) / r.parts;
    size_t at = up((size_t)B * 16 * (r.stages + 1));  // the cursors at the beginning of every stage and of the draw
    r.off_arrive = at;
    at += r.parts > 1 ? (size_t)B * kArriveBytes : 0;
    r.off_sums = at;
    at += up((size_t)B * (N + 1) * 2 * r.slices * 16);
    r.off_logits = at;
    at += up((size_t)B * N * 8);
    r.off_masses = at;
    at += up((size_t)B * r.chunks * 8);
    r.off_best = at;
    at += up((size_t)B * r.parts * 16);
    r.bytes = at + 256;
    return r;
}

}  // namespace
