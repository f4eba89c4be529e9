// What the host decides about a walk: in how many stages a tree's rows are summed, the slices of rows, the scratch.  Plain C++, no GPU.
#pragma once

#include "tree_plan.h"

namespace {

// A stage sums the first `rows` rows with children at and below the cursor, in the order of the nodes; the next one walks on over them, and
// goes on from there.  The last one takes all that are left.
constexpr int kMaxStages = 2;
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
constexpr long kAllBytes = 160l << 20, kFirstBytes = 36l << 20;
constexpr int kMostSlices = 16;                        // of a row: as many as a walk reads sums of
constexpr int kArriveBytes = 256;                      // between the counters of two sequences
inline VerifyPlan verify_plan(const ss_params& p, int units) {
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    VerifyPlan r{};
    const long B = p.batch > 0 ? p.batch : 1, N = p.k_max, esz = p.dtype == SS_BF16 ? 2 : 4, vec = 16 / esz, vecs = p.vocab / vec;
    const double pair = 2.0 * B * p.vocab * esz;  // a row of every sequence
    // About half of a tree's rows have children.  All at once where that is less than two stages and the second one's launch: 16 trees of 31 nodes,
    // V = 128256 bf16 (130 MB) 39 us a call, 45 in two stages; of 60 nodes (250 MB) 79 and 62; 64 trees of 15 84 and 68.  The first stage's rows are two
    // of each sequence or kFirstBytes of them (64 trees: one 76, two 68, four 75; 16 trees: two 65, four 62); three stages are slower throughout.
    double tasks = 2.0 * B;  // rows of a stage
    if (N == 0) {
        r.stages = 0;
    } else if (pair * (N + 1) * 0.5 <= (double)kAllBytes) {
        r.stages = 1;
        r.rows[0] = (int)N + 1;
        tasks *= (N + 1) * 0.25;
    } else {
        const double first = (double)kFirstBytes / pair;
        r.stages = 2;
        r.rows[0] = first < 2 ? 2 : first > N ? (int)N : (int)first;
        r.rows[1] = (int)N + 1;
        tasks *= r.rows[0];
    }
    // about four workgroups a unit in a stage of a few rows, of 512 vectors each at least (64 trees, two rows first: 4 slices 68 us, 8 75;
    // 4 trees in one stage: 4 32, 8 29.5)
    const long want = (long)(4.0 * units / tasks + 0.999), wide = vecs / 512 > 0 ? vecs / 512 : 1, most = wide < kMostSlices ? wide : kMostSlices;
    r.slices = (int)(want < 1 ? 1 : want > most ? most : want);
    r.slice_vecs = (int)((vecs + r.slices - 1) / r.slices);
    for (int k = 0; k < r.stages; ++k) {
        const int rows = r.rows[k] < N + 1 ? r.rows[k] : (int)N + 1;
        // a stage of any number of rows: as many as fill the chip, the others behind them (64 trees of 31 nodes: two a slice 72 us, three 67, four 68; 256
        // of 8: 127, 119, 126)
        long g = rows;
        if (k + 1 == r.stages) {
            const long fill = (6l * units + 2 * B * r.slices - 1) / (2 * B * r.slices);
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
    at += up((size_t)B * r.chunks * 16);  // and the logits that some of them are relative to
    r.off_best = at;
    at += up((size_t)B * r.parts * 16);
    r.bytes = at + 256;
    return r;
}

}  // namespace
