// How the keys of a call's sequences are dealt out to workgroups.  Plain C++ that the kernels and the host share, so that it can be checked
// without a GPU.
//
// An item is one key/value head of one sequence with one block of columns (a column: a row of the tree and a query head of the group); a unit is
// one tile of its keys, first those of the cache, then the tree's own.  Units of all items stand in one line, sequence by sequence, and every
// workgroup takes an equal share of it, wherever that begins and ends: lengths that differ from sequence to sequence cost no balance, and an item is
// cut only where a share ends.  A share's first and last items may be parts, whose sums go to two slots of the workgroup; a workgroup of a second
// launch joins those of the item that the share's beginning cuts, if it is the first to do so.
#pragma once

// begin() multiplies two numbers of shares in 32 bits; a call has fewer than 2^31 units
constexpr int kMaxShares = 1 << 15;

#ifdef __HIPCC__
#define SS_TREE_BOTH __host__ __device__ __forceinline__
#else
#define SS_TREE_BOTH inline
#endif

namespace {

struct TreeTiles {
    int tile;     // keys a unit
    int columns;  // of an item's block
    int group;    // query heads a key/value head
    int kv_heads;
};
// One sequence's items: `cached` tiles of the cache and `own` of the tree each; a sequence that is marked has one unit an item.
struct TreeItems {
    int cached, own, blocks;
    SS_TREE_BOTH int tiles() const { return cached + own; }
    SS_TREE_BOTH int units(int kv_heads) const { return tiles() * blocks * kv_heads; }
};
SS_TREE_BOTH TreeItems tree_items(const TreeTiles& t, int length, int nodes, bool bad, int max_nodes) {
    TreeItems r;
    const int columns = ((bad ? max_nodes : nodes) + 1) * t.group;
    r.cached = bad ? 0 : (int)(((unsigned)length + (unsigned)t.tile - 1) / (unsigned)t.tile);
    r.own = bad ? 1 : (nodes + t.tile) / t.tile;
    r.blocks = (columns + t.columns - 1) / t.columns;
    return r;
}
// The page of a position below 2^31 without a division: the upper half of its product with ceil(2^(31 + s) / size), shifted, with s the least for which
// 2^s >= size.  What the factor is too large by is below size <= 2^s, which 2^31 positions do not bring to a page.  A factor of 0: pages of one.
struct PageOf {
    unsigned mul;
    int shift;
    SS_TREE_BOTH unsigned operator()(unsigned position) const { return mul ? (unsigned)((unsigned long)position * mul >> 32) >> shift : position; }
};
inline PageOf page_of(int size) {
    int bits = 0;
    while (1l << bits < size) ++bits;
    return PageOf{bits ? (unsigned)(((1ul << (31 + bits)) + (unsigned long)size - 1) / (unsigned long)size) : 0u, bits - 1};
}
// The piece of a sequence's row of the table that holds the pages of tile `t` and of as many tiles behind it as `most` entries do: entries
// [from, from + entries), tiles before `until`.  t is below `cached`, whose last tile holds position length - 1.
struct TablePiece {
    int from, entries, until;
};
SS_TREE_BOTH TablePiece table_piece(int t, int tile, PageOf page_of, int page_size, int length, int cached, int most) {
    TablePiece r;
    const int first = t * tile;
    r.from = (int)page_of((unsigned)first);
    const int left = (int)page_of((unsigned)length - 1) - r.from;  // behind the first: no sum that may pass 32 bits where pages are of one position
    r.entries = left < most ? left + 1 : most;
    const long more = (((long)r.from + most) * page_size - first) / tile;
    r.until = more < cached - t ? t + (int)more : cached;
    return r;
}
// The pages that positions [length, length + rows] lie in: `more` behind the first.  length + rows is below 2^31.
struct PageRange {
    int first, more;
};
SS_TREE_BOTH PageRange pages_written(int length, int rows, int page_size) {
    PageRange r;
    r.first = length / page_size;
    r.more = (length + rows) / page_size - r.first;
    return r;
}
// The shares of all units: no share is empty.
struct Shares {
    int each;   // units of a share,
    int more;   // and one more of these of them, spread out
    int shares;
    SS_TREE_BOTH int begin(int w) const { return each * w + (int)((unsigned)more * (unsigned)w / (unsigned)shares); }
};
SS_TREE_BOTH Shares deal(int units, int most) {
    Shares r;
    r.shares = units < most ? units : most;
    r.each = r.shares ? units / r.shares : 0;
    r.more = units - r.each * r.shares;
    return r;
}

}  // namespace
