// How the keys of a call's sequences are dealt out to workgroups.  Plain C++ that the kernels and the host share, so that it can be checked
// without a GPU.
//
// An item is one key/value head of one sequence with one block of columns (a column: a row of the tree and a query head of the group); a unit is
// one tile of its keys, first those of the cache, then the tree's own.  Units of all items stand in one line, sequence by sequence, and every
// workgroup takes an equal share of it, wherever that begins and ends: lengths that differ from sequence to sequence cost no balance, and an item is
// cut only where a share ends.  A share's first and last items may be parts, whose sums go to two slots of the workgroup; a workgroup of a second
// launch joins those of the item that the share's beginning cuts, if it is the first to do so.
#pragma once

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
    SS_TREE_BOTH long units(int kv_heads) const { return (long)tiles() * blocks * kv_heads; }
};
SS_TREE_BOTH TreeItems tree_items(const TreeTiles& t, int length, int nodes, bool bad, int max_nodes) {
    TreeItems r;
    const long columns = (long)((bad ? max_nodes : nodes) + 1) * t.group;
    r.cached = bad ? 0 : (int)(((long)length + t.tile - 1) / t.tile);
    r.own = bad ? 1 : (nodes + t.tile) / t.tile;
    r.blocks = (int)((columns + t.columns - 1) / t.columns);
    return r;
}
// No share is empty.
SS_TREE_BOTH int shares_of(int most, long units) { return units < most ? (int)units : most; }
SS_TREE_BOTH long share_begin(long units, int shares, int w) {
    const long q = units / shares, r = units % shares;  // units * shares may pass 64 bits
    return q * w + r * w / shares;
}

}  // namespace
