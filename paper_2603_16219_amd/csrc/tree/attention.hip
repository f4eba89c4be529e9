// Attention of a tree's rows over a paged cache and their ancestors, for MI355X (gfx950); include/specsteer_tree.h says what it computes,
// tree_schedule.h how the work is dealt out.
//
// For a block of columns (a tree row and a query head of the group each) and a tile of keys
//     S^T = K Q^T,    P^T = 2^(c S^T - m),    l += sum P,    O^T += V^T P^T,    c = scale log2(e),
// all products by 32x32x16 matrix instructions.  With columns along the lanes, a column's maximum and sum take one exchange between the wave's
// halves, and the lanes that hold P^T's elements are those that have to give them to the second product: rows 8 a + 4 h + i of S^T lie in
// half h, so that the keys of V^T are read in that order.  The reference m rises only when a score passes it by 2^kSlack, and O is rescaled then.
// The weights are rounded to the values' type for their product, as matrix instructions take them; their sum l is of what they were before.  That is half
// a step of the type a weight, and about as much again as the rounding of the output: for bf16 outputs 2.4e-3 of their size off in all, 1.7e-3 if it were not.
//
// Keys and values go from memory to LDS without registers, half a tile at a time; in pieces of 16 bytes whose place in the row depends on the row, which
// spreads both the keys' reads and the values' transposed ones over the banks.
//
// Bytes: the cache once a call for up to 256 columns, whose products take 4 D flop a column for 4 D bytes a key.  Measured, main launch and join: 32 trees of 24
// nodes over up to 4096 tokens (32 heads over 8, D = 128, bf16; 411 MB) 112 us, 3.7 TB/s; the same without loads 101 us: products, softmax and LDS in turn.
// 8 rows (32 columns) instead of 25 over the same cache take 95 us.  4 times 64 rows over 65536 tokens (275 GFLOP) 333 to 344 us, 800 to 825 TFLOP/s; 128
// chains of 8 over up to 2000 tokens (16 heads, D = 64, fp16; 792 MB) 161 us, 4.9 TB/s.  One token over 1000 takes 14 us: a launch that finds its place in
// the batch before its first load (6 to 8 us), and the join's 4.
#include "tree_common.h"
#include "tree_schedule.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32v4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32v4 __attribute__((ext_vector_type(4)));

template <int DT> struct Half;
template <> struct Half<SS_BF16> {
    typedef __bf16 T;
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    // a weight is at most 2^kSlack
    static constexpr float kSlack = 8.f, kLift = 0.f;
    static constexpr unsigned kExponent = 0x7F80u;
};
template <> struct Half<SS_TREE_F16> {
    typedef _Float16 T;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    // weights are 2^10 times as large, so that those 2^-24 below the largest are normal numbers still, and at most 2^15
    static constexpr float kSlack = 5.f, kLift = 10.f;
    static constexpr unsigned kExponent = 0x7C00u;
};
template <int DT>
__device__ __forceinline__ f32x16 mfma(typename Half<DT>::x8 a, typename Half<DT>::x8 b, f32x16 c) {
    if constexpr (DT == SS_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// 16 bytes a lane from memory to LDS, lane i's to `to` + 16 i.  By the builtin the compiler waits for all such loads before the next read of LDS, those a
// tile ahead among them; here the wait stands before the barrier that hands the tile over.  No register is written.  m0, which nothing else in these
// kernels uses, is read one wait state behind its write.
__device__ __forceinline__ void load_lds(unsigned to, const char* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ unsigned lds_offset(const void* p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }

// Keys or values of a tile are there for all waves when each wave's loads are, of which those of up to HELD - 1 tiles may be on their way still that
// were asked for behind them: `later` tiles follow this one.
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
template <int LOADS, int HELD, bool SHARED>
__device__ __forceinline__ void arrived(int later) {
    static_assert(2 * LOADS * (HELD - 1) < 64, "what the counter counts");
    if (later >= HELD - 1) wait_loads<2 * LOADS*(HELD - 1)>();
    else if (HELD > 3 && later >= 2) wait_loads<2 * LOADS * 2>();
    else if (HELD > 2 && later >= 1) wait_loads<2 * LOADS>();
    else wait_loads<0>();
    if (SHARED) asm volatile("s_barrier" : : : "memory");
}
__device__ __forceinline__ float tree_sum16(const float (&p)[16]) {
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = p[i] + p[i + 8];
    return ((s[0] + s[4]) + (s[2] + s[6])) + ((s[1] + s[5]) + (s[3] + s[7]));
}

// Which of the 32 keys from `base` on a row sees: of the block's own rows itself and its ancestors, of the cache those there are.
__device__ __forceinline__ unsigned seen_keys(bool own, bool tree, int base, int limit, int row, int N, const unsigned short* up) {
    if (!own) return limit - base >= 32 ? ~0u : limit > base ? (1u << (limit - base)) - 1 : 0u;
    int j = min(row, N);
    if (!tree) return j < base ? 0u : j - base >= 31 ? ~0u : (2u << (j - base)) - 1;
    unsigned seen = base == 0 ? 1u : 0u;
    while (j > base + 31) j = up[j];
    while (j >= base && j > 0) {
        seen |= 1u << (j - base);
        j = up[j];
    }
    return seen;
}

// The larger of a lane's value and that of the same lane of the other half.
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

struct AttnArgs {
    const char *q, *k, *v, *kc, *vc;
    const int32_t *table, *cache_len, *parents, *tree_len;
    char* out;
    float* part_o;   // [2 * shares][columns][D]: sums of values of parts
    float2* part_ml; // [2 * shares][columns]: their references and sums of weights
    struct Cut* cuts;  // [shares]
    Strides3 qs, ks, os;
    unsigned page_step, slot_step;  // bytes
    PageOf page_of;
    long head_step;
    long ts;
    int B, N, group, kv_heads, pages, page_size, width, shares;
    float scale;  // |scale| log2(e)
    int negative; // scale < 0
};

struct Sequence {
    int L, N;
    bool bad;
};
template <bool UNIFORM>
__device__ __forceinline__ Sequence sequence(const AttnArgs& a, int b) {
    Sequence s;
    s.L = a.cache_len[b];
    s.N = a.tree_len ? a.tree_len[b] : a.N;
    if (UNIFORM) {  // which loads by vector instructions do not tell
        s.L = __builtin_amdgcn_readfirstlane(s.L);
        s.N = __builtin_amdgcn_readfirstlane(s.N);
    }
    s.bad = s.L < 0 || s.L > (long)a.width * a.page_size || s.N < 0 || s.N > a.N;
    return s;
}

// Where a unit lies: its sequence, and the units before that.
struct Place {
    int b, before, total;
};
// The sums over all sequences, by a workgroup; the unit asked for follows from them.
template <int NT, typename F>
__device__ __forceinline__ Place find_place(const AttnArgs& a, const TreeTiles& tiles, int* sh, F unit) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kWaves = NT / kWave;
    const auto of = [&](int b) {
        if (b >= a.B) return 0;
        const Sequence s = sequence<false>(a, b);
        return tree_items(tiles, s.L, s.N, s.bad, a.N).units(a.kv_heads);
    };
    const int first = of(tid);
    int sum = first;
    for (int b = tid + NT; b < a.B; b += NT) sum += of(b);
    sum = wave_sum_i32(sum);
    if (lane == 0) sh[wave] = sum;
    __syncthreads();
    Place p{0, 0, 0};
    for (int w = 0; w < kWaves; ++w) p.total += sh[w];
    p.total = __builtin_amdgcn_readfirstlane(p.total);
    const int u = unit(p.total);
    if (u < 0 || u >= p.total) return p;
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int mine = b0 == 0 ? first : of(b0 + tid), incl = wave_incl_scan_i32(mine);
        __syncthreads();
        if (lane == 63) sh[wave] = incl;
        __syncthreads();
        int start = before;
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) start += sh[w];
            before += sh[w];
        }
        if (u >= start + incl - mine && u < start + incl) {
            sh[kWaves] = b0 + tid;
            sh[kWaves + 1] = start + incl - mine;
        }
        if (u < before) break;
    }
    __syncthreads();
    p.b = __builtin_amdgcn_readfirstlane(sh[kWaves]);
    p.before = __builtin_amdgcn_readfirstlane(sh[kWaves + 1]);
    return p;
}

// What joins the parts of an item that a share's beginning cuts, written by that share if no share before it begins inside of the item.
struct Cut {
    int b, head, block, parts;  // parts: 0 if there is nothing to join; the first is the share's before, in its second slot if `second`
    int second, pad[3];
};

// A workgroup of WM x WK waves: each takes 32 columns and SUB times 32 keys of a tile; waves of the same columns take turns at the keys.  By the columns of a
// call (with_shape): no more waves over columns than there are columns for, so that none computes what nobody asked for, the others over keys.  Two
// workgroups a unit hide each other's waits: with one, 32 trees of 24 nodes took 133 us and not 113, one token 19 and not 15.  Over 128 columns a workgroup has
// eight waves, which halves what it reads of the cache, and a unit one.  Other depths of the ring and sub-tiles were within 3 per cent.
template <int D_, int WM_, int WK_, int SUB_, int HELD_, int GROUPS_>
struct Shape {
    static constexpr int D = D_, WM = WM_, WK = WK_, kSub = SUB_;
    static constexpr int kWaves = WM * WK, kThreads = kWaves * kWave, kColumns = 32 * WM;
    static constexpr int kGroups = GROUPS_;          // workgroups a compute unit
    static constexpr int kTile = 32 * WK * kSub;     // keys
    static constexpr int kLanes = D / 8;             // of 16 bytes each, a row
    static constexpr int kRows = kWave / kLanes;     // rows a load instruction
    static constexpr int kLoads = 32 * kSub / (kRows * WM);  // of a wave for the keys of a tile, and for its values; with one wave over the columns its own
    static constexpr int kRowBytes = 2 * D, kTileBytes = kTile * kRowBytes, kStage = 2 * kTileBytes;
    static constexpr int kHeld = HELD_;              // tiles in LDS
    static constexpr int kTable = 1024;              // entries of the table in LDS
    static constexpr int kPad = D + 4;               // floats of a column that waves hand over
    static constexpr int kHand = (WK - 1) * kColumns * kPad * 4;
    static constexpr int kBuffers = kHeld * kStage > kHand ? kHeld * kStage : kHand;
};

// By how much the 16-byte pieces of a row are turned round: 4 rows next to each other that a transposed read takes, and 16 whose same piece is
// read at once, lie in different banks.
template <int D>
__device__ __forceinline__ int turn(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}

template <int DT, typename C>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void attention_kernel(const AttnArgs a) {
    using H = Half<DT>;
    using x8 = typename H::x8;
    constexpr int D = C::D, kSub = C::kSub, kBlocks = D / 32, kSteps = D / 16;
    __shared__ __attribute__((aligned(1024))) char lds[C::kBuffers];
    __shared__ float2 hand_ml[C::WK][C::kColumns];
    __shared__ unsigned short up[SS_MAX_K + 1];
    __shared__ int table[C::kTable];
    __shared__ int sh[C::kWaves + 2];
    __shared__ int sh_bad[2];  // of an item and the next one
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % C::WM, wk = wave / C::WM;
    const TreeTiles tiles{C::kTile, C::kColumns, a.group, a.kv_heads};

    Shares deals{};
    const Place place = find_place<C::kThreads>(a, tiles, sh, [&](int total) {
        deals = deal(total, a.shares);
        return (int)blockIdx.x < deals.shares ? deals.begin(blockIdx.x) : -1;
    });
    int u = 0, u_end = 0;
    if ((int)blockIdx.x < deals.shares) {
        u = deals.begin(blockIdx.x);
        u_end = deals.begin(blockIdx.x + 1);
    }
    int b = place.b, rel = u - place.before;  // within the sequence
    Sequence s = sequence<true>(a, b);
    TreeItems items = tree_items(tiles, s.L, s.N, s.bad, a.N);
    if (tid == 0 && blockIdx.x > 0) {
        int parts = 0, second = 0;
        if (u < u_end) {
            const int nt = items.tiles(), item = rel / nt, start = u - (rel - item * nt);
            const int before = deals.begin(blockIdx.x - 1);
            if (start < u && before <= start) {
                int x = blockIdx.x + 1;
                while (x < deals.shares && deals.begin(x) < start + nt) ++x;
                parts = x - (int)blockIdx.x + 1;
                second = before < start ? 1 : 0;
            }
        }
        Cut* const cut = a.cuts + blockIdx.x;
        const int item = rel / max(items.tiles(), 1);
        cut->b = b;
        cut->head = item / items.blocks;
        cut->block = item % items.blocks;
        cut->parts = parts;
        cut->second = second;
    }
    int done = 0;  // items
    if (tid == 0) sh_bad[0] = 0;
    // the piece of the table that is in LDS: its sequence, the column that it begins with, the tiles whose pages it has
    int table_of = -1, table_from = 0, table_first = 0, table_until = 0;
    bool table_bad = false;  // of its sequence this thread has met a page that is none
    while (u < u_end) {
        if (rel >= items.units(a.kv_heads)) {
            ++b;
            rel = 0;
            s = sequence<true>(a, b);
            items = tree_items(tiles, s.L, s.N, s.bad, a.N);
        }
        const int nt = items.tiles();
        // the same for all lanes, which the compiler does not see: vector compares and masks around every step took 4 per cent of the long cache's time
        const int item = __builtin_amdgcn_readfirstlane(rel / nt), t0 = __builtin_amdgcn_readfirstlane(rel - item * nt);
        const int t1 = __builtin_amdgcn_readfirstlane(min(nt, t0 + (u_end - u)));
        const int head = item / items.blocks, block = item - head * items.blocks;
        // this lane's column: a row of the tree and a query head
        const int place_of = wm * 32 + (lane & 31), column = block * C::kColumns + place_of;
        const int rows = (s.bad ? a.N : s.N) + 1, row = column / a.group, query = head * a.group + column - row * a.group;
        const bool whole = t0 == 0 && t1 == nt;
        bool bad = s.bad;

        f32x16 o[kBlocks];
        float m = -1e30f, l = 0.f;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) o[i] = f32x16{};
        __syncthreads();  // the last item's hand-over is done with
        // Cleared a barrier before any wave may set it: where waves go on by themselves there is none between here and an item's end
        if (tid == 0) sh_bad[~done & 1] = 0;
        if (!s.bad) {
            // The rows of a tile that this wave loads are kMine from first_row on.  A lane finds where one of them lies, and those that load its pieces
            // ask for that: the arithmetic once for all rows, whatever the pages' size.  The pages come from a piece of the table in LDS.
            constexpr int kMine = C::kLoads * C::kRows;
            const int first_row = wave * kMine, my_row = first_row + lane % kMine;
            const auto look_up = [&](int t) {
                if (t >= items.cached || (b == table_of && t >= table_first && t < table_until)) return;
                const int32_t* const pages = a.table + b * a.ts;
                __syncthreads();
                if (b != table_of) table_bad = false;
                table_of = b;
                table_first = t;
                const TablePiece piece = table_piece(t, C::kTile, a.page_of, a.page_size, s.L, items.cached, C::kTable);
                table_from = piece.from;
                table_until = piece.until;
                for (int i = tid; i < piece.entries; i += C::kThreads) {
                    int p = pages[table_from + i];
                    if (p < 0 || p >= a.pages) {
                        table_bad = true;
                        p = 0;
                    }
                    table[i] = p;
                }
                __syncthreads();
            };
            unsigned long of_row = 0;  // the address of this lane's row, of the keys of the tile that is asked for next or was last
            const unsigned long first_key = reinterpret_cast<uintptr_t>(a.kc) + head * a.head_step, first_own = reinterpret_cast<uintptr_t>(a.k) + 2 * (b * a.ks.a + head * a.ks.c);
            const auto locate = [&](int t) {
                if (t < items.cached) {
                    look_up(t);
                    // past the end the last key again, which is masked; the end of the last tile is a multiple of kTile up to 2^31, so that my_row < kTile
                    // leaves the sum below it
                    static_assert((1u << 31) % C::kTile == 0, "tiles end at 2^31");
                    const unsigned pos = (unsigned)min(t * C::kTile + my_row, s.L - 1);
                    const unsigned col = a.page_of(pos), slot = pos - col * (unsigned)a.page_size;
                    of_row = (unsigned long)(unsigned)table[col - table_from] * a.page_step + ((unsigned long)slot * a.slot_step + first_key);
                } else {
                    of_row = first_own + 2 * (min((t - items.cached) * C::kTile + my_row, s.N) * a.ks.b);
                }
            };
            const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_offset(lds)) + wave * C::kLoads * 1024;
            const int asks = 4 * (lane / C::kLanes);
            const auto load = [&](long by, unsigned to) {
#pragma unroll
                for (int j = 0; j < C::kLoads; ++j) {
                    const unsigned lo = (unsigned)__builtin_amdgcn_ds_bpermute(asks + 4 * C::kRows * j, (int)(unsigned)of_row);
                    const unsigned hi = (unsigned)__builtin_amdgcn_ds_bpermute(asks + 4 * C::kRows * j, (int)(unsigned)(of_row >> 32));
                    const unsigned piece = 16u * ((lane % C::kLanes) ^ turn<D>(first_row + j * C::kRows + lane / C::kLanes));
                    load_lds(to + j * 1024, reinterpret_cast<const char*>(((unsigned long)hi << 32 | lo) + (by + piece)));
                }
            };
            const auto load_keys = [&](int stage) { load(0, lds0 + stage * C::kStage); };
            const auto load_values = [&](int t, int stage) { load(t < items.cached ? a.vc - a.kc : a.v - a.k, lds0 + stage * C::kStage + C::kTileBytes); };

            constexpr int kAhead = C::kHeld - 1;
            constexpr bool kShared = C::WM > 1, kTurns = C::kWaves > 4;
            const auto ask = [&](int t, int place) {  // values of t, whose keys were asked for last, and keys of t + 1
                if (t >= t1) return;
                load_values(t, place);
                if (t + 1 >= t1) return;
                locate(t + 1);
                load_keys(place == kAhead ? 0 : place + 1);
            };
            if constexpr (kTurns) {
                locate(t0);
                load_keys(0);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) ask(t0 + i, i);
            } else {
#pragma unroll
                for (int i = 0; i < C::kHeld; ++i)
                    if (t0 + i < t1) {
                        locate(t0 + i);
                        load_keys(i);
                        if (i < kAhead) load_values(t0 + i, i);
                    }
            }
            x8 q[kSteps];  // behind the first loads of keys: they are all on their way together
            {
                const char* const qp = a.q + 2 * (b * a.qs.a + min(row, s.N) * a.qs.b + query * a.qs.c) + 16 * half;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    u32v4 w = *reinterpret_cast<const u32v4*>(qp + 32 * i);
                    if (a.negative) w ^= 0x80008000u;
                    q[i] = __builtin_bit_cast(x8, w);
                }
            }
            if (t1 > items.cached && a.parents) {
                const int32_t* const parents = a.parents + (long)b * a.N;
                for (int i = tid; i < s.N; i += C::kThreads) {
                    int p = parents[i];
                    if (p < -1 || p >= i) {
                        bad = true;
                        p = -1;
                    }
                    up[i + 1] = (unsigned short)(p + 1);
                }
                __syncthreads();
            }
            const char* const mine = lds + wk * kSub * 32 * C::kRowBytes;
            f32x16 sc[kSub];
            x8 weights[kSub][2];
            // of tile t: whether it is of the block's own rows and not of the cache, the rows or positions that there are, the first of this wave's keys
            const auto is_own = [&](int t) { return t >= items.cached; };
            const auto limit_of = [&](int t) { return is_own(t) ? s.N + 1 : s.L; };
            const auto base_of = [&](int t) { return (is_own(t) ? t - items.cached : t) * C::kTile + wk * kSub * 32; };
            union Values {  // of 32 keys, transposed: 4 keys of a column each read
                s16x4 h[2];
                x8 all;
            };
            const auto read_keys = [&](int at, int sub, x8 (&k)[kSteps]) {
                const int r = lane & 31, x = half ^ turn<D>(r);
                const char* const kr = mine + at * C::kStage + (sub * 32 + r) * C::kRowBytes;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) k[i] = *reinterpret_cast<const x8*>(kr + ((2 * i) ^ x) * 16);
            };
            const auto read_values = [&](int at, int sub, Values (&v)[kBlocks][2]) {
                const char* const vt = mine + at * C::kStage + C::kTileBytes + sub * 32 * C::kRowBytes;
                const int q4 = (lane & 15) >> 2, wide = lane >> 4 & 1;
#pragma unroll
                for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * i + 4 * half + q4, piece = db * 4 + 2 * wide + ((lane & 3) >> 1);
                        v[db][i / 2].h[i % 2] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(vt + r * C::kRowBytes + (piece ^ turn<D>(r)) * 16 + (lane & 1) * 8));
                    }
            };
            const auto score = [&](int sub, const x8 (&k)[kSteps]) {
                sc[sub] = f32x16{};
#pragma unroll
                for (int i = 0; i < kSteps; ++i) sc[sub] = mfma<DT>(k[i], q[i], sc[sub]);
            };
            const auto take = [&](int sub, const Values (&v)[kBlocks][2]) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int db = 0; db < kBlocks; ++db) o[db] = mfma<DT>(v[db][kb].all, weights[sub][kb], o[db]);
            };
            const auto weigh = [&](int t) {
                const bool own = is_own(t);
                const int limit = limit_of(t), base = base_of(t);
                if (own || limit - base < 32 * kSub)
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub) {
                        const unsigned seen = seen_keys(own, a.parents != nullptr, base + 32 * sub, limit, row, s.N, up) >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(seen >> (8 * (i / 4) + i % 4) & 1)) sc[sub][i] = -__builtin_huge_valf();
                    }
                float top = sc[0][0];
#pragma unroll
                for (int sub = 0; sub < kSub; ++sub)
#pragma unroll
                    for (int i = sub == 0 ? 1 : 0; i < 16; ++i) top = fmaxf(top, sc[sub][i]);
                // one reference for all weights of the tile, which are products only later
                top = halves_max(top) * a.scale;
                const bool rise = top > m + H::kSlack;
                if (__ballot(rise)) {
                    const float to = rise ? top : m, by = __builtin_amdgcn_exp2f(m - to);
                    m = to;
                    l *= by;
#pragma unroll
                    for (int i = 0; i < kBlocks; ++i) o[i] *= by;
                }
                const float ref = H::kLift - m;
#pragma unroll
                for (int sub = 0; sub < kSub; ++sub) {
                    float p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        p[i] = __builtin_amdgcn_exp2f(fmaf(sc[sub][i], a.scale, ref));
                        weights[sub][i / 8][i % 8] = (typename H::T)p[i];
                    }
                    l += tree_sum16(p);
                }
            };
            // Values of the block that are not finite count for the rows that see them alone, which have NaN; a product with a weight of 0 is none
            const auto look_at_own = [&](int t, int at) {
                const int limit = limit_of(t), base = base_of(t);
                unsigned odd[kSub];
#pragma unroll
                for (int sub = 0; sub < kSub; ++sub) {
                    const char* const vr = mine + at * C::kStage + C::kTileBytes + (sub * 32 + (lane & 31)) * C::kRowBytes + half * D;
                    unsigned is = 0;  // an exponent of all ones carries into the sign's bit
#pragma unroll 4
                    for (int i = 0; i < D / 4; ++i) is |= (reinterpret_cast<const unsigned*>(vr)[i] & 0x7FFF7FFFu) + 0x10001u * (0x8000u - H::kExponent);
                    const unsigned long long ballot = __ballot((is & 0x80008000u) != 0);
                    odd[sub] = (unsigned)ballot | (unsigned)(ballot >> 32);
                    if (odd[sub] && limit - base > 32 * sub && (odd[sub] & seen_keys(true, a.parents != nullptr, base + 32 * sub, limit, row, s.N, up)))
                        l = __builtin_nanf("");
                }
                __syncthreads();  // other waves look at the same values
#pragma unroll
                for (int sub = 0; sub < kSub; ++sub)
                    if (odd[sub] >> (lane & 31) & 1) {
                        char* const vr = lds + (mine - lds) + at * C::kStage + C::kTileBytes + (sub * 32 + (lane & 31)) * C::kRowBytes + half * D;
                        for (int i = 0; i < D / 4; ++i) reinterpret_cast<unsigned*>(vr)[i] = 0;
                    }
                __syncthreads();
            };
            int at = 0;  // the place of tile t
            if constexpr (kTurns) {
                // Two waves a SIMD: between two barriers the first four take a tile's values, score the next one's keys and weigh them, the others weigh a
                // tile's keys, take its values and score the next one's, so that the matrix unit has one wave's products while the other's weights
                // are formed: 4 times 64 rows over 65536 tokens 330 us, 365 with all waves in step.  Keys of t and values of t - 1 are done with at the
                // barrier of t, and their places asked for again.
                const bool later = wave >= 4;
                if (t1 - t0 >= C::kHeld) wait_loads<2 * C::kLoads * kAhead>();
                else wait_loads<0>();
                asm volatile("s_barrier" : : : "memory");
                const auto score_tile = [&](int place) {
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub) {
                        x8 k[kSteps];
                        read_keys(place, sub, k);
                        __builtin_amdgcn_sched_barrier(0);
                        score(sub, k);
                    }
                };
                score_tile(0);
                if (!later) weigh(t0);
                for (int t = t0; t < t1; ++t) {
                    const int next = at == kAhead ? 0 : at + 1;
                    if (t1 - 1 - t >= kAhead) wait_loads<2 * C::kLoads*(C::kHeld - 2)>();
                    else wait_loads<0>();
                    asm volatile("s_barrier" : : : "memory");
                    if (is_own(t)) look_at_own(t, at);
                    ask(t + kAhead, at > 0 ? at - 1 : kAhead);
                    if (later) weigh(t);
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub) {
                        Values v[kBlocks][2];
                        read_values(at, sub, v);
                        __builtin_amdgcn_sched_barrier(0);
                        take(sub, v);
                    }
                    if (t + 1 < t1) score_tile(next);
                    if (!later && t + 1 < t1) weigh(t + 1);
                    at = next;
                }
            } else {
                // kHeld tiles are held, and half a tile is asked for as soon as its place is free: values of t + kHeld - 1 behind the products with the
                // values of t - 1, keys of t + kHeld behind those with the keys of t.  All but one of the halves are on their way at any time.  Waves that
                // share their keys meet at every half; others go on by themselves.
                for (int t = t0; t < t1; ++t) {
                    const bool some = base_of(t) < limit_of(t);
                    arrived<C::kLoads, C::kHeld, kShared>(t1 - 1 - t);
                    // All reads of LDS before the first product: one by one, each waited for, they took most of a tile's time
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub) {
                        x8 k[kSteps];
                        read_keys(at, sub, k);
                        __builtin_amdgcn_sched_barrier(0);
                        if (sub == 0) {
                            if (t + kAhead < t1) load_values(t + kAhead, at > 0 ? at - 1 : kAhead);
                            if (t + C::kHeld < t1) locate(t + C::kHeld);
                        }
                        score(sub, k);
                    }
                    if (some) weigh(t);
                    arrived<C::kLoads, C::kHeld, kShared>(t1 - 1 - t);
                    if (is_own(t)) look_at_own(t, at);
#pragma unroll
                    for (int sub = 0; sub < kSub; ++sub) {
                        Values v[kBlocks][2];
                        read_values(at, sub, v);
                        __builtin_amdgcn_sched_barrier(0);
                        if (sub == 0 && t + C::kHeld < t1) load_keys(at);
                        if (some) take(sub, v);
                    }
                    at = at == kAhead ? 0 : at + 1;
                }
            }
            l += __shfl_xor(l, 32, kWave);
        }
        if (bad || (table_bad && table_of == b)) sh_bad[done & 1] = 1;
        // the waves' sums over their keys to those of the first
        __syncthreads();
        float* const hand = reinterpret_cast<float*>(lds);
        if (C::WK > 1) {
            if (half == 0) hand_ml[wk][place_of] = make_float2(m, l);
            if (wk > 0) {
                float* const to = hand + ((wk - 1) * C::kColumns + place_of) * C::kPad;
#pragma unroll
                for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32v4*>(to + db * 32 + 8 * i + 4 * half) = f32v4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
            }
            __syncthreads();
        }
        if (wk == 0) {
            if (C::WK > 1) {
                float top = m;
                for (int w = 1; w < C::WK; ++w) top = fmaxf(top, hand_ml[w][place_of].x);
                const float by = __builtin_amdgcn_exp2f(m - top);
                l *= by;
                m = top;
#pragma unroll
                for (int db = 0; db < kBlocks; ++db) o[db] *= by;
                for (int w = 1; w < C::WK; ++w) {
                    const float2 ml = hand_ml[w][place_of];
                    const float f = __builtin_amdgcn_exp2f(ml.x - m);
                    l = fmaf(ml.y, f, l);
                    const float* const from = hand + ((w - 1) * C::kColumns + place_of) * C::kPad;
#pragma unroll
                    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f32v4 x = *reinterpret_cast<const f32v4*>(from + db * 32 + 8 * i + 4 * half);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[db][4 * i + j] = fmaf(x[j], f, o[db][4 * i + j]);
                        }
                }
            }
            if (sh_bad[done & 1]) l = __builtin_nanf("");
            if (row < rows) {
                if (whole) {
                    const float by = 1.f / l;
                    char* const to = a.out + 2 * (b * a.os.a + row * a.os.b + query * a.os.c + 4 * half);
#pragma unroll
                    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            typename H::T r[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) r[j] = (typename H::T)(o[db][4 * i + j] * by);
                            __builtin_memcpy(__builtin_assume_aligned(to + 2 * (db * 32 + 8 * i), 8), r, 8);
                        }
                } else {
                    const long slot = 2l * blockIdx.x + (done == 0 ? 0 : 1), at = slot * C::kColumns + place_of;
                    if (half == 0) a.part_ml[at] = make_float2(m, l);
                    float* const to = a.part_o + at * D + 4 * half;
#pragma unroll
                    for (int db = 0; db < kBlocks; ++db)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<f32v4*>(to + db * 32 + 8 * i) = f32v4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
                }
            }
        }
        ++done;
        rel += t1 - t0;
        u += t1 - t0;
    }
    if (a.tree_len) {  // rows that belong to nobody are 0
        const int pieces = a.group * a.kv_heads * (D / 8);
        for (long r = blockIdx.x; r < (long)a.B * (a.N + 1); r += gridDim.x) {
            const int b = (int)(r / (a.N + 1)), row = (int)(r % (a.N + 1));
            const Sequence s = sequence<true>(a, b);
            if (s.bad || row <= s.N) continue;
            for (int i = tid; i < pieces; i += C::kThreads)
                *reinterpret_cast<uint4*>(a.out + 2 * (b * a.os.a + row * a.os.b + (i / (D / 8)) * a.os.c) + 16 * (i % (D / 8))) = make_uint4(0, 0, 0, 0);
        }
    }
}

// The parts of the items that shares' beginnings cut, a workgroup for some columns of each.
constexpr int kJoinThreads = 256;
template <int DT, typename C>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(const AttnArgs a) {
    using H = Half<DT>;
    constexpr int D = C::D, kLanes = D / 4;
    const int w = blockIdx.x + 1, tid = threadIdx.x;
    const Cut cut = a.cuts[w];
    if (cut.parts == 0) return;
    const Sequence s = sequence<true>(a, cut.b);
    const int of_block = blockIdx.y * (kJoinThreads / kLanes) + tid / kLanes, column = cut.block * C::kColumns + of_block, row = column / a.group;
    if (row >= (s.bad ? a.N : s.N) + 1) return;
    // the share before has the item's first part
    const auto at = [&](int x) { return (2l * (w - 1 + x) + (x == 0 ? cut.second : 0)) * C::kColumns + of_block; };
    float m = -1e30f, l = 0.f;
#pragma unroll 4
    for (int x = 0; x < cut.parts; ++x) m = fmaxf(m, a.part_ml[at(x)].x);
    f32v4 o = {};
#pragma unroll 4
    for (int x = 0; x < cut.parts; ++x) {
        const float2 ml = a.part_ml[at(x)];
        const f32v4 v = *reinterpret_cast<const f32v4*>(a.part_o + at(x) * D + 4 * (tid % kLanes));
        const float f = __builtin_amdgcn_exp2f(ml.x - m);
        l = fmaf(ml.y, f, l);
        o += v * f;
    }
    typename H::T r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (typename H::T)(o[j] / l);
    char* const to = a.out + 2 * (cut.b * a.os.a + row * a.os.b + (cut.head * a.group + (column - row * a.group)) * a.os.c + 4 * (tid % kLanes));
    __builtin_memcpy(__builtin_assume_aligned(to, 8), r, 8);
}

// What a call takes: its shares, one a workgroup that runs at once, and no more than it may have units.
struct AttnPlan {
    int shares;  // 0: more units than 32 bits count
    size_t off_ml, off_cuts, bytes;
};
template <typename C>
AttnPlan plan_for(const ss_tree_params& p) {
    const TreeTiles tiles{C::kTile, C::kColumns, p.heads / p.kv_heads, p.kv_heads};
    TreeItems most = tree_items(tiles, 0, p.nodes, false, p.nodes);
    most.cached = (int)(((long)p.table_width * p.page_size + C::kTile - 1) / C::kTile);
    const double units = (double)most.tiles() * most.blocks * p.kv_heads * p.batch;
    AttnPlan r{};
    if (units >= 2147483648.0) return r;
    r.shares = device_cu_count() * C::kGroups;
    if (r.shares > kMaxShares) r.shares = kMaxShares;
    if (units < r.shares) r.shares = units < 1 ? 1 : (int)units;
    const size_t slots = 2 * (size_t)r.shares * C::kColumns;
    r.off_ml = slots * C::D * 4;
    r.off_cuts = r.off_ml + slots * 8;
    r.bytes = (r.off_cuts + (size_t)r.shares * sizeof(Cut) + 255) / 256 * 256;
    return r;
}

template <typename F>
auto with_shape(const ss_tree_params& p, F f) {
    const int columns = (p.nodes + 1) * (p.heads / p.kv_heads);
    if (p.head_dim == 64) {
        if (columns <= 32) return f(Shape<64, 1, 4, 1, 2, 2>{});
        if (columns <= 64) return f(Shape<64, 2, 2, 2, 2, 2>{});
        if (columns <= 128) return f(Shape<64, 4, 1, 2, 4, 2>{});
        return f(Shape<64, 8, 1, 2, 8, 1>{});
    }
    if (columns <= 32) return f(Shape<128, 1, 4, 1, 1, 2>{});
    if (columns <= 64) return f(Shape<128, 2, 2, 1, 2, 2>{});
    if (columns <= 128) return f(Shape<128, 4, 1, 2, 2, 2>{});
    return f(Shape<128, 8, 1, 2, 4, 1>{});
}

}  // namespace

extern "C" {

size_t specsteer_tree_attention_workspace_bytes(const ss_tree_params* params) {
    TreeShape s;
    if (tree_shape(params, true, s) != SS_OK) return 0;
    return with_shape(*params, [&](auto shape) { return plan_for<decltype(shape)>(*params).bytes; });
}

ss_status specsteer_tree_attention(const void* q, const void* k, const void* v, const void* k_cache, const void* v_cache, const int32_t* block_table,
                                   const int32_t* cache_len, const int32_t* parents, const int32_t* tree_len, const ss_tree_params* params, void* out,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    TreeShape s;
    const ss_status chk = tree_shape(params, true, s);
    if (chk != SS_OK) return chk;
    if (params->batch == 0) return SS_OK;
    const bool cached = params->pages > 0 && params->table_width > 0;
    if (!q || !k || !v || !cache_len || !out || (cached && (!k_cache || !v_cache || !block_table))) return SS_ERR_NULL;
    if (off_16(q) || off_16(k) || off_16(v) || off_16(out) || (cached && (off_16(k_cache) || off_16(v_cache)))) return SS_ERR_STRIDE;
    return with_shape(*params, [&](auto shape) {
        using C = decltype(shape);
        const AttnPlan plan = plan_for<C>(*params);
        if (plan.shares == 0) return SS_ERR_SHAPE;
        if (bad_workspace(workspace, workspace_bytes, plan.bytes)) return SS_ERR_WORKSPACE;
        const auto in = [](const void* p) { return static_cast<const char*>(p); };
        AttnArgs a{};
        a.q = in(q);
        a.k = in(k);
        a.v = in(v);
        a.kc = in(k_cache);
        a.vc = in(v_cache);
        a.table = block_table;
        a.cache_len = cache_len;
        a.parents = params->nodes ? parents : nullptr;
        a.tree_len = tree_len;
        a.out = static_cast<char*>(out);
        a.part_o = static_cast<float*>(workspace);
        a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + plan.off_ml);
        a.cuts = reinterpret_cast<Cut*>(static_cast<char*>(workspace) + plan.off_cuts);
        a.qs = s.q;
        a.ks = s.k;
        a.os = s.out;
        a.page_step = (unsigned)(2 * s.cache.a);
        a.slot_step = (unsigned)(2 * s.cache.b);
        a.head_step = 2 * s.cache.c;
        a.page_of = page_of(params->page_size);
        a.ts = s.table;
        a.B = params->batch;
        a.N = params->nodes;
        a.kv_heads = params->kv_heads;
        a.group = params->heads / params->kv_heads;
        a.pages = params->pages;
        a.page_size = params->page_size;
        a.width = cached ? params->table_width : 0;
        a.shares = plan.shares;
        // a factor of 0 would make masked scores NaN, and an infinite one scores of 0; the least normal number tells scores apart beyond 1e37 only
        a.scale = (float)std::fmin(std::fmax(std::fabs((double)params->scale) * 1.4426950408889634, 1.1754944e-38), 3.4028234e38);
        a.negative = params->scale < 0.f;
        hipStream_t st = static_cast<hipStream_t>(stream);
        const bool bf = params->dtype == SS_BF16;
        launch(bf ? attention_kernel<SS_BF16, C> : attention_kernel<SS_TREE_F16, C>, dim3((unsigned)plan.shares), dim3(C::kThreads), 0, st, (const AttnArgs)a);
        if (plan.shares > 1)
            launch(bf ? attention_join_kernel<SS_BF16, C> : attention_join_kernel<SS_TREE_F16, C>,
                   dim3((unsigned)plan.shares - 1, (unsigned)(C::kColumns * (C::D / 4) / kJoinThreads)), dim3(kJoinThreads), 0, st, (const AttnArgs)a);
        return tree_launched();
    });
}

const char* specsteer_tree_status_string(int status) {
    switch (status) {
        case SS_OK: return "ok";
        case SS_ERR_NULL: return "a required pointer is NULL";
        case SS_ERR_SHAPE: return "batch, nodes, heads, head_dim, pages or vocab out of range";
        case SS_ERR_DTYPE: return "unknown dtype";
        case SS_ERR_PARAM: return "scale, lambda, beta, temperature or flags out of range";
        case SS_ERR_STRIDE: return "strides negative, off 16 bytes or overlapping, or a pointer off its alignment";
        case SS_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case SS_ERR_DEVICE: return "HIP launch failed";
        default: return "unknown status";
    }
}

}  // extern "C"
