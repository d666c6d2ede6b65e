// The kernels of attention over a paged cache (mpv_attention.hip, mpv_prefix.hip), and what the host decides about them.
//
// With s the scaled products of a query with the keys it sees, out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), in one pass over the
// keys with a running reference m (log2 units).  The work is cut into tiles of kTile keys; a unit is what a tree's nodes read of one
// cache head: its tiles are those of the sinks, of the window (or the whole context), and of the tree.  All tiles of all units
// form one list, which is divided evenly among teams of workgroups, whatever the lengths of the contexts: a team carries on across
// units, and a unit that several teams share is put together by combine_kernel from their partial sums.  A member of a team has
// kRows of the rows (node, query head) that read the unit; the members read the same tiles at about the same time, on the
// same chiplet, so that only one of them waits for memory and the others find the tile in the chiplet's L2.
//
// A tile of keys and values goes straight from memory to LDS (16 bytes a lane), up to three tiles ahead of the one that is worked on;
// so do the entries of the block table, a batch of tiles ahead: a lane then works out where one key's rows lie.
//   products    S^T = K Q^T: keys are the rows of the matrix instruction's first operand, read from LDS; queries stay in registers
//   weights     lane l then holds 4 consecutive keys for query l % 16: the statistics of a query lie in 4 lanes, and the weights are
//               where the second product wants them (the order of keys within an instruction does not matter if both operands have it)
//   out^T = V^T W^T   16-bit values come out of LDS transposed (ds_read_b64_tr_b16), float32 ones are read a value a lane
// Rows of a tile lie in LDS with their 16-byte chunks exchanged by row, so that 16 rows' equal chunks lie in different banks.
//
// Weights are rounded to the type of the values, which the matrix instruction wants; the sum that divides them adds up the rounded
// ones, so that a common factor of their errors falls out.  Everything else (products, references, both sums) is float32.

#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstring>

#include "mpv_host.h"

namespace mpv {

struct AttentionArgs {
    mpv_attention a;
    mpv_attention_buffers b;
    int8_t parent[MPV_MAX_NODES];          // the shared shape (without tree_parent)
    int teams;
    int blocks;                            // row blocks of the largest tree: members of a team
    int group;                             // query heads of a cache head
    Divisor by_group, by_page;
    float factor;                          // |scale| log2(e): products to exponents (1 where the scale is 0)
    int sign;                              // of the scale: -1, 0, 1
    float* partial;                        // [teams][members][2][rows][columns]
    float2* partial_stats;                 // [teams][members][2][rows]: reference, sum of weights
    int4* split;                           // shared units (tree, cache head, first and last team; x < 0: none), by unit or by the first team
    int by_unit;
};

// What a kernel attends to: a tree's context and the tree (mpv_tree_attention); the same behind a prefix that others share, whose
// sums the rows begin with; such a prefix, for the nodes of all trees that follow each other and share it, up to 64 of them; or a tree's
// prefix, context and nodes, one after the other.
constexpr int kTree = 0, kBehind = 1, kPrefix = 2, kThrough = 3;

struct PrefixArgs : AttentionArgs {
    const int32_t* prefix_of;              // null: there are none
    const int32_t* prefix_table;
    const int32_t* prefix_len;
    int prefixes, prefix_width;
    float* lse;                            // null: not wanted
    float* partial_exact;                  // [teams][members][2][rows]: sums of the weights as they were before they were rounded
    int2* units;                           // kPrefix, [B][kv_heads][supers]: first and last team of a unit (last < 0: one team's alone)
    int supers;                            // units of a cache head, at most
    Divisor by_rows;                       // rows of a block
    // what a prefix gives to the rows [B,N,heads]: columns of their sums; reference and sum of weights; the same before rounding
    float* state;
    float2* state_stats;
    float* state_exact;
};
template <int KIND> struct ArgsOf { typedef PrefixArgs T; };
template <> struct ArgsOf<kTree> { typedef AttentionArgs T; };

// The prefix of a tree: which (negative: none), and how long.
__device__ __forceinline__ int prefix_of(const PrefixArgs& g, int b) {
    if (!g.prefix_of || b >= g.a.B) return -1;
    const int which = g.prefix_of[b];
    return which < g.prefixes ? which : -1;
}
__device__ __forceinline__ int prefix_length(const PrefixArgs& g, int which) {
    return which < 0 ? 0 : min(max(g.prefix_len[which], 0), g.prefix_width * g.a.page_size);
}

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short i16x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

template <int DTYPE> struct Elem;
template <> struct Elem<MPV_DTYPE_F32> {
    typedef float T;
    static constexpr int kBytes = 4;
    static constexpr float kBias = 0.0f;
    static __device__ __forceinline__ void put4(char* to, const f32x4& v) { *reinterpret_cast<f32x4*>(to) = v; }
};
template <> struct Elem<MPV_DTYPE_BF16> {
    typedef __bf16 T;
    typedef bf16x8 Vec;
    static constexpr int kBytes = 2;
    static constexpr float kBias = 0.0f;
    static constexpr uint32_t kInf = 0x7f80, kOnes = 0x3f803f80;
    static __device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void put4(char* to, const f32x4& v) {
        typedef __attribute__((ext_vector_type(4))) __bf16 x4;
        x4 r;
        for (int i = 0; i < 4; ++i) r[i] = static_cast<__bf16>(v[i]);
        *reinterpret_cast<x4*>(to) = r;
    }
};
template <> struct Elem<MPV_DTYPE_F16> {
    typedef _Float16 T;
    typedef f16x8 Vec;
    static constexpr int kBytes = 2;
    static constexpr float kBias = 6.0f;   // weights are kept 2^6 times as large, so that the small ones stay normal numbers
    static constexpr uint32_t kInf = 0x7c00, kOnes = 0x3c003c00;
    static __device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void put4(char* to, const f32x4& v) {
        typedef __attribute__((ext_vector_type(4))) _Float16 x4;
        x4 r;
        for (int i = 0; i < 4; ++i) r[i] = static_cast<_Float16>(v[i]);
        *reinterpret_cast<x4*>(to) = r;
    }
};

// What the row of a key that nobody sees is read from.
__device__ const uint4 kZeros[MPV_MAX_HEAD_DIM * 4 / 16] = {};

// 16 bytes a lane to LDS, from `to` on (the wave's first lane's place) in lane order.  Written as an instruction: the compiler would
// wait for all such loads in flight before it reads LDS through ds_read_b64_tr_b16, the next tile's among them.  Nothing but `arrive`
// waits for them.  (A load that goes to LDS may follow a write of m0 after one wait state.)
__device__ __forceinline__ void to_lds(uint64_t from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void word_to_lds(uint64_t from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
// A place in LDS.  (The pass for the host, which never runs it, has pointers of 64 bits.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Wint-to-pointer-cast"
__device__ __forceinline__ __attribute__((address_space(3))) char* lds_place(uint32_t at) {
    return reinterpret_cast<__attribute__((address_space(3))) char*>(at);
}
#pragma clang diagnostic pop
// What a wave's lanes wrote to LDS is there for its other lanes (LDS serves a wave in order; the compiler must keep that order).
__device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ unsigned long long shfl64(unsigned long long v, int lane) {
    const uint32_t lo = __shfl(static_cast<uint32_t>(v), lane), hi = __shfl(static_cast<uint32_t>(v >> 32), lane);
    return static_cast<unsigned long long>(hi) << 32 | lo;
}

// The reference of a softmax moves only where a product exceeds it by more than this (log2 units): weights are at most 2^8.
constexpr float kSlack = 8.0f;
// The logarithm of a sum of weights: `exact` of them, 2^bias as large as their reference says.
__device__ __forceinline__ float lse_of(float top, float exact, float bias) {
    return exact > 0.0f || exact != exact ? (top - bias + __builtin_amdgcn_logf(exact)) * 0.69314718055994531f : -INFINITY;
}
__device__ __forceinline__ int64_t uniform64(unsigned long long v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
    return static_cast<int64_t>(static_cast<unsigned long long>(hi) << 32 | lo);
}
// x, as if it had just been read: what depends on it is worked out where it is needed and does not occupy registers across the loops.
__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// What beginning and ending a unit takes, in tiles: workgroups with many short units would end last otherwise.  256 trees of 8 nodes,
// contexts of 16 to 256: 66 us, 91 without; the benchmark's trees 613 us, 637 without; contexts of one length: the same.
constexpr int kUnitCost = 8;
// All bits where bit `at` is set, none otherwise.  (Masks instead of conditions: those would all wait in scalar registers at once.)
__device__ __forceinline__ uint32_t spread(uint32_t bits, int at) { return static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - at)) >> 31); }

// A tree's part of the list of tiles.
struct TreeWork {
    int context, nodes;
    int sink_tiles, low, context_tiles;    // tiles of the sinks, first position (a whole tile) of the rest, its tiles
    int tiles;                             // of a unit, the tree's own among them
    int blocks;                            // row blocks
    int sinks;                             // (kBehind) those of the context
    int before;                            // (kThrough) positions of the prefix
    // (kPrefix: `context` is the prefix's length, `nodes` are all nodes of the trees that share it; no tree's own tiles.)
    int which, first, end;                 // the prefix, its first tree, the tree behind its last
    int supers;                            // units of a cache head: `blocks` row blocks each
    int latest;                            // the longest context
};

template <int KIND, int TILE, int ROWS>
__device__ __forceinline__ TreeWork tree_work(const typename ArgsOf<KIND>::T& g, int b) {
    TreeWork t;
    const mpv_attention& a = g.a;
    t.context = min(max(g.b.context_len[b], 0), a.table_width * a.page_size);
    t.nodes = g.b.num_nodes ? min(max(g.b.num_nodes[b], 0), a.N) : a.N;
    if constexpr (KIND == kThrough) {
        t.which = prefix_of(g, b);
        t.before = prefix_length(g, t.which);
        t.context += t.before;
    }
    t.low = t.sink_tiles = 0;
    t.sinks = max(a.sinks, 0);
    if constexpr (KIND == kBehind)
        if (a.window > 0 && t.sinks > 0) t.sinks = max(0, t.sinks - prefix_length(g, prefix_of(g, b)));
    if (a.window > 0) {
        t.low = max(0, t.context - a.window + 1) / TILE * TILE;
        t.sink_tiles = (min(t.sinks, t.low) + TILE - 1) / TILE;
    }
    t.context_tiles = (t.context - t.low + TILE - 1) / TILE;
    t.tiles = t.sink_tiles + t.context_tiles + (t.nodes + TILE - 1) / TILE;
    t.blocks = (t.nodes * g.group + ROWS - 1) / ROWS;
    return t;
}

// Inclusive sum over the wave.
__device__ __forceinline__ int wave_sum(int v) {
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}
// The nodes of tree `b`, a lane's each.
__device__ __forceinline__ int nodes_of(const AttentionArgs& g, int b) {
    if (b >= g.a.B) return 0;
    return g.b.num_nodes ? min(max(g.b.num_nodes[b], 0), g.a.N) : g.a.N;
}
// Of the trees from `base` on, a lane's each: those that share a prefix and follow each other, at the lane of the first of them
// (nodes = 0 at the others).  All lanes call it.
template <int TILE, int ROWS>
__device__ __forceinline__ TreeWork prefix_work(const PrefixArgs& g, int base) {
    const mpv_attention& a = g.a;
    const int lane = threadIdx.x & 63, b = base + lane;
    TreeWork t;
    t.which = prefix_of(g, b);
    t.context = prefix_length(g, t.which);
    const int mine = nodes_of(g, b);
    const int before = __shfl_up(t.which, 1);
    const unsigned long long firsts = __ballot(lane == 0 || before != t.which);
    const unsigned long long later = lane == 63 ? 0 : firsts >> (lane + 1);
    const int end = later ? lane + __ffsll(later) : 64;
    const int upto = wave_sum(mine);
    const int last = __shfl(upto, end - 1);
    t.nodes = (firsts >> lane & 1) && t.context > 0 ? last - upto + mine : 0;
    t.first = b;
    t.end = base + end;
    t.low = t.sink_tiles = t.latest = 0;
    t.sinks = max(a.sinks, 0);
    if (a.window > 0) {
        // the contexts of its trees: no node sees a position more than a window before the shortest
        int least = b < a.B ? min(max(g.b.context_len[b], 0), a.table_width * a.page_size) : 0, most = least;
        for (int d = 1; d < 64; d <<= 1) {
            const int l = __shfl_down(least, d), m = __shfl_down(most, d);
            if (lane + d < end) { least = min(least, l); most = max(most, m); }
        }
        t.latest = most;
        // (a tile at least, so that the rows get their state)
        t.low = static_cast<int>(min(static_cast<int64_t>(max(t.context - 1, 0)), max(static_cast<int64_t>(0), static_cast<int64_t>(t.context) + least - a.window + 1))) / TILE * TILE;
        t.sink_tiles = (min(t.sinks, t.low) + TILE - 1) / TILE;
    }
    t.context_tiles = (t.context - t.low + TILE - 1) / TILE;
    t.tiles = t.sink_tiles + t.context_tiles;
    const int64_t rows = static_cast<int64_t>(t.nodes) * g.group;
    t.blocks = g.blocks;
    t.supers = static_cast<int>((rows + static_cast<int64_t>(ROWS) * g.blocks - 1) / (static_cast<int64_t>(ROWS) * g.blocks));
    return t;
}

// DTYPE; DP: columns of a row in LDS (head_dim, rounded up); QT: 16-row groups of a wave; WAVES; TILE: keys; STAGES: tiles in LDS;
// SHARE: workgroups that a compute unit holds; KIND: see above.
template <int DTYPE, int DP, int QT, int WAVES, int TILE, int STAGES, int SHARE, int KIND>
struct Attention {
    typedef Elem<DTYPE> E;
    typedef typename ArgsOf<KIND>::T Args;
    static constexpr int kWaves = WAVES;
    static constexpr int kThreads = 64 * WAVES;
    static constexpr int kRows = 16 * QT * WAVES;
    static constexpr int kChunks = DP * E::kBytes / 16;            // 16-byte chunks of a row
    static constexpr int kSteps = kChunks / 4;                     // of the first product: 4 chunks of every row
    static constexpr int kGroups = TILE / 16;
    static constexpr int kColumns = DP / 16;                       // 16-column groups of the output
    static constexpr int kTileBytes = TILE * DP * E::kBytes;
    static constexpr int kRowsPerLoad = 64 / kChunks;              // rows that a wave's load brings
    static constexpr int kMyRows = TILE / WAVES;                   // keys that a wave brings, and their values
    static constexpr int kMyLoads = kMyRows / kRowsPerLoad;        // of keys; as many of values
    static constexpr int kBatch = 64 / kMyRows;                    // tiles whose rows a wave's lanes look up at a time
    static constexpr int kAheadTiles = STAGES - 1;
    static constexpr int kTile = TILE;
    static constexpr int kShare = SHARE;
    static constexpr int kWavesOfSimd = WAVES == 4 && SHARE == 3 ? 3 : 2;   // that registers have to leave room for
    static constexpr bool k16 = E::kBytes == 2;
    static_assert(kChunks >= 8 && kChunks <= 64 && kMyLoads >= 1 && kMyRows % kRowsPerLoad == 0 && 64 % kMyRows == 0, "loads");
    static_assert(TILE % (k16 ? 32 : 16) == 0 && kGroups * 4 <= 32, "tile");
    // the entries asked for with one batch are there when the next one begins: the waits of `arrive` leave fewer tiles in flight
    static_assert(kBatch >= kAheadTiles && kAheadTiles * kMyLoads * 2 < 60, "batch");

    struct Shared {
        __align__(1024) char keys[STAGES][kTileBytes];
        __align__(1024) char values[STAGES][kTileBytes];
        __align__(16) uint64_t place[2][kBatch][TILE][2];          // where a key's and its value's row lie
        __align__(16) int pages[WAVES][64];                        // entries of the block table, a lane's each
        __align__(4) uint8_t seen[2][kBatch][TILE];                // whether anybody sees the key
        __align__(8) uint8_t special[2][kBatch][8];                // whether a wave found a key that not every node sees
        int spoiled;                                               // whether a sum is no number, see run
    };

    // A tile: positions of the cache from `base` on, or nodes.
    struct Tile { int base; bool tree; };

    const Args& g;
    Shared& sh;
    const uint32_t shared_at;                                      // of `sh` in LDS
    const int lane, wave, l16, quad;
    // the unit
    int b, kv;
    TreeWork t;
    __device__ __forceinline__ int sinks() const {
        if constexpr (KIND == kBehind) return t.sinks;
        else return g.a.sinks;
    }

    __device__ Attention(const Args& args, Shared& s)
        : g(args), sh(s), shared_at(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)&s)), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), l16(lane & 15), quad(lane >> 4) {}

    static __device__ __forceinline__ int swizzle(int row) { return kChunks >= 16 ? row & 15 : (row >> 1) & 7; }

    __device__ __forceinline__ Tile tile_at(int i) const {
        Tile x;
        x.tree = KIND != kPrefix && i >= t.sink_tiles + t.context_tiles;
        x.base = i < t.sink_tiles ? i * TILE : x.tree ? (i - t.sink_tiles - t.context_tiles) * TILE : t.low + (i - t.sink_tiles) * TILE;
        return x;
    }

    // ---- a batch of tiles: lane i has row i % kMyRows of this wave's in tile i / kMyRows
    struct Row { int key, at; bool tree, seen; };                  // place in the tile, position or node; seen: as far as lengths say
    __device__ __forceinline__ Row row_of(int lane, int tile, int last) const {
        const int mine = tile + lane / kMyRows;
        const Tile x = tile_at(mine);
        Row r;
        r.key = wave * kMyRows + lane % kMyRows;
        r.at = x.base + r.key;
        r.tree = x.tree;
        if constexpr (KIND == kPrefix)
            r.seen = mine < last && r.at < t.context;
        else
            r.seen = mine < last && (x.tree ? r.at < t.nodes
                                            : r.at < t.context && (g.a.window <= 0 || r.at > t.context - g.a.window || r.at < sinks()));
        return r;
    }
    // Asks for the block table's entries of the batch that begins with `tile`.
    __device__ __forceinline__ void ask_pages(int tile, int last) {
        const Row r = row_of(fresh(lane), tile, last);
        const int32_t* entry;
        if constexpr (KIND == kPrefix) entry = g.prefix_table + static_cast<int64_t>(t.which) * g.prefix_width + g.by_page.of(r.at);
        else if constexpr (KIND == kThrough)
            entry = r.at < t.before ? g.prefix_table + static_cast<int64_t>(t.which) * g.prefix_width + g.by_page.of(r.at)
                                    : g.b.block_table + static_cast<int64_t>(b) * g.a.table_width + g.by_page.of(r.at - t.before);
        else entry = g.b.block_table + static_cast<int64_t>(b) * g.a.table_width + g.by_page.of(r.at);
        const uint64_t from = r.seen && !r.tree ? reinterpret_cast<uint64_t>(entry) : reinterpret_cast<uint64_t>(&kZeros);
        word_to_lds(from, shared_at + offsetof(Shared, pages) + wave * 256);
    }
    // The entries are there: works out the places of the batch's rows.
    __device__ __forceinline__ void look_up(int tile, int last, int half) {
        const int lane = fresh(this->lane);
        Row r = row_of(lane, tile, last);
        int64_t offset;
        const char *keys, *values;
        if (r.tree) {
            offset = (static_cast<int64_t>(b) * g.a.N + r.at) * g.a.kv_stride;
            keys = static_cast<const char*>(g.b.tree_k);
            values = static_cast<const char*>(g.b.tree_v);
        } else {
            const int page = sh.pages[wave][lane];
            r.seen = r.seen && page >= 0 && page < g.a.num_pages;
            if constexpr (KIND == kThrough)
                if (r.at >= t.before) r.at -= t.before;
            offset = page * g.a.page_stride + (r.at - g.by_page.of(r.at) * g.a.page_size) * g.a.slot_stride;
            keys = static_cast<const char*>(g.b.cache_k);
            values = static_cast<const char*>(g.b.cache_v);
        }
        offset = (offset + static_cast<int64_t>(kv) * g.a.head_dim) * E::kBytes;
        const int sub = lane / kMyRows;
        const uint64_t zeros = reinterpret_cast<uint64_t>(&kZeros);
        sh.seen[half][sub][r.key] = r.seen;
        sh.place[half][sub][r.key][0] = r.seen ? reinterpret_cast<uint64_t>(keys) + offset : zeros;
        sh.place[half][sub][r.key][1] = r.seen ? reinterpret_cast<uint64_t>(values) + offset : zeros;
        const unsigned long long mask = kMyRows == 64 ? ~0ull : (1ull << (kMyRows % 64)) - 1;
        const bool hidden = (__ballot(!r.seen) >> (sub * kMyRows % 64) & mask) != 0;
        if (lane % kMyRows == 0) sh.special[half][sub][wave] = hidden || r.tree || differs(tile_at(tile + sub));
        wave_order();
    }

    // Asks for a tile whose places are known: reads them, and later sends for the rows.  A key that nobody sees is read as zeros.
    typedef __attribute__((ext_vector_type(2))) uint64_t u64x2;
    struct Places { u64x2 of[kMyLoads]; };
    __device__ __forceinline__ Places places(int half, int sub) const {
        Places p;
#pragma unroll
        for (int j = 0; j < kMyLoads; ++j)
            p.of[j] = *reinterpret_cast<const u64x2*>(sh.place[half][sub][wave * kMyRows + j * kRowsPerLoad + lane / kChunks]);
        return p;
    }
    __device__ __forceinline__ void ask(const Places& p, int stage) {
        const uint32_t to = shared_at + stage * kTileBytes + wave * kMyLoads * 1024;
#pragma unroll
        for (int j = 0; j < kMyLoads; ++j) {
            const int row = wave * kMyRows + j * kRowsPerLoad + lane / kChunks;
            const int chunk = (lane % kChunks) ^ swizzle(row);
            uint64_t k = p.of[j][0] + chunk * 16, v = p.of[j][1] + chunk * 16;
            if (chunk * 16 >= g.a.head_dim * E::kBytes) k = v = reinterpret_cast<uint64_t>(&kZeros);
            to_lds(k, to + j * 1024);
            to_lds(v, to + STAGES * kTileBytes + j * 1024);
        }
    }

    // Waits, for all waves, for the tile that kAheadTiles - 1 others were asked for after (more: otherwise for all); all waves are
    // done with the tile before it then.
    __device__ __forceinline__ void arrive(bool more) {
        if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kMyLoads * (kAheadTiles - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    // ---- the rows of this lane's queries
    u32x4 query[QT][kSteps];
    unsigned long long line[QT];                                   // the node and its ancestors, those that it sees
    int low[QT];                                                   // first position seen (but for the sinks)
    f32x4 out[QT][kColumns];
    float top[QT], base[QT];                                       // reference; what is added to an exponent
    f32x4 weight[QT];                                              // sum of weights: in all four, or (float32) of this lane's keys in the first
    float exact[KIND == kTree || !k16 ? 1 : QT];                   // sum of this lane's keys' weights before they were rounded

    // kPrefix: the rows of all trees that share the prefix.  A lane knows one tree's nodes; `upto`: those of the trees up to its own.
    struct Place { int tree, node; };
    __device__ __forceinline__ int trees_upto() const {
        const int base = t.first & ~63, tree = base + lane;
        return wave_sum(tree >= t.first && tree < t.end ? nodes_of(g, tree) : 0);
    }
    // The `rank`-th of the nodes (a lane's each; all lanes call it; beyond the last one: some tree below t.end).
    __device__ __forceinline__ Place place_of(int rank, int upto) const {
        int at = 0;                                                // trees that end before it
#pragma unroll
        for (int d = 32; d; d >>= 1)
            if (__shfl(upto, at + d - 1) <= rank) at += d;
        const int before = __shfl(upto, max(at - 1, 0));
        return {(t.first & ~63) + at, rank - (at > 0 ? before : 0)};
    }
    __device__ __forceinline__ int depth_of(int tree, int node) const {
        int depth = 0;
        for (;;) {
            const int up = node == 0 ? -1 : g.b.tree_parent ? g.b.tree_parent[static_cast<int64_t>(tree) * g.a.N + node] : g.parent[node];
            if (up < 0 || up >= node) return depth;
            node = up;
            ++depth;
        }
    }
    __device__ __forceinline__ void begin_prefix(int block) {
        const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
        const int group = g.group, upto = trees_upto();
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = block * kRows + (wave * QT + q) * 16 + l16, rank = g.by_group.of(row);
            const bool real = rank < t.nodes;
            const Place p = place_of(min(rank, t.nodes - 1), upto);
            line[q] = 0;
            low[q] = 0;
            // (the sum of lengths may exceed 32 bits; positions of the prefix do not)
            if (g.a.window > 0) {
                const int context = min(max(g.b.context_len[p.tree], 0), g.a.table_width * g.a.page_size);
                const int64_t first = static_cast<int64_t>(t.context) + context + depth_of(p.tree, p.node) + 1 - g.a.window;
                low[q] = static_cast<int>(min(first, static_cast<int64_t>(t.context)));
            }
            const char* from = static_cast<const char*>(g.b.q) +
                ((static_cast<int64_t>(p.tree) * g.a.N + p.node) * g.a.q_stride + static_cast<int64_t>(kv * group + row - rank * group) * g.a.head_dim) * E::kBytes;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int chunk = s * 4 + quad;
                u32x4 v = {0u, 0u, 0u, 0u};
                if (real && chunk * 16 < g.a.head_dim * E::kBytes && g.sign != 0) v = *reinterpret_cast<const u32x4*>(from + chunk * 16);
                if (g.sign < 0) v ^= k16 ? 0x80008000u : 0x80000000u;
                query[q][s] = v;
            }
            top[q] = -INFINITY;
            base[q] = 0.0f;
            weight[q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (k16) exact[q] = 0.0f;
#pragma unroll
            for (int c = 0; c < kColumns; ++c) out[q][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }

    __device__ __forceinline__ void begin(int block, int first_tile) {
        if constexpr (KIND == kPrefix) return begin_prefix(block);
        const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
        const int group = g.group;
        bool behind = false;                                       // whether the rows go on from where their prefix ended
        if constexpr (KIND == kBehind) behind = first_tile == 0 && prefix_length(g, prefix_of(g, b)) > 0;
        // ancestors of node `lane`: in each round twice as many steps up
        unsigned long long mask = 1ull << lane;
        int up = -1;
        if (lane < t.nodes) {
            up = g.b.tree_parent ? g.b.tree_parent[static_cast<int64_t>(b) * g.a.N + lane] : g.parent[lane];
            if (up >= lane) up = -1;
        }
        for (int round = 0; round < 6 && __ballot(up >= 0); ++round) {
            const unsigned long long theirs = shfl64(mask, max(up, 0));
            const int further = __shfl(up, max(up, 0));
            if (up >= 0) { mask |= theirs; up = further; }
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = block * kRows + (wave * QT + q) * 16 + l16;
            const int node = g.by_group.of(row);
            const bool real = node < t.nodes;
            line[q] = shfl64(mask, real ? node : 0);
            low[q] = 0;
            if (g.a.window > 0) {
                const int depth = __popcll(line[q]) - 1, first = depth + 1 - g.a.window;
                low[q] = t.context + first;
                // ancestors before the window that are no sinks are not seen: those from the `sinks - context`-th to the `first`-th
                if (first > 0) {
                    unsigned long long rest = line[q];
                    for (int d = 0; d < first; ++d) {
                        if (t.context + d >= sinks()) line[q] &= ~(rest & -rest);
                        rest &= rest - 1;
                    }
                }
            }
            const char* from = static_cast<const char*>(g.b.q) +
                ((static_cast<int64_t>(b) * g.a.N + node) * g.a.q_stride + static_cast<int64_t>(kv * group + row - node * group) * g.a.head_dim) * E::kBytes;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int chunk = s * 4 + quad;
                u32x4 v = {0u, 0u, 0u, 0u};
                if (real && chunk * 16 < g.a.head_dim * E::kBytes && g.sign != 0) v = *reinterpret_cast<const u32x4*>(from + chunk * 16);
                if (g.sign < 0) v ^= k16 ? 0x80008000u : 0x80000000u;
                query[q][s] = v;
            }
            top[q] = -INFINITY;
            base[q] = 0.0f;
            weight[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kColumns; ++c) out[q][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (KIND != kTree && k16) exact[q] = 0.0f;
            if constexpr (KIND == kBehind)
                if (behind && real) {
                    const int64_t state = (static_cast<int64_t>(b) * g.a.N + node) * g.a.heads + kv * group + row - node * group;
                    const float2 stats = g.state_stats[state];
                    top[q] = stats.x;
                    base[q] = stats.x == -INFINITY ? 0.0f : E::kBias - stats.x;
                    if constexpr (k16) {
                        weight[q] = f32x4{stats.y, stats.y, stats.y, stats.y};
                        if (quad == 0) exact[q] = g.state_exact[state];
                    } else if (quad == 0) {
                        weight[q][0] = stats.y;
                    }
#pragma unroll
                    for (int c = 0; c < kColumns; ++c) out[q][c] = *reinterpret_cast<const f32x4*>(g.state + state * DP + c * 16 + quad * 4);
                }
        }
    }

    // ---- a tile in LDS: products, weights, and their sum over the values.
    // Operands of the products are read kAhead instructions before their use, which the order of the source alone does not bring about.
    static constexpr int kAhead = 4;
    struct First { u32x4 keys[kAhead]; unsigned long long special; };
    // (Rows begin at multiples of their length, so exchanged chunks are reached by exclusive or of a place in the first one of them.)
    template <class V> static __device__ __forceinline__ V lds(uint32_t at) {
        return *reinterpret_cast<const __attribute__((address_space(3))) V*>(lds_place(at));
    }
    __device__ __forceinline__ uint32_t keys_at(int stage) const {
        return shared_at + stage * kTileBytes + (l16 * kChunks + (quad ^ swizzle(l16))) * 16;
    }
    static __device__ __forceinline__ u32x4 read_key(uint32_t keys, int n) {
        const int k = n / kSteps, d = n % kSteps;
        return lds<u32x4>((keys ^ (d * 64)) + k * 16 * kChunks * 16);
    }
    __device__ __forceinline__ First read_first(int half, int sub, int stage) const {
        constexpr unsigned long long kBytesOfWaves = WAVES == 8 ? ~0ull : (1ull << (8 * (WAVES % 8))) - 1;
        First f;
#pragma unroll
        for (int n = 0; n < kAhead; ++n) f.keys[n] = read_key(keys_at(stage), n);
        f.special = *reinterpret_cast<const unsigned long long*>(sh.special[half][sub]) & kBytesOfWaves;
        return f;
    }
    __device__ __forceinline__ void work(int index, int half, int sub, int stage, const First& f, bool careful) {
        const uint32_t keys = keys_at(stage);
        char* values = sh.values[stage];
        f32x4 s[QT][kGroups];
        constexpr int kFirst = kGroups * kSteps;
        u32x4 a[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) a[n] = f.keys[n];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int n = 0; n < kFirst; ++n) {
            const int k = n / kSteps, d = n % kSteps;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                if (d == 0) s[q][k] = f32x4{0.f, 0.f, 0.f, 0.f};
                if constexpr (k16) {
                    s[q][k] = E::mfma(a[n % kAhead], query[q][d], s[q][k]);
                } else {
                    const f32x4 fa = __builtin_bit_cast(f32x4, a[n % kAhead]), fq = __builtin_bit_cast(f32x4, query[q][d]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[q][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[i], fq[i], s[q][k], 0, 0, 0);
                }
            }
            if (n + kAhead < kFirst) a[n % kAhead] = read_key(keys, n + kAhead);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        // ---- what is not seen
        if (uniform64(f.special) != 0) {
            const Tile x = tile_at(index);
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                const int quad = fresh(lane) >> 4;
                uint32_t bits = 0;                                 // of this lane's keys, those that its query sees
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    const int key = k * 16 + quad * 4;
                    uint32_t there = *reinterpret_cast<const uint32_t*>(&sh.seen[half][sub][key]);      // a byte each, 0 or 1
                    there = (there | there >> 7 | there >> 14 | there >> 21) & 15u;
                    bits |= (there & sees4(x, key, q)) << (k * 4);
                }
#pragma unroll
                for (int k = 0; k < kGroups; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t keep = spread(bits, k * 4 + i);
                        s[q][k][i] = __uint_as_float((__float_as_uint(s[q][k][i]) & keep) | (0xff800000u & ~keep));
                    }
            }
            // a value that is no number must not reach the nodes that do not see it
            if (careful && differs(x) && !all_numbers(values)) only_numbers(values);
        }
        // ---- references
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            float most = -INFINITY;
#pragma unroll
            for (int k = 0; k < kGroups; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s[q][k][i]);
            most *= g.factor;
            if (__ballot(most > top[q] + kSlack)) {
                const int other = fresh(lane);
                most = fmaxf(most, __shfl(most, other ^ 16));
                most = fmaxf(most, __shfl(most, other ^ 32));
                const float now = fmaxf(top[q], most);
                const float fade = now == -INFINITY ? 1.0f : exp2_of(top[q] - now);
                top[q] = now;
                base[q] = now == -INFINITY ? 0.0f : E::kBias - now;
                weight[q] *= fade;
                if constexpr (KIND != kTree && k16) exact[q] *= fade;
#pragma unroll
                for (int c = 0; c < kColumns; ++c) out[q][c] *= fade;
            }
        }
        // ---- weights
        u32x4 w16[QT][k16 ? kGroups / 2 : 1];
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            float sum = 0.0f;                                      // (float32: a tile's own sum first, over long contexts it matters)
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[q][k][i] = exp2_of(fmaf(s[q][k][i], g.factor, base[q]));
                    if constexpr (!k16) sum += s[q][k][i];
                }
                if constexpr (k16) {
                    typedef __attribute__((ext_vector_type(4))) typename E::T x4;
                    x4 r;
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] = static_cast<typename E::T>(s[q][k][i]);
                    const uint2 p = __builtin_bit_cast(uint2, r);
                    w16[q][k / 2][(k & 1) * 2] = p.x;
                    w16[q][k / 2][(k & 1) * 2 + 1] = p.y;
                }
            }
            if constexpr (!k16) weight[q][0] += sum;
            // (the rounded weights' errors, 2^-9 of the largest and more of few keys, are too much for the logarithm of their sum)
            if constexpr (KIND != kTree && k16)
                if (g.lse) {
#pragma unroll
                    for (int k = 0; k < kGroups; ++k) sum += (s[q][k][0] + s[q][k][1]) + (s[q][k][2] + s[q][k][3]);
                    exact[q] += sum;
                }
            // (a product with ones adds up the rounded weights, those that meet the values)
            if constexpr (k16)
#pragma unroll
                for (int k = 0; k < kGroups / 2; ++k) weight[q] = E::mfma(u32x4{E::kOnes, E::kOnes, E::kOnes, E::kOnes}, w16[q][k], weight[q]);
        }
        // ---- their sum over the values
        __builtin_amdgcn_s_setprio(1);
        if constexpr (k16) {
            constexpr int kSecond = kColumns * (kGroups / 2);
            const uint32_t columns = values_at(stage);
#pragma unroll
            for (int n = 0; n < kAhead; ++n) a[n] = column16(columns, n % (kGroups / 2), n / (kGroups / 2));
#pragma unroll
            for (int n = 0; n < kSecond; ++n) {
                const int k = n % (kGroups / 2), c = n / (kGroups / 2);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < QT; ++q) out[q][c] = E::mfma(a[n % kAhead], w16[q][k], out[q][c]);
                if (n + kAhead < kSecond) a[n % kAhead] = column16(columns, (n + kAhead) % (kGroups / 2), (n + kAhead) / (kGroups / 2));
            }
            __builtin_amdgcn_sched_barrier(0);
        } else {
            constexpr int kSecond = kColumns * kGroups * 4, kAhead32 = 8;
            float v[kAhead32];
            // (the places of a lane's values differ in every column and row: they are worked out again for every tile, beside the products)
            const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
            auto read_value = [&](int n) {
                const int i = n % 4, k = n / 4 % kGroups, c = n / (4 * kGroups), row = k * 16 + quad * 4 + i;
                return *reinterpret_cast<const float*>(values + (row * kChunks + ((c * 4 + (l16 >> 2)) ^ swizzle(row))) * 16 + (l16 & 3) * 4);
            };
#pragma unroll
            for (int n = 0; n < kAhead32; ++n) v[n] = read_value(n);
#pragma unroll
            for (int n = 0; n < kSecond; ++n) {
                const int i = n % 4, k = n / 4 % kGroups, c = n / (4 * kGroups);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < QT; ++q) out[q][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[n % kAhead32], s[q][k][i], out[q][c], 0, 0, 0);
                if (n + kAhead32 < kSecond) v[n % kAhead32] = read_value(n + kAhead32);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    }

    // Keys 32 k + 4 quad .. + 3 and 32 k + 16 + 4 quad .. + 3 of column 16 c + l16.
    __device__ __forceinline__ uint32_t values_at(int stage) const {
        const int row = quad * 4 + (l16 >> 2);
        return shared_at + (STAGES + stage) * kTileBytes + row * kChunks * 16 + (((l16 & 3) >> 1) ^ swizzle(row)) * 16 + (l16 & 1) * 8;
    }
    static __device__ __forceinline__ u32x4 column16(uint32_t values, int k, int c) {
        u32x4 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            typedef __attribute__((address_space(3))) i16x4 lds_x4;
            const uint32_t from = (values ^ (c * 32)) + (k * 32 + h * 16) * kChunks * 16;
            const uint2 r = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_x4*)lds_place(from)));
            v[2 * h] = r.x;
            v[2 * h + 1] = r.y;
        }
        return v;
    }
    __device__ __forceinline__ bool all_numbers(const char* values) const {
        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
        bool fine = true;
        if constexpr (k16) {
            u16x2 most = {0, 0};
#pragma unroll 4
            for (int i = fresh(lane); i < TILE * kChunks; i += 64) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(values + i * 16) & 0x7fff7fffu;
#pragma unroll
                for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, static_cast<uint32_t>(v[j])));
            }
            fine = most[0] < E::kInf && most[1] < E::kInf;
        } else {
            uint32_t most = 0;
#pragma unroll 4
            for (int i = fresh(lane); i < TILE * kChunks; i += 64) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(values + i * 16) & 0x7fffffffu;
#pragma unroll
                for (int j = 0; j < 4; ++j) most = max(most, static_cast<uint32_t>(v[j]));
            }
            fine = most < 0x7f800000u;
        }
        return __ballot(!fine) == 0;
    }

    // Values of a tile that are no numbers become 0.  (Waves that share the keys may do so at once, each for itself.)
    __device__ __forceinline__ void only_numbers(char* values) {
        for (int i = fresh(lane); i < TILE * kChunks; i += 64) {
            u32x4 v = *reinterpret_cast<u32x4*>(values + i * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (k16) {
                    uint32_t x = v[j];
                    if ((x & E::kInf) == E::kInf) x &= 0xffff0000u;
                    if ((x >> 16 & E::kInf) == E::kInf) x &= 0xffffu;
                    v[j] = x;
                } else {
                    if ((v[j] & 0x7f800000u) == 0x7f800000u) v[j] = 0;
                }
            }
            *reinterpret_cast<u32x4*>(values + i * 16) = v;
        }
    }

    __device__ __forceinline__ float value_at(const char* values, int row, int column) const {
        const int chunk = (column * E::kBytes / 16) ^ swizzle(row), in_chunk = column * E::kBytes % 16;
        return static_cast<float>(*reinterpret_cast<const typename E::T*>(values + (row * kChunks + chunk) * 16 + in_chunk));
    }

    // Tiles in which the nodes of a tree see different keys: the tree's own, and those between the first positions of the root
    // and of the deepest node.
    __device__ __forceinline__ bool differs(const Tile& x) const {
        if constexpr (KIND == kPrefix)
            return g.a.window > 0 && x.base < static_cast<int64_t>(t.context) + t.latest + g.a.N - g.a.window && x.base + TILE > g.a.sinks;
        else
            return t.nodes > 1 && (x.tree || (g.a.window > 0 && x.base < t.context + t.nodes - g.a.window && x.base + TILE > sinks()));
    }
    // Which of the four keys from `key` on the lane's query q sees, as far as tree, window and sinks say.
    __device__ __forceinline__ uint32_t sees4(const Tile& x, int key, int q) const {
        const int at = x.base + key;
        if (x.tree) return static_cast<uint32_t>(line[q] >> (at & 63)) & 15u;
        const int before = min(max(low[q] - at, 0), 4), first = min(max(sinks() - at, 0), 4);
        return (15u << before & 15u) | ((1u << first) - 1);
    }

    // Where the nodes of a tree see different keys, values that are no numbers were left out of the sums: the rows that see them get
    // them now.  The tiles in question are brought in again.
    __device__ __forceinline__ void spoil(int first, int last) {
        const int quad = fresh(lane) >> 4;
        for (int i = first; i < last; ++i) {
            const Tile x = tile_at(i);
            if (!differs(x)) continue;
            __syncthreads();
            ask_pages(i, i + 1);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            look_up(i, i + 1, 0);
            ask(places(0, 0), 0);
            arrive(false);
            const char* values = sh.values[0];
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                uint32_t up[4] = {}, down[4] = {};                 // by column group: an infinity of either sign is seen (NaN: both)
                for (int key = 0; key < TILE; ++key) {
                    if (!sh.seen[0][0][key] || !(sees4(x, key, q) & 1)) continue;
                    for (int c = 0; c < kColumns; ++c)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float v = value_at(values, key, c * 16 + quad * 4 + j);
                            up[j] |= static_cast<uint32_t>(!(v < INFINITY)) << c;
                            down[j] |= static_cast<uint32_t>(!(v > -INFINITY)) << c;
                        }
                }
#pragma unroll
                for (int c = 0; c < kColumns; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        out[q][c][j] += __uint_as_float(spread(up[j], c) & 0x7f800000u);
                        out[q][c][j] += __uint_as_float(spread(down[j], c) & 0xff800000u);
                    }
            }
        }
    }

    // The unit's part [first, last) of its tiles.  A value that is no number spoils the sums of all nodes, those that do not see it
    // too (their weights of it are 0).  Nobody looks for one; but if a sum is no number in the end, all is done again, with care.
    __device__ __forceinline__ void run(int block, int first, int last) {
        const int count = last - first;
        bool careful = false;
        for (;; careful = true) {
            if (threadIdx.x == 0) sh.spoiled = 0;                  // (read by all before the last barrier)
            ask_pages(first, last);
            begin(block, first);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            // turn n asks for tile first + n and works on the tile kAheadTiles before it
#pragma unroll 1
            for (int n = 0; n < count + kAheadTiles; ++n) {
                const int mine = n - kAheadTiles;
                if (mine >= 0) arrive(n <= count);
                if (n < count) {
                    const int sub = n % kBatch, half = n / kBatch & 1;
                    if (sub == 0) {
                        look_up(first + n, last, half);
                        if (n + kBatch < count) ask_pages(first + n + kBatch, last);
                    }
                }
                // (what is read of LDS first is asked for at once, needed or not)
                const unsigned past = static_cast<unsigned>(mine + 2 * kBatch * STAGES);
                const Places p = places(n / kBatch & 1, n % kBatch);
                const First f = read_first(past / kBatch & 1, past % kBatch, past % STAGES);
                if (n < count) ask(p, n % STAGES);
                if (mine >= 0) work(first + mine, past / kBatch & 1, past % kBatch, past % STAGES, f, careful);
            }
            if (careful || (KIND == kPrefix ? g.a.window <= 0 : t.nodes == 1)) break;
            // a spoiled column is spoiled in every row, so one group of rows will do
            float zero = 0.0f;
#pragma unroll
            for (int c = 0; c < kColumns; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) zero = fmaf(out[0][c][i], 0.0f, zero);
            if (__ballot(zero != 0.0f) && lane == 0) sh.spoiled = 1;
            __syncthreads();
            const bool again = __builtin_amdgcn_readfirstlane(sh.spoiled) != 0;
            __syncthreads();
            if (!again) break;
        }
        __syncthreads();
        if (careful) {
            spoil(first, last);
            __syncthreads();
        }
        // ---- the lanes that share rows put their sums together
        if constexpr (!k16)
#pragma unroll
            for (int q = 0; q < QT; ++q) {
                weight[q][0] += __shfl_xor(weight[q][0], 16);
                weight[q][0] += __shfl_xor(weight[q][0], 32);
            }
        else if constexpr (KIND != kTree)
            if (g.lse)
#pragma unroll
                for (int q = 0; q < QT; ++q) {
                    exact[q] += __shfl_xor(exact[q], 16);
                    exact[q] += __shfl_xor(exact[q], 32);
                }
    }
    __device__ __forceinline__ float exact_of(int q) const {
        if constexpr (k16) return exact[KIND == kTree ? 0 : q];
        else return weight[q][0];
    }

    // Rows of the output, 16 at a time: through the part of LDS that only this wave's loads fill (whole rows of its keys and values in
    // each stage), from where a row leaves in one piece.  (Written from the registers, 8 bytes a lane, it took 6 us a unit.)
    __device__ __forceinline__ char* own_row(int row) const {
        const int piece = row / kMyRows;
        static_assert(16 / kMyRows <= 2 * STAGES, "room for 16 rows");
        char* at = piece < STAGES ? sh.keys[piece] : sh.values[piece - STAGES];
        return at + (wave * kMyRows + row % kMyRows) * kChunks * 16;
    }
    __device__ __forceinline__ void finish(int block) {
        const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
        const int group = g.group;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            if constexpr (KIND != kTree)
                if (g.lse && quad == 0) {
                    const int row = block * kRows + (wave * QT + q) * 16 + l16, node = g.by_group.of(row);
                    if (node < t.nodes)
                        g.lse[(static_cast<int64_t>(b) * g.a.N + node) * g.a.heads + kv * group + row - node * group] = lse_of(top[q], exact_of(q), E::kBias);
                }
            const float whole = 1.0f / weight[q][0];
            char* mine = own_row(l16);
#pragma unroll
            for (int c = 0; c < kColumns; ++c) {
                const int byte = (c * 16 + quad * 4) * E::kBytes;
                E::put4(mine + ((byte / 16) ^ swizzle(l16)) * 16 + byte % 16, out[q][c] * whole);
            }
            wave_order();
#pragma unroll
            for (int j = 0; j < 16 / kRowsPerLoad; ++j) {
                const int local = j * kRowsPerLoad + lane / kChunks, chunk = lane % kChunks;
                const u32x4 v = *reinterpret_cast<const u32x4*>(own_row(local) + (chunk ^ swizzle(local)) * 16);
                const int row = block * kRows + (wave * QT + q) * 16 + local;
                const int node = g.by_group.of(row);
                char* to = static_cast<char*>(g.b.out) +
                    ((static_cast<int64_t>(b) * g.a.N + node) * g.a.out_stride + static_cast<int64_t>(kv * group + row - node * group) * g.a.head_dim) * E::kBytes;
                if (node < t.nodes && chunk * 16 < g.a.head_dim * E::kBytes) *reinterpret_cast<u32x4*>(to + chunk * 16) = v;
            }
            wave_order();
        }
    }

    // A prefix's unit that is this team's alone: the rows' states.
    __device__ __forceinline__ void settle(int block) {
        const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
        const int group = g.group, upto = trees_upto();
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = block * kRows + (wave * QT + q) * 16 + l16, rank = g.by_group.of(row);
            const Place p = place_of(min(rank, t.nodes - 1), upto);
            if (rank >= t.nodes) continue;
            const int64_t state = (static_cast<int64_t>(p.tree) * g.a.N + p.node) * g.a.heads + kv * group + row - rank * group;
            if (quad == 0) {
                g.state_stats[state] = make_float2(top[q], weight[q][0]);
                if (k16 && g.lse) g.state_exact[state] = exact_of(q);
            }
#pragma unroll
            for (int c = 0; c < kColumns; ++c) *reinterpret_cast<f32x4*>(g.state + state * DP + c * 16 + quad * 4) = out[q][c];
        }
    }

    __device__ __forceinline__ void keep(int block, int slot) {
        const int lane = fresh(this->lane), l16 = lane & 15, quad = lane >> 4;
        const int rows = t.nodes * g.group - block * kRows;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            if ((wave * QT + q) * 16 + l16 >= rows) continue;
            const int64_t row = static_cast<int64_t>(slot) * kRows + (wave * QT + q) * 16 + l16;
            if (quad == 0) g.partial_stats[row] = make_float2(top[q], weight[q][0]);
            if constexpr (KIND != kTree)
                if (g.lse && quad == 0) g.partial_exact[row] = exact_of(q);
#pragma unroll
            for (int c = 0; c < kColumns; ++c) *reinterpret_cast<f32x4*>(g.partial + row * DP + c * 16 + quad * 4) = out[q][c];
        }
    }

    // Inclusive sum over the wave.
    __device__ __forceinline__ int64_t wave_scan(int64_t v) const {
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t o = static_cast<int64_t>(shfl64(static_cast<unsigned long long>(v), max(lane - d, 0)));
            if (lane >= d) v += o;
        }
        return v;
    }

    // A tree's tiles and units.
    struct Count { int64_t tiles; int units; };
    __device__ __forceinline__ Count count_of(int tree) const {
        if constexpr (KIND == kPrefix) {                           // (all lanes call it, each with a tree of its own, the first one a multiple of 64)
            const TreeWork w = prefix_work<TILE, kRows>(g, tree - lane);
            if (w.nodes == 0) return {0, 0};
            const int units = w.supers * g.a.kv_heads;
            return {static_cast<int64_t>(w.tiles) * units, units};
        } else {
            if (tree >= g.a.B) return {0, 0};
            const TreeWork w = tree_work<KIND, TILE, kRows>(g, tree);
            if (w.nodes == 0) return {0, 0};
            return {static_cast<int64_t>(w.tiles) * g.a.kv_heads, g.a.kv_heads};
        }
    }
    // What tree `b` has of the list (kPrefix: as the first of those that share a prefix).
    __device__ __forceinline__ void load_unit() {
        if constexpr (KIND == kPrefix) {
            const TreeWork w = prefix_work<TILE, kRows>(g, b & ~63);
            auto mine = [&](int v) { return __builtin_amdgcn_readfirstlane(__shfl(v, b & 63)); };
            t.which = mine(w.which);
            t.context = mine(w.context);
            t.nodes = mine(w.nodes);
            t.first = mine(w.first);
            t.end = mine(w.end);
            t.low = mine(w.low);
            t.sink_tiles = mine(w.sink_tiles);
            t.context_tiles = mine(w.context_tiles);
            t.tiles = mine(w.tiles);
            t.latest = mine(w.latest);
            t.supers = mine(w.supers);
            t.sinks = w.sinks;
            t.blocks = w.blocks;
        } else {
            t = tree_work<KIND, TILE, kRows>(g, b);
        }
    }

    __device__ __forceinline__ void all() {
        // teams of one chiplet (blockIdx % 8) take neighbouring parts of the list
        const int most = g.teams, place = most % 8 == 0 ? blockIdx.x / 8 : blockIdx.x;
        const int member = place % g.blocks, team = most % 8 == 0 ? (blockIdx.x % 8) * (most / 8) + place / g.blocks : place / g.blocks;
        // every wave adds the trees' tiles up for itself, 64 trees at a time
        const int trees = g.a.B;
        Count mine = count_of(lane);
        int64_t tiles = mine.tiles, units = mine.units;
        for (int base = 64; base < trees; base += 64) {
            const Count c = count_of(base + lane);
            tiles += c.tiles;
            units += c.units;
        }
        for (int d = 32; d; d >>= 1) {
            tiles += static_cast<int64_t>(shfl64(static_cast<unsigned long long>(tiles), lane ^ d));
            units += static_cast<int64_t>(shfl64(static_cast<unsigned long long>(units), lane ^ d));
        }
        // a unit counts as `extra` tiles more than it has, all of them before its first
        const int extra = static_cast<int>(min(static_cast<int64_t>(kUnitCost), uniform64(tiles) / (2 * most)));
        const int64_t total = uniform64(tiles) + extra * uniform64(units);
        const int T = static_cast<int>(min(static_cast<int64_t>(most), total));
        if (KIND != kPrefix && member == 0 && threadIdx.x == 0 && !g.by_unit) g.split[team] = make_int4(-1, 0, 0, 0);
        if (team >= T) return;
        // the first `longer` teams have one tile more than the others
        const int64_t share = total <= UINT32_MAX ? static_cast<int64_t>(static_cast<uint32_t>(total) / static_cast<uint32_t>(T)) : total / T;
        const int64_t longer = total - share * T;
        const int64_t begin_at = share * team + min(static_cast<int64_t>(team), longer), end_at = begin_at + share + (team < longer);
        // the tree of the first tile
        int64_t start = 0;
        b = 0;
        for (int base = 0;;) {
            const int64_t weight = mine.tiles + extra * mine.units, upto = wave_scan(weight), chunk = uniform64(shfl64(upto, 63));
            if (begin_at < start + chunk) {
                const int l = __ffsll(static_cast<unsigned long long>(__ballot(begin_at < start + upto))) - 1;
                start += uniform64(shfl64(upto - weight, l));
                b = __builtin_amdgcn_readfirstlane(base + l);
                break;
            }
            start += chunk;
            base += 64;
            mine = count_of(base + lane);
        }
        int64_t at = begin_at;
        for (; at < end_at; b = KIND == kPrefix ? t.end : b + 1) {
            load_unit();
            if (t.nodes == 0) continue;
            const int length = t.tiles + extra;
            const int units = KIND == kPrefix ? t.supers * g.a.kv_heads : g.a.kv_heads;
            const int64_t tree_end = start + static_cast<int64_t>(length) * units;
            while (at < min(end_at, tree_end)) {
                // (the tiles of a tree's heads may be more than 32 bits hold, but hardly ever are)
                const int64_t into = at - start;
                kv = static_cast<int>(into <= UINT32_MAX ? static_cast<uint32_t>(into) / static_cast<uint32_t>(length) : into / length);
                const int64_t unit = start + static_cast<int64_t>(kv) * length;
                int super = 0;                                     // (the units of a cache head follow each other: they read the same tiles)
                if constexpr (KIND == kPrefix) {
                    const int number = kv;
                    kv = number / t.supers;
                    super = number - kv * t.supers;
                }
                const int first = max(static_cast<int>(at - unit) - extra, 0);
                const int last = static_cast<int>(min(static_cast<int64_t>(length), end_at - unit)) - extra;
                at = min(unit + length, end_at);
                const bool shared = first > 0 || last < t.tiles;
                if (last <= first) continue;
                if (member == 0 && first == 0 && threadIdx.x == 0 && (shared || KIND == kPrefix || g.by_unit)) {
                    const int64_t x = unit + length - 1, ahead = longer * (share + 1);       // the unit's last tile, and whose it is
                    const int64_t whose = x < ahead ? x / (share + 1) : longer + (x - ahead) / share;
                    if constexpr (KIND == kPrefix)
                        g.units[(static_cast<int64_t>(b) * g.a.kv_heads + kv) * g.supers + super] = make_int2(team, shared ? static_cast<int>(whose) : -1);
                    else g.split[g.by_unit ? b * g.a.kv_heads + kv : team] = make_int4(shared ? b : -1, kv, team, static_cast<int>(whose));
                }
                if constexpr (KIND == kPrefix) {
                    const int block = super * g.blocks + member;
                    if (static_cast<int64_t>(block) * kRows >= static_cast<int64_t>(t.nodes) * g.group) continue;
                    run(block, first, last);
                    if (shared) keep(block, (team * g.blocks + member) * 2 + (first > 0 ? 0 : 1));
                    else settle(block);
                    continue;
                }
                if (member >= t.blocks) continue;
                run(member, first, last);
                if (shared) keep(member, (team * g.blocks + member) * 2 + (first > 0 ? 0 : 1));
                else finish(member);
            }
            start = tree_end;
        }
    }
};

// Puts the shared units together.  kLanes lanes have a row (4 columns each).  Few parts, as in large batches: a wave has as many rows
// as it has such groups of lanes, twice over.  Many: the groups of a workgroup share the parts of one row.
// (Few: a workgroup a row takes 651 us instead of 613 for the benchmark's trees, 56 instead of 52 for 32 trees with a window of 1024.)
constexpr int kFewParts = 8, kFewRows = 2;

template <int KIND, int DTYPE, int DP, int ROWS>
__device__ __forceinline__ void combine(const typename ArgsOf<KIND>::T& g) {
    typedef Elem<DTYPE> E;
    constexpr int kLanes = DP / 4, kGroups = 64 / kLanes;
    const int nodes_of_unit = g.by_unit && g.b.num_nodes ? g.b.num_nodes[blockIdx.x / g.a.kv_heads] : 1;
    if (nodes_of_unit <= 0) return;                                // (nobody wrote its entry)
    const int4 s = g.split[blockIdx.x];
    if (s.x < 0) return;
    const int lane = threadIdx.x & 63, column = lane % kLanes * 4, mine = lane / kLanes;
    const int b = s.x, kv = s.y, first = s.z, last = s.w, group = g.group;
    const int parts = last - first + 1;
    const int nodes = g.b.num_nodes ? min(max(g.b.num_nodes[b], 0), g.a.N) : g.a.N;
    const int rows = nodes * group, wave = blockIdx.y * 4 + (threadIdx.x >> 6);
    // part p of a row: the second slot of team `first`, the first slot of those after it
    auto at = [&](int row, int p) {
        return ((static_cast<int64_t>(first + p) * g.blocks + row / ROWS) * 2 + (p == 0 ? 1 : 0)) * ROWS + row % ROWS;
    };
    auto put = [&](int row, const f32x4& sum, float weight, float top, float exact) {
        const int node = g.by_group.of(row);
        if constexpr (KIND != kTree)
            if (g.lse && row < rows && column == 0)
                g.lse[(static_cast<int64_t>(b) * g.a.N + node) * g.a.heads + kv * group + row - node * group] = lse_of(top, exact, E::kBias);
        char* to = static_cast<char*>(g.b.out) +
            ((static_cast<int64_t>(b) * g.a.N + node) * g.a.out_stride + static_cast<int64_t>(kv * group + row - node * group) * g.a.head_dim + column) * E::kBytes;
        if (row < rows && column < g.a.head_dim) E::put4(to, sum * (1.0f / weight));
    };
    if (parts <= kFewParts) {
        const int row0 = wave * kGroups * kFewRows;
        if (row0 >= rows) return;
        float2 stats[kFewRows][kFewParts];
        float exacts[kFewRows][KIND == kTree ? 1 : kFewParts] = {};
        f32x4 part[kFewRows][kFewParts];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
            const int row = min(row0 + r * kGroups + mine, rows - 1);
#pragma unroll
            for (int p = 0; p < kFewParts; ++p) {
                if (p >= parts) continue;
                stats[r][p] = g.partial_stats[at(row, p)];
                if constexpr (KIND != kTree)
                    if (g.lse) exacts[r][p] = g.partial_exact[at(row, p)];
                part[r][p] = *reinterpret_cast<const f32x4*>(g.partial + at(row, p) * DP + column);
            }
        }
#pragma unroll
        for (int r = 0; r < kFewRows; ++r) {
            float top = stats[r][0].x, weight = 0.0f;
#pragma unroll
            for (int p = 1; p < kFewParts; ++p) if (p < parts) top = fmaxf(top, stats[r][p].x);
            const float base = top == -INFINITY ? 0.0f : top;
            float exact = 0.0f;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < kFewParts; ++p)
                if (p < parts) {
                    const float f = exp2_of(stats[r][p].x - base);
                    weight += f * stats[r][p].y;
                    if constexpr (KIND != kTree) exact += f * exacts[r][p];
                    sum += part[r][p] * f;
                }
            put(row0 + r * kGroups + mine, sum, weight, top, exact);
        }
        return;
    }
    __shared__ float tops[4], weights[4];
    __shared__ float exact_sums[KIND == kTree ? 1 : 4];
    __shared__ f32x4 sums[4][kLanes];
    const int own = threadIdx.x >> 6;
    for (int row = blockIdx.y; row < rows; row += gridDim.y) {
        // (statistics and sums are asked for together, four parts a group at a time)
        float top = -INFINITY, weight = 0.0f, exact = 0.0f;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int p = own * kGroups + mine; p < parts; p += 16 * kGroups) {
            float2 stats[4];
            float exacts[4] = {};
            f32x4 part[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t from = at(row, min(p + j * 4 * kGroups, parts - 1));
                stats[j] = g.partial_stats[from];
                if constexpr (KIND != kTree)
                    if (g.lse) exacts[j] = g.partial_exact[from];
                part[j] = *reinterpret_cast<const f32x4*>(g.partial + from * DP + column);
            }
            float now = top;
#pragma unroll
            for (int j = 0; j < 4; ++j) if (p + j * 4 * kGroups < parts) now = fmaxf(now, stats[j].x);
            const float base = now == -INFINITY ? 0.0f : now, fade = exp2_of(top - base);
            weight *= fade;
            if constexpr (KIND != kTree) exact *= fade;
            sum *= fade;
            top = now;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (p + j * 4 * kGroups < parts) {
                    const float f = exp2_of(stats[j].x - base);
                    weight += f * stats[j].y;
                    if constexpr (KIND != kTree) exact += f * exacts[j];
                    sum += part[j] * f;
                }
        }
        float now = top;
        for (int d = kLanes; d < 64; d <<= 1) now = fmaxf(now, __shfl_xor(now, d));
        const float fade = exp2_of(top - (now == -INFINITY ? 0.0f : now));
        weight *= fade;
        if constexpr (KIND != kTree) exact *= fade;
        sum *= fade;
        for (int d = kLanes; d < 64; d <<= 1) {
            weight += __shfl_xor(weight, d);
            if constexpr (KIND != kTree) exact += __shfl_xor(exact, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], d);
        }
        __syncthreads();
        if (lane == 0) { tops[own] = now; weights[own] = weight; }
        if constexpr (KIND != kTree)
            if (lane == 0) exact_sums[own] = exact;
        if (mine == 0) sums[own][lane] = sum;
        __syncthreads();
        if (own == 0 && mine == 0) {
            float most = tops[0];
#pragma unroll
            for (int w = 1; w < 4; ++w) most = fmaxf(most, tops[w]);
            const float base = most == -INFINITY ? 0.0f : most;
            weight = exact = 0.0f;
            sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2_of(tops[w] - base);
                weight += weights[w] * f;
                if constexpr (KIND != kTree) exact += exact_sums[w] * f;
                sum += sums[w][lane] * f;
            }
            put(row, sum, weight, most, exact);
        }
    }
}

// ------------------------------------------------------------------ host side

// Workgroups of a call: as many as 256 compute units hold at a time (more only where a team alone has more).
template <class A>
constexpr int kMaxWorkgroups = 256 * A::kShare;

// The tile for a type and a row length: 8 KB of keys (16 for the longest rows) and as many of values.  Two workgroups share a compute
// unit, with four stages of 16 KB or two of 32 KB each; those of one wave are three (64 single tokens with 4096 keys: 202 us, two: 212; 256
// with 16 to 512 keys: 79 and 90); and one of eight waves has the unit for itself.
template <int DTYPE, int DP, int WAVES>
struct Family {
    static constexpr int kBytes = DP * Elem<DTYPE>::kBytes;
    static constexpr int kLeast = DTYPE == MPV_DTYPE_F32 ? 16 : 32;
    static constexpr int kMost = 8192 / kBytes < 16 * WAVES ? 8192 / kBytes : 16 * WAVES;      // (a lane looks up a row of some tiles ahead)
    static constexpr int kTile = kMost < kLeast ? kLeast : kMost;
    static constexpr int kShare = WAVES == 1 && kTile * kBytes <= 8192 ? 3 : WAVES == 8 ? 1 : 2;
    static constexpr int kStages = kTile * kBytes > 8192 ? (kShare == 1 ? 4 : 2) : WAVES == 1 ? 3 : 4;
};

// What a call needs to know of the kernel that it gets.
struct Choice {
    int rows, columns, tile;
    int64_t tiles;                         // the most that a call can have
    int teams, blocks;
};

template <class A, int DP>
inline Choice choice_of(const mpv_attention* a) {
    Choice c;
    c.rows = A::kRows;
    c.columns = DP;
    c.tile = A::kTile;
    const int64_t rows = static_cast<int64_t>(a->N) * (a->heads / a->kv_heads);
    c.blocks = static_cast<int>((rows + c.rows - 1) / c.rows);
    const int64_t room = static_cast<int64_t>(a->table_width) * a->page_size;
    int64_t seen = (room + c.tile - 1) / c.tile;
    if (a->window > 0) {
        const int64_t near = (static_cast<int64_t>(a->window) + c.tile - 1) / c.tile + 1 + (static_cast<int64_t>(a->sinks > 0 ? a->sinks : 0) + c.tile - 1) / c.tile;
        if (near < seen) seen = near;
    }
    const int64_t unit = seen + (a->N + c.tile - 1) / c.tile;
    c.tiles = unit * a->B * a->kv_heads;
    c.teams = kMaxWorkgroups<A> / c.blocks;
    if (c.teams >= 8) c.teams = c.teams / 8 * 8;
    if (c.tiles < c.teams) c.teams = static_cast<int>(c.tiles);
    if (c.teams < 1) c.teams = 1;
    return c;
}

// The launch that puts shared units together: entries, and workgroups for each of them (0: no launch).
struct Second { int64_t entries, workgroups; };
template <int DP>
inline Second second_of(const mpv_attention* a, const Choice& c, bool by_unit) {
    const int64_t rows = static_cast<int64_t>(a->N) * (a->heads / a->kv_heads);
    // A list with one tile a unit shares none.  Few parts a unit: `some` rows a workgroup, and that is all where no unit has more tiles than
    // that.  Many, as a unit can have that is one of few or much longer than the others: a row, up to 4096 workgroups, or 16 384 where units are
    // not fewer than the teams and the block table has room for long ones (300 trees of 41 nodes on 2 heads, one context of 131 072 and 299 of
    // 100: 106 us, 118 with 8192, 135 with 4096; 100 trees of 7 nodes on 8 heads with one such: 142, 141, 143; the benchmark's trees, which need none
    // of them: 616 with each, 2 % more with 65 536; 256 trees of 8 nodes, contexts of 16 to 256 in a table with room for 320: 65.7, 63.5, 62.2).
    constexpr int kLongTiles = 64;
    constexpr int kSome = kFewRows * 4 * (64 / (DP / 4));
    const int64_t units = static_cast<int64_t>(a->B) * a->kv_heads, few = (rows + kSome - 1) / kSome;
    const int64_t entries = by_unit ? units : c.teams;
    const int64_t workgroups = by_unit || c.tiles <= units * kLongTiles ? 4096 : 16384;
    const int64_t most = c.tiles > units * kFewParts ? std::min(rows, workgroups / entries) : 0;
    return {entries, c.tiles > units ? std::max(few, most) : 0};
}

inline size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Behind prefixes, 17 to 64 rows: as many workgroups a compute unit as its LDS holds with two stages each, instead of two with four.  64 rows
// (four waves, three workgroups): 48 trees with a window of 2000 35.4 us, 38.0; 64 trees of 15 nodes behind prefixes of 256 to 4096 positions
// 148, 153, and 149 with two of three stages; 256 trees of 8 nodes behind 256 to 1024 117, 130; float32, 64 trees behind 4096 414, 446.
// 32 rows (two waves, four workgroups): 200 trees of 5 nodes 123.7, 129.1, and 125.2 with three; 256 trees of 8 nodes 148, 155; float32, 64
// trees behind 256 to 4096 214, 239; at worst 2 % more (16 trees of 5 nodes, 47.0, 46.2).
template <int KIND, int DTYPE, int DP, int QT, int WAVES>
struct Shape {
    typedef Family<DTYPE, DP, WAVES> F;
    static constexpr bool kTwoStages = KIND != kTree && QT == 1 && (WAVES == 2 || WAVES == 4) && F::kTile * F::kBytes <= 8192;
    typedef Attention<DTYPE, DP, QT, WAVES, F::kTile, kTwoStages ? 2 : F::kStages, kTwoStages ? (WAVES == 2 ? 4 : 3) : F::kShare, KIND> T;
};
template <int KIND, int DTYPE, int DP, int QT, int WAVES>
using Kernel = typename Shape<KIND, DTYPE, DP, QT, WAVES>::T;

template <class K> struct Chosen { typedef K T; };

// f(Chosen<kernel>) with the kernel for units of so many rows.
template <int KIND, int DTYPE, int DP, class F>
int by_rows(int64_t rows, const F& f) {
    // as few waves as hold the rows: a wave reads all of a tile from LDS, whatever it has to do with it.  (16 rows and less on two waves:
    // 538 us instead of 505 for 8 long contexts, 44 instead of 30 in float32; 32 rows on four: 223 instead of 217 for 64 trees of 8 nodes.)
    if (rows <= 16) return f(Chosen<Kernel<KIND, DTYPE, DP, 1, 1>>());
    if (rows <= 32) return f(Chosen<Kernel<KIND, DTYPE, DP, 1, 2>>());
    if (rows <= 64) return f(Chosen<Kernel<KIND, DTYPE, DP, 1, 4>>());
    if constexpr (DP * Elem<DTYPE>::kBytes > 256) {
        // (two groups a wave of such long rows do not fit its registers)
        // Behind prefixes in float32 products take the time, so what counts is how few rows stay empty and what shares a compute unit: 64 trees
        // of 41 nodes, 164 rows, behind prefixes of 512 to 2048 positions 1099 us, 1664 with 128 rows on eight waves; 128 rows 694, 796; with 256
        // columns 356, 362.  (bfloat16 with 256 columns: 124, 115.)
        if constexpr (KIND != kTree && DTYPE == MPV_DTYPE_F32) return f(Chosen<Kernel<KIND, DTYPE, DP, 1, 4>>());
        else return f(Chosen<Kernel<KIND, DTYPE, DP, 1, 8>>());
    } else {
        // as many groups a wave as divide the rows into even blocks: every block reads the tiles again, from the chiplet's cache.  (Two
        // groups for the benchmark's 164 rows: 870 us instead of 613.)
        const int64_t blocks = (rows + 191) / 192, groups = (rows + 64 * blocks - 1) / (64 * blocks);
        if (groups > 2) return f(Chosen<Kernel<KIND, DTYPE, DP, 3, 4>>());
        return f(Chosen<Kernel<KIND, DTYPE, DP, 2, 4>>());
    }
}

inline int check_attention(const mpv_attention* a) {
    if (!a) return MPV_ERR_NULL;
    if (a->B < 0 || a->N < 1 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads != 0 || a->head_dim < 1 || a->num_pages < 0 ||
        a->page_size < 1 || a->table_width < 0)
        return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(a->dtype)) return MPV_ERR_BAD_DTYPE;
    if (!std::isfinite(a->scale)) return MPV_ERR_BAD_TEMPERATURE;
    if (a->N > MPV_MAX_NODES || a->head_dim > MPV_MAX_HEAD_DIM || a->heads > MPV_MAX_HEADS) return MPV_ERR_UNSUPPORTED;
    const int64_t row = static_cast<int64_t>(a->kv_heads) * a->head_dim, wide = static_cast<int64_t>(a->heads) * a->head_dim;
    // rows of heads that do not reach into each other
    if (a->q_stride < wide || a->out_stride < wide || a->kv_stride < row || a->slot_stride < row || a->page_stride < 0) return MPV_ERR_BAD_SHAPE;
    // positions are counted in 32 bits, addresses in 64
    const int64_t nodes = static_cast<int64_t>(a->B) * a->N;
    if (a->B > (1 << 24) || span(MPV_MAX_NODES, a->table_width, a->page_size) > INT32_MAX || span(0, span(0, nodes, a->q_stride), 4) == INT64_MAX ||
        span(0, span(0, nodes, a->out_stride), 4) == INT64_MAX || span(0, span(0, nodes, a->kv_stride), 4) == INT64_MAX ||
        span(0, span(span(0, a->num_pages, a->page_stride), a->page_size, a->slot_stride), 4) == INT64_MAX)
        return MPV_ERR_UNSUPPORTED;
    const int64_t all = a->head_dim | a->q_stride | a->out_stride | a->kv_stride | a->slot_stride | a->page_stride;
    if ((all * elem_bytes(a->dtype)) % 16 != 0) return MPV_ERR_ALIGNMENT;
    return MPV_OK;
}


// A call's arguments as the kernels take them, its tree checked.
inline int take_arguments(const mpv_attention* a, const mpv_attention_buffers* buf, AttentionArgs* g) {
    g->a = *a; g->b = *buf;
    g->a.sinks = a->sinks > 0 ? a->sinks : 0;
    g->sign = a->scale > 0.0f ? 1 : a->scale < 0.0f ? -1 : 0;
    g->factor = g->sign ? static_cast<float>(std::fabs(static_cast<double>(a->scale)) * 1.4426950408889634) : 1.0f;
    g->group = a->heads / a->kv_heads;
    g->by_group.set(static_cast<uint32_t>(g->group));
    g->by_page.set(static_cast<uint32_t>(a->page_size));
    if (buf->tree_parent) return MPV_OK;
    if (!a->parent) return MPV_ERR_NULL;
    if (a->parent[0] != -1) return MPV_ERR_BAD_TREE;
    g->parent[0] = -1;
    for (int n = 1; n < a->N; ++n) {
        if (a->parent[n] < 0 || a->parent[n] >= n) return MPV_ERR_BAD_TREE;
        g->parent[n] = static_cast<int8_t>(a->parent[n]);
    }
    return MPV_OK;
}

inline int check_buffers(const mpv_attention* a, const mpv_attention_buffers* buf) {
    if (!buf->q || !buf->tree_k || !buf->tree_v || !buf->context_len || !buf->out ||
        (a->table_width > 0 && (!buf->block_table || (a->num_pages > 0 && (!buf->cache_k || !buf->cache_v)))))
        return MPV_ERR_NULL;
    if (!aligned(buf->q, 16) || !aligned(buf->tree_k, 16) || !aligned(buf->tree_v, 16) || !aligned(buf->cache_k, 16) ||
        !aligned(buf->cache_v, 16) || !aligned(buf->out, 16))
        return MPV_ERR_ALIGNMENT;
    return MPV_OK;
}

}  // namespace mpv
