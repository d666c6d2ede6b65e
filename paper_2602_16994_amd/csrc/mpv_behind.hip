// Attention of draft trees behind prefixes that requests share: the trees' own part, and the call.
//
// A softmax over several parts of its keys needs of each part the sum of its values' weights, the sum of the weights, and the reference of both:
//   m = max m_i,  out = sum_i e^(m_i - m) o_i / sum_i e^(m_i - m) w_i,  ln sum_j e^(s_j) = m + ln sum_i e^(m_i - m) w_i.
// So prefix_kernel works out the prefix's part for the nodes of all trees that share it (mpv_prefix.hip), and a row goes on from there
// over its own context and tree as if they were the next tiles (kBehind of mpv_attention.h).  The state between the two is float32.
//
// What bounds the trees' own part, 64 single tokens with contexts of 16 to 1024: 42 us for 136 MB, of which some 12 are what comes before the
// first tile (as in mpv_tree_attention); then memory.

#include "mpv_behind.h"

namespace mpv {

// Whether the prefixes are read for all trees that share them, or by every tree for itself, from the chiplets' caches.  Reading them
// together costs two launches more (about 30 us with the second one's partial sums), the state of every row, written and read, and
// products that no loads hide behind; what it saves is a reading for every tree but one.  In us, with the rates that either reached, for 8 cache
// heads of 128 bfloat16 values (and 4 of float32), prefixes of as many positions as there is room for, contexts of 16 to 300, each for itself and
// together:
//   4 rows a cache head (single tokens):  64 trees, 8192 positions: 254, 60; 16 trees, 16 384: 156, 59; 64 trees, 1024: 50, 48
//   20 rows:   200 trees, 4096: 380, 174; 64 trees, 4096: 141, 86; 64 trees, 1024: 44, 64; 16 trees, 4096: 52, 58
//   64 rows:   64 trees, 8192: 249, 225; 64 trees, 4096: 140, 158; 200 trees, 1024: 134, 214
//   164 rows:  the benchmark's trees behind four prefixes of 512 to 2048: 529, 699
//   float32, 2 rows:  64 trees, 8192: 395, 80; 16 trees, 4096: 66, 57;   10 rows:  64 trees, 1024: 91, 74; 16 trees, 1024: 31, 57
//   float32, 64 rows: 64 trees, 4096: 381, 414;   168 rows: 64 trees, 4096: 1084, 1035 (the one of these that the rule misses, by 5 %)
// All of these (but the benchmark's trees) have one prefix, and the rule counts as if there were one: how many are in use lies on the device.  With
// 4, 16 and 64 prefixes of 8192 positions, drawn at random, 64 single tokens take 256, 80; 276, 133; 312, 274; with 1024 positions 50, 48; 54, 54; 65, 73.  Where every
// tree has a prefix of its own, so that nothing is shared, the rule costs what the second way costs besides: 382, 399; 75, 90; with 20 rows
// 64 trees, 4096: 233, 251; 200 trees, 4096: 641, 773.
static bool together(const mpv_prefixed* p) {
    const mpv_attention& a = p->attention;
    if (a.B < 2 || p->prefixes < 1 || p->prefix_width < 1) return false;
    if (static_cast<int64_t>(a.B) * a.kv_heads >= kMostWorkgroups) return false;          // (the second launch has one for each tree and head)
    const bool wide = a.dtype == MPV_DTYPE_F32;
    double positions = static_cast<double>(p->prefix_width) * a.page_size;
    if (a.window > 0) positions = std::min(positions, static_cast<double>(a.window) + std::max(a.sinks, 0));
    const double bytes = 2.0 * (a.B - 1) * positions * a.kv_heads * a.head_dim * elem_bytes(a.dtype);
    const double rows = static_cast<double>(a.B) * a.N * a.heads;
    const double products = 4.0 * rows * positions * a.head_dim, states = 8.0 * rows * columns_of(&a);
    return bytes / (wide ? 4.2e6 : 7.4e6) > 30.0 + products / (wide ? 110e6 : 600e6) + states / 4e6;
}

// Bytes of a workspace: the state of the rows (none where every tree reads its prefix), and what either half needs while it runs.
struct Room {
    size_t state, stats, exact, parts;
    size_t bytes() const { return state + stats + exact + parts; }
};
static int room_of(const mpv_prefixed* p, Room* r) {
    const mpv_attention* a = &p->attention;
    *r = {0, 0, 0, 0};
    size_t trees, prefix = 0;
    const bool shared = together(p);
    int rc = shared ? attend_trees<kBehind>(p, nullptr, nullptr, &trees, nullptr) : attend_through(p, nullptr, nullptr, &trees, nullptr);
    if (rc != MPV_OK) return rc;
    if (shared) {
        rc = attend_prefixes(a, nullptr, nullptr, &prefix, nullptr);
        if (rc != MPV_OK) return rc;
        const size_t rows = static_cast<size_t>(a->B) * a->N * a->heads;
        r->stats = whole(rows * sizeof(float2));
        r->exact = whole(rows * sizeof(float));
        r->state = whole(rows * columns_of(a) * sizeof(float));
    }
    r->parts = std::max(trees, prefix);
    return MPV_OK;
}

static int check_prefixed(const mpv_prefixed* p) {
    if (!p) return MPV_ERR_NULL;
    const int rc = check_attention(&p->attention);
    if (rc != MPV_OK) return rc;
    if (p->prefixes < 0 || p->prefix_width < 0) return MPV_ERR_BAD_SHAPE;
    const mpv_attention& a = p->attention;
    // positions are counted in 32 bits
    if (span(span(MPV_MAX_NODES, a.table_width, a.page_size), p->prefix_width, a.page_size) > INT32_MAX) return MPV_ERR_UNSUPPORTED;
    return MPV_OK;
}

}  // namespace mpv

extern "C" {

int mpv_prefix_attention_workspace_bytes(const mpv_prefixed* prefixed, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    int rc = mpv::check_prefixed(prefixed);
    if (rc != MPV_OK) return rc;
    mpv::Room room;
    rc = mpv::room_of(prefixed, &room);
    *out = room.bytes();
    return rc;
}

int mpv_prefix_attention(const mpv_prefixed* prefixed, const mpv_prefixed_buffers* buf, void* workspace, size_t workspace_bytes,
                         void* hip_stream) {
    int rc = mpv::check_prefixed(prefixed);
    if (rc != MPV_OK) return rc;
    mpv::Room room;
    rc = mpv::room_of(prefixed, &room);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    const mpv_attention* a = &prefixed->attention;
    mpv::PrefixArgs g;
    rc = mpv::take_arguments(a, &buf->attention, &g);
    if (rc != MPV_OK) return rc;
    if (a->B == 0) return MPV_OK;
    rc = mpv::check_buffers(a, &buf->attention);
    if (rc != MPV_OK) return rc;
    const bool any = prefixed->prefixes > 0 && prefixed->prefix_width > 0 && buf->prefix_of;
    // (a prefix may be all that there is in the cache)
    if (any && (!buf->prefix_table || !buf->prefix_len || (a->num_pages > 0 && (!buf->attention.cache_k || !buf->attention.cache_v)))) return MPV_ERR_NULL;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < room.bytes()) return MPV_ERR_WORKSPACE;
    g.prefix_of = any ? buf->prefix_of : nullptr;
    g.prefix_table = buf->prefix_table;
    g.prefix_len = buf->prefix_len;
    g.prefixes = prefixed->prefixes;
    g.prefix_width = prefixed->prefix_width;
    g.lse = buf->lse;
    char* at = static_cast<char*>(workspace);
    g.state = reinterpret_cast<float*>(at);
    g.state_stats = reinterpret_cast<float2*>(at + room.state);
    g.state_exact = reinterpret_cast<float*>(at + room.state + room.stats);
    at += room.state + room.stats + room.exact;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    size_t need;
    if (room.state == 0) return mpv::attend_through(prefixed, &g, at, &need, s);
    if (any) {
        rc = mpv::attend_prefixes(a, &g, at, &need, s);
        if (rc != MPV_OK) return rc;
    }
    return mpv::attend_trees<mpv::kBehind>(prefixed, &g, at, &need, s);
}

}  // extern "C"
