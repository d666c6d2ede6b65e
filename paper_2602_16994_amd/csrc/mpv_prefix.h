// The two halves of attention behind shared prefixes (mpv_prefix.hip: what the prefixes give; mpv_behind.hip: the rest, and the call).

#pragma once

#include "mpv_attention.h"

namespace mpv {

// Parts of a workspace: statistics, sums before rounding, entries of shared units, sums.
struct Parts {
    size_t stats, exact, split, sums;
    size_t bytes() const { return stats + exact + split + sums; }
    static Parts of(const Choice& c) {
        const size_t rows = static_cast<size_t>(c.teams) * c.blocks * 2 * c.rows;
        return {whole(rows * sizeof(float2)), whole(rows * sizeof(float)), whole(static_cast<size_t>(c.teams) * sizeof(int4)),
                whole(rows * c.columns * sizeof(float))};
    }
    void place(PrefixArgs* g, char* at) const {
        g->partial_stats = reinterpret_cast<float2*>(at);
        g->partial_exact = reinterpret_cast<float*>(at + stats);
        g->split = reinterpret_cast<int4*>(at + stats + exact);
        g->partial = reinterpret_cast<float*>(at + stats + exact + split);
    }
};

// Columns of a row of sums for rows of head_dim values.
inline int columns_of(const mpv_attention* a) { return a->head_dim <= 64 ? 64 : a->head_dim <= 128 ? 128 : 256; }

// What the prefixes give to the rows that have one, into g->state.  g null: the bytes that it needs besides.
int attend_prefixes(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s);

}  // namespace mpv
