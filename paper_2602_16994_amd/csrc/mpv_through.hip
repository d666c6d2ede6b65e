// Attention of draft trees that read their prefixes each for itself, as the beginning of their contexts (kThrough of mpv_attention.h).
//
// A context's positions are those of the prefix and then its own, and a tile may hold both: where a key lies is looked up key by key in any
// case.  What bounds it is what bounds mpv_tree_attention, with prefixes that come from the chiplets' caches: the benchmark's trees
// (41 nodes, 164 rows a cache head) behind four prefixes of 512 to 2048 positions, own contexts of 64 to 1024: 540 us, 650 TFLOP/s: products, exponents
// and loads take turns in a wave.  48 trees of 14 nodes with a window of 2000: 31 us (and 7 for the second launch;
// 70 MB are read; vector instructions 0.32 of the time, matrix units 0.11: the few tiles of a workgroup wait for each other, and for what
// comes before them); two requests behind 1000 positions: 16 us, two launches.

#include "mpv_behind.h"

namespace mpv {

int attend_through(const mpv_prefixed* p, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    return attend_trees<kThrough>(p, g, workspace, bytes, s);
}

}  // namespace mpv
