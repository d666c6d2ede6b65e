// Attention of draft trees that read their prefixes each for itself, as the beginning of their contexts (kThrough of mpv_attention.h).

#include "mpv_behind.h"

namespace mpv {

int attend_through(const mpv_prefixed* p, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    return attend_trees<kThrough>(p, g, workspace, bytes, s);
}

}  // namespace mpv
