// The attention weight that cached positions gather: device and host code.
//
// score_j <- decay score_j + sum over the accepted nodes n and query heads of e^(s_nj - lse_n), with the logarithm lse_n of the node's sum
// that the attention found, so nothing has to be put together: keys are read once, values not at all, and a position belongs to one
// wave.  S^T = K Q^T as in the attention, but a lane's part of a key goes from memory to the registers that the matrix instruction reads.
// A result's 16 columns are rows (node, query head): they are added up over the lanes in the end, each of 16 lanes keeping another sum.
//
// What bounds it: 16 layers of 16 contexts of 500 to 8192 keys, 8 cache heads of 128 bfloat16 values, up to 6 nodes of 4 query heads: 475 us for
// 2.3 GB that are read, 4.8 TB/s: memory.  (Without the next round's keys on their way: 797.)  One token with a context of 900: 6.6 us, a launch and lengths ->
// page -> key, one after the other.  Where a score is all heads' the keys are not asked for ahead: 16 layers of 21 contexts of up to 744, 107 us
// for 410 MB.

#include <climits>
#include <type_traits>

#include "mpv_attention.h"

namespace mpv {

struct ScoreArgs {
    mpv_scores p;
    mpv_score_buffers b;
    int group, parts;                      // query heads of a cache head; parts of a row of scores, a wave's each
    Divisor by_group, by_page;
};

constexpr int kScoreWaves = 4;
// Groups of 16 keys that a wave reads at a time, for rows of so many bytes.
constexpr int keys_together(int bytes) { return bytes <= 256 ? 4 : bytes <= 512 ? 2 : 1; }

// Sums over 16 neighbouring lanes of v[0 .. n): the lane's is v[lane % n].
template <int n>
__device__ __forceinline__ float spread_sum(float (&v)[n]) {
    const int lane = threadIdx.x & 15;
    auto step = [&](auto control, auto size, int bit) {
        constexpr int kControl = decltype(control)::value, kNow = decltype(size)::value;      // values before the step
        auto other = [&](float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kControl, 0xf, 0xf, true)); };
        if constexpr (kNow > n) {
#pragma unroll
            for (int i = 0; i < n; ++i) v[i] += other(v[i]);
        } else {
            const bool high = lane & bit;
#pragma unroll
            for (int i = 0; i < kNow / 2; ++i) {
                const float keep = high ? v[i + kNow / 2] : v[i], give = high ? v[i] : v[i + kNow / 2];
                v[i] = keep + other(give);
            }
        }
    };
    step(std::integral_constant<int, 0x140>(), std::integral_constant<int, 16>(), 8);         // mirrored: every bit of the lane differs
    step(std::integral_constant<int, 0x141>(), std::integral_constant<int, 8>(), 4);          // mirrored in eights
    step(std::integral_constant<int, 0x4e>(), std::integral_constant<int, 4>(), 2);           // pairs
    step(std::integral_constant<int, 0xb1>(), std::integral_constant<int, 2>(), 1);           // neighbours
    return v[0];
}

// QT: groups of 16 rows that a wave keeps; 0: any number, read again for every round (and for every cache head where those share a score).
template <int DTYPE, int DP, int QT>
__global__ __launch_bounds__(64 * kScoreWaves) __attribute__((amdgpu_waves_per_eu(2))) void score_kernel(ScoreArgs g) {
    typedef Elem<DTYPE> E;
    constexpr int kSteps = DP * E::kBytes / 64, U = keys_together(DP * E::kBytes), kKeys = 16 * U;
    const mpv_scores& p = g.p;
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = p.score_heads;
    // (a wave has nothing to do with the others of its workgroup: lists may be shorter than what four of them take)
    const unsigned number = blockIdx.x * kScoreWaves + wave;
    unsigned unit = number / static_cast<unsigned>(g.parts);
    const int part = number - unit * g.parts;
    const int head = unit % heads;
    unit /= heads;
    const int b = unit % p.B, layer = unit / p.B;
    if (layer >= p.layers) return;
    const int context = min(max(g.b.context_len[b], 0), p.table_width * p.page_size);
    const int path = g.b.accept_len ? min(min(max(g.b.accept_len[b], 0), p.N - 1), g.b.path_nodes ? p.max_depth : p.N - 1) + 1 : 1;
    const int64_t whole = static_cast<int64_t>(context) + path;
    const int total = static_cast<int>(min(whole, p.score_width));
    // (the rounds of a list go to its parts in turn: they end together whatever the length, and read side by side)
    const int begin = part * kKeys, step = g.parts * kKeys;
    if (begin >= total) return;
    float* scores = g.b.scores + ((static_cast<int64_t>(layer) * p.B + b) * heads + head) * p.score_width;
    auto node_of = [&](int i) {            // of the path's i-th row; out of range: none
        const int n = i == 0 ? 0 : g.b.path_nodes ? g.b.path_nodes[static_cast<int64_t>(b) * p.max_depth + i - 1] : i;
        return n >= 0 && n < p.N ? n : -1;
    };
    const int64_t tree = static_cast<int64_t>(layer) * p.B + b;
    const char* q = static_cast<const char*>(g.b.q) + (static_cast<int64_t>(layer) * p.q_layer_stride + static_cast<int64_t>(b) * p.N * p.q_stride) * E::kBytes;
    const char* tree_k = static_cast<const char*>(g.b.tree_k) + (static_cast<int64_t>(layer) * p.tree_layer_stride + static_cast<int64_t>(b) * p.N * p.tree_stride) * E::kBytes;
    const char* cache = static_cast<const char*>(g.b.cache_k) + static_cast<int64_t>(layer) * p.cache_layer_stride * E::kBytes;
    const int rows = path * g.group, row_bytes = p.head_dim * E::kBytes;
    const int first_head = heads == 1 ? 0 : head, last_head = heads == 1 ? p.kv_heads : head + 1;

    // 16 rows of queries: this lane's is row base + l16, its part of every step
    struct Queries { u32x4 part[kSteps]; float lse; int upto; };   // upto: its place in the path (INT_MIN: it gives nothing)
    auto queries = [&](int kv, int base) {
        Queries r;
        const int row = base + l16, i = g.by_group.of(row), node = row < rows ? node_of(i) : -1;
        const int query_head = kv * g.group + row - i * g.group;
        r.lse = -INFINITY;
        if (node >= 0) r.lse = g.b.lse[(tree * p.N + node) * p.heads + query_head];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int byte = (s * 4 + quad) * 16;
            r.part[s] = u32x4{0u, 0u, 0u, 0u};
            if (node >= 0 && byte < row_bytes)
                r.part[s] = *reinterpret_cast<const u32x4*>(q + (static_cast<int64_t>(node) * p.q_stride + static_cast<int64_t>(query_head) * p.head_dim) * E::kBytes + byte);
        }
        r.upto = r.lse == -INFINITY ? INT_MIN : i;
        return r;
    };
    Queries kept[QT ? QT : 1];
    if constexpr (QT > 0)
#pragma unroll
        for (int t = 0; t < QT; ++t) kept[t] = queries(first_head, t * 16);

    // a round's keys: the pages that they lie in, where their rows lie (null: nowhere), the rows, and the score so far of this lane's position
    struct Keys { const char* from[U]; u32x4 part[U][kSteps]; float old; };
    struct Pages { int of[U]; };
    const int mine = l16 % (4 * U), own_key = (mine >> 2) * 16 + quad * 4 + (mine & 3);
    auto pages = [&](int first) {
        Pages r;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = first + u * 16 + l16;
            r.of[u] = -1;
            if (at < context) r.of[u] = g.b.block_table[static_cast<int64_t>(b) * p.table_width + g.by_page.of(at)];
            else if (at < total) r.of[u] = node_of(at - context);
        }
        return r;
    };
    auto places = [&](int first, const Pages& r, Keys& k) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = first + u * 16 + l16;
            k.from[u] = nullptr;
            if (at < context) {
                if (r.of[u] >= 0 && r.of[u] < p.num_pages)
                    k.from[u] = cache + (r.of[u] * p.page_stride + (at - g.by_page.of(at) * p.page_size) * p.slot_stride) * E::kBytes;
            } else if (r.of[u] >= 0) {
                k.from[u] = tree_k + r.of[u] * p.tree_stride * E::kBytes;
            }
        }
    };
    auto ask = [&](int first, int kv, Keys& k) {
        const int at = first + own_key;
        k.old = l16 < 4 * U && at < context ? scores[at] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int byte = (s * 4 + quad) * 16;
                k.part[u][s] = u32x4{0u, 0u, 0u, 0u};
                if (k.from[u] && byte < row_bytes) k.part[u][s] = *reinterpret_cast<const u32x4*>(k.from[u] + static_cast<int64_t>(kv) * row_bytes + byte);
            }
    };
    auto add = [&](int first, const Keys& k, const Queries& r, float (&sum)[4 * U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if constexpr (E::kBytes == 2) {
                    c = E::mfma(k.part[u][s], r.part[s], c);
                } else {
                    const f32x4 fk = __builtin_bit_cast(f32x4, k.part[u][s]), fq = __builtin_bit_cast(f32x4, r.part[s]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fk[x], fq[x], c, 0, 0, 0);
                }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int ahead = first + u * 16 + quad * 4 + x - context;                 // of the path's rows, those behind it see it
                const float w = exp2_of(fmaf(c[x], p.scale, -r.lse) * 1.4426950408889634f);
                sum[u * 4 + x] += ahead <= r.upto ? w : 0.0f;
            }
        }
    };
    auto finish = [&](int first, const Keys& k, float (&sum)[4 * U]) {
        const float given = spread_sum(sum);
        const int at = first + own_key;
        // (whether the key is there is known at the lane that looked for it)
        bool seen = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool x = __shfl(static_cast<int>(k.from[u] != nullptr), own_key & 15);
            if (own_key >> 4 == u) seen = x;
        }
        if (l16 < 4 * U && at < total) scores[at] = (at < context ? p.decay * k.old : 0.0f) + (seen ? given : 0.0f);
    };

    if constexpr (QT > 0) {
        // the next round's keys, and the pages of the one after it, are on their way while one is worked on
        Keys keys[2];
        Pages next = pages(begin);
        places(begin, next, keys[0]);
        ask(begin, first_head, keys[0]);
        next = pages(begin + step);
        for (int first = begin; first < total;) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (first >= total) break;
                if (first + step < total) {
                    places(first + step, next, keys[1 - h]);
                    ask(first + step, first_head, keys[1 - h]);
                    next = pages(first + 2 * step);
                }
                float sum[4 * U] = {};
#pragma unroll
                for (int t = 0; t < QT; ++t) add(first, keys[h], kept[t], sum);
                finish(first, keys[h], sum);
                first += step;
            }
        }
    } else {
        for (int first = begin; first < total; first += step) {
            Keys keys;
            places(first, pages(first), keys);
            float sum[4 * U] = {};
            for (int kv = first_head; kv < last_head; ++kv) {
                ask(first, kv, keys);
                for (int base = 0; base < rows; base += 16) add(first, keys, queries(kv, base), sum);
            }
            finish(first, keys, sum);
        }
    }
}

// ------------------------------------------------------------------ host side

static int check_scores(const mpv_scores* p) {
    if (!p) return MPV_ERR_NULL;
    if (p->layers < 0 || p->B < 0 || p->N < 1 || p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads != 0 || p->head_dim < 1 ||
        (p->score_heads != 1 && p->score_heads != p->kv_heads) || p->max_depth < 0 || p->num_pages < 0 || p->page_size < 1 || p->table_width < 0 ||
        p->score_width < 0)
        return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(p->dtype)) return MPV_ERR_BAD_DTYPE;
    if (!std::isfinite(p->scale) || !std::isfinite(p->decay)) return MPV_ERR_BAD_TEMPERATURE;
    if (p->N > MPV_MAX_NODES || p->head_dim > MPV_MAX_HEAD_DIM || p->heads > MPV_MAX_HEADS) return MPV_ERR_UNSUPPORTED;
    const int64_t row = static_cast<int64_t>(p->kv_heads) * p->head_dim, wide = static_cast<int64_t>(p->heads) * p->head_dim;
    if (p->q_stride < wide || p->tree_stride < row || p->slot_stride < row || p->page_stride < 0 || p->q_layer_stride < 0 || p->tree_layer_stride < 0 ||
        p->cache_layer_stride < 0 || p->score_width < span(0, p->table_width, p->page_size))
        return MPV_ERR_BAD_SHAPE;
    const int64_t nodes = static_cast<int64_t>(p->B) * p->N;
    const int64_t lists = span(0, span(0, p->layers, p->B), p->score_heads);
    if (p->B > (1 << 24) || span(MPV_MAX_NODES, p->table_width, p->page_size) > INT32_MAX || p->score_width > (1 << 29) ||
        lists > kMostWorkgroups ||
        span(0, span(span(0, nodes, p->q_stride), p->layers, p->q_layer_stride), 4) == INT64_MAX ||
        span(0, span(span(0, nodes, p->tree_stride), p->layers, p->tree_layer_stride), 4) == INT64_MAX ||
        span(0, span(span(span(0, p->num_pages, p->page_stride), p->page_size, p->slot_stride), p->layers, p->cache_layer_stride), 4) == INT64_MAX)
        return MPV_ERR_UNSUPPORTED;
    const int64_t all = p->head_dim | p->q_stride | p->tree_stride | p->slot_stride | p->page_stride | p->q_layer_stride | p->tree_layer_stride |
                        p->cache_layer_stride;
    if ((all * elem_bytes(p->dtype)) % 16 != 0) return MPV_ERR_ALIGNMENT;
    return MPV_OK;
}

template <int DTYPE, int DP, int QT>
static void launch_groups(const ScoreArgs& g, int64_t lists, hipStream_t s) {
    const int64_t workgroups = (lists * g.parts + kScoreWaves - 1) / kScoreWaves;
    hipLaunchKernelGGL((score_kernel<DTYPE, DP, QT>), dim3(static_cast<unsigned>(workgroups)), dim3(64 * kScoreWaves), 0, s, g);
}

template <int DTYPE, int DP>
static int launch_scores(ScoreArgs& g, hipStream_t s) {
    constexpr int kRound = 16 * keys_together(DP * Elem<DTYPE>::kBytes);
    const mpv_scores& p = g.p;
    const int64_t positions = std::min(span(p.N, p.table_width, p.page_size), p.score_width);
    const int64_t lists = static_cast<int64_t>(p.layers) * p.B * p.score_heads, rounds = (positions + kRound - 1) / kRound;
    if (rounds == 0 || lists == 0) return MPV_OK;
    // as many rounds a wave as leave enough waves for all compute units (16 layers of 16 contexts of up to 8192: 460 us with eight, 485 with
    // four, 481 with sixteen)
    const int64_t most = kMostWorkgroups * kScoreWaves;
    const int64_t each = std::max(std::max<int64_t>(1, std::min<int64_t>(8, rounds * lists / 8192)), (rounds + most / lists - 1) / (most / lists));
    g.parts = static_cast<int>((rounds + each - 1) / each);
    const int64_t deepest = g.b.accept_len ? std::min(p.N - 1, g.b.path_nodes ? p.max_depth : p.N - 1) + 1 : 1, rows = deepest * g.group;
    const bool alone = p.score_heads == p.kv_heads;
    constexpr bool kLongest = DP * Elem<DTYPE>::kBytes > 512;      // (two groups of such rows do not fit the registers)
    (void)hipGetLastError();
    if (alone && rows <= 16) launch_groups<DTYPE, DP, 1>(g, lists, s);
    else if (!kLongest && alone && rows <= 32) launch_groups<DTYPE, DP, kLongest ? 1 : 2>(g, lists, s);
    else launch_groups<DTYPE, DP, 0>(g, lists, s);
    return launched();
}

template <int DTYPE>
static int score(ScoreArgs& g, hipStream_t s) {
    if (g.p.head_dim <= 64) return launch_scores<DTYPE, 64>(g, s);
    if (g.p.head_dim <= 128) return launch_scores<DTYPE, 128>(g, s);
    return launch_scores<DTYPE, 256>(g, s);
}

}  // namespace mpv

extern "C" {

int mpv_score_positions(const mpv_scores* scores, const mpv_score_buffers* buf, void* hip_stream) {
    const int rc = mpv::check_scores(scores);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    if (scores->layers == 0 || scores->B == 0) return MPV_OK;
    if (!buf->q || !buf->tree_k || !buf->context_len || !buf->lse || (scores->score_width > 0 && !buf->scores) ||
        (scores->table_width > 0 && (!buf->block_table || (scores->num_pages > 0 && !buf->cache_k))))
        return MPV_ERR_NULL;
    if (!mpv::aligned(buf->q, 16) || !mpv::aligned(buf->tree_k, 16) || !mpv::aligned(buf->cache_k, 16)) return MPV_ERR_ALIGNMENT;
    mpv::ScoreArgs g;
    g.p = *scores;
    g.b = *buf;
    g.group = scores->heads / scores->kv_heads;
    g.by_group.set(static_cast<uint32_t>(g.group));
    g.by_page.set(static_cast<uint32_t>(scores->page_size));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (scores->dtype == MPV_DTYPE_F32) return mpv::score<MPV_DTYPE_F32>(g, s);
    if (scores->dtype == MPV_DTYPE_BF16) return mpv::score<MPV_DTYPE_BF16>(g, s);
    return mpv::score<MPV_DTYPE_F16>(g, s);
}

}  // extern "C"
