// Attention of draft-tree nodes over a paged cache: device and host code.

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <cmath>
#include <cstring>

#include "mpv_host.h"

namespace mpv {

struct AttentionArgs {
    mpv_attention a;
    mpv_attention_buffers b;
    int8_t parent[MPV_MAX_NODES];          // the shared shape (without tree_parent)
};

__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float value(const uint16_t* p, int64_t i) { return __uint_as_float(static_cast<uint32_t>(p[i]) << 16); }
__device__ __forceinline__ float value(const __half* p, int64_t i) { return __half2float(p[i]); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(uint16_t* p, float v) {
    const __hip_bfloat16 h = __float2bfloat16(v);
    *reinterpret_cast<__hip_bfloat16*>(p) = h;
}
__device__ __forceinline__ void store(__half* p, float v) { *p = __float2half(v); }

// A wave per (tree, node, head): 64 keys at a time, a lane each; then the lanes share the values' columns.
template <class T>
__global__ __launch_bounds__(64) void tree_attention_kernel(AttentionArgs g) {
    const mpv_attention& a = g.a;
    const int lane = threadIdx.x;
    const int h = blockIdx.x % a.heads, n = blockIdx.x / a.heads, b = blockIdx.y;
    const int nodes = g.b.num_nodes ? min(max(g.b.num_nodes[b], 0), a.N) : a.N;
    if (n >= nodes) return;
    auto parent_of = [&](int m) {
        const int p = g.b.tree_parent ? g.b.tree_parent[static_cast<int64_t>(b) * a.N + m] : g.parent[m];
        return p >= 0 && p < m ? p : -1;
    };
    unsigned long long line = 0;                              // ancestors and the node itself
    for (int m = n; m >= 0; m = parent_of(m)) line |= 1ull << m;
    const int depth = __popcll(line) - 1;
    const int64_t context = min(static_cast<int64_t>(max(g.b.context_len[b], 0)), static_cast<int64_t>(a.table_width) * a.page_size);
    const int64_t at = context + depth;
    const int64_t low = a.window > 0 ? at - a.window + 1 : 0;
    const int64_t tree = static_cast<int64_t>(b) * a.N;
    const int kv = h / (a.heads / a.kv_heads);
    const T* q = static_cast<const T*>(g.b.q) + (tree + n) * a.q_stride + static_cast<int64_t>(h) * a.head_dim;
    float top = -INFINITY, sum = 0.0f, out[MPV_MAX_HEAD_DIM / 64] = {};

    auto take = [&](bool seen, const T* k, const T* v) {      // 64 keys
        float s = -INFINITY;
        if (seen) {
            s = 0.0f;
            for (int d = 0; d < a.head_dim; ++d) s += value(q, d) * value(k, d);
            s *= a.scale;
        }
        float m = s;
        for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
        const float now = fmaxf(top, m), base = now == -INFINITY ? 0.0f : now;
        const float fade = expf(top - base);
        const float w = seen ? expf(s - base) : 0.0f;
        top = now;
        sum *= fade;
        for (int c = 0; c < MPV_MAX_HEAD_DIM / 64; ++c) out[c] *= fade;
        float all = w;
        for (int x = 32; x; x >>= 1) all += __shfl_xor(all, x);
        sum += all;
        for (unsigned long long m2 = __ballot(seen); m2; m2 &= m2 - 1) {
            const int l = __ffsll(m2) - 1;
            const float wl = __shfl(w, l);
            const T* vl = reinterpret_cast<const T*>(__shfl(reinterpret_cast<unsigned long long>(v), l));
            for (int c = 0; c < MPV_MAX_HEAD_DIM / 64; ++c)
                if (lane + 64 * c < a.head_dim) out[c] += wl * value(vl, lane + 64 * c);
        }
    };

    const int64_t sinks = a.window > 0 ? min(static_cast<int64_t>(max(a.sinks, 0)), context) : 0;
    for (int64_t base = 0; base < context; base += 64) {
        if (base >= sinks && base + 64 <= low) base = low / 64 * 64;     // nothing is seen between the sinks and the window
        if (base >= context) break;
        const int64_t j = base + lane;
        bool seen = j < context && (j >= low || j < sinks);
        const T *k = nullptr, *v = nullptr;
        if (seen) {
            const int64_t page = g.b.block_table[static_cast<int64_t>(b) * a.table_width + j / a.page_size];
            seen = page >= 0 && page < a.num_pages;
            const int64_t where = page * a.page_stride + j % a.page_size * a.slot_stride + static_cast<int64_t>(kv) * a.head_dim;
            k = static_cast<const T*>(g.b.cache_k) + where;
            v = static_cast<const T*>(g.b.cache_v) + where;
        }
        take(seen, k, v);
    }
    {
        bool seen = lane < nodes && ((line >> lane) & 1);
        const int64_t place = context + __popcll(line & ((1ull << lane) - 1));
        seen = seen && (place >= low || place < max(a.sinks, 0));
        const int64_t where = (tree + lane) * a.kv_stride + static_cast<int64_t>(kv) * a.head_dim;
        take(seen, static_cast<const T*>(g.b.tree_k) + where, static_cast<const T*>(g.b.tree_v) + where);
    }
    T* to = static_cast<T*>(g.b.out) + (tree + n) * a.out_stride + static_cast<int64_t>(h) * a.head_dim;
    for (int c = 0; c < MPV_MAX_HEAD_DIM / 64; ++c)
        if (lane + 64 * c < a.head_dim) store(to + lane + 64 * c, out[c] / sum);
}

static int check_attention(const mpv_attention* a) {
    if (!a) return MPV_ERR_NULL;
    if (a->B < 0 || a->N < 1 || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads != 0 || a->head_dim < 1 || a->num_pages < 0 ||
        a->page_size < 1 || a->table_width < 0)
        return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(a->dtype)) return MPV_ERR_BAD_DTYPE;
    if (!std::isfinite(a->scale)) return MPV_ERR_BAD_TEMPERATURE;
    if (a->N > MPV_MAX_NODES || a->head_dim > MPV_MAX_HEAD_DIM || a->heads > 65535) return MPV_ERR_UNSUPPORTED;
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

template <class T>
static int launch_attention(const AttentionArgs& g, hipStream_t s) {
    (void)hipGetLastError();
    hipLaunchKernelGGL(tree_attention_kernel<T>, dim3(static_cast<unsigned>(g.a.N * g.a.heads), static_cast<unsigned>(g.a.B)), dim3(64), 0, s, g);
    return launched();
}

}  // namespace mpv

extern "C" {

int mpv_tree_attention_workspace_bytes(const mpv_attention* attention, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_attention(attention);
    if (rc != MPV_OK) return rc;
    *out = 256;
    return MPV_OK;
}

int mpv_tree_attention(const mpv_attention* attention, const mpv_attention_buffers* buf, void* workspace, size_t workspace_bytes,
                       void* hip_stream) {
    size_t need;
    const int rc = mpv_tree_attention_workspace_bytes(attention, &need);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    mpv::AttentionArgs g;
    g.a = *attention; g.b = *buf;
    if (!buf->tree_parent) {
        if (!attention->parent) return MPV_ERR_NULL;
        if (attention->parent[0] != -1) return MPV_ERR_BAD_TREE;
        g.parent[0] = -1;
        for (int n = 1; n < attention->N; ++n) {
            if (attention->parent[n] < 0 || attention->parent[n] >= n) return MPV_ERR_BAD_TREE;
            g.parent[n] = static_cast<int8_t>(attention->parent[n]);
        }
    }
    if (attention->B == 0) return MPV_OK;
    if (!buf->q || !buf->tree_k || !buf->tree_v || !buf->context_len || !buf->out ||
        (attention->table_width > 0 && (!buf->block_table || !buf->cache_k || !buf->cache_v)))
        return MPV_ERR_NULL;
    if (!mpv::aligned(buf->q, 16) || !mpv::aligned(buf->tree_k, 16) || !mpv::aligned(buf->tree_v, 16) || !mpv::aligned(buf->cache_k, 16) ||
        !mpv::aligned(buf->cache_v, 16) || !mpv::aligned(buf->out, 16))
        return MPV_ERR_ALIGNMENT;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < need) return MPV_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (attention->dtype == MPV_DTYPE_F32) return mpv::launch_attention<float>(g, s);
    if (attention->dtype == MPV_DTYPE_BF16) return mpv::launch_attention<uint16_t>(g, s);
    return mpv::launch_attention<__half>(g, s);
}

}  // extern "C"
