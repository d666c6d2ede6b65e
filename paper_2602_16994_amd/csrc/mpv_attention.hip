// Attention of draft-tree nodes over a paged cache: the call.  Its kernels are those of mpv_attention.h.
//
// What bounds it, with 32 query heads on 8 cache heads of 128 bfloat16 values:
//   256 trees of 41 nodes, contexts of 512 to 4096: 164 rows read every key, 613 us, 2.6 GB at 4.2 TB/s and 645 TFLOP/s (the floor of
//     either alone: 540 us, 350 us).  Loads, the exponents' vector instructions and matrix instructions take turns in a wave, and two
//     workgroups a compute unit do not fill all of the gaps.  With all pages the same (no memory): 12 % less.
//   8 single tokens, contexts of 20 000 to 131 072: 505 us for 2.9 GB, 5.8 TB/s: memory.
//   one tree of 7 nodes, a context of 900: 11.2 us, two launches and the loads that depend on each other (lengths, page, key).
// Contexts of medium size that many teams share are bound by their partial sums as much as by the cache: 32 trees with a window of 1024
// keys of 4 heads of 256 float16 values, 52 us for 144 MB.  float32 is bound by its matrix instruction (154 TFLOP/s at most; 16x16x4).

#include "mpv_attention.h"

namespace mpv {

template <class A>
__global__ __launch_bounds__(A::kThreads) __attribute__((amdgpu_waves_per_eu(2))) void attention_kernel(AttentionArgs g) {
    extern __shared__ __align__(1024) char memory[];
    A a(g, *reinterpret_cast<typename A::Shared*>(memory));
    a.all();
}

template <int DTYPE, int DP, int ROWS>
__global__ __launch_bounds__(256) void combine_kernel(AttentionArgs g) {
    combine<kTree, DTYPE, DP, ROWS>(g);
}

// ------------------------------------------------------------------ host side

// One call: the size of its workspace (g null) or its launches.
template <class A, int DTYPE, int DP>
static int with_kernel(const mpv_attention* a, AttentionArgs* g, void* workspace, size_t* bytes, hipStream_t s) {
    const Choice c = choice_of<A, DP>(a);
    const size_t stats = whole(static_cast<size_t>(c.teams) * c.blocks * 2 * c.rows * sizeof(float2));
    const size_t split = whole(static_cast<size_t>(c.teams) * sizeof(int4));
    const size_t sums = whole(static_cast<size_t>(c.teams) * c.blocks * 2 * c.rows * DP * sizeof(float));
    *bytes = stats + split + sums;
    if (!g) return MPV_OK;
    char* at = static_cast<char*>(workspace);
    g->teams = c.teams;
    g->blocks = c.blocks;
    // (units that are fewer than the teams are joined by unit: 14.6 us by team instead of 11.2 for one tree, 37 instead of 30 in float32)
    g->by_unit = static_cast<int64_t>(a->B) * a->kv_heads < c.teams;
    g->partial_stats = reinterpret_cast<float2*>(at);
    g->split = reinterpret_cast<int4*>(at + stats);
    g->partial = reinterpret_cast<float*>(at + stats + split);
    (void)hipGetLastError();
    if (!hip_fine(hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_kernel<A>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(sizeof(typename A::Shared)))))
        return MPV_ERR_HIP;
    hipLaunchKernelGGL(attention_kernel<A>, dim3(static_cast<unsigned>(c.teams) * c.blocks), dim3(A::kThreads), sizeof(typename A::Shared), s, *g);
    const Second second = second_of<DP>(a, c, g->by_unit);
    if (second.workgroups)
        hipLaunchKernelGGL((combine_kernel<DTYPE, DP, A::kRows>), dim3(static_cast<unsigned>(second.entries), static_cast<unsigned>(second.workgroups)),
                           dim3(256), 0, s, *g);
    return launched();
}

template <int DTYPE, int DP>
static int with_columns(const mpv_attention* a, AttentionArgs* g, void* workspace, size_t* bytes, hipStream_t s) {
    return by_rows<kTree, DTYPE, DP>(static_cast<int64_t>(a->N) * (a->heads / a->kv_heads), [&](auto kernel) {
        return with_kernel<typename decltype(kernel)::T, DTYPE, DP>(a, g, workspace, bytes, s);
    });
}

template <int DTYPE>
static int with_type(const mpv_attention* a, AttentionArgs* g, void* workspace, size_t* bytes, hipStream_t s) {
    if (a->head_dim <= 64) return with_columns<DTYPE, 64>(a, g, workspace, bytes, s);
    if (a->head_dim <= 128) return with_columns<DTYPE, 128>(a, g, workspace, bytes, s);
    return with_columns<DTYPE, 256>(a, g, workspace, bytes, s);
}

static int attend(const mpv_attention* a, AttentionArgs* g, void* workspace, size_t* bytes, hipStream_t s) {
    if (a->dtype == MPV_DTYPE_F32) return with_type<MPV_DTYPE_F32>(a, g, workspace, bytes, s);
    if (a->dtype == MPV_DTYPE_BF16) return with_type<MPV_DTYPE_BF16>(a, g, workspace, bytes, s);
    return with_type<MPV_DTYPE_F16>(a, g, workspace, bytes, s);
}

}  // namespace mpv

extern "C" {

int mpv_tree_attention_workspace_bytes(const mpv_attention* attention, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_attention(attention);
    if (rc != MPV_OK) return rc;
    return mpv::attend(attention, nullptr, nullptr, out, nullptr);
}

int mpv_tree_attention(const mpv_attention* attention, const mpv_attention_buffers* buf, void* workspace, size_t workspace_bytes,
                       void* hip_stream) {
    size_t need;
    const int rc = mpv_tree_attention_workspace_bytes(attention, &need);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    mpv::AttentionArgs g;
    int status = mpv::take_arguments(attention, buf, &g);
    if (status != MPV_OK) return status;
    if (attention->B == 0) return MPV_OK;
    status = mpv::check_buffers(attention, buf);
    if (status != MPV_OK) return status;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < need) return MPV_ERR_WORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return mpv::attend(attention, &g, workspace, &need, s);
}

}  // extern "C"
