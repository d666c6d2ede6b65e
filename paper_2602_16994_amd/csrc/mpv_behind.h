// The launches for trees behind prefixes: their own part (mpv_behind.hip), or prefix and all (mpv_through.hip).

#pragma once

#include "mpv_prefix.h"

namespace mpv {

template <class A>
__global__ __launch_bounds__(A::kThreads) __attribute__((amdgpu_waves_per_eu(A::kWavesOfSimd))) void behind_kernel(PrefixArgs g) {
    extern __shared__ __align__(1024) char memory[];
    A a(g, *reinterpret_cast<typename A::Shared*>(memory));
    a.all();
}

// Puts the units together that several teams share.
template <int KIND, int DTYPE, int DP, int ROWS>
__global__ __launch_bounds__(256) void join_behind_kernel(PrefixArgs g) {
    combine<KIND, DTYPE, DP, ROWS>(g);
}

template <class A, int KIND, int DTYPE, int DP>
int with_kernel(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    const Choice c = choice_of<A, DP>(a);
    const Parts parts = Parts::of(c);
    *bytes = parts.bytes();
    if (!g) return MPV_OK;
    parts.place(g, workspace);
    g->teams = c.teams;
    g->blocks = c.blocks;
    g->by_unit = static_cast<int64_t>(a->B) * a->kv_heads < c.teams;
    const int64_t rows = static_cast<int64_t>(a->N) * (a->heads / a->kv_heads);
    (void)hipGetLastError();
    if (!hip_fine(hipFuncSetAttribute(reinterpret_cast<const void*>(&behind_kernel<A>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(sizeof(typename A::Shared)))))
        return MPV_ERR_HIP;
    hipLaunchKernelGGL(behind_kernel<A>, dim3(static_cast<unsigned>(c.teams) * c.blocks), dim3(A::kThreads), sizeof(typename A::Shared), s, *g);
    const Second second = second_of<DP>(a, c, g->by_unit);
    if (second.workgroups)
        hipLaunchKernelGGL((join_behind_kernel<KIND, DTYPE, DP, A::kRows>), dim3(static_cast<unsigned>(second.entries), static_cast<unsigned>(second.workgroups)),
                           dim3(256), 0, s, *g);
    return launched();
}

template <int KIND, int DTYPE, int DP>
int with_columns(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    return by_rows<KIND, DTYPE, DP>(static_cast<int64_t>(a->N) * (a->heads / a->kv_heads), [&](auto kernel) {
        return with_kernel<typename decltype(kernel)::T, KIND, DTYPE, DP>(a, g, workspace, bytes, s);
    });
}

template <int KIND, int DTYPE>
int with_type(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    if (a->head_dim <= 64) return with_columns<KIND, DTYPE, 64>(a, g, workspace, bytes, s);
    if (a->head_dim <= 128) return with_columns<KIND, DTYPE, 128>(a, g, workspace, bytes, s);
    return with_columns<KIND, DTYPE, 256>(a, g, workspace, bytes, s);
}

// The launches of a call for its trees (g null: the bytes that they need).
template <int KIND>
int attend_trees(const mpv_prefixed* p, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    mpv_attention a = p->attention;
    if (KIND == kThrough) a.table_width += p->prefix_width;        // (as far as a context's length goes)
    if (a.dtype == MPV_DTYPE_F32) return with_type<KIND, MPV_DTYPE_F32>(&a, g, workspace, bytes, s);
    if (a.dtype == MPV_DTYPE_BF16) return with_type<KIND, MPV_DTYPE_BF16>(&a, g, workspace, bytes, s);
    return with_type<KIND, MPV_DTYPE_F16>(&a, g, workspace, bytes, s);
}

// attend_trees<kThrough> (mpv_through.hip)
int attend_through(const mpv_prefixed* p, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s);

}  // namespace mpv
