// What shared prefixes give to the rows behind them: device and host code.
//
// A unit is what the nodes of up to 64 trees that follow each other and share a prefix read of one cache head (kPrefix of
// mpv_attention.h): their rows, blocks of kRows, read the prefix's tiles together.  So a prefix is read once for each block of rows
// instead of once a tree.

#include "mpv_prefix.h"

namespace mpv {

template <class A>
__global__ __launch_bounds__(A::kThreads) __attribute__((amdgpu_waves_per_eu(2))) void prefix_kernel(PrefixArgs g) {
    extern __shared__ __align__(1024) char memory[];
    A a(g, *reinterpret_cast<typename A::Shared*>(memory));
    a.all();
}

// Puts the units together that several teams share.
template <int DTYPE, int DP, int ROWS>
__global__ __launch_bounds__(256) void join_prefix_kernel(PrefixArgs g) {
    combine<kPrefix, DTYPE, DP, ROWS>(g);
}

// Row blocks of a team.
constexpr int kMostMembers = 8;

template <class A, int DTYPE, int DP>
static int with_kernel(const mpv_attention* a, PrefixArgs* g, int64_t rows, char* workspace, size_t* bytes, hipStream_t s) {
    Choice c;
    c.rows = A::kRows;
    c.columns = DP;
    c.tile = A::kTile;
    const int64_t blocks = (rows + c.rows - 1) / c.rows, supers = (blocks + kMostMembers - 1) / kMostMembers;
    c.blocks = static_cast<int>((blocks + supers - 1) / supers);
    c.teams = kMaxWorkgroups<A> / c.blocks / 8 * 8;
    const Parts parts = Parts::of(c);
    *bytes = parts.bytes();
    if (!g) return MPV_OK;
    parts.place(g, workspace);
    g->teams = c.teams;
    g->blocks = c.blocks;
    g->by_unit = 0;
    (void)hipGetLastError();
    if (!hip_fine(hipFuncSetAttribute(reinterpret_cast<const void*>(&prefix_kernel<A>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(sizeof(typename A::Shared)))))
        return MPV_ERR_HIP;
    hipLaunchKernelGGL(prefix_kernel<A>, dim3(static_cast<unsigned>(c.teams) * c.blocks), dim3(A::kThreads), sizeof(typename A::Shared), s, *g);
    constexpr int kSome = kFewRows * 4 * (64 / (DP / 4));
    const int64_t together = std::min<int64_t>(rows, static_cast<int64_t>(c.blocks) * c.rows);
    const int64_t few = (together + kSome - 1) / kSome, most = std::min<int64_t>(together, std::max<int64_t>(16384 / c.teams, 1));
    hipLaunchKernelGGL((join_prefix_kernel<DTYPE, DP, A::kRows>), dim3(static_cast<unsigned>(c.teams), static_cast<unsigned>(std::max(few, most))),
                       dim3(256), 0, s, *g);
    return launched();
}

template <int DTYPE, int DP>
static int with_columns(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    const int64_t rows = static_cast<int64_t>(std::min(a->B, 64)) * a->N * (a->heads / a->kv_heads);
    return by_rows<kPrefix, DTYPE, DP>(rows, [&](auto kernel) {
        return with_kernel<typename decltype(kernel)::T, DTYPE, DP>(a, g, rows, workspace, bytes, s);
    });
}

template <int DTYPE>
static int with_type(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    if (a->head_dim <= 64) return with_columns<DTYPE, 64>(a, g, workspace, bytes, s);
    if (a->head_dim <= 128) return with_columns<DTYPE, 128>(a, g, workspace, bytes, s);
    return with_columns<DTYPE, 256>(a, g, workspace, bytes, s);
}

int attend_prefixes(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    if (a->dtype == MPV_DTYPE_F32) return with_type<MPV_DTYPE_F32>(a, g, workspace, bytes, s);
    if (a->dtype == MPV_DTYPE_BF16) return with_type<MPV_DTYPE_BF16>(a, g, workspace, bytes, s);
    return with_type<MPV_DTYPE_F16>(a, g, workspace, bytes, s);
}

}  // namespace mpv
