// What shared prefixes give to the rows behind them: device and host code.
//
// A unit is what the nodes of up to 64 trees that follow each other and share a prefix read of one cache head (kPrefix of
// mpv_attention.h): their rows, blocks of kRows, read the prefix's tiles together.  So a prefix is read once for each block of rows
// instead of once a tree.
//
// What bounds it, 64 single tokens of 32 query heads on 8 cache heads of 128 bfloat16 values behind 8192 positions: 31 us (and 9 for the
// joining launch) where memory would take 7 and the products as many.  What each further 8192 positions
// take, 17 to 20 us, says that some 11 are what comes before a workgroup's first tile and after its last: the trees' numbers, lengths, pages and
// rows, one load after the other; partial sums.  In between each of the four waves reads all of a tile's keys and values from LDS for 16 rows.

#include "mpv_prefix.h"

namespace mpv {

template <class A>
__global__ __launch_bounds__(A::kThreads) __attribute__((amdgpu_waves_per_eu(A::kWavesOfSimd))) void prefix_kernel(PrefixArgs g) {
    extern __shared__ __align__(1024) char memory[];
    A a(g, *reinterpret_cast<typename A::Shared*>(memory));
    a.all();
}

constexpr int kRowsOfWave = 4;
// Puts the units together that several teams share: a wave has a row, its groups of kLanes lanes some of the parts each.
template <int DTYPE, int DP>
__global__ __launch_bounds__(256) void join_prefix_kernel(PrefixArgs g) {
    constexpr int kLanes = DP / 4, kGroups = 64 / kLanes, kAtOnce = 8;
    const int b = blockIdx.x / g.a.kv_heads, kv = blockIdx.x - b * g.a.kv_heads;
    const int lane = threadIdx.x & 63, column = lane % kLanes * 4, mine = lane / kLanes;
    const int wave = threadIdx.x >> 6;
    // the tree's place among those that share its prefix
    const int tree = (b & ~63) + lane, which = prefix_of(g, tree), nodes = nodes_of(g, tree), upto = wave_sum(nodes);
    const int before = __shfl_up(which, 1);
    const unsigned long long firsts = __ballot(lane == 0 || before != which);
    const int at = b & 63, start = 63 - __clzll(firsts & (at == 63 ? ~0ull : (1ull << (at + 1)) - 1));
    const int rows = __shfl(nodes, at) * g.group, offset = (__shfl(upto - nodes, at) - __shfl(upto - nodes, start)) * g.group;
    if (prefix_length(g, __shfl(which, at)) == 0) return;
    const int last = min(rows, static_cast<int>(blockIdx.y + 1) * (4 * kRowsOfWave));
    for (int row = blockIdx.y * (4 * kRowsOfWave) + wave; row < last; row += 4) {
        const int together = g.blocks * static_cast<int>(g.by_rows.d), super = (offset + row) / together, local = offset + row - super * together;
        const int2 teams = g.units[(static_cast<int64_t>((b & ~63) + start) * g.a.kv_heads + kv) * g.supers + super];
        if (teams.y < 0) continue;
        const int parts = teams.y - teams.x + 1, block = g.by_rows.of(local);
        // part p: the second slot of the first team, the first slot of those after it
        const int64_t first = (static_cast<int64_t>(teams.x) * g.blocks + block) * 2 * g.by_rows.d + (local - block * static_cast<int>(g.by_rows.d));
        const int64_t step = static_cast<int64_t>(g.blocks) * 2 * g.by_rows.d;
        float top = -INFINITY, weight = 0.0f, exact = 0.0f;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int p0 = mine; p0 < parts; p0 += kGroups * kAtOnce) {
            float2 stats[kAtOnce];
            float exacts[kAtOnce] = {};
            f32x4 part[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int p = min(p0 + j * kGroups, parts - 1);
                const int64_t from = first + p * step + (p == 0 ? static_cast<int64_t>(g.by_rows.d) : 0);
                stats[j] = g.partial_stats[from];
                if (g.lse) exacts[j] = g.partial_exact[from];
                part[j] = *reinterpret_cast<const f32x4*>(g.partial + from * DP + column);
            }
            float now = top;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (p0 + j * kGroups < parts) now = fmaxf(now, stats[j].x);
            const float base = now == -INFINITY ? 0.0f : now, fade = exp2_of(top - base);
            weight *= fade;
            exact *= fade;
            sum *= fade;
            top = now;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (p0 + j * kGroups < parts) {
                    const float f = exp2_of(stats[j].x - base);
                    weight += f * stats[j].y;
                    exact += f * exacts[j];
                    sum += part[j] * f;
                }
        }
        float now = top;
        for (int d = kLanes; d < 64; d <<= 1) now = fmaxf(now, __shfl_xor(now, d));
        const float fade = exp2_of(top - (now == -INFINITY ? 0.0f : now));
        weight *= fade;
        exact *= fade;
        sum *= fade;
        for (int d = kLanes; d < 64; d <<= 1) {
            weight += __shfl_xor(weight, d);
            exact += __shfl_xor(exact, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], d);
        }
        if (mine != 0) continue;
        const int node = g.by_group.of(row);
        const int64_t state = (static_cast<int64_t>(b) * g.a.N + node) * g.a.heads + kv * g.group + row - node * g.group;
        *reinterpret_cast<f32x4*>(g.state + state * DP + column) = sum;
        if (column == 0) {
            g.state_stats[state] = make_float2(now, weight);
            if (Elem<DTYPE>::kBytes == 2 && g.lse) g.state_exact[state] = exact;
        }
    }
}

template <class A, int DTYPE, int DP>
static int with_kernel(const mpv_attention* a, PrefixArgs* g, int64_t rows, char* workspace, size_t* bytes, hipStream_t s) {
    Choice c;
    c.rows = A::kRows;
    c.columns = DP;
    c.tile = A::kTile;
    // (a unit is one block of rows, a team one workgroup: those that read the same tiles are neighbours)
    const int64_t supers = (rows + c.rows - 1) / c.rows;
    c.blocks = 1;
    c.teams = kMaxWorkgroups<A>;
    const Parts parts = Parts::of(c);
    const size_t units = whole(static_cast<size_t>(a->B) * a->kv_heads * supers * sizeof(int2));
    *bytes = parts.bytes() + units;
    if (!g) return MPV_OK;
    parts.place(g, workspace);
    g->units = reinterpret_cast<int2*>(workspace + parts.bytes());
    g->supers = static_cast<int>(supers);
    g->by_rows.set(static_cast<uint32_t>(c.rows));
    g->teams = c.teams;
    g->blocks = c.blocks;
    g->by_unit = 0;
    (void)hipGetLastError();
    if (!hip_fine(hipFuncSetAttribute(reinterpret_cast<const void*>(&prefix_kernel<A>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                      static_cast<int>(sizeof(typename A::Shared)))))
        return MPV_ERR_HIP;
    hipLaunchKernelGGL(prefix_kernel<A>, dim3(static_cast<unsigned>(c.teams) * c.blocks), dim3(A::kThreads), sizeof(typename A::Shared), s, *g);
    const int64_t rows_of_tree = static_cast<int64_t>(a->N) * (a->heads / a->kv_heads);
    hipLaunchKernelGGL((join_prefix_kernel<DTYPE, DP>), dim3(static_cast<unsigned>(a->B) * a->kv_heads, static_cast<unsigned>((rows_of_tree + 4 * kRowsOfWave - 1) / (4 * kRowsOfWave))), dim3(256), 0, s, *g);
    return launched();
}

template <int DTYPE, int DP>
static int with_columns(const mpv_attention* a, PrefixArgs* g, char* workspace, size_t* bytes, hipStream_t s) {
    const int64_t rows_of_tree = static_cast<int64_t>(a->N) * (a->heads / a->kv_heads), rows = std::min(a->B, 64) * rows_of_tree;
    const int64_t all = a->B * rows_of_tree * a->kv_heads;
    auto go = [&](auto kernel) { return with_kernel<typename decltype(kernel)::T, DTYPE, DP>(a, g, rows, workspace, bytes, s); };
    // Blocks as large as leave enough of them: a unit that many workgroups share costs partial sums of all its rows from each.  (200 trees
    // with 20 rows a cache head behind 4096 positions: 172 us with blocks of 192 rows, 194 with 64; 64 single tokens with 4 behind 8192: 71 with
    // 128, 64 with 64; 64 trees with 64 behind 8192: 224 with 192, 255 with 64; float32, 200 trees with 20: 990 with 64, 1071 with 128.)
    constexpr int64_t kEnough = 128;
    if (rows <= 16) return go(Chosen<Kernel<kPrefix, DTYPE, DP, 1, 1>>());
    if (rows <= 32) return go(Chosen<Kernel<kPrefix, DTYPE, DP, 1, 2>>());
    if constexpr (DP * Elem<DTYPE>::kBytes > 256) {
        if constexpr (DTYPE != MPV_DTYPE_F32)
            if (rows > 64 && all >= 128 * kEnough) return go(Chosen<Kernel<kPrefix, DTYPE, DP, 1, 8>>());
    } else {
        if (rows > 128 && all >= 192 * kEnough) return go(Chosen<Kernel<kPrefix, DTYPE, DP, 3, 4>>());
        if (rows > 64 && all >= 128 * kEnough) return go(Chosen<Kernel<kPrefix, DTYPE, DP, 2, 4>>());
    }
    return go(Chosen<Kernel<kPrefix, DTYPE, DP, 1, 4>>());
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
