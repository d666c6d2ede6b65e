// Block tables and slot maps from request lengths, and the move of accepted rows into the paged cache: device and host code.

#include "mpv_host.h"

namespace mpv {

// ------------------------------------------------------------------ tables

// What a call has to move is small (8 bytes a token and the pages' numbers): it costs launches and loads that depend on each other
// (length -> place in the list of free pages -> page -> slot).  So one launch where one workgroup can do it all, and no load of a thread
// waits for another one of the same kind.  64 requests, 1 to 6 new tokens each: 7.2 us; 300 prompts of up to 8192 tokens (1.2 million
// slots, 10 MB): 12.6 us.
constexpr int kPlanBlock = 1024;
constexpr int kFillBlock = 256;
// Slots of a thread of the fill kernels, their pages asked for together (300 prompts: 12.6 us, 13.7 with eight).
constexpr int kFillTogether = 4;
constexpr int kFillSlots = kFillBlock * kFillTogether;
// Up to so many slots (of requests that take one round of the plan's workgroup) that workgroup fills them itself, in one launch:
// 1024 slots in 8.0 us against 8.8 with a second launch, 4000 packed ones in 8.5 against 10.8, 4096 in rows in 10.5 against 10.4;
// 16384 in 34 against 10.4.
constexpr int64_t kFillAtOnce = 4096;

struct PlanEntry {                         // what the fill needs of a request
    int32_t old, given;                    // cached tokens before the call, tokens placed (0 or more)
    int32_t have;                          // pages before the call
    int32_t top;                           // place in the list of free pages of its first new page; the next ones lie before it
};

struct TableArgs {
    mpv_tables t;
    mpv_table_buffers b;
    PlanEntry* plan;                       // [B]
    Divisor by_page;
};

// Inclusive sums of two numbers over the workgroup, the sums of all in total[2].  `part`: LDS, two values a wave.
__device__ __forceinline__ void block_scan(int64_t (&v)[2], int64_t (&total)[2], int64_t (*part)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t a = __shfl_up(v[0], d), b = __shfl_up(v[1], d);
        if (lane >= d) { v[0] += a; v[1] += b; }
    }
    __syncthreads();
    if (lane == 63) { part[wave][0] = v[0]; part[wave][1] = v[1]; }
    __syncthreads();
    total[0] = total[1] = 0;
    for (int w = 0; w < waves; ++w) {
        if (w == wave) { v[0] += total[0]; v[1] += total[1]; }
        total[0] += part[w][0];
        total[1] += part[w][1];
    }
}

// The page of a request's new token i, as it stands in the block table or in the list of free pages.
__device__ __forceinline__ const int32_t* page_of(const TableArgs& a, int b, const PlanEntry& e, int i) {
    const int column = a.by_page.of(e.old + i);
    return column < e.have ? a.b.block_table + static_cast<int64_t>(b) * a.t.table_width + column : a.b.free_pages + e.top - (column - e.have);
}
// Its slot; a new page enters the block table with its first slot, which is always a new token's.
__device__ __forceinline__ int64_t slot_of(const TableArgs& a, int b, const PlanEntry& e, int i, int page) {
    const int at = e.old + i, column = a.by_page.of(at), place = at - column * a.t.page_size;
    if (column >= e.have && place == 0) a.b.block_table[static_cast<int64_t>(b) * a.t.table_width + column] = page;
    return page >= 0 && page < a.t.num_pages ? static_cast<int64_t>(page) * a.t.page_size + place : -1;
}
// A place of the slot map: request, its new token, where its slot goes (null: nowhere).
struct Place {
    int b, i;
    PlanEntry e;
    int64_t* to;
};
// A thread's places, their pages asked for together.
template <int N>
__device__ __forceinline__ void fill_places(const TableArgs& a, const Place (&p)[N]) {
    int page[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        page[j] = -1;
        if (p[j].to && p[j].i < p[j].e.given) page[j] = *page_of(a, p[j].b, p[j].e, p[j].i);
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (p[j].to) *p[j].to = p[j].i < p[j].e.given ? slot_of(a, p[j].b, p[j].e, p[j].i, page[j]) : -1;
}

// One workgroup: who gets what (sums over the requests in their order), and the pages of finished requests.
__global__ __launch_bounds__(kPlanBlock) void plan_tables_kernel(TableArgs a, int fill) {
    __shared__ int64_t part[kPlanBlock / 64][2];
    __shared__ PlanEntry plan[kPlanBlock];                          // with fill: of the only round
    const int B = a.t.B, lane = threadIdx.x & 63, threads = blockDim.x;
    const int64_t width = a.t.table_width;
    auto pages_of = [&](int64_t length) { return length > 0 ? static_cast<int64_t>(a.by_page.of(static_cast<int>(length - 1))) + 1 : 0; };
    int64_t count = min(max(a.b.free_count[0], 0), a.t.num_pages);
    int64_t v[2], total[2];
    for (int base = 0; base < B; base += threads) {
        const int b = base + threadIdx.x;
        int64_t back = 0;
        if (b < B && a.b.new_len[b] < 0)
            back = min(pages_of(max(a.b.context_len[b], 0)), width);
        if (!__syncthreads_or(back > 0)) continue;
        v[0] = back;
        v[1] = 0;
        block_scan(v, total, part);
        const int64_t begin = count + v[0] - back;
        count += total[0];
        for (uint64_t m = __ballot(back > 0); m; m &= m - 1) {
            const int l = __ffsll(static_cast<unsigned long long>(m)) - 1;
            const int64_t pages = __shfl(back, l), to = __shfl(begin, l);
            const int32_t* row = a.b.block_table + (static_cast<int64_t>(b) - lane + l) * width;
            for (int64_t i = lane; i < pages; i += 64)
                if (to + i < a.t.num_pages) a.b.free_pages[to + i] = row[i];
        }
    }
    count = min(count, static_cast<int64_t>(a.t.num_pages));
    int64_t asked = 0, tokens = 0, placed = 0, taken = 0;          // sums over the requests before this round's
    for (int base = 0; base < B; base += threads) {
        const int b = base + threadIdx.x;
        int64_t old = 0, n = 0, have = 0, need = 0;
        bool done = false, never = true;
        if (b < B) {
            const int64_t more = a.b.new_len[b];
            old = max(a.b.context_len[b], 0);
            done = more < 0;
            n = done ? 0 : more + a.t.extra;
            have = pages_of(old);
            const int64_t want = old + n <= INT32_MAX ? pages_of(old + n) : width + 1;       // (a row holds no more than that)
            never = done || want > width || (!a.t.packed && n > a.t.slot_width);
            need = never ? 0 : want - have;
        }
        v[0] = need;
        v[1] = never ? 0 : n;
        block_scan(v, total, part);
        const int64_t upto = asked + v[0], token = tokens + v[1];
        asked += total[0];
        tokens += total[1];
        const bool fits = !never && (need == 0 || upto <= count) && (!a.t.packed || n == 0 || token <= a.t.slot_width);
        const int64_t given = fits ? n : 0;
        v[0] = given;
        v[1] = fits ? need : 0;
        block_scan(v, total, part);
        const int64_t begin = placed + v[0] - given;
        placed += total[0];
        taken += total[1];
        if (b < B) {
            a.b.granted[b] = static_cast<int32_t>(fits ? n : done ? 0 : -1);
            a.b.context_len_out[b] = static_cast<int32_t>(done ? 0 : old + given);
            if (a.b.offsets) a.b.offsets[b] = static_cast<int32_t>(begin);
            PlanEntry e;
            e.old = static_cast<int32_t>(old);
            e.given = static_cast<int32_t>(given);
            e.have = static_cast<int32_t>(have);
            e.top = static_cast<int32_t>(count - 1 - (upto - need));
            if (fill) plan[threadIdx.x] = e; else a.plan[b] = e;
        }
    }
    if (threadIdx.x == 0) {
        a.b.free_count_out[0] = static_cast<int32_t>(count - taken);
        if (a.b.offsets) a.b.offsets[B] = static_cast<int32_t>(placed);
    }
    if (!fill) return;
    __syncthreads();
    if (a.t.packed) {
        for (int b = threadIdx.x >> 6; b < B; b += threads / 64) {
            const PlanEntry e = plan[b];
            const int64_t begin = a.b.offsets[b];
            for (int base = lane; base < e.given; base += 64 * kFillTogether) {
                Place p[kFillTogether];
#pragma unroll
                for (int j = 0; j < kFillTogether; ++j) {
                    const int i = base + 64 * j;
                    p[j] = {b, i, e, i < e.given ? a.b.slot_map + begin + i : nullptr};
                }
                fill_places(a, p);
            }
        }
    } else {
        const int slot_width = static_cast<int>(a.t.slot_width), slots = B * slot_width;
        for (int base = threadIdx.x; base < slots; base += threads * kFillTogether) {
            Place p[kFillTogether];
#pragma unroll
            for (int j = 0; j < kFillTogether; ++j) {
                const int x = base + threads * j, b = x < slots ? x / slot_width : 0;
                p[j] = {b, x - b * slot_width, plan[b], x < slots ? a.b.slot_map + x : nullptr};
            }
            fill_places(a, p);
        }
    }
}

__global__ __launch_bounds__(kFillBlock) void fill_rows_kernel(TableArgs a) {
    const int64_t slots = a.t.slot_width * a.t.B;
    Place p[kFillTogether];
#pragma unroll
    for (int j = 0; j < kFillTogether; ++j) {
        const int64_t x = static_cast<int64_t>(blockIdx.x) * kFillSlots + kFillBlock * j + threadIdx.x;
        const int b = x < slots ? static_cast<int>(static_cast<uint32_t>(x) / static_cast<uint32_t>(a.t.slot_width)) : 0;
        p[j] = {b, static_cast<int>(x - b * a.t.slot_width), a.plan[b], x < slots ? a.b.slot_map + x : nullptr};
    }
    fill_places(a, p);
}

// Requests of a workgroup's slots: the number of requests that end at or before the first of them, found by counting, and at or
// before the last.  Where they are few, as they are where tokens are many, their entries lie in LDS and the request of a slot is found
// there; otherwise by bisection of the offsets.
constexpr int kFewRequests = 8;
__global__ __launch_bounds__(kFillBlock) void fill_packed_kernel(TableArgs a) {
    __shared__ int lo_hi[2];
    __shared__ PlanEntry plan[kFewRequests];
    __shared__ int offset[kFewRequests + 1];
    const int B = a.t.B;
    const int64_t total = a.b.offsets[B];
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kFillSlots;
    if (first >= total) return;
    const int64_t last = min(first + kFillSlots, total) - 1;
    if (threadIdx.x < 2) lo_hi[threadIdx.x] = 0;
    __syncthreads();
    int lo = 0, hi = 0;
    for (int b = threadIdx.x; b < B; b += kFillBlock) {
        const int end = a.b.offsets[b + 1];
        lo += end <= first;
        hi += end <= last;
    }
    for (int d = 32; d; d >>= 1) { lo += __shfl_xor(lo, d); hi += __shfl_xor(hi, d); }
    if ((threadIdx.x & 63) == 0) { atomicAdd(&lo_hi[0], lo); atomicAdd(&lo_hi[1], hi); }
    __syncthreads();
    const int first_request = lo_hi[0], requests = lo_hi[1] - lo_hi[0] + 1;
    if (requests <= kFewRequests) {
        if (static_cast<int>(threadIdx.x) <= requests) offset[threadIdx.x] = a.b.offsets[first_request + threadIdx.x];
        if (static_cast<int>(threadIdx.x) < requests) plan[threadIdx.x] = a.plan[first_request + threadIdx.x];
        __syncthreads();
        Place p[kFillTogether];
#pragma unroll
        for (int j = 0; j < kFillTogether; ++j) {
            const int64_t x = first + j * kFillBlock + threadIdx.x;
            int r = 0;
            for (int k = 1; k < requests; ++k) r += offset[k] <= x;
            p[j] = {first_request + r, static_cast<int>(x - offset[r]), plan[r], x <= last ? a.b.slot_map + x : nullptr};
        }
        fill_places(a, p);
        return;
    }
    for (int64_t x = first + threadIdx.x; x <= last; x += kFillBlock) {
        int l = first_request, h = first_request + requests - 1;           // the request lies in [l, h]
        while (l < h) {
            const int m = (l + h) >> 1;
            if (a.b.offsets[m + 1] <= x) l = m + 1; else h = m;
        }
        const Place p[1] = {{l, static_cast<int>(x - a.b.offsets[l]), a.plan[l], a.b.slot_map + x}};
        fill_places(a, p);
    }
}

// ------------------------------------------------------------------ append

constexpr int kAppendBlock = 256;
constexpr int kAppendLayers = 2;           // layers of one workgroup: a (layer, keys or values) for each of its waves

struct AppendArgs {
    mpv_append p;
    mpv_append_buffers b;
    int rows;                              // rows a tree can have: what slot_map, path_nodes and N allow
    int bytes;                             // of an element
};

// A copy, bound by memory where it is large: a workgroup moves one row of one tree, keys and values, for kAppendLayers layers, a wave
// one of them.  What a wave needs first (accept_len, path, slot) are loads that depend on each other, so many short workgroups hide them
// better than few long ones: 256 trees of 41 nodes and 16 layers of rows of 2 KB, 117 MB read and written, 25.9 us (4.5 TB/s), 27.8 with
// eight layers a workgroup; 4 trees, 32 layers: 3.2 us against 4.0.
__global__ __launch_bounds__(kAppendBlock) void append_kernel(AppendArgs a) {
    const int b = blockIdx.x / a.rows, i = blockIdx.x - b * a.rows;
    if (i > a.b.accept_len[b]) return;
    int node = i;
    if (i > 0 && a.b.path_nodes) node = a.b.path_nodes[static_cast<int64_t>(b) * a.p.max_depth + i - 1];
    const int64_t slot = a.b.slot_map[static_cast<int64_t>(b) * a.p.slot_width + i];
    const int64_t page = slot / a.p.page_size;
    if (slot < 0 || page >= a.p.num_pages || node < 0 || node >= a.p.N) return;
    const int64_t from = (static_cast<int64_t>(b) * a.p.N + node) * a.p.tree_stride;
    const int64_t to = page * a.p.page_stride + (slot - page * a.p.page_size) * a.p.slot_stride;
    const int vectors = a.p.row * a.bytes / 16, lane = threadIdx.x & 63;
    const int layer0 = blockIdx.y * kAppendLayers;
    const int layers = min(kAppendLayers, a.p.layers - layer0);
    for (int j = threadIdx.x >> 6; j < 2 * layers; j += kAppendBlock / 64) {
        const int64_t layer = layer0 + (j >> 1);
        const char* src = static_cast<const char*>(j & 1 ? a.b.tree_v : a.b.tree_k) + (layer * a.p.tree_layer_stride + from) * a.bytes;
        char* dst = static_cast<char*>(j & 1 ? a.b.cache_v : a.b.cache_k) + (layer * a.p.cache_layer_stride + to) * a.bytes;
        for (int x = lane; x < vectors; x += 64) reinterpret_cast<uint4*>(dst)[x] = reinterpret_cast<const uint4*>(src)[x];
    }
}

static int check_tables(const mpv_tables* t) {
    if (!t) return MPV_ERR_NULL;
    if (t->B < 0 || t->page_size < 1 || t->table_width < 0 || t->num_pages < 0 || t->extra < 0 || t->slot_width < 0 ||
        (t->packed != 0 && t->packed != 1))
        return MPV_ERR_BAD_SHAPE;
    // positions, tokens and slots are counted in 32 bits on the device, sums of them in 64
    if (span(0, t->table_width, t->page_size) > INT32_MAX || span(0, t->packed ? 1 : t->B, t->slot_width) > INT32_MAX ||
        t->B > (1 << 30))
        return MPV_ERR_UNSUPPORTED;
    return MPV_OK;
}

}  // namespace mpv

extern "C" {

int mpv_extend_tables_workspace_bytes(const mpv_tables* tables, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_tables(tables);
    if (rc != MPV_OK) return rc;
    *out = (static_cast<size_t>(tables->B) * sizeof(mpv::PlanEntry) + 255) / 256 * 256;
    return MPV_OK;
}

int mpv_extend_tables(const mpv_tables* tables, const mpv_table_buffers* buf, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
    size_t need;
    const int rc = mpv_extend_tables_workspace_bytes(tables, &need);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    if (tables->B == 0) return MPV_OK;
    if (!buf->new_len || !buf->context_len || !buf->free_count || !buf->context_len_out || !buf->free_count_out || !buf->granted ||
        (!buf->block_table && tables->table_width > 0) || (!buf->free_pages && tables->num_pages > 0) ||
        (!buf->slot_map && tables->slot_width > 0) || (!buf->offsets && tables->packed))
        return MPV_ERR_NULL;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < need) return MPV_ERR_WORKSPACE;
    mpv::TableArgs a;
    a.t = *tables; a.b = *buf; a.plan = static_cast<mpv::PlanEntry*>(workspace);
    a.by_page.set(static_cast<uint32_t>(tables->page_size));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int64_t slots = tables->slot_width * (tables->packed ? 1 : tables->B);
    // a wave for 64 requests; as they fill the slots, too, four at least, and eight where slots are many (4096 in rows: 10.5 us against
    // 12.7 with four and 11.5 with sixteen; 512 in rows: the same)
    const int least = slots >= 1024 && slots <= mpv::kFillAtOnce ? 512 : 256;
    const int threads = tables->B >= mpv::kPlanBlock ? mpv::kPlanBlock : tables->B <= least ? least : (tables->B + 63) / 64 * 64;
    const int fill = slots <= mpv::kFillAtOnce && tables->B <= threads;
    (void)hipGetLastError();
    hipLaunchKernelGGL(mpv::plan_tables_kernel, dim3(1), dim3(threads), 0, s, a, fill);
    if (!fill && slots > 0) {
        const dim3 grid(static_cast<unsigned>((slots + mpv::kFillSlots - 1) / mpv::kFillSlots));
        if (tables->packed) hipLaunchKernelGGL(mpv::fill_packed_kernel, grid, dim3(mpv::kFillBlock), 0, s, a);
        else hipLaunchKernelGGL(mpv::fill_rows_kernel, grid, dim3(mpv::kFillBlock), 0, s, a);
    }
    return mpv::launched();
}

int mpv_append_paths(const mpv_append* p, const mpv_append_buffers* buf, void* hip_stream) {
    if (!p || !buf) return MPV_ERR_NULL;
    if (p->layers < 0 || p->B < 0 || p->N < 1 || p->row < 1 || p->max_depth < 0 || p->slot_width < 0 || p->num_pages < 0 || p->page_size < 1)
        return MPV_ERR_BAD_SHAPE;
    if (!mpv::known_dtype(p->dtype)) return MPV_ERR_BAD_DTYPE;
    if (p->N > MPV_MAX_NODES || p->row > (1 << 24)) return MPV_ERR_UNSUPPORTED;
    mpv::AppendArgs a;
    a.p = *p; a.b = *buf; a.bytes = mpv::elem_bytes(p->dtype);
    const int64_t most = buf->path_nodes ? static_cast<int64_t>(p->max_depth) + 1 : p->N;
    a.rows = static_cast<int>(most < p->slot_width ? most : p->slot_width);
    if (p->layers == 0 || p->B == 0 || a.rows == 0 || p->num_pages == 0) return MPV_OK;
    // a row must not reach into the next one
    if (p->tree_stride < p->row || p->slot_stride < p->row || (p->layers > 1 && (p->tree_layer_stride < 0 || p->cache_layer_stride < 0)) ||
        p->page_stride < 0)
        return MPV_ERR_BAD_SHAPE;
    const int64_t layers = (p->layers + mpv::kAppendLayers - 1) / mpv::kAppendLayers;
    if (layers > 65535 || static_cast<int64_t>(p->B) * a.rows >= (1 << 24) || mpv::span(0, p->num_pages, p->page_size) == INT64_MAX ||
        mpv::span(0, mpv::span(mpv::span(0, p->layers, p->tree_layer_stride), static_cast<int64_t>(p->B) * p->N, p->tree_stride), 4) == INT64_MAX ||
        mpv::span(0, mpv::span(mpv::span(mpv::span(0, p->layers, p->cache_layer_stride), p->num_pages, p->page_stride), p->page_size, p->slot_stride), 4) == INT64_MAX)
        return MPV_ERR_UNSUPPORTED;
    if (!buf->tree_k || !buf->tree_v || !buf->cache_k || !buf->cache_v || !buf->slot_map || !buf->accept_len) return MPV_ERR_NULL;
    const int64_t strides = p->row | p->tree_stride | p->slot_stride | p->page_stride | (p->layers > 1 ? p->tree_layer_stride | p->cache_layer_stride : 0);
    if (!mpv::aligned(buf->tree_k, 16) || !mpv::aligned(buf->tree_v, 16) || !mpv::aligned(buf->cache_k, 16) || !mpv::aligned(buf->cache_v, 16) ||
        (strides * a.bytes) % 16 != 0)
        return MPV_ERR_ALIGNMENT;
    (void)hipGetLastError();
    hipLaunchKernelGGL(mpv::append_kernel, dim3(static_cast<unsigned>(p->B * a.rows), static_cast<unsigned>(layers)), dim3(mpv::kAppendBlock),
                       0, static_cast<hipStream_t>(hip_stream), a);
    return mpv::launched();
}

}  // extern "C"
