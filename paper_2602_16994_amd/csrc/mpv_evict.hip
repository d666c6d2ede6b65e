// Eviction of cached positions that gathered little weight: device and host code.
//
// select_kernel: a workgroup has one list (layer, request, score head).  The budget's worth of best scores is found some bits of their
// order at a time; then the kept positions are written in order, and the slots that their rows lie in.  Its first workgroups work out
// where the returned pages go, and whether all of them are pages.
// move_kernel: kept rows move forward in order.  The i-th kept position s_i is at least i and the s_i ascend, so that what is written to the
// rows [c, c + n) was read with them or before: a workgroup that takes a slice of a list's rows, some rows a round, all loads before the
// stores, needs no other copy, and may ask for the next round's rows before it writes.  Different slices (of different bytes) do not
// meet.  Its first workgroups return the pages.  (The same holds for any number of rounds ahead: a later round's rows come from its own first
// row on.)
//
// What bounds it: 8 layers of 16 requests, 8 cache heads of 128 bfloat16 values, cut from 2048 to 6000 positions to 2048: 371 us for the rows that
// move, 1.77 GB read and written at 4.8 TB/s (a large copy: 4.9), and 34 us for the 1024 lists (tables of counts in LDS; 50 us with ballots, 70
// with eight bits a round and the scores read again).  One request, 1100 to 1000 positions in 4 layers: 11 us and 10, lengths ->
// scores -> limit -> page, then slot -> row.  24 requests of whole slots of 960 bytes, 0 to 2500 to 700: 106 us for 390 MB, 3.7 TB/s: of 768
// workgroups some 550 have anything to move, up to six rounds, and 512 fit the chip at a time; a round's look-ups come after the stores of the
// round before it, and memory operations are counted in order.

#include <algorithm>
#include <type_traits>

#include "mpv_host.h"
#include "mpv_select.h"

namespace mpv {

constexpr int kSelectBlock = 512;          // of the long lists
// Positions that are kept, or in a row of the block table: loops over them take 32 bits, and the last step of one goes beyond them.
constexpr int64_t kMostPositions = INT32_MAX - (1 << 16);
constexpr int kMostReturning = 64;         // workgroups that return pages, at most
constexpr int kMostLooking = 256;          // and that look at them before
constexpr int kLookTogether = 4;           // entries of a thread on their way

struct EvictArgs {
    mpv_eviction p;
    mpv_eviction_buffers b;
    int lists, slices;
    int64_t row_bytes, lead;               // of a moved row; elements from a head's row to the next (a list's: 0 where a list has whole slots)
    Divisor by_page;
    int32_t* slots;                        // [lists][budget] slot of a kept row, -1: none
    int32_t* moved;                        // [lists] first row that moves (budget: none does)
    struct Plan {
        int32_t free;                      // pages that were free
        int32_t strange[kMostLooking];   // whether a part of the tables' entries behind the kept pages holds one that is no page
    } * plan;
    int64_t* first_page;                   // [B+1] where a request's pages go in the list of free ones
    int32_t* lengths;                      // [B] new ones
    int returning, looking;                // workgroups that return pages, and that look at them before
};

__device__ __forceinline__ int context_of(const EvictArgs& a, int b) { return min(max(a.b.context_len[b], 0), a.p.table_width * a.p.page_size); }

// Pages of so many positions.  (Their sum with a page's may be more than 32 bits hold.)
__device__ __forceinline__ int pages_of(const EvictArgs& a, int positions) { return positions > 0 ? a.by_page.of(positions - 1) + 1 : 0; }

// Order of the scores; NaN comes last, both zeros are the same.
__device__ __forceinline__ uint32_t score_order(float z) {
    const uint32_t u = __float_as_uint(z + 0.0f);
    return z != z ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sums of two numbers over the workgroup, the sums of all in total[2].
__device__ __forceinline__ void before(int (&v)[2], int (&total)[2], int (*part)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto[2] = {v[0], v[1]};
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(upto[0], d), y = __shfl_up(upto[1], d);
        if (lane >= d) { upto[0] += x; upto[1] += y; }
    }
    __syncthreads();
    if (lane == 63) { part[wave][0] = upto[0]; part[wave][1] = upto[1]; }
    __syncthreads();
    v[0] = upto[0] - v[0];
    v[1] = upto[1] - v[1];
    total[0] = total[1] = 0;
    for (int w = 0; w < static_cast<int>(blockDim.x >> 6); ++w) {
        if (w < wave) { v[0] += part[w][0]; v[1] += part[w][1]; }
        total[0] += part[w][0];
        total[1] += part[w][1];
    }
}

// What returns the pages behind the kept positions to the end of the list of free ones, in request order: a workgroup of the first launch works
// out where each request's begin, since lengths and count may be written by the second one.
__device__ __forceinline__ void plan_pages(const EvictArgs& a) {
    const mpv_eviction& p = a.p;
    __shared__ int part[16][2];
    int64_t count = min(max(a.b.free_count[0], 0), p.num_pages);
    if (threadIdx.x == 0) a.plan->free = static_cast<int32_t>(count);
    const int have = pages_of(a, p.budget);
    for (int base = 0; base < p.B; base += blockDim.x) {
        const int b = base + threadIdx.x;
        const int context = b < p.B ? context_of(a, b) : 0;
        const int pages = context > p.trigger ? pages_of(a, context) - have : 0;
        int at[2] = {pages, 0}, total[2];
        before(at, total, part);
        if (b < p.B) {
            a.first_page[b] = count + at[0];
            a.lengths[b] = context > p.trigger ? p.budget : context;
        }
        count += total[0];
    }
    if (threadIdx.x == 0) a.first_page[p.B] = count;
}
// Part `number` of `looking` of the tables' entries: whether one that is to be returned is no page.
__device__ __forceinline__ void look_at_pages(const EvictArgs& a, int number) {
    const mpv_eviction& p = a.p;
    const int have = pages_of(a, p.budget), width = max(p.table_width, 1), step = a.looking * static_cast<int>(blockDim.x);
    const int rows = step / width, columns = step - rows * width;
    const int first = number * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x);
    int b = p.table_width > 0 ? first / width : p.B, column = first % width;
    bool strange = false;
    while (b < p.B) {
        int at[kLookTogether], in[kLookTogether], context[kLookTogether], page[kLookTogether];
#pragma unroll
        for (int j = 0; j < kLookTogether; ++j) {
            at[j] = b;
            in[j] = column;
            const bool next = column >= width - columns;
            b += rows + next;
            column += next ? columns - width : columns;
        }
#pragma unroll
        for (int j = 0; j < kLookTogether; ++j) context[j] = at[j] < p.B ? context_of(a, at[j]) : 0;
#pragma unroll
        for (int j = 0; j < kLookTogether; ++j) {
            page[j] = 0;
            if (context[j] > p.trigger && in[j] >= have && in[j] < pages_of(a, context[j]))
                page[j] = a.b.block_table[static_cast<int64_t>(at[j]) * p.table_width + in[j]];
        }
#pragma unroll
        for (int j = 0; j < kLookTogether; ++j) strange = strange || page[j] < 0 || page[j] >= p.num_pages;      // (0 is one, if there are any)
    }
    const bool any = __syncthreads_or(strange);
    if (threadIdx.x == 0) a.plan->strange[number] = any;
}
// The first workgroups of a launch that selects have the pages.
__device__ __forceinline__ bool plan(const EvictArgs& a) {
    if (blockIdx.x > static_cast<unsigned>(a.looking)) return false;
    if (blockIdx.x == 0) plan_pages(a);
    else look_at_pages(a, blockIdx.x - 1);
    return true;
}
// The entry that has a place in the list (pages and what is none together).
__device__ __forceinline__ int page_at(const EvictArgs& a, int64_t place, int have) {
    int low = 0, high = a.p.B;                                     // the last request whose pages begin at or before the place
    while (high - low > 1) {
        const int middle = (low + high) >> 1;
        if (a.first_page[middle] <= place) low = middle;
        else high = middle;
    }
    return a.b.block_table[static_cast<int64_t>(low) * a.p.table_width + have + static_cast<int>(place - a.first_page[low])];
}
__device__ __forceinline__ void return_pages(const EvictArgs& a) {
    const mpv_eviction& p = a.p;
    const int have = pages_of(a, p.budget);
    const int64_t free = a.plan->free, all = a.first_page[p.B];
    const int64_t step = static_cast<int64_t>(a.returning) * blockDim.x;
    const int64_t mine = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    int64_t end = min(all, static_cast<int64_t>(p.num_pages));
    bool strange = false;
#pragma unroll
    for (int i = 0; i < kMostLooking; i += 64) {
        const int part = i + static_cast<int>(threadIdx.x & 63);
        if (part < a.looking) strange = strange || a.plan->strange[part];
    }
    if (!__ballot(strange)) {
        for (int64_t place = free + mine; place < end; place += step) a.b.free_pages[place] = page_at(a, place, have);
    } else if (blockIdx.x == 0) {
        // some are no pages (which nobody should have to hurry with): one workgroup leaves them out
        __shared__ int part[16][2];
        int64_t to = free;
        for (int64_t base = free; base < all; base += blockDim.x) {
            const int64_t place = base + threadIdx.x;
            const int page = place < all ? page_at(a, place, have) : -1;
            const bool real = page >= 0 && page < p.num_pages;
            int at[2] = {real, 0}, total[2];
            before(at, total, part);
            if (real && to + at[0] < p.num_pages) a.b.free_pages[to + at[0]] = page;
            to += total[0];
        }
        end = min(to, static_cast<int64_t>(p.num_pages));
    }
    for (int64_t b = mine; b < p.B; b += step) a.b.context_len_out[b] = a.lengths[b];
    if (mine == 0) a.b.free_count_out[0] = static_cast<int32_t>(end);
}

// A request that is not cut: its scores stay.
__device__ __forceinline__ void leave(const EvictArgs& a, int list, int context) {
    const float* scores = a.b.scores + static_cast<int64_t>(list) * a.p.score_width;
    float* out = a.b.scores_out + static_cast<int64_t>(list) * a.p.score_width;
    int32_t* kept = a.b.kept + static_cast<int64_t>(list) * a.p.budget;
    for (int i = threadIdx.x; i < a.p.budget; i += blockDim.x) kept[i] = -1;
    if (out != scores)
        for (int i = threadIdx.x; i < context; i += blockDim.x) out[i] = scores[i];
    if (threadIdx.x == 0) a.moved[list] = a.p.budget;
}

// A list whose scores a workgroup holds in registers.
template <int BLOCK, int HELD>
__global__ __launch_bounds__(BLOCK) void select_kernel(EvictArgs a) {
    typedef Select<BLOCK, HELD, 0> S;
    __shared__ typename S::Shared sh;
    __shared__ typename std::conditional<BLOCK == 64, int, typename S::Table>::type table;
    (void)table;
    __shared__ int stay;
    const mpv_eviction& p = a.p;
    if (plan(a)) return;
    const int list = blockIdx.x - 1 - a.looking, b = list / p.score_heads % p.B;
    const int context = context_of(a, b);
    if (context <= p.trigger) return leave(a, list, context);
    const float* scores = a.b.scores + static_cast<int64_t>(list) * p.score_width;
    float* out = a.b.scores_out + static_cast<int64_t>(list) * p.score_width;
    const int64_t first = static_cast<int64_t>(list) * p.budget;
    const int rounds = (context + BLOCK - 1) / BLOCK;
    float score[HELD];
    uint32_t key[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int at = i * BLOCK + threadIdx.x;
        score[i] = at < context ? scores[at] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int at = i * BLOCK + threadIdx.x;
        // (what is kept in any case is larger than every score)
        key[i] = at >= context ? 0u : at < p.sinks || at >= context - p.recent ? 0xffffffffu : score_order(score[i]);
    }
    if (threadIdx.x == 0) stay = 0;
    uint32_t limit;
    int above;
    // (all scores are here when it returns: `out` may be `scores`)
    if constexpr (BLOCK == 64) S::largest(key, rounds, p.budget, sh, limit, above);
    else S::largest_by_table(key, rounds, p.budget, table, limit, above);
    int mine = 0;
    S::chosen(key, rounds, context, limit, p.budget - above, sh, [&](int i, int place) {
        const int at = i * BLOCK + threadIdx.x, column = a.by_page.of(at);
        const int page = a.b.block_table[static_cast<int64_t>(b) * p.table_width + column];
        a.b.kept[first + place] = at;
        a.slots[first + place] = page >= 0 && page < p.num_pages ? page * p.page_size + at - column * p.page_size : -1;
        out[place] = score[i];
        mine += at == place;
    });
    if (mine) atomicAdd(&stay, mine);
    __syncthreads();
    if (threadIdx.x == 0) a.moved[list] = stay;
}

// The same for lists of any length, read again for each byte of the limit.
__global__ __launch_bounds__(kSelectBlock) void select_long_kernel(EvictArgs a) {
    const mpv_eviction& p = a.p;
    if (plan(a)) return;
    const int list = blockIdx.x - 1 - a.looking, b = list / p.score_heads % p.B;
    const int context = context_of(a, b);
    const float* scores = a.b.scores + static_cast<int64_t>(list) * p.score_width;
    float* out = a.b.scores_out + static_cast<int64_t>(list) * p.score_width;
    int32_t* kept = a.b.kept + static_cast<int64_t>(list) * p.budget;
    if (context <= p.trigger) return leave(a, list, context);
    __shared__ int counts[256];
    __shared__ int part[kSelectBlock / 64][2];
    __shared__ int chosen_digit, chosen_above;
    const int from = p.sinks, to = context - p.recent, want = p.budget - p.sinks - p.recent;
    // the want-th largest; `above`: those larger than it
    uint32_t limit = 0;
    int above = 0;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        if (threadIdx.x < 256) counts[threadIdx.x] = 0;
        __syncthreads();
        for (int j = from + threadIdx.x; j < to; j += kSelectBlock) {
            const uint32_t k = score_order(scores[j]);
            if (shift == 24 || k >> (shift + 8) == limit >> (shift + 8)) atomicAdd(&counts[k >> shift & 255], 1);
        }
        __syncthreads();
        int mine[2] = {threadIdx.x < 256 ? counts[255 - threadIdx.x] : 0, 0}, total[2];
        const int count = mine[0];
        before(mine, total, part);
        if (above + mine[0] < want && above + mine[0] + count >= want) { chosen_digit = 255 - threadIdx.x; chosen_above = above + mine[0]; }
        __syncthreads();
        limit |= static_cast<uint32_t>(chosen_digit) << shift;
        above = chosen_above;
        __syncthreads();
    }
    // the kept positions in order: of equal ones the first
    const int equal = want - above;
    int larger_before = 0, equal_before = 0;
    for (int i = threadIdx.x; i < p.sinks; i += kSelectBlock) kept[i] = i;
    for (int base = from; base < to && want > 0; base += kSelectBlock) {
        const int j = base + threadIdx.x;
        const uint32_t k = j < to ? score_order(scores[j]) : 0u;
        const bool is_larger = j < to && k > limit, is_equal = j < to && k == limit;
        int at[2] = {is_larger, is_equal}, total[2];
        before(at, total, part);
        const int e = equal_before + at[1];
        if (is_larger || (is_equal && e < equal)) kept[p.sinks + larger_before + at[0] + min(e, equal)] = j;
        larger_before += total[0];
        equal_before += total[1];
    }
    for (int i = threadIdx.x; i < p.recent; i += kSelectBlock) kept[p.budget - p.recent + i] = to + i;
    __threadfence_block();
    __syncthreads();
    // their scores and slots
    __shared__ int stay;
    if (threadIdx.x == 0) stay = 0;
    __syncthreads();
    for (int base = 0; base < p.budget; base += kSelectBlock) {
        const int i = base + threadIdx.x;
        float score = 0.0f;
        if (i < p.budget) {
            const int j = kept[i], column = a.by_page.of(j);
            const int page = a.b.block_table[static_cast<int64_t>(b) * p.table_width + column];
            a.slots[static_cast<int64_t>(list) * p.budget + i] = page >= 0 && page < p.num_pages ? page * p.page_size + j - column * p.page_size : -1;
            score = scores[j];
            if (j == i) atomicAdd(&stay, 1);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (`out` may be `scores`)
        __syncthreads();
        if (i < p.budget) out[i] = score;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.moved[list] = stay;
}

// A slice of a list's rows, LANES 16-byte pieces wide.  A round's rows are asked for before those of the round before it are written, and the
// slots a round earlier still.
template <int BLOCK, int LANES>
__global__ __launch_bounds__(BLOCK) void move_kernel(EvictArgs a) {
    constexpr int kLoads = BLOCK == 1024 ? 4 : 8;                  // rows of a thread in a round (1024 threads have 128 registers each)
    constexpr int kStep = BLOCK / LANES, kRound = kStep * kLoads;
    const mpv_eviction& p = a.p;
    if (blockIdx.x < static_cast<unsigned>(a.returning)) return return_pages(a);
    const int part = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    unsigned number = blockIdx.x - a.returning;
    const bool values = number & 1;
    number >>= 1;
    const int list = number / a.slices, slice = number - static_cast<unsigned>(list) * a.slices;
    const int begin = a.moved[list];
    if (begin >= p.budget) return;
    const int head = list % p.score_heads, b = list / p.score_heads % p.B, layer = list / p.score_heads / p.B;
    const int bytes = p.dtype == MPV_DTYPE_F32 ? 4 : 2;
    const int64_t byte = (static_cast<int64_t>(slice) * LANES + part) * 16;
    char* cache = static_cast<char*>(values ? a.b.cache_v : a.b.cache_k) + (layer * p.cache_layer_stride + head * a.lead) * bytes + byte;
    const bool inside = byte < a.row_bytes;
    const int32_t* slots = a.slots + static_cast<int64_t>(list) * p.budget;
    const int32_t* table = a.b.block_table + static_cast<int64_t>(b) * p.table_width;
    struct Rows { int from[kLoads], page[kLoads]; };
    auto look = [&](int first, Rows& r) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = first + j * kStep + mine;
            r.from[j] = -1;
            r.page[j] = -1;
            if (i < p.budget && inside) {
                r.from[j] = slots[i];
                r.page[j] = table[a.by_page.of(i)];
            }
        }
    };
    auto whole = [&](const Rows& r, int j) { return r.from[j] >= 0 && r.page[j] >= 0 && r.page[j] < p.num_pages; };
    auto ask = [&](const Rows& r, uint4 (&v)[kLoads]) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (whole(r, j)) {
                const int page = a.by_page.of(r.from[j]);
                v[j] = *reinterpret_cast<const uint4*>(cache + (page * p.page_stride + (r.from[j] - page * p.page_size) * p.slot_stride) * bytes);
            }
    };
    auto store = [&](int first, const Rows& r, const uint4 (&v)[kLoads]) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (whole(r, j)) {
                const int i = first + j * kStep + mine, place = i - a.by_page.of(i) * p.page_size;
                *reinterpret_cast<uint4*>(cache + (r.page[j] * p.page_stride + place * p.slot_stride) * bytes) = v[j];
            }
    };
    // all threads' rows of a round are here
    auto arrive = [&](uint4 (&v)[kLoads]) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
        __syncthreads();
    };
    Rows r[2];
    uint4 v[2][kLoads] = {};
    look(begin, r[0]);
    ask(r[0], v[0]);
    look(begin + kRound, r[1]);
    for (int first = begin;; first += 2 * kRound) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = first + h * kRound;
            if (at >= p.budget) return;
            arrive(v[h]);
            ask(r[1 - h], v[1 - h]);
            store(at, r[h], v[h]);
            look(at + 2 * kRound, r[h]);
        }
    }
}

// ------------------------------------------------------------------ host side

// Bytes of a row that moves as one.
static int64_t row_bytes(const mpv_eviction* p) {
    return static_cast<int64_t>(p->score_heads == 1 ? p->kv_heads : 1) * p->head_dim * elem_bytes(p->dtype);
}
static int64_t slices_of(int64_t bytes, int lanes) { return (bytes + lanes * 16 - 1) / (lanes * 16); }
// Workgroups that move rows.
static int64_t movers_of(int64_t lists, int64_t bytes, int lanes) { return lists * slices_of(bytes, lanes) * 2; }
// 16-byte pieces of a slice: as wide as a row, up to 1024 bytes (592 requests' lists of 14 positions of 384 bytes: 54 us, 109 with 128 bytes), but
// not wider than a cache line where that makes 512 workgroups or saves many rounds (16 requests to 2048 positions: 401 us, 419 with 256 bytes;
// 32 to 2048 slots of 2048 bytes: 603, 617 with 256 and 686 with 1024; 20 to 533 positions of 512 bytes, four rounds: 180, and 173 as one
// slice).  Half a line where there are few workgroups: 96 of them 86 us, twice as
// many 74; 256 and 512, 68 and 85; 128 and 256, 20 and 23.
static int lanes_of(int64_t lists, int64_t bytes, int64_t budget) {
    int lanes = 64;
    auto workgroups = [&] { return movers_of(lists, bytes, lanes); };
    auto many_rounds = [&] { return budget > 6 * 4 * (1024 / lanes) && workgroups() < 8192; };
    while (lanes > 8 && (lanes * 8 >= bytes || workgroups() < 512 || many_rounds())) lanes /= 2;
    if (lanes == 8 && (lanes * 8 >= bytes || workgroups() < 128)) lanes = 4;
    return lanes;
}

// Many rounds of 256 threads (or few lists): 1024 threads, more rows a round, unless that is more threads than a launch can have.  (16 requests to 2048
// positions: 433 us with 1024 threads, 491 with 256, which take 16 rounds; 42 requests to 12 108 slots of 1024 bytes: 232, 407; 41 requests
// to 48: 60, 44.)
static bool large_workgroups(int64_t lists, int64_t bytes, int lanes, int64_t budget) {
    const int64_t workgroups = movers_of(lists, bytes, lanes), round = 256 / lanes * 8;
    return (budget > 4 * round || (workgroups < 512 && budget > round)) && workgroups + kMostReturning <= kMostWorkgroups / 4;
}

static int check_eviction(const mpv_eviction* p) {
    if (!p) return MPV_ERR_NULL;
    if (p->layers < 0 || p->B < 0 || p->kv_heads < 1 || p->head_dim < 1 || (p->score_heads != 1 && p->score_heads != p->kv_heads) || p->num_pages < 0 ||
        p->page_size < 1 || p->table_width < 0 || p->budget < 1 || p->trigger < p->budget || p->sinks < 0 || p->recent < 0 ||
        static_cast<int64_t>(p->sinks) + p->recent > p->budget || p->score_width < span(0, p->table_width, p->page_size))
        return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(p->dtype)) return MPV_ERR_BAD_DTYPE;
    if (p->head_dim > MPV_MAX_HEAD_DIM || p->kv_heads > MPV_MAX_HEADS) return MPV_ERR_UNSUPPORTED;
    const int64_t row = static_cast<int64_t>(p->kv_heads) * p->head_dim;
    if (p->slot_stride < row || p->page_stride < 0 || p->cache_layer_stride < 0) return MPV_ERR_BAD_SHAPE;
    const int64_t lists = span(0, span(0, p->layers, p->B), p->score_heads);
    if (span(0, p->num_pages, p->page_size) > INT32_MAX || span(0, p->table_width, p->page_size) > kMostPositions || p->budget > kMostPositions ||
        p->score_width > INT32_MAX ||
        lists > INT32_MAX / 1024 || p->B > (1 << 24) || span(0, lists, p->budget) > (static_cast<int64_t>(1) << 40) ||
        movers_of(lists, row_bytes(p), lanes_of(lists, row_bytes(p), p->budget)) > kMostWorkgroups - kMostReturning ||
        span(0, span(span(span(0, p->num_pages, p->page_stride), p->page_size, p->slot_stride), p->layers, p->cache_layer_stride), 4) == INT64_MAX)
        return MPV_ERR_UNSUPPORTED;
    const int64_t all = p->head_dim | p->slot_stride | p->page_stride | p->cache_layer_stride;
    if ((all * elem_bytes(p->dtype)) % 16 != 0) return MPV_ERR_ALIGNMENT;
    return MPV_OK;
}

static void launch_select(EvictArgs& a, hipStream_t s) {
    const int64_t room = static_cast<int64_t>(a.p.table_width) * a.p.page_size, entries = static_cast<int64_t>(a.p.B) * a.p.table_width;
    auto go = [&](auto kernel, int threads) {
        a.looking = static_cast<int>(std::min<int64_t>(kMostLooking, 1 + entries / (threads * kLookTogether)));
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(a.lists) + 1 + a.looking), dim3(threads), 0, s, a);
    };
    if (room <= 64 * 16) go(select_kernel<64, 16>, 64);
    else if (room <= 512 * 16) go(select_kernel<512, 16>, 512);
    else if (room <= 1024 * 32) go(select_kernel<1024, 32>, 1024);
    else go(select_long_kernel, kSelectBlock);
}

template <int LANES>
static void launch_slices(EvictArgs& a, hipStream_t s) {
    a.slices = static_cast<int>(slices_of(a.row_bytes, LANES));
    const dim3 grid(static_cast<unsigned>(movers_of(a.lists, a.row_bytes, LANES) + a.returning));
    if (large_workgroups(a.lists, a.row_bytes, LANES, a.p.budget)) hipLaunchKernelGGL((move_kernel<1024, LANES>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((move_kernel<256, LANES>), grid, dim3(256), 0, s, a);
}
static void launch_move(EvictArgs& a, hipStream_t s) {
    const int lanes = lanes_of(a.lists, a.row_bytes, a.p.budget);
    if (lanes == 64) launch_slices<64>(a, s);
    else if (lanes == 32) launch_slices<32>(a, s);
    else if (lanes == 16) launch_slices<16>(a, s);
    else if (lanes == 8) launch_slices<8>(a, s);
    else launch_slices<4>(a, s);
}

// Parts of a workspace.
struct EvictRoom {
    size_t slots, moved, plan, pages, lengths;
    size_t bytes() const { return slots + moved + plan + pages + lengths; }
};
static EvictRoom room_of(const mpv_eviction* p) {
    auto whole = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    const size_t lists = static_cast<size_t>(p->layers) * p->B * p->score_heads;
    return {whole(lists * p->budget * sizeof(int32_t)), whole(lists * sizeof(int32_t)), whole(sizeof(EvictArgs::Plan)), whole((static_cast<size_t>(p->B) + 1) * sizeof(int64_t)),
            whole(static_cast<size_t>(p->B) * sizeof(int32_t))};
}

}  // namespace mpv

extern "C" {

int mpv_evict_positions_workspace_bytes(const mpv_eviction* eviction, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_eviction(eviction);
    if (rc != MPV_OK) return rc;
    *out = mpv::room_of(eviction).bytes();
    return MPV_OK;
}

int mpv_evict_positions(const mpv_eviction* eviction, const mpv_eviction_buffers* buf, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
    size_t need;
    const int rc = mpv_evict_positions_workspace_bytes(eviction, &need);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    const mpv_eviction* p = eviction;
    if (p->B == 0) return MPV_OK;
    const bool any = p->layers > 0;
    if (!buf->context_len || !buf->context_len_out || !buf->free_count || !buf->free_count_out || (p->num_pages > 0 && !buf->free_pages) ||
        (p->table_width > 0 && !buf->block_table) ||
        (any && (!buf->kept || (p->score_width > 0 && (!buf->scores || !buf->scores_out)) || (p->num_pages > 0 && (!buf->cache_k || !buf->cache_v)))))
        return MPV_ERR_NULL;
    if (!mpv::aligned(buf->cache_k, 16) || !mpv::aligned(buf->cache_v, 16)) return MPV_ERR_ALIGNMENT;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < need) return MPV_ERR_WORKSPACE;
    mpv::EvictArgs a;
    a.p = *p;
    a.b = *buf;
    a.lists = p->layers * p->B * p->score_heads;
    a.row_bytes = mpv::row_bytes(p);
    a.lead = p->score_heads == 1 ? 0 : p->head_dim;
    a.by_page.set(static_cast<uint32_t>(p->page_size));
    const mpv::EvictRoom room = mpv::room_of(p);
    char* at = static_cast<char*>(workspace);
    a.slots = reinterpret_cast<int32_t*>(at);
    a.moved = reinterpret_cast<int32_t*>(at += room.slots);
    a.plan = reinterpret_cast<mpv::EvictArgs::Plan*>(at += room.moved);
    a.first_page = reinterpret_cast<int64_t*>(at += room.plan);
    a.lengths = reinterpret_cast<int32_t*>(at += room.pages);
    // (eight pages a thread, if every request had all that it has room for)
    a.returning = static_cast<int>(std::min<int64_t>(mpv::kMostReturning, 1 + static_cast<int64_t>(p->B) * p->table_width / 2048));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    mpv::launch_select(a, s);
    mpv::launch_move(a, s);
    return mpv::launched();
}

}  // extern "C"
