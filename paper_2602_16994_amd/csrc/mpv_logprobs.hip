// Log probabilities of given tokens, entropy and the most likely tokens of logit rows: device and host code.

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "mpv_host.h"
#include "mpv_select.h"

namespace mpv {

// With c = log2(e) / T, m = max z, d = c (z - m), S = sum 2^d, A = sum 2^d d:
//   log2 p_t = d_t - log2 S,    entropy = log2 S - A / S  (log2 units)
// Every sum's reference is m itself, never the rounded product c m: that is off by 2^-24 |c m|, 12.7 nats for a logit of 1e9.  (So the
// difference comes before the factor; where a round's exponents are c z - fl(c m), the round's sums are brought to m, see sweep_kernel.)
// S and A of parts are put together by powers of 2, as the statistics of a softmax are.  The best tokens are found through the maxima
// of segments of 64 tokens: the `top` best lie in the `top` segments with the largest maxima (of equal ones the first), so the row is
// read once, and those segments again.
//
// sweep_kernel: a workgroup has a part of a row; finish_kernel: one has a row, its parts and its segments' maxima.
//
// What bounds it: 900 rows of 151 936 bfloat16 logits (the emitted tokens of 256 trees) take 68 us for 272 MB, 4.0 TB/s, with vector
// instructions 0.71 of the time (13 a logit: unpacking, maximum, comparison, exponential, two sums), and 16 in the second launch, loads that depend on each other: row, maxima, segments, their logits.  1024 rows of 128 257 float32 logits: 101 us for 525 MB, 5.2 TB/s,
// memory, and 16.  One request's four rows of 32 000: 13 us, two launches.

constexpr int kSweepBlock = 256;
constexpr int kSegment = 64;
constexpr int kListed = 256;               // segments that are looked at, at most
constexpr int kMany = 1024;                // tokens of them that there is room for (where equal logits make more, at most `top` whole segments)
constexpr int kOrdered = 160;              // tokens that are put in order by comparing each with each
constexpr int kChunks = 4;                 // 16-byte loads of a thread in flight

// Tokens that there has to be room for: `top` whole segments, where they are more.
__host__ __device__ constexpr int room_of_candidates(int top) { return top * kSegment > kMany ? top * kSegment : kMany; }

// c (z - m).  (Halves: the difference of two numbers of opposite sign may be larger than any.)
__device__ __forceinline__ float apart_of(float z, float m, float c2) { return (0.5f * z - 0.5f * m) * c2; }

struct PartSums { float m, sum, weighted; int32_t better; };

// S and A from the reference `from` to the larger `to`.  (What fades to nothing may be infinitely far away: 0 times the lowest number is 0.)
__device__ __forceinline__ void bring(float from, float to, float c2, float& sum, float& weighted) {
    const float apart = apart_of(from, to, c2), fade = exp2f(apart);
    sum *= fade;
    weighted = fmaf(sum, fmaxf(apart, -FLT_MAX), fade * weighted);
}

struct RowArgs {
    mpv_logprobs p;
    mpv_logprob_buffers b;
    int rows, width, parts, part;          // output rows in all and of a tree; parts of a row, segments of each
    int segments;
    float c2, twice;                       // 2 log2(e) / T, 2 / T
    PartSums* sums;                        // [rows][parts]
    float* best;                           // [rows][segments] (top > 0)
};

__device__ __forceinline__ float logit(float z) { return z; }
__device__ __forceinline__ float logit(uint16_t z) { return __uint_as_float(static_cast<uint32_t>(z) << 16); }
__device__ __forceinline__ float logit(__half z) { return __half2float(z); }

// Numbers in the order of the logits, -inf at 0x007fffff; both zeros are the same.
__device__ __forceinline__ uint32_t order_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
constexpr uint32_t kNothing = 0x007fffffu;
// The next smaller float32; none is below -inf: NaN, which no number is less than or equal to.
__device__ __forceinline__ float next_below(float z) {
    if (z == -INFINITY || z != z) return NAN;
    if (z == 0.0f) return __uint_as_float(0x80000001u);
    return __uint_as_float(z > 0.0f ? __float_as_uint(z) - 1 : __float_as_uint(z) + 1);
}

// Maximum, NaN if one is.
__device__ __forceinline__ float maximum(float x, float y, float z) {
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
}

// Maximum over the lanes of a segment, 8 or 16 neighbours.
template <int LANES>
__device__ __forceinline__ float segment_max(float v) {
    auto with = [&](auto control) {
        constexpr int kControl = decltype(control)::value;
        return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kControl, 0xf, 0xf, true)));
    };
    v = with(std::integral_constant<int, 0xb1>());                 // neighbours
    v = with(std::integral_constant<int, 0x4e>());                 // pairs
    v = with(std::integral_constant<int, 0x141>());                // fours, mirrored
    if (LANES == 16) v = with(std::integral_constant<int, 0x140>());
    return v;
}

// An output row: where its logits are and its token; node < 0: there is none.
struct Row { int64_t at; int token; bool real; };
__device__ __forceinline__ Row row_of(const RowArgs& a, int row) {
    const int b = row / a.width, i = row - b * a.width;
    Row r{0, -1, false};
    int node = i;
    if (a.p.paths) {
        const int length = min(max(a.b.accept_len[b], 0), a.p.max_depth);
        if (i > length) return r;
        node = i == 0 ? 0 : a.b.path_nodes[static_cast<int64_t>(b) * a.p.max_depth + i - 1];
        r.token = i == length ? a.b.bonus_token[b] : a.b.tokens[static_cast<int64_t>(b) * a.p.max_depth + i];
    } else {
        if (a.b.num_nodes && i >= a.b.num_nodes[b]) return r;
        r.token = a.b.tokens[row];
    }
    if (node < 0 || node >= a.p.N) return r;
    r.real = true;
    r.at = (static_cast<int64_t>(b) * a.p.N + node) * a.p.stride;
    return r;
}

template <class T>
__global__ __launch_bounds__(kSweepBlock) void sweep_kernel(RowArgs a) {
    constexpr int N = 16 / sizeof(T), kLanes = kSegment / N;
    const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
    const Row r = row_of(a, row);
    if (!r.real) return;
    const T* z = static_cast<const T*>(a.b.logits) + r.at;
    const int V = a.p.V, whole = V / N;
    const bool known = r.token >= 0 && r.token < V;
    const float c = 0.5f * a.c2;
    const float mine = known ? logit(z[r.token]) : INFINITY;
    const int from = part * a.part * kLanes, to = min(from + a.part * kLanes, a.segments * kLanes);      // chunks of N
    float m = -INFINITY, sum = 0.0f, weighted = 0.0f;
    int better = 0, equals = 0;            // of the wave, and of this lane
    const float below = next_below(mine);
    const int full = min(to, whole);
    // where this lane writes a maximum: that of its segment in the round's chunk `lane % kLanes`, if there are so many
    constexpr int kPerRound = kSweepBlock / kLanes;
    const int chunk_of = threadIdx.x % kLanes;
    float* mine_best = a.best + static_cast<int64_t>(row) * a.segments + chunk_of * kPerRound + threadIdx.x / kLanes;
    const int token_chunk = known ? r.token / N : INT_MAX;
    // a round of chunks; kWhole: all of them are there; kPlain: the given token's is none of them
    auto round = [&](int first, auto all, auto elsewhere) {
        constexpr bool kWhole = decltype(all)::value, kPlain = decltype(elsewhere)::value;
        T raw[kChunks][N];
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int chunk = first + j * kSweepBlock + threadIdx.x;
            if (kWhole || chunk < full) __builtin_memcpy(raw[j], z + static_cast<int64_t>(chunk) * N, 16);
        }
        float v[kChunks][N], now = m, best = -INFINITY;
#pragma unroll
        for (int j = 0; j < kChunks; ++j) {
            const int chunk = first + j * kSweepBlock + threadIdx.x;
            if (kWhole || chunk < full) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[j][i] = logit(raw[j][i]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int at = chunk * N + i;
                    v[j][i] = chunk < to && at < V ? logit(z[at]) : -INFINITY;
                }
            }
            float most = maximum(v[j][0], v[j][1], v[j][2]);
#pragma unroll
            for (int i = 3; i < N; i += 2) most = maximum(most, v[j][i], v[j][i + 1 < N ? i + 1 : i]);
            now = maximum(now, most, most);
            if (a.p.top > 0) {
                const float segment = segment_max<kLanes>(most);
                best = chunk_of == j ? segment : best;
            }
            // tokens before the given one are better if they are not smaller: if they are larger than the number below it
            if constexpr (kPlain) {
                const float least = token_chunk != INT_MAX && token_chunk > first ? below : mine;
#pragma unroll
                for (int i = 0; i < N; ++i) better += __popcll(__ballot(!(v[j][i] <= least)));
            } else {
                const bool there = kWhole || chunk < to;           // (what lies behind the part is not counted)
                const float least = token_chunk != INT_MAX && chunk < token_chunk && there ? below : mine;
#pragma unroll
                for (int i = 0; i < N; ++i) better += __popcll(__ballot(!(v[j][i] <= least)));
                if (chunk == token_chunk && there)
                    for (int i = 0; i < N; ++i) equals += chunk * N + i < r.token && v[j][i] == mine;
            }
            asm volatile("" : "+s"(better));                       // (counted here: the ballots would all wait in scalar registers)
        }
        if (a.p.top > 0 && chunk_of < kChunks && (kWhole || first + chunk_of * kSweepBlock + static_cast<int>(threadIdx.x) < to)) mine_best[first / kLanes] = best;
        const float base = now == -INFINITY ? 0.0f : now, shift = base * c;
        if (m != -INFINITY) bring(m, now, a.c2, sum, weighted);
        m = now;
        if (fabsf(shift) < 65536.0f && c > 1e-30f) {
            // (exponents c z - shift are one fma each.  Their reference is `shift`, which is c m rounded, while sums are put together by m
            // itself: `rest` = c m - shift, exact as an fma, at most 2^-9 here, brings a round's sums from one to the other.
            // What lies further than 200 log2 units below adds nothing, and 0 times -inf would be NaN.)
            const float lowest = base - 200.0f * (1.0f / c), rest = fmaf(base, c, -shift);
            float in_log2 = 0.0f, now_sum = 0.0f;
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float d = fmaf(__builtin_amdgcn_fmed3f(v[j][i], lowest, INFINITY), c, -shift), e = __builtin_amdgcn_exp2f(d);
                    now_sum += e;
                    in_log2 = fmaf(e, d, in_log2);
                }
            const float back = __builtin_amdgcn_exp2f(-rest);
            sum = fmaf(back, now_sum, sum);
            weighted = fmaf(back, fmaf(-rest, now_sum, in_log2), weighted);
        } else {
            // (far from zero, where c m is off by too much, the difference comes first; so for masks of the lowest number alone, c times
            // which is -inf, and for what is no number)
#pragma unroll
            for (int j = 0; j < kChunks; ++j)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float d = apart_of(v[j][i], base, a.c2), e = __builtin_amdgcn_exp2f(d);
                    sum += e;
                    weighted = fmaf(e, fmaxf(d, -FLT_MAX), weighted);
                }
        }
    };
    int first = from;
    for (; first + kChunks * kSweepBlock <= full; first += kChunks * kSweepBlock) {
        if (token_chunk < first || token_chunk >= first + kChunks * kSweepBlock) round(first, std::true_type(), std::true_type());
        else round(first, std::true_type(), std::false_type());
    }
    for (; first < to; first += kChunks * kSweepBlock) round(first, std::false_type(), std::false_type());
    // over the workgroup
    __shared__ float ms[kSweepBlock / 64], sums[kSweepBlock / 64], weights[kSweepBlock / 64];
    __shared__ int betters[kSweepBlock / 64];
    float top = m;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));       // (a lane without a number has no sum, either)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (m != -INFINITY) bring(m, top, a.c2, sum, weighted);
    for (int d = 32; d; d >>= 1) {
        sum += __shfl_xor(sum, d);
        weighted += __shfl_xor(weighted, d);
        equals += __shfl_xor(equals, d);
    }
    better += equals;
    if (lane == 0) { ms[wave] = top; sums[wave] = sum; weights[wave] = weighted; betters[wave] = better; }
    __syncthreads();
    if (threadIdx.x == 0) {
        PartSums s{ms[0], 0.0f, 0.0f, 0};
        for (int w = 1; w < kSweepBlock / 64; ++w) s.m = fmaxf(s.m, ms[w]);
        for (int w = 0; w < kSweepBlock / 64; ++w) {
            if (ms[w] != -INFINITY) bring(ms[w], s.m, a.c2, sums[w], weights[w]);
            s.sum += sums[w];
            s.weighted += weights[w];
            s.better += betters[w];
        }
        a.sums[static_cast<int64_t>(row) * a.parts + part] = s;
    }
}

// Lowest bits in which no two numbers of a type's order differ.
template <class T> struct Unused { static constexpr int kBits = 0; };
template <> struct Unused<uint16_t> { static constexpr int kBits = 16; };
template <> struct Unused<__half> { static constexpr int kBits = 12; };

// HELD: segments of a thread.
template <class T, int kFinishBlock, int HELD>
__global__ __launch_bounds__(kFinishBlock) void finish_kernel(RowArgs a) {
    constexpr int N = 16 / sizeof(T), LOW = Unused<T>::kBits;
    typedef Select<kFinishBlock, HELD, LOW> S;
    typedef Select<kFinishBlock, 1, LOW> Single;
    const int row = blockIdx.x, top = a.p.top;
    const Row r = row_of(a, row);
    int32_t* tokens = top > 0 ? a.b.top_tokens + static_cast<int64_t>(row) * top : nullptr;
    float* logprobs = top > 0 ? a.b.top_logprobs + static_cast<int64_t>(row) * top : nullptr;
    if (!r.real) {
        if (threadIdx.x == 0) {
            a.b.logprob[row] = 0.0f;
            a.b.entropy[row] = 0.0f;
            a.b.rank[row] = -1;
        }
        for (int i = threadIdx.x; i < top; i += kFinishBlock) { tokens[i] = -1; logprobs[i] = -INFINITY; }
        return;
    }
    const T* z = static_cast<const T*>(a.b.logits) + r.at;
    const bool known = r.token >= 0 && r.token < a.p.V;
    // (what does not depend on anything is asked for at once)
    const float* best = a.best + static_cast<int64_t>(row) * a.segments;
    float segment[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int s = i * kFinishBlock + threadIdx.x;
        segment[i] = top > 0 && s < a.segments ? best[s] : -INFINITY;
    }
    const float mine = known ? logit(z[r.token]) : 0.0f;
    // (the turn to natural logarithms before the product: the lowest number's log probability at T = 1 is the lowest number)
    constexpr float kLn2 = 0.69314718055994531f;
    auto logprob_of = [&](float z, float m, float log) { return fmaf(log, -kLn2, apart_of(z, m, a.twice)); };
    __shared__ float shared_m, shared_log, shared_sum;
    if (threadIdx.x < 64) {
        // (all lanes have parts: their number is not limited by the wave)
        const PartSums* s = a.sums + static_cast<int64_t>(row) * a.parts;
        float m = -INFINITY, sum = 0.0f, weighted = 0.0f;
        int better = 0;
        for (int p = threadIdx.x; p < a.parts; p += 64) m = fmaxf(m, s[p].m);
        for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        for (int p = threadIdx.x; p < a.parts; p += 64) {
            PartSums x = s[p];
            if (x.m != -INFINITY) bring(x.m, m, a.c2, x.sum, x.weighted);
            sum += x.sum;
            weighted += x.weighted;
            better += x.better;
        }
        for (int d = 32; d; d >>= 1) {
            sum += __shfl_xor(sum, d);
            weighted += __shfl_xor(weighted, d);
            better += __shfl_xor(better, d);
        }
        if (threadIdx.x == 0) {
            const float log = log2f(sum);
            const bool number = sum == sum;
            float logprob = -INFINITY, entropy = (log - weighted / sum) * kLn2;
            if (!number) logprob = entropy = NAN;
            else if (sum == 0.0f) entropy = 0.0f;
            else if (known) logprob = logprob_of(mine, m, log);
            a.b.logprob[row] = logprob;
            a.b.entropy[row] = entropy;
            a.b.rank[row] = known && number ? better + 1 : -1;
            shared_m = m;
            shared_log = log;
            shared_sum = sum;
        }
    }
    if (top == 0) return;
    __syncthreads();
    const float m = shared_m, log = shared_log;
    if (!(shared_sum > 0.0f)) {                                    // no tokens, or no numbers
        const float v = shared_sum == 0.0f ? -INFINITY : NAN;
        for (int i = threadIdx.x; i < top; i += kFinishBlock) { tokens[i] = -1; logprobs[i] = v; }
        return;
    }
    // No token of the best is smaller than the top-th largest of the threads' largest maxima: the segments that reach it are few, and hold
    // them all.  (Where they are many, because of equal logits, the `top` segments with the largest maxima, of equal ones the first, are
    // looked for among all: the second launch took 36 us for 900 rows of 151 936 tokens, 22 without.)
    const int rounds = (a.segments + kFinishBlock - 1) / kFinishBlock;
    __shared__ typename S::Shared sh;
    __shared__ typename Single::Shared single;
    __shared__ int segments[kListed];
    __shared__ int found, take;
    extern __shared__ unsigned long long candidates[];             // [room_of_candidates]
    const int room = room_of_candidates(top);
    uint32_t key[HELD], most[1] = {0};
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const uint32_t k = order_of(segment[i]);
        key[i] = k > kNothing ? k : 0u;                            // (tokens of no probability are no alternatives)
        most[0] = max(most[0], key[i]);
    }
    if (threadIdx.x == 0) found = take = 0;
    uint32_t limit;
    int above;
    Single::largest(most, 1, top, single, limit, above);
    if (most[0] >> LOW >= limit >> LOW)
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (key[i] != 0 && key[i] >> LOW >= limit >> LOW) {
                const int at = atomicAdd(&take, 1);
                if (at < kListed) segments[at] = i * kFinishBlock + threadIdx.x;
            }
    __syncthreads();
    // their tokens that are not smaller, in any order
    auto collect = [&](int segments_of) {
        constexpr int kLanes = kSegment / N;
        for (int i = threadIdx.x; i < segments_of * kLanes; i += kFinishBlock) {
            const int token = segments[i / kLanes] * kSegment + i % kLanes * N;
            T raw[N];
            if (token + N <= a.p.V) {
                __builtin_memcpy(raw, z + token, 16);
            } else {
                for (int j = 0; j < N; ++j)
                    if (token + j < a.p.V) raw[j] = z[token + j];
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const uint32_t k = order_of(logit(raw[j]));
                if (token + j < a.p.V && k > kNothing && k >> LOW >= limit >> LOW) {
                    const int at = atomicAdd(&found, 1);
                    if (at < room) candidates[at] = static_cast<unsigned long long>(k) << 32 | static_cast<uint32_t>(~(token + j));
                }
            }
        }
        __syncthreads();
    };
    bool many = take > kListed;
    if (!many) {
        collect(take);
        many = found > room;
    }
    if (many) {
        __syncthreads();
        if (threadIdx.x == 0) found = 0;
        S::largest(key, rounds, top, sh, limit, above);
        S::chosen(key, rounds, limit >> LOW ? a.segments : 0, limit, top - above, sh,
                  [&](int i, int place) { segments[place] = i * kFinishBlock + threadIdx.x; });
        __syncthreads();
        collect(min(take, top));                                   // (fewer, if fewer have a token at all: they are all among the first)
    }
    int count = found;
    if (count > kOrdered) {
        // (few tokens or equal logits) the best of them by their logits, of equal ones by their place (6586 rows of 1969 tokens, 64 of each: 166 us,
        // 2849 where all are compared with each other)
        typedef Select<kFinishBlock, MPV_MAX_TOP * kSegment / kFinishBlock, 0> Refine;
        __shared__ typename Refine::Shared refine;
        constexpr int kOf = MPV_MAX_TOP * kSegment / kFinishBlock;
        uint32_t high[kOf], low[kOf], same[kOf];
#pragma unroll
        for (int i = 0; i < kOf; ++i) {
            const int at = i * kFinishBlock + threadIdx.x;
            const unsigned long long k = at < count ? candidates[at] : 0ull;
            high[i] = static_cast<uint32_t>(k >> 32);
            low[i] = static_cast<uint32_t>(k);
        }
        const int rounds_of = (count + kFinishBlock - 1) / kFinishBlock;
        int larger, first = 0;
        uint32_t least, last = 0;
        Refine::largest(high, rounds_of, top, refine, least, larger);
#pragma unroll
        for (int i = 0; i < kOf; ++i) same[i] = high[i] == least ? low[i] : 0u;
        if (larger < top) Refine::largest(same, rounds_of, top - larger, refine, last, first);
        if (threadIdx.x == 0) found = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kOf; ++i)
            if (high[i] > least || (larger < top && same[i] != 0 && (same[i] > last || (same[i] == last && first < top - larger))))
                candidates[atomicAdd(&found, 1)] = static_cast<unsigned long long>(high[i]) << 32 | low[i];
        __syncthreads();
        count = found;
    }
    for (int i = threadIdx.x; i < count; i += kFinishBlock) {
        const unsigned long long k = candidates[i];
        int place = 0;
        for (int j = 0; j < count; ++j) place += candidates[j] > k;
        if (place < top) {
            tokens[place] = static_cast<int>(~static_cast<uint32_t>(k));
            logprobs[place] = logprob_of(from_order(static_cast<uint32_t>(k >> 32)), m, log);
        }
    }
    for (int i = count + threadIdx.x; i < top; i += kFinishBlock) { tokens[i] = -1; logprobs[i] = -INFINITY; }
}

// ------------------------------------------------------------------ host side

// Segments of a part, whole rounds of a workgroup: one where the card is not full otherwise, up to four (the emitted tokens of 256 trees, 151 936
// tokens in bfloat16: 106 us with four, 108 with two, 110 with one, 114 with eight, the second launch as it was then included).
static void parts_of(const mpv_logprobs* p, int64_t rows, int* parts, int* part) {
    const int64_t segments = (p->V + kSegment - 1) / kSegment;
    const int64_t round = kChunks * kSweepBlock * (16 / elem_bytes(p->dtype)) / kSegment;         // segments of a round
    const int64_t all = (segments + round - 1) / round;
    const int64_t rounds = std::max<int64_t>(1, std::min<int64_t>(4, rows * all / 2048));
    *part = static_cast<int>(std::min(rounds * round, segments));
    *parts = static_cast<int>((segments + *part - 1) / *part);
}

static int check_logprobs(const mpv_logprobs* p) {
    if (!p) return MPV_ERR_NULL;
    if (p->B < 0 || p->N < 1 || p->V < 1 || p->top < 0 || p->stride < p->V || (p->paths != 0 && p->paths != 1) || (p->paths && p->max_depth < 1))
        return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(p->dtype)) return MPV_ERR_BAD_DTYPE;
    // (of smaller ones the factors log2(e) / T and 1 / T are infinite in float32)
    if (!std::isfinite(p->temperature) || !(p->temperature >= FLT_MIN)) return MPV_ERR_BAD_TEMPERATURE;
    if (p->V > MPV_MAX_VOCAB || p->top > MPV_MAX_TOP) return MPV_ERR_UNSUPPORTED;
    const int64_t width = p->paths ? static_cast<int64_t>(p->max_depth) + 1 : p->N, rows = width * p->B;
    int parts = 1, part;
    if (rows > 0 && rows <= kMostWorkgroups) parts_of(p, rows, &parts, &part);
    // (a row's second workgroup may have 1024 threads)
    if (rows > kMostWorkgroups / 4 || rows * parts > kMostWorkgroups || span(0, static_cast<int64_t>(p->B) * p->N, p->stride) > INT64_MAX / 8) return MPV_ERR_UNSUPPORTED;
    return MPV_OK;
}

struct LogprobRoom { size_t sums, best; };
static LogprobRoom room_of(const mpv_logprobs* p, RowArgs* a) {
    const int64_t width = p->paths ? static_cast<int64_t>(p->max_depth) + 1 : p->N, rows = width * p->B;
    a->rows = static_cast<int>(rows);
    a->width = static_cast<int>(width);
    a->segments = (p->V + kSegment - 1) / kSegment;
    parts_of(p, std::max<int64_t>(rows, 1), &a->parts, &a->part);
    const size_t sums = (static_cast<size_t>(rows) * a->parts * sizeof(PartSums) + 255) / 256 * 256;
    return {sums, p->top > 0 ? static_cast<size_t>(rows) * a->segments * sizeof(float) : 0};
}

template <class T>
static int launch_rows(const RowArgs& a, hipStream_t s) {
    (void)hipGetLastError();
    hipLaunchKernelGGL(sweep_kernel<T>, dim3(static_cast<unsigned>(a.rows) * a.parts), dim3(kSweepBlock), 0, s, a);
    const dim3 rows(static_cast<unsigned>(a.rows));
    const unsigned lds = a.p.top > 0 ? room_of_candidates(a.p.top) * sizeof(unsigned long long) : 0;
    if (a.segments <= 256 * 16) hipLaunchKernelGGL((finish_kernel<T, 256, 16>), rows, dim3(256), lds, s, a);
    else hipLaunchKernelGGL((finish_kernel<T, 1024, 32>), rows, dim3(1024), lds, s, a);
    return launched();
}

}  // namespace mpv

extern "C" {

int mpv_token_logprobs_workspace_bytes(const mpv_logprobs* logprobs, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_logprobs(logprobs);
    if (rc != MPV_OK) return rc;
    mpv::RowArgs a;
    const mpv::LogprobRoom room = mpv::room_of(logprobs, &a);
    *out = room.sums + room.best;
    return MPV_OK;
}

int mpv_token_logprobs(const mpv_logprobs* logprobs, const mpv_logprob_buffers* buf, void* workspace, size_t workspace_bytes,
                       void* hip_stream) {
    const int rc = mpv::check_logprobs(logprobs);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    if (logprobs->B == 0) return MPV_OK;
    if (!buf->logits || !buf->tokens || !buf->logprob || !buf->rank || !buf->entropy ||
        (logprobs->paths && (!buf->accept_len || !buf->path_nodes || !buf->bonus_token)) ||
        (logprobs->top > 0 && (!buf->top_tokens || !buf->top_logprobs)))
        return MPV_ERR_NULL;
    if (!mpv::aligned(buf->logits, mpv::elem_bytes(logprobs->dtype))) return MPV_ERR_ALIGNMENT;
    mpv::RowArgs a;
    a.p = *logprobs;
    a.b = *buf;
    const mpv::LogprobRoom room = mpv::room_of(logprobs, &a);
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < room.sums + room.best) return MPV_ERR_WORKSPACE;
    a.c2 = static_cast<float>(2.0 * 1.4426950408889634 / static_cast<double>(logprobs->temperature));
    a.twice = static_cast<float>(2.0 / static_cast<double>(logprobs->temperature));
    a.sums = static_cast<mpv::PartSums*>(workspace);
    a.best = reinterpret_cast<float*>(static_cast<char*>(workspace) + room.sums);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (logprobs->dtype == MPV_DTYPE_F32) return mpv::launch_rows<float>(a, s);
    if (logprobs->dtype == MPV_DTYPE_BF16) return mpv::launch_rows<uint16_t>(a, s);
    return mpv::launch_rows<__half>(a, s);
}

}  // extern "C"
