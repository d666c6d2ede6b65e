// Verification of drafted chains from probabilities: device and host code.

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "mpv_host.h"

namespace mpv {

// The tests cost a few dependent loads; what is read in earnest is one row of p (and of q) a chain, for the sum of its masses, and a
// small part of it again, where the drawn point lies.  Masses are taken and added in double: the differences of two rows are exact
// and a border of the cumulative mass lies where it does in the definition, but for sums' rounding (2^-53).
//
// One workgroup a chain (chain_kernel) where that is enough; with fewer chains than compute units and long rows the sums are
// made by `parts` workgroups a chain (part_kernel), and draw_kernel goes on from there.
//
// Large batches are bound by memory: 64 chains of 128 256 float32 tokens with a draft (66 MB) take 18.7 us, 256 of 151 937 bfloat16
// tokens without (78 MB) 24.4 us, 3.5 and 3.2 TB/s, launches and the draw's second look included.  Small ones are bound by two launches
// and loads that depend on each other (length, token, its masses, the row, the point's place): one chain of 32 000 tokens, 8.8 us.

constexpr int kChainBlock = 1024;
constexpr int kPartBlock = 256;

struct ChainArgs {
    mpv_chains c;
    mpv_chain_buffers b;
    int parts, part;                       // workgroups a chain, elements of each
    double* sums;                          // [B][parts]
};

// A probability as a double; what is not positive counts as 0 (fmax: NaN too).
__device__ __forceinline__ double mass_of(float v) { return static_cast<double>(fmaxf(v, 0.0f)); }
__device__ __forceinline__ float prob(float p) { return p; }
__device__ __forceinline__ float prob(uint16_t p) { return __uint_as_float(static_cast<uint32_t>(p) << 16); }
__device__ __forceinline__ float prob(__half p) { return __half2float(p); }

// 16 bytes of a row, at any element's address
template <class T>
struct Vector {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
    __device__ __forceinline__ void load(const T* from) { __builtin_memcpy(v, from, 16); }
};

// What the bonus token is drawn from: token t has the mass (p_t - q_t)_+, p_t without a draft row, nothing where t is `without`.
template <class T>
struct Rest {
    const T* p;
    const T* q;
    int without;
    __device__ __forceinline__ double operator()(int t) const {
        if (t == without) return 0.0;
        const double m = mass_of(prob(p[t]));
        return q ? fmax(m - mass_of(prob(q[t])), 0.0) : m;
    }
    // Mass of N tokens from t on.  The token left out is looked for a group at a time.
    template <bool Q>
    __device__ __forceinline__ double group_sum(const Vector<T>& a, const Vector<T>& d, int t) const {
        constexpr int N = Vector<T>::N;
        double s[2] = {};
        if (!Q && static_cast<unsigned>(without - t) < static_cast<unsigned>(N)) {
            for (int i = 0; i < N; ++i) s[0] += (*this)(t + i);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (Q) s[i & 1] += fmax(mass_of(prob(a.v[i])) - mass_of(prob(d.v[i])), 0.0);
                else s[i & 1] += mass_of(prob(a.v[i]));
            }
        }
        return s[0] + s[1];
    }
    // Mass of the 16-byte groups lane, lane + lanes, .. of [from, to), four of them asked for at a time.
    template <bool Q>
    __device__ __forceinline__ double lane_sum_of(int from, int to, int lane, int lanes) const {
        constexpr int N = Vector<T>::N, kAtOnce = 4;
        double s = 0.0;
        int t = from + lane * N;
        const int step = lanes * N;
        for (; t + (kAtOnce - 1) * step + N <= to; t += kAtOnce * step) {
            Vector<T> a[kAtOnce], d[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                a[j].load(p + t + j * step);
                if constexpr (Q) d[j].load(q + t + j * step);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) s += group_sum<Q>(a[j], d[j], t + j * step);
        }
        {
            Vector<T> a[kAtOnce - 1], d[kAtOnce - 1];
#pragma unroll
            for (int j = 0; j < kAtOnce - 1; ++j)
                if (t + j * step + N <= to) {
                    a[j].load(p + t + j * step);
                    if constexpr (Q) d[j].load(q + t + j * step);
                }
#pragma unroll
            for (int j = 0; j < kAtOnce - 1; ++j)
                if (t + N <= to) {
                    s += group_sum<Q>(a[j], d[j], t);
                    t += step;
                }
        }
        for (; t < to; ++t) s += (*this)(t);                // (only the lane at the end has some left)
        return s;
    }
    __device__ __forceinline__ double lane_sum(int from, int to, int lane, int lanes) const {
        return q ? lane_sum_of<true>(from, to, lane, lanes) : lane_sum_of<false>(from, to, lane, lanes);
    }
};

__device__ __forceinline__ double wave_sum(double v) {
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A chain's rows.
template <class T>
struct Chain {
    const int32_t* tokens;
    const float* u;
    const T* target;
    const T* draft;
    int nodes;
    __device__ __forceinline__ Chain(const ChainArgs& a, int b) {
        const int N = a.c.N;
        nodes = a.b.num_nodes ? min(max(a.b.num_nodes[b], 1), N) : N;
        tokens = a.b.tokens + static_cast<int64_t>(b) * N;
        u = a.b.uniforms + static_cast<int64_t>(b) * N;
        target = static_cast<const T*>(a.b.target_probs) + static_cast<int64_t>(b) * N * a.c.target_stride;
        draft = a.b.draft_probs ? static_cast<const T*>(a.b.draft_probs) + static_cast<int64_t>(b) * N * a.c.draft_stride : nullptr;
    }
    // Accepted tokens: lane n - 1 tests token n.  A whole wave calls it.
    __device__ __forceinline__ int test(const ChainArgs& a, int lane) const {
        // (what does not depend on the chain's length is asked for together with it)
        const int n = lane + 1;
        const int x = n < a.c.N ? tokens[n] : -1;
        const float un = n < a.c.N ? u[n] : 0.0f;
        bool passed = false;
        if (n < nodes && x >= 0 && x < a.c.V) {
            const double p = mass_of(prob(target[(n - 1) * a.c.target_stride + x]));
            const double q = draft ? mass_of(prob(draft[(n - 1) * a.c.draft_stride + x])) : 1.0;
            passed = static_cast<double>(un) * q < p;
        }
        return __ffsll(~static_cast<unsigned long long>(__ballot(passed))) - 1;
    }
    __device__ __forceinline__ Rest<T> rest(const ChainArgs& a, int length, bool* bad) const {
        const bool rejected = length + 1 < nodes;
        const int x = rejected ? tokens[length + 1] : -1;
        *bad = rejected && (x < 0 || x >= a.c.V);
        Rest<T> r;
        r.p = target + length * a.c.target_stride;
        r.q = rejected && draft ? draft + length * a.c.draft_stride : nullptr;
        r.without = rejected && !draft && !*bad ? x : -1;
        return r;
    }
    __device__ __forceinline__ void write_path(const ChainArgs& a, int b, int length, int lane) const {
        for (int i = lane; i < a.c.max_depth; i += 64) {
            const int64_t at = static_cast<int64_t>(b) * a.c.max_depth + i;
            a.b.path_nodes[at] = i < length ? i + 1 : -1;
            a.b.path_tokens[at] = i < length ? tokens[i + 1] : -1;
        }
        if (lane == 0) a.b.accept_len[b] = length;
    }
};

// A workgroup's share of a draw.
struct Draw {
    static constexpr int kWaves = kChainBlock / 64;
    struct Shared {
        double part[kWaves];
        int first, last;
        int token;
    };
    Shared& sh;
    const int lane, wave;

    // sums of the waves' parts [from + w * step, from + (w + 1) * step) below `to` in sh.part; returns their total
    template <class T>
    __device__ __forceinline__ double parts(const Rest<T>& rest, int from, int to, int step) {
        const int begin = from + wave * step;
        const double s = wave_sum(rest.lane_sum(min(begin, to), min(begin + step, to), lane, 64));
        __syncthreads();
        if (lane == 0) sh.part[wave] = s;
        __syncthreads();
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) all += sh.part[w];
        return all;
    }
    static __device__ __forceinline__ double upto(double s, int lane) {
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(s, d);
            if (lane >= d) s += o;
        }
        return s;
    }
    // The sum of n sums.  A whole wave calls it.
    static __device__ __forceinline__ double total_of(const double* sums, int n, int lane) {
        double s = 0.0;
        for (int w = lane; w < n; w += 64) s += sums[w];
        return wave_sum(s);
    }
    // The first of n sums that passes the point, or the last with mass; *before: the sums ahead of it.  A whole wave calls it.
    static __device__ __forceinline__ int pick(const double* sums, int n, double point, int lane, double* before) {
        double ahead = 0.0;
        int at = 0;
        *before = 0.0;
        for (int base = 0; base < n; base += 64) {
            const double mine = base + lane < n ? sums[base + lane] : 0.0;
            const double to = ahead + upto(mine, lane);
            const unsigned long long some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && to > point);
            if (some) {
                const int l = past ? __ffsll(past) - 1 : 63 - __clzll(static_cast<long long>(some));
                at = base + l;
                *before = __shfl(to - mine, l);
            }
            if (past) break;
            ahead = __shfl(to, 63);
        }
        return at;
    }
    // The token of [from, to) in which the cumulative mass passes `point`, the last one with mass if none does: neighbouring tokens
    // to a lane, whole 16-byte groups.  Thread 0 has the answer.
    template <class T>
    __device__ __forceinline__ int token(const Rest<T>& rest, int from, int to, double point) {
        constexpr int N = Vector<T>::N;
        const int mine = (to - from + kChainBlock * N - 1) / (kChainBlock * N) * N;
        const int begin = min(from + static_cast<int>(threadIdx.x) * mine, to), end = min(begin + mine, to);
        const double sum = rest.lane_sum(begin, end, 0, 1);
        double end_at = upto(sum, lane);
        __syncthreads();
        if (lane == 63) sh.part[wave] = end_at;
        if (threadIdx.x == 0) { sh.first = kChainBlock; sh.last = 0; sh.token = from; }
        __syncthreads();
        for (int w = 0; w < wave; ++w) end_at += sh.part[w];
        const unsigned long long some = __ballot(sum > 0.0), past = __ballot(sum > 0.0 && end_at > point);
        if (lane == 0 && past) atomicMin(&sh.first, wave * 64 + __ffsll(past) - 1);
        if (lane == 0 && some) atomicMax(&sh.last, wave * 64 + 63 - __clzll(static_cast<long long>(some)));
        __syncthreads();
        if (static_cast<int>(threadIdx.x) == (sh.first < kChainBlock ? sh.first : sh.last)) {
            double run = end_at - sum;
            int last = begin;
            bool found = false;
            for (int t = begin; t < end && !found; t += N) {
                double m[N];
                if (t + N <= end) {
                    Vector<T> a, d;
                    a.load(rest.p + t);
                    if (rest.q) d.load(rest.q + t);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        m[i] = mass_of(prob(a.v[i]));
                        if (rest.q) m[i] = fmax(m[i] - mass_of(prob(d.v[i])), 0.0);
                        if (t + i == rest.without) m[i] = 0.0;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) m[i] = t + i < end ? rest(t + i) : 0.0;
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (found) continue;
                    run += m[i];
                    if (m[i] > 0.0) {
                        last = t + i;
                        found = run > point;
                    }
                }
            }
            sh.token = last;
        }
        __syncthreads();
        return sh.token;
    }
};

// The draw over the whole row.
template <class T>
__device__ __forceinline__ void draw_row(const ChainArgs& a, int b, const Chain<T>& chain, Rest<T> rest, Draw& draw) {
    const int V = a.c.V, step = (V + Draw::kWaves - 1) / Draw::kWaves;
    double total = draw.parts(rest, 0, V, step);
    if (!(total > 0.0)) {
        if (threadIdx.x == 0) atomicAdd(&a.b.counters[MPV_COUNTER_ZERO_MASS], 1u);
        rest.q = nullptr;
        rest.without = -1;
        total = draw.parts(rest, 0, V, step);
    }
    int token = 0;
    if (total > 0.0) {
        double before;
        const double point = static_cast<double>(chain.u[0]) * total;
        const int from = Draw::pick(draw.sh.part, Draw::kWaves, point, draw.lane, &before) * step;
        token = draw.token(rest, from, min(from + step, V), point - before);
    }
    if (threadIdx.x == 0) a.b.bonus_token[b] = token;
}

template <class T>
__global__ __launch_bounds__(kChainBlock) void chain_kernel(ChainArgs a) {
    __shared__ Draw::Shared shared;
    __shared__ int stop;
    const int b = blockIdx.x;
    Draw draw{shared, static_cast<int>(threadIdx.x & 63), static_cast<int>(threadIdx.x >> 6)};
    const Chain<T> chain(a, b);
    if (draw.wave == 0) {
        const int length = chain.test(a, draw.lane);
        chain.write_path(a, b, length, draw.lane);
        if (draw.lane == 0) stop = length;
    }
    __syncthreads();
    bool bad;
    const Rest<T> rest = chain.rest(a, stop, &bad);
    if (threadIdx.x == 0 && bad) atomicAdd(&a.b.counters[MPV_COUNTER_BAD_TOKEN], 1u);
    draw_row(a, b, chain, rest, draw);
}

// A part's sum.  Every workgroup of a chain tests its tokens for itself.
template <class T>
__global__ __launch_bounds__(kPartBlock) void part_kernel(ChainArgs a) {
    __shared__ double part[kPartBlock / 64];
    const int b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Chain<T> chain(a, b);
    const int length = chain.test(a, lane);
    bool bad;
    const Rest<T> rest = chain.rest(a, length, &bad);
    const int from = blockIdx.x * a.part, to = min(from + a.part, a.c.V);
    const double s = wave_sum(rest.lane_sum(from, to, threadIdx.x, kPartBlock));
    if (lane == 0) part[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[static_cast<int64_t>(b) * a.parts + blockIdx.x] = part[0] + part[1] + part[2] + part[3];
    if (blockIdx.x == 0 && wave == 1) chain.write_path(a, b, length, lane);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < MPV_COUNTER_COUNT) a.b.counters[threadIdx.x] = 0;
}

template <class T>
__global__ __launch_bounds__(kChainBlock) void draw_kernel(ChainArgs a) {
    __shared__ Draw::Shared shared;
    const int b = blockIdx.x;
    Draw draw{shared, static_cast<int>(threadIdx.x & 63), static_cast<int>(threadIdx.x >> 6)};
    const Chain<T> chain(a, b);
    bool bad;
    const Rest<T> rest = chain.rest(a, a.b.accept_len[b], &bad);
    if (threadIdx.x == 0 && bad) atomicAdd(&a.b.counters[MPV_COUNTER_BAD_TOKEN], 1u);
    const double* sums = a.sums + static_cast<int64_t>(b) * a.parts;
    const double total = Draw::total_of(sums, a.parts, draw.lane);
    if (!(total > 0.0)) {
        draw_row(a, b, chain, rest, draw);
        return;
    }
    double before;
    const double point = static_cast<double>(chain.u[0]) * total;
    const int from = Draw::pick(sums, a.parts, point, draw.lane, &before) * a.part;
    const int token = draw.token(rest, from, min(from + a.part, a.c.V), point - before);
    if (threadIdx.x == 0) a.b.bonus_token[b] = token;
}

__global__ void clear_counters_kernel(uint32_t* counters) {
    if (threadIdx.x < MPV_COUNTER_COUNT) counters[threadIdx.x] = 0;
}

// Workgroups a chain.  One (of 1024 threads) where the chains alone nearly fill the device; more of them are needed where a chain has two
// long rows to read, so that those of the compute units that would have none are missed.  us with one / with parts, rows of 128 256 tokens
// (in brackets: of 32 000),
//   with a draft     float32: 128 chains 38.6 / 32.2, 192: 35.6 / 32.7 (15.4 / 15.4), 239: 40.3 / 39.5 (16.5 / 17.7), 256: 41.9 / 41.8 (17.0 / 17.8)
//                    bfloat16: 192 chains 28.0 / 23.8 (15.0 / 15.4), 239: 29.8 / 27.4 (15.8 / 16.5), 256: 30.3 / 29.5 (16.2 / 16.2)
//                    (of 262 144 tokens, float32: 208 chains 74.1 / 74.8, 240: 77.4 / 83.4; bfloat16: 43.1 / 40.2, 46.2 / 45.2)
//   without          float32: 96 chains 18.7 / 18.5 (11.5 / 10.7), 144: 21.2 / 22.4 (12.2 / 13.1), 256: 29.8 / 33.4 (14.5 / 16.0)
//                    bfloat16: 96 chains 18.1 / 16.8 (11.8 / 11.5), 144: 18.8 / 19.6 (12.1 / 13.4), 256: 21.5 / 25.4 (12.5 / 15.4)
// One of 151 937 tokens takes 22.2 us with one, 9.4 with parts.  Otherwise 2048 workgroups in all (half as many: 64 chains of 128 256 tokens in
// 19.3 us against 18.7), none with fewer than 2048 tokens (4096: 16 chains of 32 000 tokens in 10.4 us against 9.5; 1024: 9.2, but 9.8
// against 9.4 for one of 151 937, whose sums the draw then has to add up).
static int parts_of(const mpv_chains* c, bool draft) {
    if (c->B >= (!draft ? 144 : c->V < 65536 ? 192 : 240)) return 1;
    const int most = (c->V + 2047) / 2048, wanted = c->B > 0 ? (2048 + c->B - 1) / c->B : 1;
    return most < wanted ? most : wanted;
}

template <class T>
static void launch_chains(ChainArgs& a, hipStream_t s) {
    const dim3 chains(static_cast<unsigned>(a.c.B));
    if (a.parts > 1) {
        hipLaunchKernelGGL(part_kernel<T>, dim3(static_cast<unsigned>(a.parts), chains.x), dim3(kPartBlock), 0, s, a);
        hipLaunchKernelGGL(draw_kernel<T>, chains, dim3(kChainBlock), 0, s, a);
    } else {
        hipLaunchKernelGGL(clear_counters_kernel, dim3(1), dim3(64), 0, s, a.b.counters);
        hipLaunchKernelGGL(chain_kernel<T>, chains, dim3(kChainBlock), 0, s, a);
    }
}

static int check_chains(const mpv_chains* c) {
    if (!c) return MPV_ERR_NULL;
    if (c->B < 0 || c->N < 1 || c->V < 1 || c->max_depth < 1 || c->max_depth < c->N - 1) return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(c->dtype)) return MPV_ERR_BAD_DTYPE;
    if (c->N > MPV_MAX_NODES || c->V > MPV_MAX_VOCAB || c->B > (1 << 21) || c->max_depth > (1 << 20)) return MPV_ERR_UNSUPPORTED;
    if (c->target_stride < c->V || c->draft_stride < 0) return MPV_ERR_BAD_SHAPE;
    const int64_t rows = static_cast<int64_t>(c->B) * c->N;
    if (span(0, span(0, rows, c->target_stride), 4) == INT64_MAX || span(0, span(0, rows, c->draft_stride), 4) == INT64_MAX) return MPV_ERR_UNSUPPORTED;
    return MPV_OK;
}

}  // namespace mpv

extern "C" {

int mpv_verify_chains_workspace_bytes(const mpv_chains* chains, size_t* out) {
    if (!out) return MPV_ERR_NULL;
    const int rc = mpv::check_chains(chains);
    if (rc != MPV_OK) return rc;
    const size_t sums = static_cast<size_t>(chains->B) * mpv::parts_of(chains, true) * sizeof(double);      // (without a draft: no more)
    *out = (sums + 255) / 256 * 256 + 256;
    return MPV_OK;
}

int mpv_verify_chains(const mpv_chains* chains, const mpv_chain_buffers* buf, void* workspace, size_t workspace_bytes,
                      void* hip_stream) {
    size_t need;
    const int rc = mpv_verify_chains_workspace_bytes(chains, &need);
    if (rc != MPV_OK) return rc;
    if (!buf) return MPV_ERR_NULL;
    if (chains->B == 0) return MPV_OK;
    if (!buf->target_probs || !buf->tokens || !buf->uniforms || !buf->accept_len || !buf->path_nodes || !buf->path_tokens ||
        !buf->bonus_token || !buf->counters)
        return MPV_ERR_NULL;
    if (buf->draft_probs && chains->draft_stride < chains->V) return MPV_ERR_BAD_SHAPE;
    const int bytes = mpv::elem_bytes(chains->dtype);
    if (!mpv::aligned(buf->target_probs, bytes) || !mpv::aligned(buf->draft_probs, bytes)) return MPV_ERR_ALIGNMENT;
    if (!workspace || !mpv::aligned(workspace, 256) || workspace_bytes < need) return MPV_ERR_WORKSPACE;
    mpv::ChainArgs a;
    a.c = *chains; a.b = *buf;
    a.parts = mpv::parts_of(chains, buf->draft_probs != nullptr);
    a.part = (chains->V + a.parts - 1) / a.parts;
    a.part = (a.part + 7) / 8 * 8;
    a.sums = static_cast<double*>(workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    if (chains->dtype == MPV_DTYPE_F32) mpv::launch_chains<float>(a, s);
    else if (chains->dtype == MPV_DTYPE_BF16) mpv::launch_chains<uint16_t>(a, s);
    else mpv::launch_chains<__half>(a, s);
    return mpv::launched();
}

}  // extern "C"
