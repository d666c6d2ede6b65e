// Verification of drafted chains from probabilities: device and host code.

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "mpv_host.h"

namespace mpv {

constexpr int kChainBlock = 1024;

struct ChainArgs {
    mpv_chains c;
    mpv_chain_buffers b;
};

// A probability as a double; what is not positive counts as 0.
__device__ __forceinline__ double mass_of(float v) { return v > 0.0f ? static_cast<double>(v) : 0.0; }
__device__ __forceinline__ float prob(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float prob(const uint16_t* p, int64_t i) { return __uint_as_float(static_cast<uint32_t>(p[i]) << 16); }
__device__ __forceinline__ float prob(const __half* p, int64_t i) { return __half2float(p[i]); }

// What the bonus token is drawn from: token t has the mass (p_t - q_t)_+, p_t without a draft row, nothing where t is `without`.
template <class T>
struct Rest {
    const T* p;
    const T* q;
    int without;
    __device__ __forceinline__ double operator()(int t) const {
        double m = mass_of(prob(p, t));
        if (q) m -= mass_of(prob(q, t));
        return m > 0.0 && t != without ? m : 0.0;
    }
};

__device__ __forceinline__ double wave_sum(double v) {
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A workgroup per chain: the tests (a lane each), then the draw.  The row is divided among the waves, the part in which the
// cumulative mass passes the drawn point is divided again, and one wave walks through what is left.
template <class T>
__global__ __launch_bounds__(kChainBlock) void chains_kernel(ChainArgs a) {
    constexpr int kWaves = kChainBlock / 64;
    __shared__ double part[kWaves];
    __shared__ int stop;
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int N = a.c.N, V = a.c.V;
    const int nodes = a.b.num_nodes ? min(max(a.b.num_nodes[b], 1), N) : N;
    const int32_t* tokens = a.b.tokens + static_cast<int64_t>(b) * N;
    const float* u = a.b.uniforms + static_cast<int64_t>(b) * N;
    const T* target = static_cast<const T*>(a.b.target_probs) + static_cast<int64_t>(b) * N * a.c.target_stride;
    const T* draft = a.b.draft_probs ? static_cast<const T*>(a.b.draft_probs) + static_cast<int64_t>(b) * N * a.c.draft_stride : nullptr;
    if (wave == 0) {
        const int n = lane + 1;
        bool passed = false;
        if (n < nodes) {
            const int x = tokens[n];
            if (x >= 0 && x < V) {
                const double p = mass_of(prob(target + (n - 1) * a.c.target_stride, x));
                const double q = draft ? mass_of(prob(draft + (n - 1) * a.c.draft_stride, x)) : 1.0;
                passed = static_cast<double>(u[n]) * q < p;
            }
        }
        const int length = __ffsll(~static_cast<unsigned long long>(__ballot(passed))) - 1;
        if (lane < a.c.max_depth) {
            const int64_t at = static_cast<int64_t>(b) * a.c.max_depth + lane;
            a.b.path_nodes[at] = lane < length ? n : -1;
            a.b.path_tokens[at] = lane < length ? tokens[n] : -1;
        }
        for (int i = 64 + lane; i < a.c.max_depth; i += 64) {
            const int64_t at = static_cast<int64_t>(b) * a.c.max_depth + i;
            a.b.path_nodes[at] = -1;
            a.b.path_tokens[at] = -1;
        }
        if (lane == 0) {
            a.b.accept_len[b] = length;
            stop = length;
        }
    }
    __syncthreads();
    const int length = stop;
    const bool rejected = length + 1 < nodes;
    const int x = rejected ? tokens[length + 1] : -1;
    const bool bad = rejected && (x < 0 || x >= V);
    Rest<T> rest;
    rest.p = target + length * a.c.target_stride;
    rest.q = rejected && draft ? draft + length * a.c.draft_stride : nullptr;
    rest.without = rejected && !draft && !bad ? x : -1;
    if (threadIdx.x == 0 && bad) atomicAdd(&a.b.counters[MPV_COUNTER_BAD_TOKEN], 1u);

    // sums of the waves' parts [w * step, (w + 1) * step) of [from, to)
    auto parts = [&](int from, int to, int step) {
        double s = 0.0;
        const int end = min(from + (wave + 1) * step, to);
        for (int t = from + wave * step + lane; t < end; t += 64) s += rest(t);
        s = wave_sum(s);
        __syncthreads();
        if (lane == 0) part[wave] = s;
        __syncthreads();
    };
    auto total_of = [&]() {
        double s = 0.0;
        for (int w = 0; w < kWaves; ++w) s += part[w];
        return s;
    };
    int from = 0, to = V, step = (V + kWaves - 1) / kWaves;
    parts(from, to, step);
    double total = total_of();
    if (!(total > 0.0)) {
        if (threadIdx.x == 0) atomicAdd(&a.b.counters[MPV_COUNTER_ZERO_MASS], 1u);
        rest.q = nullptr;
        rest.without = -1;
        parts(from, to, step);
        total = total_of();
    }
    if (!(total > 0.0)) {
        if (threadIdx.x == 0) a.b.bonus_token[b] = 0;
        return;
    }
    double point = static_cast<double>(u[0]) * total;      // the token sought is the first with more than that up to it
    for (int level = 0; level < 2; ++level) {
        // the first part that passes the point, or the last with mass
        double before = 0.0, at = 0.0;
        int pick = -1;
        for (int w = 0; w < kWaves; ++w) {
            if (part[w] > 0.0) {
                pick = w;
                at = before;
                if (before + part[w] > point) break;
            }
            before += part[w];
        }
        if (pick < 0) pick = 0;                              // (cannot be: the range has mass)
        point -= at;
        from += pick * step;
        to = min(from + step, to);
        step = (to - from + kWaves - 1) / kWaves;
        if (level == 0) parts(from, to, step);
    }
    if (wave != 0) return;
    double before = 0.0;
    int last = from;
    for (int base = from; base < to; base += 64) {
        const int t = base + lane;
        const double m = t < to ? rest(t) : 0.0;
        double s = m;
        for (int d = 1; d < 64; d <<= 1) {
            const double o = __shfl_up(s, d);
            if (lane >= d) s += o;
        }
        const unsigned long long some = __ballot(m > 0.0);
        const unsigned long long past = __ballot(m > 0.0 && before + s > point);
        if (past) {
            last = base + __ffsll(past) - 1;
            break;
        }
        if (some) last = base + 63 - __clzll(static_cast<long long>(some));
        before += __shfl(s, 63);
    }
    if (lane == 0) a.b.bonus_token[b] = last;
}

__global__ void clear_counters_kernel(uint32_t* counters) {
    if (threadIdx.x < MPV_COUNTER_COUNT) counters[threadIdx.x] = 0;
}

static int check_chains(const mpv_chains* c) {
    if (!c) return MPV_ERR_NULL;
    if (c->B < 0 || c->N < 1 || c->V < 1 || c->max_depth < 1 || c->max_depth < c->N - 1) return MPV_ERR_BAD_SHAPE;
    if (!known_dtype(c->dtype)) return MPV_ERR_BAD_DTYPE;
    if (c->N > MPV_MAX_NODES || c->V > MPV_MAX_VOCAB || c->B > (1 << 24) || c->max_depth > (1 << 20)) return MPV_ERR_UNSUPPORTED;
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
    *out = 256;
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
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();
    hipLaunchKernelGGL(mpv::clear_counters_kernel, dim3(1), dim3(64), 0, s, buf->counters);
    const dim3 grid(static_cast<unsigned>(chains->B)), block(mpv::kChainBlock);
    if (chains->dtype == MPV_DTYPE_F32) hipLaunchKernelGGL(mpv::chains_kernel<float>, grid, block, 0, s, a);
    else if (chains->dtype == MPV_DTYPE_BF16) hipLaunchKernelGGL(mpv::chains_kernel<uint16_t>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(mpv::chains_kernel<__half>, grid, block, 0, s, a);
    return mpv::launched();
}

}  // extern "C"
