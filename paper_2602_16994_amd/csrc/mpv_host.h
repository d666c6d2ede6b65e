// Helpers shared by the translation units of the library.

#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mpv.h"

namespace mpv {

extern thread_local int g_last_hip_error;      // mpv.hip

inline bool hip_fine(hipError_t e) {
    if (e == hipSuccess) return true;
    g_last_hip_error = static_cast<int>(e);
    return false;
}

// Workgroups of 256 threads that a launch can have: 2^32 threads in a dimension are too many.
constexpr int64_t kMostWorkgroups = (1 << 24) - 1;

// The outcome of the launches since the last hipGetLastError().
inline int launched() { return hip_fine(hipGetLastError()) ? MPV_OK : MPV_ERR_HIP; }

inline int elem_bytes(int32_t dtype) { return dtype == MPV_DTYPE_F32 ? 4 : 2; }
inline bool known_dtype(int32_t dtype) { return dtype == MPV_DTYPE_F32 || dtype == MPV_DTYPE_BF16 || dtype == MPV_DTYPE_F16; }
inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// a + b * c where it stays below 2^62, otherwise a number above it
inline int64_t span(int64_t a, int64_t b, int64_t c) {
    int64_t r;
    if (__builtin_mul_overflow(b, c, &r) || __builtin_add_overflow(a, r, &r)) return INT64_MAX;
    return r;
}

// Division of numbers below 2^31 by one that the host knows (Granlund and Montgomery, Division by invariant integers using
// multiplication, 1994, figure 4.1).
struct Divisor {
    uint32_t d, factor, shift1, shift2;
    __host__ void set(uint32_t by) {
        int log = 0;
        while ((1ull << log) < by) ++log;
        d = by;
        factor = static_cast<uint32_t>(((1ull << 32) * ((1ull << log) - by)) / by + 1);
        shift1 = log < 1 ? log : 1;
        shift2 = log < 1 ? 0 : log - 1;
    }
    __device__ __forceinline__ int of(int n) const {
        const uint32_t x = static_cast<uint32_t>(n), high = __umulhi(factor, x);
        return static_cast<int>((high + ((x - high) >> shift1)) >> shift2);
    }
};

}  // namespace mpv
