// Host-side helpers shared by the translation units of the library.

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

}  // namespace mpv
