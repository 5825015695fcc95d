// Shared by the kernels at the ends of a training step (embedding.hip, log_probs.hip, adamw.hip): storage types, checks of arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "libra.h"

namespace libra {

constexpr int WAVE_LANES = 64;

template <class T> __device__ inline float load_as_float(T x) { return (float)x; }
// one rounding to nearest even; NaN stays NaN, what is too large for the type becomes infinite
template <class T> __device__ inline T round_to(float x) { return (T)x; }

inline bool known_dtype(int dtype) { return dtype == LIBRA_F16 || dtype == LIBRA_BF16 || dtype == LIBRA_F32; }
inline size_t dtype_bytes(int dtype) { return dtype == LIBRA_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline int last_launch() { return hipGetLastError() == hipSuccess ? LIBRA_OK : LIBRA_ERR_HIP; }

// f(a value of the storage type)
template <class F> inline int for_dtype(int dtype, F &&f) {
    if (dtype == LIBRA_F16) return f(_Float16{});
    if (dtype == LIBRA_BF16) return f(__bf16{});
    return f(float{});
}

// index `i` of an array of 32- or 64-bit whole numbers
__device__ inline int64_t index_at(const void *index, int index_type, int64_t i) {
    return index_type == LIBRA_INDEX_I64 ? reinterpret_cast<const int64_t *>(index)[i] : (int64_t)reinterpret_cast<const int32_t *>(index)[i];
}

inline bool known_index(int index_type) { return index_type == LIBRA_INDEX_I32 || index_type == LIBRA_INDEX_I64; }
inline size_t index_bytes(int index_type) { return index_type == LIBRA_INDEX_I64 ? 8 : 4; }

}  // namespace libra
