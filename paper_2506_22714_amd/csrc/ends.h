// Shared by the kernels at the ends of a training step (embedding.hip, log_probs.hip, adamw.hip): storage types, checks of arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "libra.h"

namespace libra {

constexpr int WAVE_LANES = 64;

template <class T> __device__ inline float load_as_float(T x) { return (float)x; }
// One rounding of an fp32 number to nearest even; NaN stays NaN, what is too large for the type becomes infinite.  The compiler may not look
// behind the number: it would merge a product or a sum with its rounding to fp16 into one instruction that rounds the exact value (not that to
// bf16), and the last place of a result would go by how the code around it was compiled.
template <class T> __device__ inline T round_to(float x) {
    if constexpr (std::is_same_v<T, _Float16>) asm("" : "+v"(x));
    return (T)x;
}

// 16 bytes of a row as numbers, and back
template <class T> constexpr int VECTOR = 16 / (int)sizeof(T);
template <class T> __device__ inline void unpack(uint4 v, float *f) {
    const T *t = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int k = 0; k < VECTOR<T>; ++k) f[k] = load_as_float(t[k]);
}
template <class T> __device__ inline uint4 pack(const float *f) {
    uint4 v;
    T *t = reinterpret_cast<T *>(&v);
#pragma unroll
    for (int k = 0; k < VECTOR<T>; ++k) t[k] = round_to<T>(f[k]);
    return v;
}

// 16 bytes that begin at any element: one load or store too (memory accesses need no alignment here)
struct __attribute__((packed, aligned(2))) Unaligned { uint32_t x[4]; };

// What the lane `STEP` further (by exclusive or of lane numbers, once the steps below it have been taken) holds: moves inside a row of
// 16 lanes, shuffles beyond.
template <int STEP> __device__ inline uint32_t lane_across(uint32_t x) {
    if constexpr (STEP == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true);             // quad_perm [1,0,3,2]
    else if constexpr (STEP == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true);        // quad_perm [2,3,0,1]
    else if constexpr (STEP == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true);       // row_half_mirror
    else if constexpr (STEP == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true);       // row_mirror
    else return (uint32_t)__shfl_xor((int)x, STEP);
}
template <int STEP> __device__ inline float lane_across(float x) { return __uint_as_float(lane_across<STEP>(__float_as_uint(x))); }
template <int STEP> __device__ inline uint64_t lane_across(uint64_t x) {
    return (uint64_t)lane_across<STEP>((uint32_t)(x >> 32)) << 32 | lane_across<STEP>((uint32_t)x);
}
// f over a group of L neighbouring lanes (a power of two up to 64); every lane gets the result
template <int L, int STEP = 1, class V, class F> __device__ inline V over_group(V x, F &&f) {
    if constexpr (STEP >= L) return x;
    else {
        x = f(x, lane_across<STEP>(x));
        return over_group<L, STEP * 2>(x, f);
    }
}

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

// N of them, index_of(k) for each: the loads are issued together
template <int N, class F> __device__ inline void indices_at(const void *index, int index_type, F &&index_of, int64_t *out) {
    if (index_type == LIBRA_INDEX_I64) {
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = reinterpret_cast<const int64_t *>(index)[index_of(k)];
    } else {
        int32_t x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = reinterpret_cast<const int32_t *>(index)[index_of(k)];
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = x[k];
    }
}

inline bool known_index(int index_type) { return index_type == LIBRA_INDEX_I32 || index_type == LIBRA_INDEX_I64; }
inline size_t index_bytes(int index_type) { return index_type == LIBRA_INDEX_I64 ? 8 : 4; }

}  // namespace libra
