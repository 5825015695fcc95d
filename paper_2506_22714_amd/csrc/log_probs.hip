// Log probabilities of given classes, entropy and the most likely classes of rows of logits, and the gradient.  With
// z_j = scale * (x_j - max x) and s = sum exp(z_j):
//   log p_j = z_j - log s          H = log s - sum exp(z_j) z_j / s
//   dx_j = scale * ([j = target] d + sum_a [j = top_a] d_a - p_j (d + sum_a d_a + e (log p_j + H)))
// where d, d_a and e are the gradients of the target's, the alternatives' log probabilities and the entropy.
#include <algorithm>
#include <cmath>

#include "ends.h"

using namespace libra;

namespace {

constexpr float INF = __builtin_inff();

// Whole numbers in the order of the logits, NaN last; a larger one comes first among the alternatives.  Zeros are equal.
__device__ inline uint32_t rank_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
// ... and among equal ones the lower class
__device__ inline uint64_t rank_of(float x, uint32_t j) { return (uint64_t)rank_of(x) << 32 | (0xffffffffu - j); }

__device__ inline float wave_sum(float x) {
    for (int d = 32; d; d /= 2) x += __shfl_xor(x, d);
    return x;
}
__device__ inline uint64_t wave_most(uint64_t x) {
    for (int d = 32; d; d /= 2) {
        const uint64_t y = __shfl_xor((unsigned long long)x, d);
        x = x > y ? x : y;
    }
    return x;
}

// a workgroup per row
template <class T>
__global__ __launch_bounds__(256) void log_probs_kernel(const T *logits, int64_t n, int64_t classes, int64_t ld, const void *targets, int index_type, int32_t top, float scale,
                                                        float *target_out, float *entropy, float *top_out, int64_t *top_index, float *stats) {
    __shared__ uint64_t best[4];
    __shared__ float part[4][2];
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const T *x = logits + i * ld;
    // the largest logit that comes after `limit`
    auto next = [&](uint64_t limit) {
        uint64_t most = 0;
        for (int64_t j = threadIdx.x; j < classes; j += 256) {
            const uint64_t r = rank_of(load_as_float(x[j]), (uint32_t)j);
            if (r < limit && r > most) most = r;
        }
        most = wave_most(most);
        __syncthreads();
        if (lane == 0) best[wave] = most;
        __syncthreads();
        for (int w = 0; w < 4; ++w) most = most > best[w] ? most : best[w];
        return most;
    };
    uint64_t r = next(~0ull);
    const float most = load_as_float(x[0xffffffffu - (uint32_t)r]);
    const bool empty = most == -INF;
    float s = 0.f, t = 0.f;
    for (int64_t j = threadIdx.x; j < classes; j += 256) {
        const float z = scale * (load_as_float(x[j]) - (empty ? 0.f : most)), e = expf(z);
        s += e;
        if (e != 0.f) t += e * z;
    }
    s = wave_sum(s);
    t = wave_sum(t);
    if (lane == 0) part[wave][0] = s, part[wave][1] = t;
    __syncthreads();
    s = t = 0.f;
    for (int w = 0; w < 4; ++w) s += part[w][0], t += part[w][1];
    const float logs = empty ? 0.f : logf(s);
    auto logp = [&](int64_t j) { return scale * (load_as_float(x[j]) - (empty ? 0.f : most)) - logs; };
    if (threadIdx.x == 0) {
        entropy[i] = empty ? 0.f : logs - t / s;
        stats[2 * i] = most;
        stats[2 * i + 1] = logs;
        if (targets) {
            const int64_t j = index_at(targets, index_type, i);
            target_out[i] = j >= 0 && j < classes ? logp(j) : j == -1 ? 0.f : __builtin_nanf("");
        }
    }
    for (int32_t a = 0; a < top; ++a) {
        const int64_t j = 0xffffffffu - (uint32_t)r;
        if (threadIdx.x == 0) {
            top_out[i * top + a] = logp(j);
            top_index[i * top + a] = j;
        }
        if (a + 1 < top) r = next(r);
    }
    __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(256) void log_probs_backward_kernel(const T *logits, int64_t n, int64_t classes, int64_t ld, const void *targets, int index_type, int32_t top,
                                                                 float scale, const float *entropy, const float *stats, const int64_t *top_index, const float *d_target,
                                                                 const float *d_entropy, const float *d_top, T *dlogits, int64_t ld_dlogits) {
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const T *x = logits + i * ld;
    const float most = stats[2 * i], logs = stats[2 * i + 1], h = entropy[i];
    const int64_t target = targets ? index_at(targets, index_type, i) : -1;
    const bool given = target >= 0 && target < classes;
    const float e = d_entropy ? d_entropy[i] : 0.f;
    const float d = target == -1 || !d_target ? 0.f : given ? d_target[i] : __builtin_nanf("");
    float all = d;
    if (d_top)
        for (int a = 0; a < top; ++a) all += d_top[i * top + a];
    for (int64_t j = threadIdx.x; j < classes; j += 256) {
        const float logp = scale * (load_as_float(x[j]) - most) - logs, p = expf(logp);
        float g = p == 0.f ? 0.f * all : -p * (all + e * (logp + h));
        if (j == target) g += d;
        if (d_top)
            for (int a = 0; a < top; ++a)
                if (top_index[i * top + a] == j) g += d_top[i * top + a];
        dlogits[i * ld_dlogits + j] = round_to<T>(most == -INF ? 0.f : scale * g);
    }
    }
}

int shape(int64_t n, int64_t classes, int32_t top) {
    if (n < 0 || classes < 1 || top < 0 || top > classes) return LIBRA_ERR_SHAPE;
    if (n > INT32_MAX || classes > INT32_MAX) return LIBRA_ERR_TOO_LARGE;
    if (top > LIBRA_LOG_PROBS_MAX_TOP) return LIBRA_ERR_UNSUPPORTED;
    return LIBRA_OK;
}

}  // namespace

extern "C" int libra_log_probs_workspace(int64_t n, int64_t classes, int32_t top, size_t *bytes) {
    if (!bytes) return LIBRA_ERR_NULL;
    if (int rc = shape(n, classes, top)) return rc;
    *bytes = 0;
    return LIBRA_OK;
}

extern "C" int libra_log_probs(const void *logits, int64_t n, int64_t classes, int64_t ld, int dtype, const void *targets, int index_type, int32_t top, float scale,
                               float *target_out, float *entropy, float *top_out, int64_t *top_index, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = shape(n, classes, top)) return rc;
    if (ld < classes) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if ((targets && !known_index(index_type)) || !(scale > 0.f && std::isfinite(scale))) return LIBRA_ERR_OPTION;
    if (n == 0) return LIBRA_OK;
    if (!logits || !entropy || !stats || (targets && !target_out) || (top && (!top_out || !top_index))) return LIBRA_ERR_NULL;
    if (!aligned_to(logits, dtype_bytes(dtype)) || (targets && !aligned_to(targets, index_bytes(index_type))) || !aligned_to(target_out, 4) || !aligned_to(entropy, 4) ||
        !aligned_to(top_out, 4) || !aligned_to(top_index, 8) || !aligned_to(stats, 4))
        return LIBRA_ERR_BUFFER;
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((log_probs_kernel<T>), dim3((unsigned)std::min<int64_t>(n, 1 << 20)), dim3(256), 0, (hipStream_t)stream, (const T *)logits, n, classes, ld, targets, index_type, top, scale,
                           target_out, entropy, top_out, top_index, stats);
        return last_launch();
    });
}

extern "C" int libra_log_probs_backward(const void *logits, int64_t n, int64_t classes, int64_t ld, int dtype, const void *targets, int index_type, int32_t top, float scale,
                                        const float *entropy, const float *stats, const int64_t *top_index, const float *d_target, const float *d_entropy, const float *d_top,
                                        void *dlogits, int64_t ld_dlogits, void *stream) {
    if (int rc = shape(n, classes, top)) return rc;
    if (ld < classes || ld_dlogits < classes) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if ((targets && !known_index(index_type)) || !(scale > 0.f && std::isfinite(scale))) return LIBRA_ERR_OPTION;
    if (n == 0) return LIBRA_OK;
    if (!logits || !entropy || !stats || !dlogits || (d_target && !targets) || (top && d_top && !top_index)) return LIBRA_ERR_NULL;
    if (!aligned_to(logits, dtype_bytes(dtype)) || !aligned_to(dlogits, dtype_bytes(dtype)) || (targets && !aligned_to(targets, index_bytes(index_type))) ||
        !aligned_to(entropy, 4) || !aligned_to(stats, 4) || !aligned_to(top_index, 8) || !aligned_to(d_target, 4) || !aligned_to(d_entropy, 4) || !aligned_to(d_top, 4))
        return LIBRA_ERR_BUFFER;
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((log_probs_backward_kernel<T>), dim3((unsigned)std::min<int64_t>(n, 1 << 20)), dim3(256), 0, (hipStream_t)stream, (const T *)logits, n, classes, ld, targets, index_type, top,
                           scale, entropy, stats, top_index, d_target, d_entropy, top ? d_top : nullptr, (T *)dlogits, ld_dlogits);
        return last_launch();
    });
}
