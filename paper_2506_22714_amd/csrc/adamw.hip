// One AdamW step over many tensors (decoupled weight decay), states in 32 bits or in 8:
//   m <- b1 m + (1 - b1) g      v <- b2 v + (1 - b2) g g      p <- (1 - lr wd) p - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8 bits: m and r = sqrt(v) as e4m3 numbers (OCP, finite ones up to 448) times a power of two for every 256 elements, the smallest
// that keeps the block's largest number within 448.  The root has twice the range of v in octaves.  A number goes up or down to a
// neighbour by chance, in proportion to its distance, because a nearest one would never move: an average over 1,000 steps changes by
// 0.1 % a step, and e4m3 numbers are 6 to 12 % apart.  The chances are a hash of (seed, step, tensor, element), so a step gives the same
// result every time.  A root above zero never becomes zero: it divides.  The new parameter is made from the states before they are rounded.
// No product is contracted with a sum: what is rounded to 8 bits is then the same on every machine with IEEE arithmetic.
#include <algorithm>
#include <cmath>

#include "ends.h"

using namespace libra;

namespace {

constexpr int STATE_BLOCK = LIBRA_ADAMW_BLOCK, LAUNCH_TENSORS = 32;
constexpr int64_t LAUNCH_BLOCKS = 1 << 22;      // the threads of a launch are counted in 32 bits

struct Tensors {                    // of one launch, in its arguments: nothing is copied to the device beforehand
    libra_adamw_tensor_t t[LAUNCH_TENSORS];
    int32_t first[LAUNCH_TENSORS];  // workgroup that each begins with
    int64_t begin[LAUNCH_TENSORS];  // and the block of the tensor that this workgroup takes
    int32_t count;
};

struct Step {
    float b1, b2, c1, c2, eps;      // c = 1 - b
    float keep, size, root;         // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    double lr, decay, log_b1, log_b2;
    const int64_t *step_dev;
    const float *lr_dev;
    uint32_t seed;
    uint32_t step;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6C8E9CF5u;
    x ^= x >> 15;
    x *= 0x58AC4D6Bu;
    return x ^ (x >> 16);
}

// The step's own numbers where they are in device memory (a captured step counts on).
__device__ inline void read_step(Step &s) {
    if (!s.step_dev && !s.lr_dev) return;
    __shared__ float got[3];
    __shared__ uint32_t number;
    if (threadIdx.x == 0) {
        const int64_t t = s.step_dev ? *s.step_dev : (int64_t)s.step;
        const double lr = s.lr_dev ? (double)*s.lr_dev : s.lr;
        got[0] = (float)(1.0 - lr * s.decay);
        got[1] = (float)(lr / -expm1((double)t * s.log_b1));
        got[2] = (float)(1.0 / sqrt(-expm1((double)t * s.log_b2)));
        number = (uint32_t)t;
    }
    __syncthreads();
    s.keep = got[0];
    s.size = got[1];
    s.root = got[2];
    s.step = number;
}

__device__ inline float e4m3_value(uint8_t code) {
    const uint32_t e = (code >> 3) & 15, f = code & 7;
    const float a = (code & 127) == 127 ? __builtin_nanf("") : e ? __uint_as_float((e + 120) << 23 | f << 20) : (float)f * 0x1p-9f;
    return code & 128 ? -a : a;
}

// |x| / scale, 0 .. 448, to one of its two neighbours; `inverse` is the power of two 1 / scale
__device__ inline uint32_t e4m3_code(float x, float inverse, float chance, bool root) {
    const float y = fabsf(x) * inverse;
    if (!(y <= 448.f)) return 127;                                       // Inf and NaN
    const int e = max((int)(__float_as_uint(y) >> 23) - 127, -6);
    uint32_t q = (uint32_t)(y * __uint_as_float((uint32_t)(130 - e) << 23) + chance);
    if (root && q == 0 && x > 0.f) q = 1;
    return (uint32_t)(e + 6) * 8 + q;
}

struct Element {
    float p, m, v;
};

// r: sqrt of the new v
__device__ inline Element updated(const Step &s, float p, float g, float m, float v, float &r) {
#pragma clang fp contract(off)
    Element e;
    e.m = s.b1 * m + s.c1 * g;
    e.v = s.b2 * v + s.c2 * (g * g);
    r = sqrtf(e.v);
    e.p = s.keep * p - s.size * (e.m / (s.root * r + s.eps));
    return e;
}

// a workgroup per 256 elements
template <class T, bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(Tensors list, Step s) {
    __shared__ uint32_t most[2][4];
    read_step(s);
    int k = 0;
    while (k + 1 < list.count && list.first[k + 1] <= (int)blockIdx.x) ++k;
    const libra_adamw_tensor_t t = list.t[k];
    const int64_t block = list.begin[k] + (blockIdx.x - list.first[k]), i = block * STATE_BLOCK + threadIdx.x;
    const bool real = i < t.n;
    float p = 0.f, g = 0.f, m = 0.f, v = 0.f, r;
    if (real) {
        p = t.master ? t.master[i] : load_as_float(((T *)t.param)[i]);
        g = load_as_float(((const T *)t.grad)[i]);
        if (BITS8) {
            m = e4m3_value(((uint8_t *)t.first)[i]) * t.first_scales[block];
            r = e4m3_value(((uint8_t *)t.second)[i]) * t.second_scales[block];
            v = r * r;
        } else {
            m = ((float *)t.first)[i];
            v = ((float *)t.second)[i];
        }
    }
    const Element e = updated(s, p, g, m, v, r);
    if (real) {
        if (t.master) t.master[i] = e.p;
        ((T *)t.param)[i] = round_to<T>(e.p);
    }
    if (!BITS8) {
        if (real) {
            ((float *)t.first)[i] = e.m;
            ((float *)t.second)[i] = e.v;
        }
        return;
    }
    float scale[2];
    const float x[2] = {e.m, r};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t a = __float_as_uint(fabsf(x[j]));
        if (!real || a >= 0x7f800000u) a = 0;
        for (int d = 32; d; d /= 2) a = max(a, (uint32_t)__shfl_xor((int)a, d));
        if (threadIdx.x % 64 == 0) most[j][threadIdx.x / 64] = a;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t a = max(max(most[j][0], most[j][1]), max(most[j][2], most[j][3]));
        const int ex = max((int)(a >> 23) - 135 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
        scale[j] = __uint_as_float((uint32_t)(ex + 127) << 23);
    }
    if (!real) return;
    const uint32_t key = mix(mix(mix(s.seed) + s.step) + t.number), h = mix(key + (uint32_t)i + (uint32_t)(i >> 32) * 0x9E3779B1u);
    const float chance[2] = {(float)(h & 0xffff) * 0x1p-16f, (float)(h >> 16) * 0x1p-16f};
    const uint32_t sign = __float_as_uint(e.m) >> 31 << 7;
    ((uint8_t *)t.first)[i] = (uint8_t)(e4m3_code(e.m, 1.f / scale[0], chance[0], false) | sign);
    ((uint8_t *)t.second)[i] = (uint8_t)e4m3_code(r, 1.f / scale[1], chance[1], true);
    if (threadIdx.x == 0) {
        t.first_scales[block] = scale[0];
        t.second_scales[block] = scale[1];
    }
}

int check(const libra_adamw_tensor_t &t, bool bits8) {
    if (t.n < 0) return LIBRA_ERR_SHAPE;
    if (t.n > (int64_t)STATE_BLOCK * INT32_MAX / 2) return LIBRA_ERR_TOO_LARGE;
    if (!known_dtype(t.dtype)) return LIBRA_ERR_DTYPE;
    if (t.n == 0) return LIBRA_OK;
    if (!t.param || !t.grad || !t.first || !t.second || (bits8 && (!t.first_scales || !t.second_scales))) return LIBRA_ERR_NULL;
    const size_t state = bits8 ? 1 : 4;
    if (!aligned_to(t.param, dtype_bytes(t.dtype)) || !aligned_to(t.grad, dtype_bytes(t.dtype)) || !aligned_to(t.first, state) || !aligned_to(t.second, state) ||
        !aligned_to(t.master, 4) || (bits8 && (!aligned_to(t.first_scales, 4) || !aligned_to(t.second_scales, 4))))
        return LIBRA_ERR_BUFFER;
    return LIBRA_OK;
}

}  // namespace

extern "C" int libra_adamw(const libra_adamw_tensor_t *tensors, int32_t count, const libra_adamw_opts_t *o, void *stream) {
    if (count < 0) return LIBRA_ERR_SHAPE;
    if (!o || (!tensors && count > 0)) return LIBRA_ERR_NULL;
    if (o->struct_size != sizeof *o || (o->state_bits != 8 && o->state_bits != 32)) return LIBRA_ERR_OPTION;
    if (!(o->beta1 >= 0 && o->beta1 < 1) || !(o->beta2 >= 0 && o->beta2 < 1) || !(o->eps >= 0 && std::isfinite(o->eps)) || !std::isfinite(o->weight_decay) ||
        (!o->lr_dev && !std::isfinite(o->lr)) || (!o->step_dev && o->step < 1))
        return LIBRA_ERR_OPTION;
    if (!aligned_to(o->step_dev, 8) || !aligned_to(o->lr_dev, 4)) return LIBRA_ERR_BUFFER;
    const bool bits8 = o->state_bits == 8;
    for (int32_t k = 0; k < count; ++k)
        if (int rc = check(tensors[k], bits8)) return rc;
    Step s{};
    s.b1 = (float)o->beta1;
    s.b2 = (float)o->beta2;
    s.c1 = (float)(1 - o->beta1);
    s.c2 = (float)(1 - o->beta2);
    s.eps = (float)o->eps;
    s.log_b1 = std::log(o->beta1);
    s.log_b2 = std::log(o->beta2);
    s.lr = o->lr;
    s.decay = o->weight_decay;
    if (!o->step_dev && !o->lr_dev) {
        s.keep = (float)(1 - o->lr * o->weight_decay);
        s.size = (float)(o->lr / (1 - std::pow(o->beta1, (double)o->step)));
        s.root = (float)(1 / std::sqrt(1 - std::pow(o->beta2, (double)o->step)));
    }
    s.step_dev = o->step_dev;
    s.lr_dev = o->lr_dev;
    s.seed = o->seed;
    s.step = (uint32_t)o->step;
    for (int dtype = LIBRA_F16; dtype <= LIBRA_F32; ++dtype) {
        Tensors list;
        int64_t blocks = 0;
        list.count = 0;
        auto launch = [&]() {
            if (!list.count) return LIBRA_OK;
            const int rc = for_dtype(dtype, [&](auto tag) {
                typedef decltype(tag) T;
                if (bits8) hipLaunchKernelGGL((adamw_kernel<T, true>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, list, s);
                else hipLaunchKernelGGL((adamw_kernel<T, false>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, list, s);
                return last_launch();
            });
            list.count = 0;
            blocks = 0;
            return rc;
        };
        for (int32_t k = 0; k < count; ++k) {
            if (tensors[k].dtype != dtype || tensors[k].n == 0) continue;
            const int64_t all = (tensors[k].n + STATE_BLOCK - 1) / STATE_BLOCK;
            for (int64_t begin = 0; begin < all;) {
                if (list.count == LAUNCH_TENSORS || blocks == LAUNCH_BLOCKS)
                    if (int rc = launch()) return rc;
                const int64_t some = std::min(all - begin, LAUNCH_BLOCKS - blocks);
                list.t[list.count] = tensors[k];
                list.first[list.count] = (int32_t)blocks;
                list.begin[list.count++] = begin;
                blocks += some;
                begin += some;
            }
        }
        if (int rc = launch()) return rc;
    }
    return LIBRA_OK;
}
