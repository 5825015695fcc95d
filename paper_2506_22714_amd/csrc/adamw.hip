// One AdamW step over many tensors (decoupled weight decay), states in 32 bits or in 8:
//   m <- b1 m + (1 - b1) g      v <- b2 v + (1 - b2) g g      p <- (1 - lr wd) p - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8 bits: m and r = sqrt(v) as e4m3 numbers (OCP, finite ones up to 448) times a power of two for every 256 elements, the smallest
// that keeps the block's largest number within 448.  The root has twice the range of v in octaves.  A number goes up or down to a
// neighbour by chance, in proportion to its distance, because a nearest one would never move: an average over 1,000 steps changes by
// 0.1 % a step, and e4m3 numbers are 6 to 12 % apart.  The chances are a hash of (seed, step, tensor, element), so a step gives the same
// result every time.  A root above zero never becomes zero: it divides.  The new parameter is made from the states before they are rounded.
// No product is contracted with a sum: what is rounded to 8 bits is then the same on every machine with IEEE arithmetic.
//
// Bound by memory: 16.8 M fp32 elements with 32-bit states 90 us, 67 M bf16 with copies in 32 bits and 8-bit states 204 us (5.3 TB/s),
// wherever the tensors begin (by single elements where they are not aligned: 484 us, not 218).  Without the copies 8-bit states are bound
// by the vector ALUs: 167 us, 4.0 TB/s.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "ends.h"

using namespace libra;

namespace {

constexpr int STATE_BLOCK = LIBRA_ADAMW_BLOCK, LAUNCH_TENSORS = 32;
static_assert(LAUNCH_TENSORS % 4 == 0, "searched by fours");
constexpr int64_t LAUNCH_BLOCKS = 1 << 22;      // the threads of a launch are counted in 32 bits

struct Tensors {                    // of one launch, in its arguments: nothing is copied to the device beforehand
    libra_adamw_tensor_t t[LAUNCH_TENSORS];
    int32_t first[LAUNCH_TENSORS];  // workgroup that each begins with
    int64_t begin[LAUNCH_TENSORS];  // and the workgroup of the tensor that this one is
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

// Four e4m3 numbers
__device__ inline void e4m3_values(uint32_t codes, float *x) {
    const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    x[0] = low[0];
    x[1] = low[1];
    x[2] = high[0];
    x[3] = high[1];
}

// |x| / scale, 0 .. 448, to one of its two neighbours; `inverse` is the power of two 1 / scale, the chance is c / 2^16.  From 2^-6 on, where
// a number has four digits, the chance is added below the last of them and what is carried is kept; below 2^-6 the steps are all 2^-9.
__device__ inline uint32_t e4m3_code(float x, float inverse, uint32_t c) {
    const float y = fabsf(x) * inverse;
    uint32_t code = ((__float_as_uint(y) + (c << 4)) >> 20) - (120u << 3);
    if (y < 0x1p-6f) code = (uint32_t)(y * 0x1p9f + (float)c * 0x1p-16f);
    return code;
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
    const float den = s.root * r + s.eps;
    // (the quotient goes into the parameter alone: a reciprocal of one unit in the last place will do, but for numbers it flushes to zero)
    const float q = den > 0x1p-100f && den < 0x1p100f ? e.m * __builtin_amdgcn_rcpf(den) : e.m / den;
    e.p = s.keep * p - s.size * q;
    return e;
}

// N neighbouring numbers from `i` on, in pieces of up to 16 bytes that begin anywhere if `whole`; those from `n` on are zeros, and are not written
template <class T, int N> struct Run {
    T x[N];
    static constexpr int PIECE = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16, PIECES = N * (int)sizeof(T) / PIECE;
    struct __attribute__((packed, aligned(1))) Piece { uint32_t x[PIECE / 4]; };
    __device__ void load(const T *p, int64_t i, int64_t n, bool whole) {
        if (whole) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const Piece q = reinterpret_cast<const Piece *>(p + i)[k];
                __builtin_memcpy(x + k * (N / PIECES), &q, PIECE);
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = i + k < n ? p[i + k] : T(0);
        }
    }
    __device__ void store(T *p, int64_t i, int64_t n, bool whole) const {
        if (whole) {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                Piece q;
                __builtin_memcpy(&q, x + k * (N / PIECES), PIECE);
                reinterpret_cast<Piece *>(p + i)[k] = q;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (i + k < n) p[i + k] = x[k];
        }
    }
};

// Codes of N elements, four in a word
template <int N> __device__ inline void load_codes(Run<uint32_t, N / 4> &r, const uint8_t *p, int64_t i, int64_t n, bool whole) {
    if (whole) r.load(reinterpret_cast<const uint32_t *>(p + i), 0, 0, true);
    else {
        Run<uint8_t, N> bytes;
        bytes.load(p, i, n, false);
        __builtin_memcpy(r.x, bytes.x, N);
    }
}
template <int N> __device__ inline void store_codes(const Run<uint32_t, N / 4> &r, uint8_t *p, int64_t i, int64_t n, bool whole) {
    if (whole) r.store(reinterpret_cast<uint32_t *>(p + i), 0, 0, true);
    else {
        Run<uint8_t, N> bytes;
        __builtin_memcpy(bytes.x, r.x, N);
        bytes.store(p, i, n, false);
    }
}

// A workgroup takes eight blocks of 256 elements, a thread eight neighbouring elements: 32 lanes have a block of 8-bit states.
constexpr int EACH = 8, GROUP_BLOCKS = 256 * EACH / STATE_BLOCK, BLOCK_LANES = STATE_BLOCK / EACH;

template <class T, bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(Tensors list, Step s) {
    read_step(s);
    // the last tensor that begins at this workgroup or before: four at a time (all 32: 14 us of scalar instructions for 67 M elements)
    int k = -1;
    for (int j = 0; j < LAUNCH_TENSORS && list.first[j] <= (int)blockIdx.x; j += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) k += list.first[j + u] <= (int)blockIdx.x;
    const libra_adamw_tensor_t &t = list.t[k];
    const int64_t i = (list.begin[k] + (blockIdx.x - list.first[k])) * (GROUP_BLOCKS * STATE_BLOCK) + threadIdx.x * EACH, n = t.n;
    const bool whole = i + EACH <= n;
    const int64_t block = min(i, n - 1) / STATE_BLOCK;
    Run<T, EACH> p, g;
    Run<float, EACH> w, m, v;
    Run<uint32_t, EACH / 4> first, second;          // four codes each
    float scale[2];
    g.load((const T *)t.grad, i, n, whole);
    if (t.master) w.load(t.master, i, n, whole);
    else p.load((const T *)t.param, i, n, whole);
    if constexpr (BITS8) {
        load_codes<EACH>(first, (const uint8_t *)t.first, i, n, whole);
        load_codes<EACH>(second, (const uint8_t *)t.second, i, n, whole);
        scale[0] = t.first_scales[block];
        scale[1] = t.second_scales[block];
    } else {
        m.load((const float *)t.first, i, n, whole);
        v.load((const float *)t.second, i, n, whole);
    }
    if (!t.master)
#pragma unroll
        for (int e = 0; e < EACH; ++e) w.x[e] = load_as_float(p.x[e]);
    float r[EACH];
    if constexpr (BITS8) {
#pragma unroll
        for (int e = 0; e < EACH; e += 4) {
            e4m3_values(first.x[e / 4], m.x + e);
            e4m3_values(second.x[e / 4], v.x + e);
        }
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if constexpr (BITS8) {
            m.x[e] *= scale[0];
            v.x[e] *= scale[1];
            v.x[e] *= v.x[e];
        }
        const Element u = updated(s, w.x[e], load_as_float(g.x[e]), m.x[e], v.x[e], r[e]);
        w.x[e] = u.p;
        m.x[e] = u.m;
        v.x[e] = u.v;
        p.x[e] = round_to<T>(u.p);
    }
    p.store((T *)t.param, i, n, whole);
    if (t.master) w.store(t.master, i, n, whole);
    if constexpr (!BITS8) {
        m.store((float *)t.first, i, n, whole);
        v.store((float *)t.second, i, n, whole);
    } else {
        const uint32_t key = mix(mix(mix(s.seed) + s.step) + t.number);
        uint32_t most[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < EACH; ++e) {            // (what lies behind the end is zero)
            most[0] = max(most[0], __float_as_uint(fabsf(m.x[e])));
            most[1] = max(most[1], __float_as_uint(r[e]) & 0x7fffffffu);
        }
        const bool odd = __ballot(max(most[0], most[1]) >= 0x7f800000u) != 0;       // an Inf or NaN in this wave
        if (odd) {
            most[0] = most[1] = 0;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const uint32_t a = __float_as_uint(fabsf(m.x[e])), b = __float_as_uint(r[e]) & 0x7fffffffu;
                most[0] = max(most[0], a < 0x7f800000u ? a : 0);
                most[1] = max(most[1], b < 0x7f800000u ? b : 0);
            }
        }
        float inverse[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t a = over_group<BLOCK_LANES>(most[j], [](uint32_t x, uint32_t y) { return max(x, y); });
            const int ex = max((int)(a >> 23) - 135 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
            scale[j] = __uint_as_float((uint32_t)(127 + ex) << 23);
            inverse[j] = __uint_as_float((uint32_t)(127 - ex) << 23);
        }
        const uint32_t place = key + (uint32_t)i + (uint32_t)(i >> 32) * 0x9E3779B1u;      // (eight neighbours have one high word)
#pragma unroll
        for (int q = 0; q < EACH / 4; ++q) {
            uint32_t one = 0, two = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = 4 * q + k;
                const uint32_t h = mix(place + e);
                uint32_t a = e4m3_code(m.x[e], inverse[0], h & 0xffff), b = max(e4m3_code(r[e], inverse[1], h >> 16), min(__float_as_uint(r[e]), 1u));
                if (odd) {
                    if (!(fabsf(m.x[e]) < INFINITY)) a = 127;
                    if (!(r[e] < INFINITY)) b = 127;
                }
                one |= (a | __float_as_uint(m.x[e]) >> 31 << 7) << (8 * k);
                two |= b << (8 * k);
            }
            first.x[q] = one;
            second.x[q] = two;
        }
        store_codes<EACH>(first, (uint8_t *)t.first, i, n, whole);
        store_codes<EACH>(second, (uint8_t *)t.second, i, n, whole);
        if (threadIdx.x % BLOCK_LANES == 0 && i < n) {
            t.first_scales[block] = scale[0];
            t.second_scales[block] = scale[1];
        }
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

// Every array that is written lies apart from all others.  (Gradients may lie on each other, and a copy on its parameter where that is fp32:
// both get the same numbers from the same threads.)  19 tensors: 1 us.
struct Place {
    uintptr_t begin, end;
    bool written;
};
int check_places(const libra_adamw_tensor_t *tensors, int32_t count, bool bits8) {
    Place few[LAUNCH_TENSORS * 7];
    std::unique_ptr<Place[]> many;
    Place *place = few;
    if (count > LAUNCH_TENSORS) {
        many.reset(new (std::nothrow) Place[(size_t)count * 7]);
        if (!(place = many.get())) return LIBRA_ERR_NOMEM;
    }
    size_t places = 0;
    auto add = [&](const void *p, size_t bytes, bool written) { place[places++] = {(uintptr_t)p, (uintptr_t)p + bytes, written}; };
    for (int32_t k = 0; k < count; ++k) {
        const libra_adamw_tensor_t &t = tensors[k];
        if (t.n == 0) continue;
        const size_t n = (size_t)t.n, scales = (n + STATE_BLOCK - 1) / STATE_BLOCK * 4, state = bits8 ? 1 : 4;
        add(t.param, n * dtype_bytes(t.dtype), true);
        add(t.grad, n * dtype_bytes(t.dtype), false);
        add(t.first, n * state, true);
        add(t.second, n * state, true);
        if (bits8) add(t.first_scales, scales, true), add(t.second_scales, scales, true);
        if (t.master && !(t.dtype == LIBRA_F32 && t.master == t.param)) add(t.master, n * 4, true);
    }
    std::sort(place, place + places, [](const Place &a, const Place &b) { return a.begin < b.begin; });
    uintptr_t end = 0, written_end = 0;         // of what begins before
    for (size_t k = 0; k < places; ++k) {
        if (place[k].begin < (place[k].written ? end : written_end)) return LIBRA_ERR_BUFFER;
        end = std::max(end, place[k].end);
        if (place[k].written) written_end = std::max(written_end, place[k].end);
    }
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
    if (int rc = check_places(tensors, count, bits8)) return rc;
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
        int listed = 0;
        auto launch = [&]() {
            if (!listed) return LIBRA_OK;
            for (int j = listed; j < LAUNCH_TENSORS; ++j) list.first[j] = INT32_MAX;
            const int rc = for_dtype(dtype, [&](auto tag) {
                typedef decltype(tag) T;
                if (bits8) hipLaunchKernelGGL((adamw_kernel<T, true>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, list, s);
                else hipLaunchKernelGGL((adamw_kernel<T, false>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, list, s);
                return last_launch();
            });
            listed = 0;
            blocks = 0;
            return rc;
        };
        for (int32_t k = 0; k < count; ++k) {
            if (tensors[k].dtype != dtype || tensors[k].n == 0) continue;
            const libra_adamw_tensor_t &t = tensors[k];
            const int64_t all = (t.n + GROUP_BLOCKS * STATE_BLOCK - 1) / (GROUP_BLOCKS * STATE_BLOCK);
            for (int64_t begin = 0; begin < all;) {
                if (listed == LAUNCH_TENSORS || blocks == LAUNCH_BLOCKS)
                    if (int rc = launch()) return rc;
                const int64_t some = std::min(all - begin, LAUNCH_BLOCKS - blocks);
                list.t[listed] = t;
                list.first[listed] = (int32_t)blocks;
                list.begin[listed++] = begin;
                blocks += some;
                begin += some;
            }
        }
        if (int rc = launch()) return rc;
    }
    return LIBRA_OK;
}
