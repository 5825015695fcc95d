// Rows of a learned table, scaled, and the gradient of the table.
//   out[i] = scale * table[index[i]]            dtable[v] = scale * sum over i with index[i] = v of dout[i]
#include <algorithm>

#include "ends.h"

using namespace libra;

namespace {

template <class T>
__global__ __launch_bounds__(256) void embedding_kernel(const T *table, int64_t rows, int32_t width, int64_t ld_table, const void *index, int index_type, int64_t n,
                                                        float scale, T *out, int64_t ld_out) {
    const int lane = threadIdx.x % WAVE_LANES;
    for (int64_t i = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE_LANES; i < n; i += (int64_t)gridDim.x * 4) {
        const int64_t v = index_at(index, index_type, i);
        const bool known = v >= 0 && v < rows;
        const float other = v == -1 ? 0.f : __builtin_nanf("");
        for (int32_t c = lane; c < width; c += WAVE_LANES)
            out[i * ld_out + c] = round_to<T>(known ? scale * load_as_float(table[v * ld_table + c]) : other);
    }
}

// ---- sorting (key, place) pairs by key, eight bits at a time; equal keys keep their order ----
constexpr int DIGITS = 256, SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / WAVE_LANES, SORT_BATCHES = 16, SORT_TILE = SORT_THREADS * SORT_BATCHES, SORT_BLOCKS = 64;

struct Keys {                       // of one pass: the ids themselves in the first one, pairs afterwards
    const void *index;
    int index_type;
    int64_t rows;
    const uint32_t *key;
    const int32_t *place;
    __device__ uint32_t at(int64_t i) const {
        if (key) return key[i];
        const int64_t v = index_at(index, index_type, i);
        return v >= 0 && v < rows ? (uint32_t)v : (uint32_t)rows;       // what is no row comes last
    }
    __device__ int32_t place_of(int64_t i) const { return key ? place[i] : (int32_t)i; }
};

__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(Keys in, int64_t n, int64_t each, int shift, int32_t *count) {
    __shared__ int32_t seen[DIGITS];
    seen[threadIdx.x] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * each, end = min(n, begin + each);
    for (int64_t i = begin + threadIdx.x; i < end; i += SORT_THREADS) atomicAdd(&seen[(in.at(i) >> shift) & (DIGITS - 1)], 1);
    __syncthreads();
    count[threadIdx.x * gridDim.x + blockIdx.x] = seen[threadIdx.x];
}

// exclusive prefix sums of n counts, one workgroup
__global__ __launch_bounds__(1024) void sort_scan_kernel(int32_t *count, int n) {
    __shared__ int32_t part[1024];
    const int each = (n + 1023) / 1024, begin = min(n, (int)threadIdx.x * each), end = min(n, begin + each);
    int32_t sum = 0;
    for (int i = begin; i < end; ++i) sum += count[i];
    part[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 1; d < 1024; d *= 2) {
        const int32_t before = (int)threadIdx.x >= d ? part[threadIdx.x - d] : 0;
        __syncthreads();
        part[threadIdx.x] += before;
        __syncthreads();
    }
    sum = part[threadIdx.x] - sum;
    for (int i = begin; i < end; ++i) {
        const int32_t c = count[i];
        count[i] = sum;
        sum += c;
    }
}

__global__ __launch_bounds__(SORT_THREADS) void sort_place_kernel(Keys in, int64_t n, int64_t each, int shift, const int32_t *first, uint32_t *key_out, int32_t *place_out) {
    __shared__ int32_t next[DIGITS], mine[SORT_WAVES][DIGITS];
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES;
    next[threadIdx.x] = first[threadIdx.x * gridDim.x + blockIdx.x];
    const int64_t begin = (int64_t)blockIdx.x * each, end = min(n, begin + each);
    for (int64_t tile = begin; tile < end; tile += SORT_TILE) {
        for (int w = 0; w < SORT_WAVES; ++w) mine[w][threadIdx.x] = 0;
        __syncthreads();
        uint32_t key[SORT_BATCHES];
        int32_t rank[SORT_BATCHES];
        const int64_t at = tile + (int64_t)wave * (SORT_BATCHES * WAVE_LANES) + lane;
#pragma unroll
        for (int b = 0; b < SORT_BATCHES; ++b) key[b] = at + b * WAVE_LANES < end ? in.at(at + b * WAVE_LANES) : 0;
#pragma unroll
        for (int b = 0; b < SORT_BATCHES; ++b) {
            const bool real = at + b * WAVE_LANES < end;
            const uint32_t digit = (key[b] >> shift) & (DIGITS - 1);
            uint64_t same = __ballot(real);             // lanes with this lane's digit
#pragma unroll
            for (int bit = 0; bit < 8; ++bit) {
                const uint64_t set = __ballot((digit >> bit) & 1);
                same &= (digit >> bit) & 1 ? set : ~set;
            }
            const int before = __popcll(same & ((1ull << lane) - 1));
            int32_t base = 0;
            if (real && before == 0) base = atomicAdd(&mine[wave][digit], (int32_t)__popcll(same));
            rank[b] = __shfl(base, real ? __ffsll((unsigned long long)same) - 1 : 0) + before;
        }
        __syncthreads();
        int32_t place = next[threadIdx.x];
        for (int w = 0; w < SORT_WAVES; ++w) {
            const int32_t c = mine[w][threadIdx.x];
            mine[w][threadIdx.x] = place;
            place += c;
        }
        next[threadIdx.x] = place;
        __syncthreads();
#pragma unroll
        for (int b = 0; b < SORT_BATCHES; ++b) {
            const int64_t i = at + b * WAVE_LANES;
            if (i >= end) continue;
            const int32_t to = mine[wave][(key[b] >> shift) & (DIGITS - 1)] + rank[b];
            key_out[to] = key[b];
            place_out[to] = in.place_of(i);
        }
        __syncthreads();
    }
}

// first of n sorted keys that is not below `v`
__device__ inline int64_t first_not_below(const uint32_t *key, int64_t n, uint32_t v) {
    int64_t low = 0, high = n;
    while (low < high) {
        const int64_t mid = (low + high) / 2;
        if (key[mid] < v) low = mid + 1;
        else high = mid;
    }
    return low;
}

// a wave per row of the table
template <class T>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const T *dout, int64_t ld_dout, const uint32_t *key, const int32_t *place, int64_t n, int64_t rows, int32_t width,
                                                            float scale, T *dtable, int64_t ld_dtable) {
    const int lane = threadIdx.x % WAVE_LANES;
    for (int64_t v = (int64_t)blockIdx.x * 4 + threadIdx.x / WAVE_LANES; v < rows; v += (int64_t)gridDim.x * 4) {
        const int64_t begin = first_not_below(key, n, (uint32_t)v), end = first_not_below(key, n, (uint32_t)v + 1);
        for (int32_t c = lane; c < width; c += WAVE_LANES) {
            float sum = 0.f;
            for (int64_t q = begin; q < end; q += 8) {
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = load_as_float(dout[(int64_t)place[min(q + k, end - 1)] * ld_dout + c]);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (q + k < end) sum += x[k];
            }
            dtable[v * ld_dtable + c] = round_to<T>(scale * sum);
        }
    }
}

struct BackwardWork {
    uint32_t *key[2];
    int32_t *place[2], *count;
    size_t bytes;
};

BackwardWork backward_work(void *base, int64_t n) {
    BackwardWork w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = reinterpret_cast<char *>(base) + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    for (int k = 0; k < 2; ++k) {
        w.key[k] = (uint32_t *)take((size_t)n * 4);
        w.place[k] = (int32_t *)take((size_t)n * 4);
    }
    w.count = (int32_t *)take((size_t)DIGITS * SORT_BLOCKS * 4);
    w.bytes = at;
    return w;
}

int backward_shape(int64_t n, int64_t rows, int32_t width) {
    if (n < 0 || rows < 0 || width < 1) return LIBRA_ERR_SHAPE;
    if (n > INT32_MAX || rows >= INT32_MAX) return LIBRA_ERR_TOO_LARGE;
    return LIBRA_OK;
}

}  // namespace

extern "C" int libra_embedding(const void *table, int64_t rows, int32_t width, int64_t ld_table, int dtype, const void *index, int index_type, int64_t n, float scale,
                               void *out, int64_t ld_out, void *stream) {
    if (n < 0 || rows < 0 || width < 1 || ld_table < width || ld_out < width) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if (!known_index(index_type)) return LIBRA_ERR_OPTION;
    if (n == 0) return LIBRA_OK;
    if (!index || !out || (!table && rows > 0)) return LIBRA_ERR_NULL;
    if (!aligned_to(table, dtype_bytes(dtype)) || !aligned_to(out, dtype_bytes(dtype)) || !aligned_to(index, index_bytes(index_type))) return LIBRA_ERR_BUFFER;
    const unsigned blocks = (unsigned)std::min<int64_t>((n + 3) / 4, 1 << 16);
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((embedding_kernel<T>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, (const T *)table, rows, width, ld_table, index, index_type, n, scale,
                           (T *)out, ld_out);
        return last_launch();
    });
}

extern "C" int libra_embedding_backward_workspace(int64_t n, int64_t rows, int32_t width, size_t *bytes) {
    if (!bytes) return LIBRA_ERR_NULL;
    if (int rc = backward_shape(n, rows, width)) return rc;
    *bytes = backward_work(nullptr, n).bytes;
    return LIBRA_OK;
}

extern "C" int libra_embedding_backward(const void *dout, int64_t ld_dout, int dtype, const void *index, int index_type, int64_t n, int64_t rows, int32_t width, float scale,
                                        void *dtable, int64_t ld_dtable, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = backward_shape(n, rows, width)) return rc;
    if (ld_dout < width || ld_dtable < width) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if (!known_index(index_type)) return LIBRA_ERR_OPTION;
    if (rows == 0) return LIBRA_OK;
    if (!dtable || ((!dout || !index || !workspace) && n > 0)) return LIBRA_ERR_NULL;
    if (!aligned_to(dout, dtype_bytes(dtype)) || !aligned_to(dtable, dtype_bytes(dtype)) || !aligned_to(index, index_bytes(index_type))) return LIBRA_ERR_BUFFER;
    const BackwardWork w = backward_work(workspace, n);
    if (n > 0 && (workspace_bytes < w.bytes || !aligned_to(workspace, 256))) return LIBRA_ERR_BUFFER;
    hipStream_t s = (hipStream_t)stream;
    int at = 0;
    if (n > 0) {
        const int64_t tiles = (n + SORT_TILE - 1) / SORT_TILE, blocks = std::min<int64_t>(tiles, SORT_BLOCKS), each = (tiles + blocks - 1) / blocks * SORT_TILE;
        Keys in{index, index_type, rows, nullptr, nullptr};
        for (int shift = 0; shift == 0 || rows >> shift; shift += 8, at ^= 1) {
            hipLaunchKernelGGL(sort_count_kernel, dim3((unsigned)blocks), dim3(SORT_THREADS), 0, s, in, n, each, shift, w.count);
            hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, s, w.count, DIGITS * (int)blocks);
            hipLaunchKernelGGL(sort_place_kernel, dim3((unsigned)blocks), dim3(SORT_THREADS), 0, s, in, n, each, shift, w.count, w.key[at], w.place[at]);
            in.key = w.key[at];
            in.place = w.place[at];
        }
        at ^= 1;
    }
    const unsigned blocks = (unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16);
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((embedding_sum_kernel<T>), dim3(blocks), dim3(256), 0, s, (const T *)dout, ld_dout, w.key[at], w.place[at], n, rows, width, scale, (T *)dtable,
                           ld_dtable);
        return last_launch();
    });
}
