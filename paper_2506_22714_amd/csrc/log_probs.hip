// Log probabilities of given classes, entropy and the most likely classes of rows of logits, and the gradient.  With
// z_j = scale * (x_j - max x) and s = sum exp(z_j):
//   log p_j = z_j - log s          H = log s - sum exp(z_j) z_j / s
//   dx_j = scale * ([j = target] d + sum_a [j = top_a] d_a - p_j (d + sum_a d_a + e (log p_j + H)))
// where d, d_a and e are the gradients of the target's, the alternatives' log probabilities and the entropy.
//
// The forward pass reads the logits once: maximum, s and sum exp(z) z run along and are rescaled where the maximum grows, and the best
// logits are kept in the lanes of a wave.  The backward pass reads them once more and writes as much.  Both are bound by memory, but 16-bit
// logits and lists of alternatives by the vector ALUs.
#include <algorithm>

#include "ends.h"

using namespace libra;

namespace {

constexpr float INF = __builtin_inff(), LOWEST = -0x1.fffffep127f, LOG2E = 1.44269504088896340736f;
constexpr int MAX_TOP = LIBRA_LOG_PROBS_MAX_TOP, SHORT_CLASSES = 2048 - 7, MAX_PARTS = 64;
constexpr int64_t WAVE_CLASSES = 16384, WAVE_ROWS = 1024;
static_assert(MAX_TOP <= WAVE_LANES, "a list of the best logits has a lane for each");

// NaN if one of them is
__device__ inline float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Whole numbers in the order of the logits, NaN last; a larger one comes first among the alternatives.  Zeros are equal.  Zero is no logit's.
__device__ inline uint32_t rank_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0xffffffffu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float logit_of(uint32_t rank) { return __uint_as_float(rank == 0xffffffffu ? 0x7fc00000u : rank & 0x80000000u ? rank ^ 0x80000000u : ~rank); }
// ... and among equal ones the lower class
__device__ inline uint64_t key_of(float x, uint32_t j) { return (uint64_t)rank_of(x) << 32 | (0xffffffffu - j); }
__device__ inline uint32_t class_of(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ inline uint64_t read_lane(uint64_t x, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

// Maximum, sum of exp(scale (x - maximum)) and sum of exp(scale (x - maximum)) (x - maximum) of some logits
struct Sums {
    float m = -INF, s = 0.f, t = 0.f;
    // these sums with the maximum `m2`, which is not below m
    __device__ void raise(float m2, float c) {
        const float d = m == -INF ? 0.f : m - m2, f = m == -INF ? 0.f : __builtin_amdgcn_exp2f(d * c);
        t = f == 0.f && s == s ? 0.f : f * (t + d * s);
        s *= f;
        m = m2;
    }
    __device__ void join(Sums o, float c) {
        const float m2 = larger(m, o.m);
        raise(m2, c);
        o.raise(m2, c);
        s += o.s;
        t += o.t;
    }
    // N more logits; what is no logit comes as -Inf.  c = scale * log2 e
    template <int N> __device__ void add(const float *x, float most, float c) {
        raise(larger(m, most), c);
        const float base = m == -INF ? 0.f : m;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float d = x[k] - base, e = __builtin_amdgcn_exp2f(d * c);
            s += e;
            t = fmaf(e, fmaxf(d, LOWEST), t);       // 0 where the class is masked; NaN comes with e
        }
    }
};

template <int L> __device__ inline Sums over_group_sums(Sums a, float c) {
    if constexpr (L > 1) {
        const float m = over_group<L>(a.m, larger);
        a.raise(m, c);
        auto add = [](float x, float y) { return x + y; };
        a.s = over_group<L>(a.s, add);
        a.t = over_group<L>(a.t, add);
    }
    return a;
}

struct Forward {
    int64_t n, classes, ld;
    const void *targets;
    int index_type;
    int32_t top;
    float scale;
    float *target_out, *entropy, *top_out, *stats;
    int64_t *top_index;
};

struct Finished {
    float m, logs;
    __device__ float logp(float x, float scale) const { return scale * (x - m) - logs; }
};

// What a row of -Inf has is 0 for the sums' sake: log p = -Inf - 0.
__device__ inline Finished finish(const Sums &a) {
    const bool empty = a.m == -INF;
    return {empty ? 0.f : a.m, empty ? 0.f : logf(a.s)};
}

template <class T> __device__ inline void write_row(const Forward &f, const T *x, int64_t i, const Sums &a, const Finished &r) {
    f.entropy[i] = a.m == -INF ? 0.f : r.logs - f.scale * (a.t / a.s);
    f.stats[2 * i] = a.m;
    f.stats[2 * i + 1] = r.logs;
    if (f.targets) {
        const int64_t j = index_at(f.targets, f.index_type, i);
        f.target_out[i] = j >= 0 && j < f.classes ? r.logp(load_as_float(x[j]), f.scale) : j == -1 ? 0.f : __builtin_nanf("");
    }
}
__device__ inline void write_alternative(const Forward &f, int64_t i, int a, uint64_t key, const Finished &r) {
    f.top_out[i * f.top + a] = r.logp(logit_of((uint32_t)(key >> 32)), f.scale);
    f.top_index[i * f.top + a] = class_of(key);
}

// ---- short rows: L lanes hold a row in registers, E numbers each ----
// They load the 16-byte pieces of memory that the row touches; a piece at an end of the row holds numbers of its neighbours, which count for
// nothing.  (A load for every number where rows are not aligned: 65,536 x 500 bf16 46 us, where these took 22.)
template <class T> struct Span {        // of all rows, and its whole pieces
    const T *low, *high;
    const T *first, *last;              // last < first: there is none
    __device__ Span(const T *p, int64_t n, int64_t classes, int64_t ld) {
        low = p;
        high = p + (n - 1) * ld + classes;
        first = reinterpret_cast<const T *>(((uintptr_t)low + 15) & ~(uintptr_t)15);
        last = reinterpret_cast<const T *>((uintptr_t)high & ~(uintptr_t)15) - VECTOR<T>;
    }
};

template <class T, int L, int E> struct ShortRow {
    static constexpr int W = VECTOR<T>, PIECES = E / W;
    float x[E];
    int before;                         // numbers in the first piece that are not the row's
    __device__ int class_at(int lane, int e) const { return (lane + L * (e / W)) * W + e % W - before; }
    __device__ void load(const Span<T> &span, const T *row, int classes, int lane) {
        before = (int)((uintptr_t)row % 16 / sizeof(T));
        const int end = (before + classes - 1) / W * W - before;        // the row's last piece: also for lanes beyond it
        const T *at[PIECES];
        uint4 raw[PIECES];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            at[p] = row + min(class_at(lane, p * W), end);
            const T *a = at[p] < span.first ? span.first : at[p] > span.last ? span.last : at[p];
            if (span.first <= span.last) raw[p] = *reinterpret_cast<const uint4 *>(a);
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            unpack<T>(raw[p], x + p * W);
            const int j = class_at(lane, p * W);
            if ((at[p] < span.first || at[p] > span.last) && j + W > 0 && j < classes) {       // the ends of the first and the last row
#pragma unroll
                for (int k = 0; k < W; ++k) x[p * W + k] = j + k >= 0 && j + k < classes ? load_as_float(row[j + k]) : -INF;
            }
#pragma unroll
            for (int k = 0; k < W; ++k)
                if (j + k < 0 || j + k >= classes) x[p * W + k] = -INF;
        }
    }
};

// What orders the logits of a short row, larger ones first and lower classes among equals: their 16 bits and the class, or 32 and the class
template <class T> struct ShortKey {
    typedef uint32_t type;
    __device__ static uint32_t of(float x, int j) {
        const T t = round_to<T>(x + 0.f);
        const uint32_t u = __builtin_bit_cast(uint16_t, t);
        return (x != x ? 0xffffu : u & 0x8000u ? ~u & 0xffffu : u | 0x8000u) << 16 | (0xffffu - (uint32_t)j);
    }
    __device__ static float logit(uint32_t key) {
        const uint32_t r = key >> 16;
        return load_as_float(__builtin_bit_cast(T, (uint16_t)(r == 0xffffu ? (uint32_t)__builtin_bit_cast(uint16_t, T(__builtin_nanf(""))) : r & 0x8000u ? r ^ 0x8000u : ~r)));
    }
    __device__ static int64_t class_at(uint32_t key) { return 0xffffu - (key & 0xffffu); }
};
template <> struct ShortKey<float> {
    typedef uint64_t type;
    __device__ static uint64_t of(float x, int j) { return key_of(x, (uint32_t)j); }
    __device__ static float logit(uint64_t key) { return logit_of((uint32_t)(key >> 32)); }
    __device__ static int64_t class_at(uint64_t key) { return class_of(key); }
};

// The best logits one after another: the best of each lane's, then of the group's.  All keys of classes differ.
template <class T, int L, int E> __device__ inline void short_alternatives(const Forward &f, const ShortRow<T, L, E> &row, int64_t i, int lane, bool there, const Finished &r) {
    typedef ShortKey<T> Key;
    typename Key::type key[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int j = row.class_at(lane, e);
        key[e] = j >= 0 && j < f.classes ? Key::of(row.x[e], j) : 0;
    }
    typename Key::type best = 0;
    for (int a = 0; a < f.top; ++a) {
        // key - best wraps round for the keys below the last best, so that the next one has the largest difference
        typename Key::type most = key[0] - best;
#pragma unroll
        for (int e = 1; e < E; ++e) most = key[e] - best > most ? key[e] - best : most;
        best += over_group<L>(most, [](auto p, auto q) { return p > q ? p : q; });
        if (there && lane == a % L) {
            f.top_out[i * f.top + a] = r.logp(Key::logit(best), f.scale);
            f.top_index[i * f.top + a] = Key::class_at(best);
        }
    }
}

// What lane (this ^ MASK) holds
template <int MASK> __device__ inline uint32_t lane_xor(uint32_t x) {
    if constexpr (MASK == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true);             // quad_perm [1,0,3,2]
    else if constexpr (MASK == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true);        // quad_perm [2,3,0,1]
    else if constexpr (MASK == 3) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x1B, 0xf, 0xf, true);        // quad_perm [3,2,1,0]
    else if constexpr (MASK == 4) return lane_xor<7>(lane_xor<3>(x));
    else if constexpr (MASK == 7) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true);       // row_half_mirror
    else if constexpr (MASK == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);       // row_ror:8
    else if constexpr (MASK == 15) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true);      // row_mirror
    else return (uint32_t)__shfl_xor((int)x, MASK);
}
// The larger of the two in the lower lane, the smaller one in the upper
template <int MASK> __device__ inline uint64_t ordered(uint64_t x) {
    const uint64_t other = (uint64_t)lane_xor<MASK>((uint32_t)(x >> 32)) << 32 | lane_xor<MASK>((uint32_t)x);
    const bool upper = ((int)(threadIdx.x % WAVE_LANES) ^ MASK) < (int)(threadIdx.x % WAVE_LANES);
    return (x > other) != upper ? x : other;
}
// A wave's keys into descending order if every half of L lanes is: the halves' pairs from outside in, then smaller and smaller halves
template <int L> __device__ inline uint64_t cleaned(uint64_t x) {
    if constexpr (L == 1) return x;
    else return cleaned<L / 2>(ordered<L / 2>(x));
}
template <int L> __device__ inline uint64_t sorted(uint64_t x) {
    if constexpr (L == 1) return x;
    else return cleaned<L / 2>(ordered<L - 1>(sorted<L / 2>(x)));
}

// The best logits that a wave has seen, in descending order, one in each of the first `top` lanes.
struct Best {
    uint64_t key = 0;               // this lane's
    uint64_t limit = 0;             // the last one of the list; 0 while it is not full
    // every lane brings a key, or 0
    __device__ void insert(uint64_t brought, int top) {
        for (;;) {
            const uint64_t those = __ballot(brought > limit);
            if (!those) return;
            const int lane = 63 - __builtin_clzll(those);
            const uint64_t x = read_lane(brought, lane);
            if ((int)(threadIdx.x % WAVE_LANES) == lane) brought = 0;
            // the list with x: b_k = max(a_k, min(a_(k-1), x))
            const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)(uint32_t)(key >> 32), 0x138, 0xf, 0xf, false);    // wave_shr:1
            const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)(uint32_t)key, 0x138, 0xf, 0xf, false);
            const uint64_t above = (uint64_t)high << 32 | low, place = above < x ? above : x;
            key = key > place ? key : place;
            limit = read_lane(key, top - 1);
        }
    }
    // All of them at once: of two descending lists, one turned round, the larger of each pair of lanes are the best 64, rising and falling once
    __device__ void join(uint64_t brought, int top) {
        const uint64_t x = sorted<WAVE_LANES>(brought), turned = (uint64_t)lane_xor<63>((uint32_t)(x >> 32)) << 32 | lane_xor<63>((uint32_t)x);
        key = cleaned<WAVE_LANES>(key > turned ? key : turned);
        limit = read_lane(key, top - 1);
    }
};

// Logits on their way into a wave's list: one by one, or up to 64 in LDS and then sorted, for a wave with a whole row and a long list.
// Inserting takes some 14 instructions for each, sorting 64 and joining them 230.  65,536 x 1,000 bf16 with 10 / 20 / 64 alternatives
// 76 / 117 / 496 us one by one, 89 / 96 / 226 sorted.  (One kernel with both: 10 % slower where few are asked for.)
constexpr int SORTED_TOP = 14;
template <bool SORTED> struct Waiting {
    uint64_t *keys;                 // of this wave
    int many = 0;
    __device__ void add(bool near, uint64_t key, Best &best, int top) {
        const uint64_t those = __ballot(near);
        if (!those) return;
        if constexpr (SORTED) {
            const int more = (int)__popcll(those);
            if (many + more > WAVE_LANES) flush(best, top);
            if (near) keys[many + __popcll(those & ((1ull << (threadIdx.x % WAVE_LANES)) - 1))] = key;
            many += more;
        } else best.insert(near ? key : 0, top);
    }
    __device__ void flush(Best &best, int top) {
        if constexpr (SORTED) {
            if (!many) return;
            __builtin_amdgcn_wave_barrier();            // a wave's LDS accesses keep their order
            const int lane = threadIdx.x % WAVE_LANES;
            const uint64_t brought = lane < many ? keys[lane] : 0;
            __builtin_amdgcn_wave_barrier();
            if (many > SORTED_TOP) best.join(brought, top);
            else best.insert(brought, top);
            many = 0;
        }
    }
};

// The largest rank of the wave, in a scalar register
__device__ inline uint32_t wave_most(uint32_t x) {
    x = over_group<16>(x, [](uint32_t p, uint32_t q) { return max(p, q); });
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, true));     // row_bcast:15
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, true));     // row_bcast:31
    return (uint32_t)__builtin_amdgcn_readlane((int)x, WAVE_LANES - 1);
}
// The k-th largest of the lanes' ranks
__device__ inline uint32_t wave_kth(uint32_t x, int k) {
    for (;;) {
        const uint32_t most = wave_most(x);
        const uint64_t those = __ballot(x == most);
        k -= (int)__popcll(those);
        if (k <= 0 || most == 0) return most;
        if (x == most) x = 0;
    }
}

// The `top` best of `lists` descending lists of `top` keys in LDS, by one wave: f(a, key), the same key in every lane.
template <class F> __device__ inline void merge_lists(const uint64_t *keys, int lists, int top, F &&f) {
    const int lane = threadIdx.x % WAVE_LANES;
    int at = 0;
    uint64_t head = lane < lists ? keys[lane * top] : 0;
    for (int a = 0; a < top; ++a) {
        const uint32_t rank = wave_most((uint32_t)(head >> 32));
        uint64_t those = __ballot((uint32_t)(head >> 32) == rank);
        if (those & (those - 1)) {                      // several: the lowest class, which has the largest low word
            const uint32_t low = wave_most((uint32_t)(head >> 32) == rank ? (uint32_t)head : 0);
            those = __ballot((uint32_t)(head >> 32) == rank && (uint32_t)head == low);
        }
        const int from = __ffsll((unsigned long long)those) - 1;
        const uint64_t best = read_lane(head, from);
        if (lane == from) {
            ++at;
            head = lane < lists && at < top ? keys[lane * top + at] : 0;
        }
        f(a, best);
    }
}

// All rows of a wave at once.  80 M logits without alternatives, four arrays in turn: 40 classes fp32 83 us (3.8 TB/s), bf16 63 (2.5); 1,000
// classes fp32 64 us (5.0 TB/s), bf16 47 (3.4).  bf16 takes 21 vector instructions for each logit, and the ALUs are busy all the time: unpacking,
// the comparisons with the ends of the row, maximum, difference and its bound, product, exponential, two sums.  131,072 x 40 fp32 8.0 us.
template <class T, int L, int E, bool SORTED> __global__ __launch_bounds__(256) void short_rows_kernel(Forward f, const T *logits) {
    const int lane = threadIdx.x % L;
    const float c = f.scale * LOG2E;
    const Span<T> span(logits, f.n, f.classes, f.ld);
    constexpr int ROWS = 256 / L;
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < f.n; base += (int64_t)gridDim.x * ROWS) {
        const bool there = base + threadIdx.x / L < f.n;
        const int64_t i = there ? base + threadIdx.x / L : f.n - 1;
        ShortRow<T, L, E> row;
        row.load(span, logits + i * f.ld, (int)f.classes, lane);
        float mine = row.x[0];
#pragma unroll
        for (int e = 1; e < E; ++e) mine = larger(mine, row.x[e]);
        Sums a;
        a.template add<E>(row.x, over_group<L>(mine, larger), c);
        auto add = [](float x, float y) { return x + y; };
        a.s = over_group<L>(a.s, add);
        a.t = over_group<L>(a.t, add);
        const Finished r = finish(a);
        if (there && lane == 0) write_row(f, logits + i * f.ld, i, a, r);
        if constexpr (L < WAVE_LANES) {
            if (f.top) short_alternatives(f, row, i, lane, there, r);
        } else if (f.top) {
            // `top` lanes have a maximum that reaches this rank: no logit below it is among the alternatives, and few others reach it.
            // (One after another, as for shorter rows: 65,536 x 1,000 bf16 with 20 251 us, not 96.)
            __shared__ uint64_t keys[SORTED ? 256 / WAVE_LANES : 1][WAVE_LANES];
            const float limit = logit_of(wave_kth(rank_of(mine), f.top));
            Best best;
            Waiting<SORTED> waiting{keys[SORTED ? threadIdx.x / WAVE_LANES : 0]};
#pragma unroll
            for (int e = E - 1; e >= 0; --e) {
                const int j = row.class_at(lane, e);
                const bool near = !(row.x[e] < limit) && j >= 0 && j < f.classes;
                waiting.add(near, key_of(row.x[e], (uint32_t)j), best, f.top);
            }
            waiting.flush(best, f.top);
            if (there && lane < f.top) write_alternative(f, i, lane, best.key, r);
        }
    }
}

// ---- long rows: a workgroup walks a row, or a part of it where there are few rows ----
struct Parts {                      // of rows that several workgroups share
    int32_t count;
    float *sums;                    // 3 for each part of each row
    uint64_t *keys;                 // top for each
};

constexpr int LONG_THREADS = 256, ROUNDS = 16;
enum List { NONE, ONE_BY_ONE, SORTED };      // how the alternatives come

// LDS of the waves of a row: what they exchange
template <int WAVES> struct RowShared {
    float sums[WAVES][3];
    uint64_t keys[WAVES * MAX_TOP];
    uint32_t floor[WAVES];
};
template <> struct RowShared<1> {};
template <int WAVES> __device__ inline void row_barrier() {
    if constexpr (WAVES > 1) __syncthreads();
}
// Which of the workgroup's rows this wave works on, in a scalar register, and with it all that follows from the row
template <int WAVES> __device__ inline int row_of_wave() { return WAVES * WAVE_LANES == LONG_THREADS ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / (WAVES * WAVE_LANES)); }

// WAVES waves for a row or a part of it, 4 / WAVES rows for a workgroup.  A thread takes 16 logits a round.  The alternatives are looked for
// after every sixteen rounds: each thread has kept the maximum of each of its rounds, and if every wave has `share` maxima that reach a rank,
// the row has `top` logits that do, so that only the few rounds of a thread that reach it are read again, a lane each, and their logits go
// through the list.  (After every eight rounds: 5,000 x 50,000 bf16 with 20 alternatives 137 us, not 123.)
// 8,191 x 32,768 fp16, forward, in us with 0 / 1 / 5 / 20 / 64 alternatives: 100 / 110 / 118 / 138 / 188.  When this way was chosen it took
// 94 / 122 / 123 / 145 / 216; looking at every logit as it comes by, with the same bound, 99 / 129 / 151 / 203 / 350, with each wave's own
// list as the bound 97 / 129 / 191 / 364 / 757.  (Two rounds in flight instead of one: 5 to 14 % slower, fewer waves fit.)
// A kernel of its own without alternatives has 60 registers, not 79 (16-bit logits): 20,000 classes 5.4 TB/s, not 5.0.  With them six waves on a
// SIMD are asked for where that spills nothing: 16-bit logits, 12,000 classes by workgroups 3.0 TB/s, not 2.9; 32-bit ones would spill.
template <class T, int WAVES, List LIST> __global__ __launch_bounds__(LONG_THREADS, LIST != NONE && sizeof(T) == 2 ? 6 : 1) void long_rows_kernel(Forward f, const T *logits, Parts parts) {
    constexpr int W = VECTOR<T>, U = 16 / W, N = U * W, THREADS = WAVES * WAVE_LANES, ROUND = U * THREADS, ROWS = LONG_THREADS / THREADS;
    __shared__ RowShared<WAVES> shared;
    __shared__ float maxima[ROUNDS][LONG_THREADS];
    __shared__ uint16_t reaching[LONG_THREADS / WAVE_LANES][ROUNDS * WAVE_LANES];
    __shared__ uint64_t keys[LIST == SORTED ? LONG_THREADS / WAVE_LANES : 1][WAVE_LANES];
    const int share = (f.top + WAVES - 1) / WAVES;
    const int lane = threadIdx.x % WAVE_LANES, in_group = threadIdx.x / WAVE_LANES, wave = in_group % WAVES, thread = threadIdx.x % THREADS;
    const float c = f.scale * LOG2E;
    for (int64_t unit = (int64_t)blockIdx.x * ROWS + row_of_wave<WAVES>(); unit < f.n * parts.count; unit += (int64_t)gridDim.x * ROWS) {
        const int64_t i = unit / parts.count;
        const int part = (int)(unit % parts.count);
        const T *x = logits + i * f.ld;
        // 16-byte pieces of memory.  The first and the last, which hold other things beside the row, are loaded from where all is the row's; so is
        // what lies behind: every lane loads.  The numbers of other pieces are left out when they come.
        const int before = (int)((uintptr_t)x % 16 / sizeof(T));
        const int32_t pieces = (int32_t)((before + f.classes + W - 1) / W), each = (pieces + parts.count - 1) / parts.count, begin = part * each, end = min(pieces, begin + each);
        const int32_t first_whole = before ? 1 : 0, last_whole = min(end, (int32_t)((before + f.classes) / W)) - ROUND;
        auto class_of_piece = [&](int32_t p) { return min(max((int64_t)p * W - before, (int64_t)0), f.classes - W); };
        auto is_of_piece = [&](int32_t p, int64_t j) { return p < end && j >= (int64_t)p * W - before && j < (int64_t)p * W - before + W; };
        auto inside = [&](int32_t v0) { return v0 >= first_whole && v0 <= last_whole; };
        auto fetch = [&](int32_t v0, uint4 *raw) {
            if (v0 >= end) return;
            if (inside(v0)) {
                const uint4 *from = reinterpret_cast<const uint4 *>(x - before) + v0;
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = from[u * THREADS + thread];
                return;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = __builtin_bit_cast(uint4, *reinterpret_cast<const Unaligned *>(x + class_of_piece(v0 + thread + u * THREADS)));
        };
        Sums a;
        Best best;
        Waiting<LIST == SORTED> waiting{keys[LIST == SORTED ? in_group : 0]};
        uint32_t floor = 0;             // what this wave has shown of the row
        uint4 raw[U], next[U];
        fetch(begin, raw);
        for (int32_t super = begin; super < end; super += ROUNDS * ROUND) {
            int rounds = 0;
            float super_most = -INF;
            for (int32_t v0 = super; rounds < ROUNDS && v0 < end; v0 += ROUND, ++rounds) {
                fetch(v0 + ROUND, next);                // on its way while this one is worked on
                float y[N];
#pragma unroll
                for (int u = 0; u < U; ++u) unpack<T>(raw[u], y + u * W);
                if (!inside(v0)) {
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int32_t p = v0 + thread + (k / W) * THREADS;
                        if (!is_of_piece(p, class_of_piece(p) + k % W)) y[k] = -INF;
                    }
                }
                float most = y[0];
#pragma unroll
                for (int k = 1; k < N; ++k) most = larger(most, y[k]);
                a.template add<N>(y, most, c);
                if constexpr (LIST != NONE) {
                    maxima[rounds][threadIdx.x] = most;
                    super_most = rounds ? larger(super_most, most) : most;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = next[u];
            }
            if constexpr (LIST == NONE) continue;
            const uint32_t largest = rank_of(super_most);
            floor = max(floor, wave_kth(largest, share));
            uint32_t least = floor;
            if constexpr (WAVES > 1) {
                if (lane == 0) shared.floor[wave] = floor;
                __syncthreads();
                least = shared.floor[0];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) least = min(least, shared.floor[w]);
                // (a wave with masked classes alone, or none, shows nothing: then this wave's own)
                if (least <= rank_of(-INF)) least = max(least, wave_kth(largest, f.top));
            }
            least = max(least, (uint32_t)(best.limit >> 32));
            int many = 0;
            for (int r = 0; r < rounds; ++r) {
                const bool there = rank_of(maxima[r][threadIdx.x]) >= least;
                const uint64_t those = __ballot(there);
                if (there) reaching[in_group][many + __popcll(those & ((1ull << lane) - 1))] = (uint16_t)(r * WAVE_LANES + lane);
                many += (int)__popcll(those);
            }
            __builtin_amdgcn_wave_barrier();
            for (int q = 0; q < many; q += WAVE_LANES) {
                const int at = reaching[in_group][min(q + lane, many - 1)];
                const int32_t v = super + (at / WAVE_LANES) * ROUND + wave * WAVE_LANES + at % WAVE_LANES;
                // the best that these logits can be: their maximum, of the lowest class (rows of equal logits, masked ones among them, have little to read)
                const uint32_t lowest = (uint32_t)max((int64_t)v * W - before, (int64_t)0);
                const bool there = q + lane < many && ((uint64_t)rank_of(maxima[at / WAVE_LANES][in_group * WAVE_LANES + at % WAVE_LANES]) << 32 | (0xffffffffu - lowest)) > best.limit;
                if (!__ballot(there)) continue;
                uint4 again[U];
                float y[N];
#pragma unroll
                for (int u = 0; u < U; ++u) again[u] = __builtin_bit_cast(uint4, *reinterpret_cast<const Unaligned *>(x + class_of_piece(v + u * THREADS)));
#pragma unroll
                for (int u = 0; u < U; ++u) unpack<T>(again[u], y + u * W);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int32_t p = v + (k / W) * THREADS;
                    const int64_t j = class_of_piece(p) + k % W;
                    const bool near = there && rank_of(y[k]) >= least && is_of_piece(p, j);
                    waiting.add(near, key_of(y[k], (uint32_t)j), best, f.top);
                }
            }
            waiting.flush(best, f.top);
            floor = max(floor, (uint32_t)(read_lane(best.key, share - 1) >> 32));
            row_barrier<WAVES>();           // the bounds have been read
        }
        a = over_group_sums<WAVE_LANES>(a, c);
        if constexpr (WAVES == 1) {         // (never a part)
            const Finished r = finish(a);
            if (lane == 0) write_row(f, x, i, a, r);
            if (LIST != NONE && lane < f.top) write_alternative(f, i, lane, best.key, r);
        } else {
            if (lane == 0) shared.sums[wave][0] = a.m, shared.sums[wave][1] = a.s, shared.sums[wave][2] = a.t;
            if (LIST != NONE && lane < f.top) shared.keys[wave * f.top + lane] = best.key;
            __syncthreads();
            if (wave == 0) {
                a = Sums{};
                for (int w = 0; w < WAVES; ++w) a.join(Sums{shared.sums[w][0], shared.sums[w][1], shared.sums[w][2]}, c);
                if (parts.count == 1) {
                    const Finished r = finish(a);
                    if (lane == 0) write_row(f, x, i, a, r);
                    if (LIST != NONE) merge_lists(shared.keys, WAVES, f.top, [&](int k, uint64_t key) {
                        if (lane == 0) write_alternative(f, i, k, key, r);
                    });
                } else {
                    if (lane == 0) parts.sums[3 * unit] = a.m, parts.sums[3 * unit + 1] = a.s, parts.sums[3 * unit + 2] = a.t;
                    if (LIST != NONE) merge_lists(shared.keys, WAVES, f.top, [&](int k, uint64_t key) {
                        if (lane == 0) parts.keys[unit * f.top + k] = key;
                    });
                }
            }
            __syncthreads();
        }
    }
}

// a workgroup joins the parts of a row
template <class T> __global__ __launch_bounds__(256) void join_parts_kernel(Forward f, const T *logits, Parts parts) {
    extern __shared__ uint64_t keys[];
    const int lane = threadIdx.x % WAVE_LANES;
    const float c = f.scale * LOG2E;
    for (int64_t i = blockIdx.x; i < f.n; i += gridDim.x) {
        for (int k = threadIdx.x; k < parts.count * f.top; k += 256) keys[k] = parts.keys[i * parts.count * f.top + k];
        __syncthreads();
        if (threadIdx.x < WAVE_LANES) {
            Sums a;
            if (lane < parts.count) {
                const float *p = parts.sums + 3 * (i * parts.count + lane);
                a = Sums{p[0], p[1], p[2]};
            }
            a = over_group_sums<WAVE_LANES>(a, c);
            const Finished r = finish(a);
            if (lane == 0) write_row(f, logits + i * f.ld, i, a, r);
            if (f.top) merge_lists(keys, parts.count, f.top, [&](int k, uint64_t key) {
                if (lane == 0) write_alternative(f, i, k, key, r);
            });
        }
        __syncthreads();
    }
}

// ---- gradient ----
struct Backward {
    int64_t n, classes, ld, ld_out;
    const void *targets;
    int index_type;
    int32_t top;
    float scale;
    const float *entropy, *stats, *d_target, *d_entropy, *d_top;
    const int64_t *top_index;
};

// dx_j = p_j (a + b log p_j) plus what the target and the alternatives get on top; a = -scale (d + sum d_a + e H), b = -scale e
struct RowGradient {
    float m, logs, a, b, d;
    int64_t target;
    bool empty;
    // L lanes, which all come here, for a row; the rows' lanes share the alternatives
    template <int L> __device__ void load(const Backward &g, int64_t i, int lane) {
        const float e = g.d_entropy ? g.d_entropy[i] : 0.f, h = g.entropy[i], given = g.d_target ? g.d_target[i] : 0.f;
        float all = 0.f;
        if (g.d_top) {
            for (int k = lane; k < g.top; k += L) all += g.d_top[i * g.top + k];
            all = over_group<L>(all, [](float x, float y) { return x + y; });
        }
        m = g.stats[2 * i];
        logs = g.stats[2 * i + 1];
        empty = m == -INF;
        target = g.targets ? index_at(g.targets, g.index_type, i) : -1;
        d = target == -1 ? 0.f : target >= 0 && target < g.classes ? given : __builtin_nanf("");
        if (!g.d_target) d = 0.f;
        a = -g.scale * fmaf(e, h, d + all);
        b = -g.scale * e;
    }
    __device__ float at(float x, float scale) const {
        const float logp = fmaf(scale, x - m, -logs), p = __builtin_amdgcn_exp2f(logp * LOG2E);
        // p = 0 below -104, for masked classes too, where b log p must not become infinite; NaN comes with p
        return empty ? 0.f : p * fmaf(b, fmaxf(logp, -128.f), a);
    }
};

// The alternatives' classes are written a second time, whole, by a lane each.  (In the registers that hold them: 65,536 x 1,000 bf16 with 20
// alternatives 186 us, not 70.)
template <class T, int L, int E> __global__ __launch_bounds__(256) void short_rows_backward_kernel(Backward g, const T *logits, T *out) {
    typedef ShortRow<T, L, E> Row;
    const int lane = threadIdx.x % L;
    const Span<T> span(logits, g.n, g.classes, g.ld);
    constexpr int ROWS = 256 / L;
    for (int64_t base = (int64_t)blockIdx.x * ROWS; base < g.n; base += (int64_t)gridDim.x * ROWS) {
        const bool there = base + threadIdx.x / L < g.n;
        const int64_t i = there ? base + threadIdx.x / L : g.n - 1;
        const T *x = logits + i * g.ld;
        T *o = out + i * g.ld_out;
        Row row;
        row.load(span, x, (int)g.classes, lane);
        RowGradient r;
        r.template load<L>(g, i, lane);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            row.x[e] = r.at(row.x[e], g.scale);
            if (row.class_at(lane, e) == r.target && !r.empty) row.x[e] = fmaf(g.scale, r.d, row.x[e]);
        }
        if (there) {
#pragma unroll
            for (int p = 0; p < Row::PIECES; ++p) {
                const int j = row.class_at(lane, p * Row::W);
                if (j >= 0 && j + Row::W <= g.classes) *reinterpret_cast<Unaligned *>(o + j) = __builtin_bit_cast(Unaligned, pack<T>(row.x + p * Row::W));
                else {
#pragma unroll
                    for (int k = 0; k < Row::W; ++k)
                        if (j + k >= 0 && j + k < g.classes) o[j + k] = round_to<T>(row.x[p * Row::W + k]);
                }
            }
        }
        if (g.d_top) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");      // behind what this wave has written
            for (int k = lane; k < g.top; k += L) {
                const int64_t j = g.top_index[i * g.top + k];
                if (there && !r.empty && j >= 0 && j < g.classes)
                    o[j] = round_to<T>(fmaf(g.scale, g.d_top[i * g.top + k] + (j == r.target ? r.d : 0.f), r.at(load_as_float(x[j]), g.scale)));
            }
        }
    }
}

// WAVES waves take a run of pieces of a row; the target and the alternatives, which get more than p_j times a sum, are written a second time,
// whole.  Rows are taken from the last to the first: the forward pass has just read the last ones.  8,191 x 32,768 bf16: 185 us, a copy of
// these bytes 203.  (The ends of a row with a load for every piece and number in a branch: 2,677 classes bf16 3.1 TB/s, not 5.1.)
template <class T, int WAVES> __global__ __launch_bounds__(LONG_THREADS) void long_rows_backward_kernel(Backward g, const T *logits, T *out, int32_t runs) {
    constexpr int W = VECTOR<T>, U = 32 / W, THREADS = WAVES * WAVE_LANES, ROWS = LONG_THREADS / THREADS;
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES % WAVES, thread = threadIdx.x % THREADS;
    for (int64_t unit = (int64_t)blockIdx.x * ROWS + row_of_wave<WAVES>(); unit < g.n * runs; unit += (int64_t)gridDim.x * ROWS) {
        const int64_t i = g.n - 1 - unit / runs, run = unit % runs;
        const T *x = logits + i * g.ld;
        T *o = out + i * g.ld_out;
        const int before = (int)((uintptr_t)x % 16 / sizeof(T));
        const int64_t first = run * (U * THREADS), low = first * W - before, high = low + (int64_t)U * THREADS * W;
        RowGradient r;
        if (low >= 0 && high <= g.classes) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = *reinterpret_cast<const uint4 *>(x + low + (u * THREADS + thread) * W);
            r.load<WAVE_LANES>(g, i, lane);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float y[W];
                unpack<T>(raw[u], y);
#pragma unroll
                for (int k = 0; k < W; ++k) y[k] = r.at(y[k], g.scale);
                *reinterpret_cast<Unaligned *>(o + low + (u * THREADS + thread) * W) = __builtin_bit_cast(Unaligned, pack<T>(y));
            }
        } else {
            // the first and the last run of a row: a piece that it shares with its neighbours is loaded from where it is the row's alone, and
            // what belongs to it is stored element by element
            uint4 raw[U];
            int64_t c[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                c[u] = min(max(low + (u * THREADS + thread) * W, (int64_t)0), g.classes - W);
                if (low + u * THREADS * W < g.classes) raw[u] = __builtin_bit_cast(uint4, *reinterpret_cast<const Unaligned *>(x + c[u]));
            }
            r.load<WAVE_LANES>(g, i, lane);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (low + u * THREADS * W >= g.classes) break;
                const int64_t j = low + (u * THREADS + thread) * W;
                float y[W];
                unpack<T>(raw[u], y);
#pragma unroll
                for (int k = 0; k < W; ++k) y[k] = r.at(y[k], g.scale);
                if (j == c[u]) *reinterpret_cast<Unaligned *>(o + j) = __builtin_bit_cast(Unaligned, pack<T>(y));
                else {
#pragma unroll
                    for (int k = 0; k < W; ++k)
                        if (c[u] + k >= j && c[u] + k < j + W) o[c[u] + k] = round_to<T>(y[k]);
                }
            }
        }
        if (r.empty || (r.target < 0 && !g.d_top)) continue;        // the same for all waves of the row
        row_barrier<WAVES>();
        if constexpr (WAVES == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        // the alternatives by a lane each, and the target unless it is among them
        if (wave == 0) {
            const bool listed = g.d_top && lane < g.top;
            const int64_t j = listed ? g.top_index[i * g.top + lane] : -1;
            const bool among = __ballot(listed && j == r.target) != 0;
            auto write = [&](int64_t j, float more) {
                if (j >= 0 && j >= low && j < high && j < g.classes) o[j] = round_to<T>(fmaf(g.scale, more, r.at(load_as_float(x[j]), g.scale)));
            };
            if (listed) write(j, g.d_top[i * g.top + lane] + (j == r.target ? r.d : 0.f));
            if (lane == 0 && !among) write(r.target, r.d);
        }
        row_barrier<WAVES>();
    }
}

int shape(int64_t n, int64_t classes, int32_t top) {
    if (n < 0 || classes < 1 || top < 0 || top > classes) return LIBRA_ERR_SHAPE;
    if (n > INT32_MAX || classes > INT32_MAX) return LIBRA_ERR_TOO_LARGE;
    if (top > MAX_TOP) return LIBRA_ERR_UNSUPPORTED;
    return LIBRA_OK;
}

// A wave for a row of few rounds, if there are rows for all compute units then; otherwise a workgroup, whose waves have to wait for each other.
// In us with 0 / 1 / 10 alternatives, bf16, by waves and by workgroups: 8,192 x 2,100 14 / 20 / 25 and 25 / 51 / 66, 8,192 x 8,192 27 / 34 / 39
// and 28 / 51 / 66, 4,096 x 12,000 19 / 25 / 31 and 21 / 34 / 42; 1,024 x 4,000 5.1 / 8.3 / 10.2 and 5.4 / 10.3 / 13.8, but 1,024 x 12,000
// 9.2 / 14.9 / 18.6 and 8.2 / 12.7 / 16.2, 256 x 20,000 13 / 21 / 26 and 9 / 14 / 19.
bool wave_rows(int64_t n, int64_t classes) { return n >= WAVE_ROWS && classes <= std::min(WAVE_CLASSES, 4 * n); }

// Parts of a long row: as many as keep all workgroups on the compute units at once (six on each of 256: their registers), a part having a
// round of loads at least.  (Rounded up to 2,048: 1,000 x 50,000 bf16 26.5 us and with 20 alternatives 51.6, not 20.8 and 36.9; to 1,792: 800 x 20,000 14.1,
// not 10.0.)
int32_t part_count(int64_t n, int64_t classes) {
    if (classes <= SHORT_CLASSES || wave_rows(n, classes)) return 1;
    const int64_t wanted = 1536 / n, most = (classes + 4095) / 4096;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min(wanted, most), MAX_PARTS));
}

// (times log2 e a larger one is infinite)
bool known_scale(float scale) { return scale > 0.f && scale <= 0x1p127f; }

size_t part_bytes(int64_t n, int32_t count, int32_t top) { return count == 1 ? 0 : ((size_t)n * count * 12 + 255) / 256 * 256 + (size_t)n * count * top * 8; }

// f(lanes of a row, numbers of a lane) for rows that with their neighbours' numbers in the first piece have `numbers`; a lane has EACH or
// half as many again of rows of 17 to 768.  (Without the halves 300 classes bf16 2.5 TB/s, not 3.2, 1,100 2.3, not 3.0: idle lanes.)
template <int EACH, class F> int for_short(int64_t numbers, F &&f) {
#define LIBRA_SHORT(L, E) \
    if (numbers <= L * E) return f(std::integral_constant<int, L>{}, std::integral_constant<int, E>{});
    LIBRA_SHORT(1, 16)
    LIBRA_SHORT(32 / EACH, EACH)
    if constexpr (EACH == 16) LIBRA_SHORT(2, 24)        // (three pieces for 8: 40 classes, backward, 4.3 TB/s, not 5.2)
    LIBRA_SHORT(64 / EACH, EACH)
    if constexpr (EACH == 16) LIBRA_SHORT(4, 24)
    LIBRA_SHORT(128 / EACH, EACH)
    LIBRA_SHORT(128 / EACH, EACH * 3 / 2)
    LIBRA_SHORT(256 / EACH, EACH)
    LIBRA_SHORT(256 / EACH, EACH * 3 / 2)
    LIBRA_SHORT(512 / EACH, EACH)
    LIBRA_SHORT(512 / EACH, EACH * 3 / 2)
    LIBRA_SHORT(64, 16)
    LIBRA_SHORT(64, 24)
#undef LIBRA_SHORT
    return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 32>{});
}
template <class T> int64_t short_numbers(const T *x, int64_t classes, int64_t ld) { return classes + (aligned_to(x, 16) && ld % VECTOR<T> == 0 ? 0 : VECTOR<T> - 1); }

constexpr int64_t MOST_WORKGROUPS = 1 << 23;        // the threads of a launch are counted in 32 bits

}  // namespace

extern "C" int libra_log_probs_workspace(int64_t n, int64_t classes, int32_t top, size_t *bytes) {
    if (!bytes) return LIBRA_ERR_NULL;
    if (int rc = shape(n, classes, top)) return rc;
    *bytes = n ? part_bytes(n, part_count(n, classes), top) : 0;
    return LIBRA_OK;
}

extern "C" int libra_log_probs(const void *logits, int64_t n, int64_t classes, int64_t ld, int dtype, const void *targets, int index_type, int32_t top, float scale,
                               float *target_out, float *entropy, float *top_out, int64_t *top_index, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = shape(n, classes, top)) return rc;
    if (ld < classes) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if ((targets && !known_index(index_type)) || !known_scale(scale)) return LIBRA_ERR_OPTION;
    if (n == 0) return LIBRA_OK;
    if (!logits || !entropy || !stats || (targets && !target_out) || (top && (!top_out || !top_index))) return LIBRA_ERR_NULL;
    if (!aligned_to(logits, dtype_bytes(dtype)) || (targets && !aligned_to(targets, index_bytes(index_type))) || !aligned_to(target_out, 4) || !aligned_to(entropy, 4) ||
        !aligned_to(top_out, 4) || !aligned_to(top_index, 8) || !aligned_to(stats, 4))
        return LIBRA_ERR_BUFFER;
    Parts parts{part_count(n, classes), nullptr, nullptr};
    if (const size_t need = part_bytes(n, parts.count, top)) {
        if (!workspace) return LIBRA_ERR_NULL;
        if (workspace_bytes < need || !aligned_to(workspace, 256)) return LIBRA_ERR_BUFFER;
        parts.sums = (float *)workspace;
        parts.keys = (uint64_t *)((char *)workspace + ((size_t)n * parts.count * 12 + 255) / 256 * 256);
    }
    const Forward f{n, classes, ld, targets, index_type, top, scale, target_out, entropy, top_out, stats, top_index};
    hipStream_t s = (hipStream_t)stream;
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        const T *x = (const T *)logits;
        if (classes <= SHORT_CLASSES) {
            const int64_t numbers = short_numbers(x, classes, ld);
            auto launch = [&](auto lanes, auto each) {
                constexpr int L = decltype(lanes)::value, E = decltype(each)::value;
                const unsigned blocks = (unsigned)std::min<int64_t>((n * L + 255) / 256, MOST_WORKGROUPS);
                if constexpr (L == WAVE_LANES) if (top > SORTED_TOP) {
                    hipLaunchKernelGGL((short_rows_kernel<T, L, E, true>), dim3(blocks), dim3(256), 0, s, f, x);
                    return last_launch();
                }
                hipLaunchKernelGGL((short_rows_kernel<T, L, E, false>), dim3(blocks), dim3(256), 0, s, f, x);
                return last_launch();
            };
            // A wave's list takes several alternatives of 32-bit logits sooner than 32 lanes with keys of 64 bits: 512 classes, 10 of them, 2.2 TB/s,
            // not 1.6, but 4.8 without alternatives, not 5.9
            if constexpr (sizeof(T) == 4) if (numbers > 256 && numbers <= 768 && top > 1)
                return numbers <= 512 ? launch(std::integral_constant<int, 64>{}, std::integral_constant<int, 8>{})
                                      : launch(std::integral_constant<int, 64>{}, std::integral_constant<int, 12>{});
            return for_short<16>(numbers, launch);
        }
        auto launch = [&](auto waves, auto list) {
            constexpr int WAVES = decltype(waves)::value, ROWS = LONG_THREADS / WAVE_LANES / WAVES;
            const int64_t groups = (n * parts.count + ROWS - 1) / ROWS;
            hipLaunchKernelGGL((long_rows_kernel<T, WAVES, decltype(list)::value>), dim3((unsigned)std::min(groups, MOST_WORKGROUPS)), dim3(LONG_THREADS), 0, s, f, x, parts);
        };
        const std::integral_constant<int, 1> wave;
        const std::integral_constant<int, 4> workgroup;
        const std::integral_constant<List, NONE> none;
        const std::integral_constant<List, ONE_BY_ONE> one_by_one;
        if (!wave_rows(n, classes)) top ? launch(workgroup, one_by_one) : launch(workgroup, none);
        else if (top > SORTED_TOP) launch(wave, std::integral_constant<List, SORTED>{});
        else top ? launch(wave, one_by_one) : launch(wave, none);
        if (parts.count > 1)
            hipLaunchKernelGGL((join_parts_kernel<T>), dim3((unsigned)std::min<int64_t>(n, MOST_WORKGROUPS)), dim3(256), (size_t)parts.count * top * 8, s, f, x, parts);
        return last_launch();
    });
}

extern "C" int libra_log_probs_backward(const void *logits, int64_t n, int64_t classes, int64_t ld, int dtype, const void *targets, int index_type, int32_t top, float scale,
                                        const float *entropy, const float *stats, const int64_t *top_index, const float *d_target, const float *d_entropy, const float *d_top,
                                        void *dlogits, int64_t ld_dlogits, void *stream) {
    if (int rc = shape(n, classes, top)) return rc;
    if (ld < classes || ld_dlogits < classes) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if ((targets && !known_index(index_type)) || !known_scale(scale)) return LIBRA_ERR_OPTION;
    if (n == 0) return LIBRA_OK;
    if (!logits || !entropy || !stats || !dlogits || (d_target && !targets) || (top && d_top && !top_index)) return LIBRA_ERR_NULL;
    if (!aligned_to(logits, dtype_bytes(dtype)) || !aligned_to(dlogits, dtype_bytes(dtype)) || (targets && !aligned_to(targets, index_bytes(index_type))) ||
        !aligned_to(entropy, 4) || !aligned_to(stats, 4) || !aligned_to(top_index, 8) || !aligned_to(d_target, 4) || !aligned_to(d_entropy, 4) || !aligned_to(d_top, 4))
        return LIBRA_ERR_BUFFER;
    const Backward g{n, classes, ld, ld_dlogits, targets, index_type, top, scale, entropy, stats, d_target, d_entropy, top ? d_top : nullptr, top_index};
    hipStream_t s = (hipStream_t)stream;
    return for_dtype(dtype, [&](auto tag) {
        typedef decltype(tag) T;
        const T *x = (const T *)logits;
        T *o = (T *)dlogits;
        // (with more than 16 logits a lane fewer waves fit: 1,100 classes bf16 2.9 TB/s, not 4.3 as below; 768 classes 5.1, not 4.2)
        if (classes <= SHORT_CLASSES / 2) return for_short<2 * VECTOR<T>>(short_numbers(x, classes, ld), [&](auto lanes, auto each) {
            constexpr int L = decltype(lanes)::value, E = decltype(each)::value;
            const unsigned blocks = (unsigned)std::min<int64_t>((n * L + 255) / 256, MOST_WORKGROUPS);
            hipLaunchKernelGGL((short_rows_backward_kernel<T, L, E>), dim3(blocks), dim3(256), 0, s, g, x, o);
            return last_launch();
        });
        const int64_t pieces = (classes + 2 * VECTOR<T> - 2) / VECTOR<T>;
        auto launch = [&](auto waves) {
            constexpr int WAVES = decltype(waves)::value, ROWS = LONG_THREADS / WAVE_LANES / WAVES;
            const int64_t run = 32 / VECTOR<T> * WAVES * WAVE_LANES, runs = (pieces + run - 1) / run;
            hipLaunchKernelGGL((long_rows_backward_kernel<T, WAVES>), dim3((unsigned)std::min<int64_t>((n * runs + ROWS - 1) / ROWS, MOST_WORKGROUPS)), dim3(LONG_THREADS), 0, s, g, x, o,
                               (int32_t)runs);
            return last_launch();
        };
        // (a workgroup's run is 8,192 logits, of which a row that ends in the middle leaves much idle: 12,003 classes bf16 4.5 TB/s, not 5.7; in
        // long rows the loads of what a row has are shared: 131,072 with 10 alternatives 5.7, not 5.3)
        return classes <= WAVE_CLASSES ? launch(std::integral_constant<int, 1>{}) : launch(std::integral_constant<int, 4>{});
    });
}
