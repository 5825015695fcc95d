// Rows of a learned table, scaled, and the gradient of the table.
//   out[i] = scale * table[index[i]]            dtable[v] = scale * sum over i with index[i] = v of dout[i]
// Both are bound by memory.
#include <algorithm>
#include <type_traits>

#include "ends.h"

using namespace libra;

namespace {

// What a lane moves of a row: 16 bytes at a multiple of 16; 16 bytes anywhere, where rows are not aligned (the last piece of a row then ends
// with the row and overlaps the one before: both lanes hold and write the same numbers there); an element, where rows are shorter.
// (Elements instead of 16 bytes anywhere: lookup of 1,000,003 rows of 63 bf16 85 us, not 57, their gradient 181, not 153.  Rows of 64 take 44: one
// of 126 bytes lies on two lines of memory, and 212 MiB come from it, not 110.)
enum Access { ELEMENTS, ANYWHERE, ALIGNED };

template <class T, int ACCESS> struct Piece {
    static constexpr int W = ACCESS == ELEMENTS ? 1 : VECTOR<T>;
    float x[W];
    // where the piece that a row of `width` elements has at `at`, a multiple of W below the width, begins
    __device__ static int32_t column(int32_t at, int32_t width) { return ACCESS == ANYWHERE ? min(at, width - W) : at; }
    // as it is in memory
    typedef std::conditional_t<ACCESS == ELEMENTS, T, uint4> Stored;
    __device__ static Stored fetch(const T *p) {
        if constexpr (ACCESS == ALIGNED) return *reinterpret_cast<const uint4 *>(p);
        else if constexpr (ACCESS == ANYWHERE) return __builtin_bit_cast(uint4, *reinterpret_cast<const Unaligned *>(p));
        else return p[0];
    }
    __device__ void take(Stored s) {
        if constexpr (ACCESS == ELEMENTS) x[0] = load_as_float(s);
        else unpack<T>(s, x);
    }
    __device__ void load(const T *p) { take(fetch(p)); }
    __device__ void store(T *p) const {
        if constexpr (ACCESS == ALIGNED) *reinterpret_cast<uint4 *>(p) = pack<T>(x);
        else if constexpr (ACCESS == ANYWHERE) *reinterpret_cast<Unaligned *>(p) = __builtin_bit_cast(Unaligned, pack<T>(x));
        else p[0] = round_to<T>(x[0]);
    }
    __device__ void fill(float v) {
#pragma unroll
        for (int k = 0; k < W; ++k) x[k] = v;
    }
    __device__ void scale(float s) {
#pragma unroll
        for (int k = 0; k < W; ++k) x[k] *= s;
    }
    __device__ void add(const Piece &o) {
#pragma unroll
        for (int k = 0; k < W; ++k) x[k] += o.x[k];
    }
};

// ---- lookup ----
// Four rows of each group of lanes in flight, as they are in memory (as fp32 they take the registers of two waves): 1,000,003 rows of 128 bytes
// in 40 us, 5 TB/s (one row of a wave at a time: 137 us).
constexpr int LOOKUP_ROWS = 4;

template <class T, int ACCESS>
__global__ __launch_bounds__(256) void embedding_kernel(const T *table, int64_t rows, int32_t width, int64_t ld_table, const void *index, int index_type, int64_t n,
                                                        float scale, T *out, int64_t ld_out, int lanes) {
    typedef Piece<T, ACCESS> P;
    const int groups = 256 / lanes, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
    for (int64_t first = (int64_t)blockIdx.x * (groups * LOOKUP_ROWS); first < n; first += (int64_t)gridDim.x * (groups * LOOKUP_ROWS)) {
        int64_t v[LOOKUP_ROWS];
        indices_at<LOOKUP_ROWS>(index, index_type, [&](int u) { return min(first + u * groups + group, n - 1); }, v);
        for (uint32_t at = lane * P::W; at < (uint32_t)width; at += lanes * P::W) {      // (unsigned: it passes the end of a row of up to 2^31 - 1)
            const int32_t c = P::column((int32_t)at, width);
            typename P::Stored stored[LOOKUP_ROWS];
            if (rows > 0) {                 // (loads from some row even where there is none to load: a load in a branch would wait for those before it)
#pragma unroll
                for (int u = 0; u < LOOKUP_ROWS; ++u) stored[u] = P::fetch(table + (v[u] >= 0 && v[u] < rows ? v[u] : 0) * ld_table + c);
            }
#pragma unroll
            for (int u = 0; u < LOOKUP_ROWS; ++u) {
                P p;
                p.take(stored[u]);
                p.scale(scale);
                if (v[u] < 0 || v[u] >= rows) p.fill(v[u] == -1 ? 0.f : __builtin_nanf(""));
                if (first + u * groups + group < n) p.store(out + (first + u * groups + group) * ld_out + c);
            }
        }
    }
}

// ---- gradient ----
// Few ids: every workgroup owns a run of the table's rows.  It reads all ids, keeps those of its rows in LDS, brings them into the order
// of their rows, adds the rows of dout up and writes its rows of the table, zeros among them: one launch, no array between.
// Many ids: (row, place) pairs are sorted by row, the pairs are cut into runs of equal length whatever rows they name, the sums of rows
// that a run holds whole are written, those of rows that go on beyond a run are joined by another launch.  The zeros are written
// while the sort, which is bound by latency, runs.  (Owners for many ids too, to whom one pass of the sort deals the pairs out: 116 us
// for 2^20 uniform ids on as many rows instead of 126, but 266 instead of 131 with popular rows, and 1,900 instead of 136 for 2^21 on 2^16:
// a row's ids are too uneven a share of work.)

__device__ inline uint32_t key_at(const void *index, int index_type, int64_t rows, int64_t i) {
    const int64_t v = index_at(index, index_type, i);
    return v >= 0 && v < rows ? (uint32_t)v : (uint32_t)rows;           // what is no row comes last
}

// Which lanes of the wave hold this lane's digit (0 for a lane without one)
__device__ inline uint64_t same_digit(uint32_t digit, int bits, bool real) {
    uint64_t same = __ballot(real);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
    }
    return real ? same : 0;
}
// Number of this digit in the wave so far (counted in LDS, where only this wave counts), among earlier batches and lower lanes
template <class C> __device__ inline int32_t rank_in_wave(uint32_t digit, int bits, bool real, C *count) {
    const int lane = threadIdx.x % WAVE_LANES;
    const uint64_t same = same_digit(digit, bits, real);
    const int before = __popcll(same & ((1ull << lane) - 1));
    volatile C *c = count + digit;
    const int32_t base = real ? *c : 0;
    __builtin_amdgcn_wave_barrier();                // all lanes have read before one writes: a wave's LDS accesses keep their order
    if (real && before == 0) *c = (C)(base + __popcll(same));
    __builtin_amdgcn_wave_barrier();
    return base + before;
}

// -- few ids --
// 8,191 ids on 2^17 rows of 256 bytes: 17 us, of which the zeros are 6.4 at the rate of memory; the rest is latency, the same for all
// workgroups, which run at once: ids from the L2s, LDS sort, rows of dout.  Loads are issued together, outside branches (24 us before).
constexpr int OWNER_THREADS = 1024, OWNER_WAVES = OWNER_THREADS / WAVE_LANES, OWNER_PLACE_BITS = 14, OWNER_MAX_IDS = 1 << OWNER_PLACE_BITS;
constexpr int OWNER_ROW_BITS = 10, OWNER_ROWS = 1 << OWNER_ROW_BITS, OWNER_LONG = 32;    // rows with more ids than that are added up by the whole workgroup

template <class T, int ACCESS, int MOST>
__global__ __launch_bounds__(OWNER_THREADS) void owner_kernel(const T *dout, int64_t ld_dout, const void *index, int index_type, int32_t n, int64_t rows, int32_t width,
                                                              int32_t owned, int row_bits, float scale, T *dtable, int64_t ld_dtable, int lanes) {
    typedef Piece<T, ACCESS> P;
    constexpr int IDS = MOST / OWNER_THREADS;
    __shared__ uint32_t list[MOST];                             // row in this run << OWNER_PLACE_BITS | place, n at most
    __shared__ int32_t start[OWNER_ROWS], total[OWNER_WAVES], long_rows[OWNER_MAX_IDS / OWNER_LONG], longs;
    __shared__ uint8_t named[OWNER_ROWS];                       // the row has ids
    __shared__ union {                                          // first the one, then the other
        uint16_t count[OWNER_WAVES][OWNER_ROWS];
        float part[OWNER_THREADS * 8];
    } shared;
    uint16_t(&count)[OWNER_WAVES][OWNER_ROWS] = shared.count;
    float(&part)[OWNER_THREADS * 8] = shared.part;
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES;
    const int64_t low = (int64_t)blockIdx.x * owned;
    const int32_t mine = (int32_t)min((int64_t)owned, rows - low);

    const int groups = OWNER_THREADS / lanes, group = threadIdx.x / lanes;
    const int32_t at_column = (blockIdx.y * lanes + threadIdx.x % lanes) * P::W, c = P::column(at_column, width);      // this lane's columns
    const bool there = at_column < width;
    for (int r = threadIdx.x; r < OWNER_ROWS; r += OWNER_THREADS) named[r] = 0;

    // the ids of these rows, in the order of their places
    int32_t m = 0;
    {
        uint32_t row[IDS];
        int64_t v[IDS];
        int32_t found = 0;
        const int32_t each = (n + OWNER_THREADS - 1) / OWNER_THREADS, at = wave * each * WAVE_LANES + lane;
        if (n > 0) indices_at<IDS>(index, index_type, [&](int b) { return min(at + min(b, each - 1) * WAVE_LANES, n - 1); }, v);
#pragma unroll
        for (int b = 0; b < IDS; ++b) {
            row[b] = b < each && at + b * WAVE_LANES < n && v[b] >= low && v[b] < low + mine ? (uint32_t)(v[b] - low) : ~0u;
            found += __popcll(__ballot(row[b] != ~0u));
        }
        if (lane == 0) total[wave] = found;
        __syncthreads();
        int32_t to = 0;
        for (int w = 0; w < OWNER_WAVES; ++w) {
            const int32_t t = total[w];
            to += w < wave ? t : 0;
            m += t;
        }
#pragma unroll
        for (int b = 0; b < IDS; ++b) {
            const uint64_t those = __ballot(row[b] != ~0u);
            if (row[b] != ~0u) {
                list[to + __popcll(those & ((1ull << lane) - 1))] = row[b] << OWNER_PLACE_BITS | (uint32_t)(at + b * WAVE_LANES);
                named[row[b]] = 1;
            }
            to += __popcll(those);
        }
    }
    for (int r = threadIdx.x; r < OWNER_WAVES * OWNER_ROWS / 2; r += OWNER_THREADS) reinterpret_cast<uint32_t *>(count)[r] = 0;
    if (threadIdx.x == 0) longs = 0;
    __syncthreads();
    if (there) {                                                // the zeros, on their way while the list is sorted
        P zero;
        zero.fill(0.f);
        for (int32_t r = group; r < mine; r += groups)
            if (!named[r]) zero.store(dtable + (low + r) * ld_dtable + c);
    }
    if (m == 0) return;                                         // the same for the whole workgroup

    // into the order of their rows (`start`: where a row's ids begin)
    {
        const int32_t each = (m + OWNER_THREADS - 1) / OWNER_THREADS;
        uint32_t item[IDS];
        int32_t rank[IDS];
#pragma unroll
        for (int b = 0; b < IDS; ++b) {
            if (b < each) {
                const int32_t q = (wave * each + b) * WAVE_LANES + lane;
                item[b] = q < m ? list[q] : 0;
                rank[b] = rank_in_wave(item[b] >> OWNER_PLACE_BITS, row_bits, q < m, count[wave]);
            }
        }
        __syncthreads();
        // a row's number over all waves, then the sum of the rows before
        static_assert(OWNER_ROWS == OWNER_THREADS, "a thread for each row");
        int32_t sum = 0;
        {
            uint16_t in[OWNER_WAVES];
#pragma unroll
            for (int w = 0; w < OWNER_WAVES; ++w) in[w] = count[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < OWNER_WAVES; ++w) {
                count[w][threadIdx.x] = (uint16_t)sum;
                sum += in[w];
            }
        }
        int32_t up_to = sum;
        for (int d = 1; d < WAVE_LANES; d *= 2) {
            const int32_t y = __shfl_up(up_to, d);
            if (lane >= d) up_to += y;
        }
        if (lane == WAVE_LANES - 1) total[wave] = up_to;
        __syncthreads();
        for (int w = 0; w < wave; ++w) up_to += total[w];
        start[threadIdx.x] = up_to - sum;
        __syncthreads();
#pragma unroll
        for (int b = 0; b < IDS; ++b) {
            const int32_t q = (wave * each + b) * WAVE_LANES + lane;
            if (b < each && q < m) {
                const int32_t r = item[b] >> OWNER_PLACE_BITS;
                list[start[r] + count[wave][r] + rank[b]] = item[b];
            }
        }
        __syncthreads();
    }

    auto end_of = [&](int32_t r) { return r + 1 < OWNER_ROWS ? start[r + 1] : m; };
    auto sum_of = [&](int32_t q, int32_t end, P &sum) {                          // four rows in flight
        for (; q < end; q += 4) {
            P p[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) p[u].load(dout + (int64_t)(list[min(q + u, end - 1)] & (OWNER_MAX_IDS - 1)) * ld_dout + c);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (q + u < end) sum.add(p[u]);
        }
    };
    for (int32_t r = group; r < mine; r += groups) {
        const int32_t begin = start[r], end = end_of(r);
        if (end - begin > OWNER_LONG) {
            if (threadIdx.x % lanes == 0) long_rows[atomicAdd(&longs, 1)] = r;
            continue;
        }
        if (!there || begin == end) continue;
        P sum;
        sum.fill(0.f);
        sum_of(begin, end, sum);
        sum.scale(scale);
        sum.store(dtable + (low + r) * ld_dtable + c);
    }
    __syncthreads();
    const int32_t all = longs;
    for (int32_t k = 0; k < all; ++k) {
        const int32_t r = long_rows[k], begin = start[r], end = end_of(r), each = (end - begin + groups - 1) / groups;
        P sum;
        sum.fill(0.f);
        if (there) sum_of(begin + group * each, min(end, begin + (group + 1) * each), sum);
#pragma unroll
        for (int w = 0; w < P::W; ++w) part[w * OWNER_THREADS + threadIdx.x] = sum.x[w];
        __syncthreads();
        for (int half = groups / 2; half > 0; half /= 2) {       // the groups' sums in pairs
            if (group < half)
#pragma unroll
                for (int w = 0; w < P::W; ++w) part[w * OWNER_THREADS + threadIdx.x] += part[w * OWNER_THREADS + half * lanes + threadIdx.x];
            __syncthreads();
        }
        if (group == 0 && there) {
#pragma unroll
            for (int w = 0; w < P::W; ++w) sum.x[w] = part[w * OWNER_THREADS + threadIdx.x];
            sum.scale(scale);
            sum.store(dtable + (low + r) * ld_dtable + c);
        }
        __syncthreads();
    }
}

// -- many ids: pairs sorted by row, up to 11 bits at a time; equal rows keep the order of their places --
constexpr int DIGIT_BITS = 11, DIGITS = 1 << DIGIT_BITS, SORT_THREADS = 256, PLACE_THREADS = 1024, PLACE_WAVES = PLACE_THREADS / WAVE_LANES, PLACE_BATCHES = 4;
constexpr int SORT_TILE = PLACE_THREADS * PLACE_BATCHES, SORT_BLOCKS = 512, SCAN_DIGITS = WAVE_LANES;

struct Keys {                       // of one pass: the ids themselves in the first one, pairs afterwards
    const void *index;
    int index_type;
    int64_t rows;
    const uint2 *pair;
    __device__ uint2 at(int64_t i) const { return pair ? pair[i] : uint2{key_at(index, index_type, rows, i), (uint32_t)i}; }
};

// A share of the table's zeros, written by workgroups behind those of a sorting launch: these wait for chains of loads and LDS accesses and
// leave the memory to others (all zeros in the first launch: 143 us for 2^20 skewed ids on 2^20 rows of 128 bytes, not 131).
struct Zeros {
    char *base;
    int64_t rows, width_bytes, ld_bytes;
    unsigned blocks;
    int share, shares;
};
__device__ inline void write_zeros(const Zeros &z, unsigned block, int threads) {
    const int64_t first = (int64_t)block * threads + threadIdx.x, step = (int64_t)z.blocks * threads;
    if (z.width_bytes == z.ld_bytes && ((uintptr_t)z.base & 15) == 0) {
        const int64_t bytes = z.rows * z.width_bytes, all = bytes / 16, from = all / z.shares * z.share, to = z.share + 1 < z.shares ? all / z.shares * (z.share + 1) : all;
        uint4 *p = reinterpret_cast<uint4 *>(z.base);
        for (int64_t k = from + first; k < to; k += step) p[k] = uint4{0, 0, 0, 0};
        if (to == all && first < bytes % 16) z.base[all * 16 + first] = 0;
        return;
    }
    const int64_t halves = z.width_bytes / 2, from = z.rows / z.shares * z.share, to = z.share + 1 < z.shares ? z.rows / z.shares * (z.share + 1) : z.rows;
    for (int64_t r = from + first / WAVE_LANES; r < to; r += step / WAVE_LANES)      // a wave per row
        for (int64_t k = threadIdx.x % WAVE_LANES; k < halves; k += WAVE_LANES) reinterpret_cast<uint16_t *>(z.base + r * z.ld_bytes)[k] = 0;
}

// count[block][digit]
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(Keys in, int64_t n, int64_t each, int shift, int bits, unsigned blocks, int32_t *count, Zeros zeros) {
    __shared__ int32_t seen[DIGITS];
    if (blockIdx.x >= blocks) {
        write_zeros(zeros, blockIdx.x - blocks, SORT_THREADS);
        return;
    }
    for (int d = threadIdx.x; d < DIGITS; d += SORT_THREADS) seen[d] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * each, end = min(n, begin + each);
    for (int64_t i = begin + threadIdx.x; i < end; i += 8 * SORT_THREADS) {
        uint32_t key[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) key[u] = in.at(min(i + u * SORT_THREADS, end - 1)).x;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u * SORT_THREADS < end) atomicAdd(&seen[(key[u] >> shift) & ((1u << bits) - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += SORT_THREADS) count[(int64_t)blockIdx.x * DIGITS + d] = seen[d];
}

// For 64 digits: number of the digit in earlier blocks in place of the counts, and the digit's total.  Sixteen waves share the blocks.
__global__ __launch_bounds__(1024) void sort_scan_kernel(int32_t *count, int blocks, int32_t *totals) {
    __shared__ int32_t part[16][WAVE_LANES];
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES, each = (blocks + 15) / 16;
    const int digit = blockIdx.x * SCAN_DIGITS + lane, begin = min(blocks, wave * each), end = min(blocks, begin + each);
    constexpr int MOST = SORT_BLOCKS / 16;
    int32_t c[MOST], sum = 0;
#pragma unroll
    for (int b = 0; b < MOST; ++b) c[b] = begin + b < end ? count[(int64_t)(begin + b) * DIGITS + digit] : 0;
#pragma unroll
    for (int b = 0; b < MOST; ++b) sum += c[b];
    part[wave][lane] = sum;
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        before += w < wave ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (wave == 0) totals[digit] = all;
#pragma unroll
    for (int b = 0; b < MOST; ++b) {
        if (begin + b < end) count[(int64_t)(begin + b) * DIGITS + digit] = before;
        before += c[b];
    }
}

// A tile of 4,096 pairs at a time: their numbers among the tile's pairs of the same digit, wave by wave, and from there their places.
// Many waves of few pairs: ranking is a chain of ballots and LDS accesses (four waves of 16 pairs a lane took 15 us for a tile, not 7).
__global__ __launch_bounds__(PLACE_THREADS) void sort_place_kernel(Keys in, int64_t n, int64_t each, int shift, int bits, unsigned blocks, const int32_t *count, const int32_t *totals, uint2 *out, Zeros zeros) {
    __shared__ int32_t next[DIGITS], part[PLACE_WAVES];
    __shared__ uint16_t mine[PLACE_WAVES][DIGITS];               // pairs of each wave, then of the waves before it: below 4,096
    const int lane = threadIdx.x % WAVE_LANES, wave = threadIdx.x / WAVE_LANES, digits = 1 << bits;
    constexpr int EACH = DIGITS / PLACE_THREADS;
    if (blockIdx.x >= blocks) {
        write_zeros(zeros, blockIdx.x - blocks, PLACE_THREADS);
        return;
    }
    {   // where this block's first pair of each digit goes: totals of the digits before, and what earlier blocks have
        int32_t t[EACH], earlier[EACH], sum = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int d = threadIdx.x * EACH + k;
            t[k] = earlier[k] = 0;
            if (d < digits && totals) {
                t[k] = totals[d];
                earlier[k] = count[(int64_t)blockIdx.x * DIGITS + d];
            } else if (d < digits) {
#pragma unroll 8
                for (int b = 0; b < (int)blocks; ++b) {
                    const int32_t x = count[(int64_t)b * DIGITS + d];
                    t[k] += x;
                    earlier[k] += b < (int)blockIdx.x ? x : 0;
                }
            }
            sum += t[k];
        }
        int32_t up_to = sum;
        for (int d = 1; d < WAVE_LANES; d *= 2) {
            const int32_t y = __shfl_up(up_to, d);
            if (lane >= d) up_to += y;
        }
        if (lane == WAVE_LANES - 1) part[wave] = up_to;
        __syncthreads();
        for (int w = 0; w < wave; ++w) up_to += part[w];
        up_to -= sum;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int d = threadIdx.x * EACH + k;
            next[d] = up_to + earlier[k];
            up_to += t[k];
        }
    }
    const int64_t begin = (int64_t)blockIdx.x * each, end = min(n, begin + each);
    for (int64_t tile = begin; tile < end; tile += SORT_TILE) {
        uint2 pair[PLACE_BATCHES];
        int32_t rank[PLACE_BATCHES], all[EACH];
        const int64_t at = tile + (int64_t)wave * (PLACE_BATCHES * WAVE_LANES) + lane;
#pragma unroll
        for (int b = 0; b < PLACE_BATCHES; ++b) pair[b] = in.at(min(at + b * WAVE_LANES, end - 1));
        for (int w = 0; w < PLACE_WAVES; ++w)
            for (int d = threadIdx.x; d < (digits + 1) / 2; d += PLACE_THREADS) reinterpret_cast<uint32_t *>(mine[w])[d] = 0;
        __syncthreads();
#pragma unroll
        for (int b = 0; b < PLACE_BATCHES; ++b) rank[b] = rank_in_wave((pair[b].x >> shift) & (digits - 1), bits, at + b * WAVE_LANES < end, mine[wave]);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int d = k * PLACE_THREADS + threadIdx.x;
            uint16_t c[PLACE_WAVES];
            all[k] = 0;
            if (d >= digits) continue;
#pragma unroll
            for (int w = 0; w < PLACE_WAVES; ++w) c[w] = mine[w][d];
#pragma unroll
            for (int w = 0; w < PLACE_WAVES; ++w) {
                mine[w][d] = (uint16_t)all[k];
                all[k] += c[w];
            }
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < PLACE_BATCHES; ++b) {
            const int d = (pair[b].x >> shift) & (digits - 1);
            if (at + b * WAVE_LANES < end) out[next[d] + mine[wave][d] + rank[b]] = pair[b];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) next[k * PLACE_THREADS + threadIdx.x] += all[k];
    }
}

// Runs of `run` pairs, a group of lanes each, eight rows of dout in flight: 41 us for 2^20 rows of 128 bytes, 5 TB/s with what is written.
// The row that a run begins in the middle of, and the one that goes on behind it, leave their sums in `part` (two rows of fp32 for each run);
// a row that fills the whole run and goes on at both ends leaves the first of them.
template <class T, int ACCESS>
__global__ __launch_bounds__(256) void run_sums_kernel(const T *dout, int64_t ld_dout, const uint2 *pair, int64_t n, int32_t run, int64_t rows, int32_t width, float scale,
                                                       T *dtable, int64_t ld_dtable, float *part, int32_t part_width, int lanes) {
    typedef Piece<T, ACCESS> P;
    constexpr int U = 8;
    const int64_t k = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes, begin = k * run, end = min(n, begin + run);
    const int32_t at_column = (blockIdx.y * lanes + threadIdx.x % lanes) * P::W, c = P::column(at_column, width);
    if (begin >= n || at_column >= width) return;
    uint32_t row = pair[begin].x;
    bool whole = begin == 0 || pair[begin - 1].x != row;            // the current row began here
    P sum;
    sum.fill(0.f);
    auto leave = [&](bool ends) {
        if (row >= (uint32_t)rows) return;
        if (whole && ends) {
            sum.scale(scale);
            sum.store(dtable + (int64_t)row * ld_dtable + c);
        } else {
            float *to = part + (2 * k + (whole ? 1 : 0)) * part_width + c;
#pragma unroll
            for (int w = 0; w < P::W; ++w) to[w] = sum.x[w];
        }
    };
    for (int64_t q = begin; q < end; q += U) {
        uint2 item[U];
        P p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) item[u] = pair[min(q + u, end - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) p[u].load(dout + (int64_t)item[u].y * ld_dout + c);       // (also of padding: its sum goes nowhere)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q + u < end) {
                if (item[u].x != row) {
                    leave(true);
                    row = item[u].x;
                    whole = true;
                    sum.fill(0.f);
                }
                sum.add(p[u]);
            }
        }
    }
    leave(end == n || pair[end].x != row);
}

// Rows of several runs.  A workgroup looks at as many runs as it has groups of lanes (16 at least) and adds up the rows that begin in one of
// them and go on behind it: a group each, which walks on while runs begin with the row; all groups together those that reach over more
// than 32 runs.
constexpr int LONG_JOIN = 32;
__host__ __device__ constexpr int join_runs(int lanes) { return 256 / lanes < 16 ? 16 : 256 / lanes < WAVE_LANES ? 256 / lanes : WAVE_LANES; }

template <class T, int ACCESS>
__global__ __launch_bounds__(256) void join_runs_kernel(const uint2 *pair, int64_t n, int32_t run, int64_t runs, int64_t rows, int32_t width, float scale, T *dtable,
                                                        int64_t ld_dtable, const float *part, int32_t part_width, int lanes) {
    typedef Piece<T, ACCESS> P;
    constexpr int U = 4;
    __shared__ int64_t head[WAVE_LANES];                        // row; as ~row if it is a long one; 2^40 for none
    __shared__ float shared[256 * P::W];
    __shared__ uint64_t shorts, longs;                          // which of the runs
    __shared__ unsigned equal;
    constexpr int64_t NONE = 1ll << 40;
    const int many = join_runs(lanes);
    const int64_t first = (int64_t)blockIdx.x * many;
    if (threadIdx.x < WAVE_LANES) {
        const int64_t k = first + threadIdx.x;
        int64_t h = NONE;
        if ((int)threadIdx.x < many && k + 1 < runs) {
            const int64_t beyond = min(k + 1 + LONG_JOIN, runs - 1);
            const uint32_t row = pair[(k + 1) * run].x, end = pair[(k + 1) * run - 1].x, begin = pair[k * run].x, before = pair[max(k * run - 1, (int64_t)0)].x, far = pair[beyond * run].x;
            if (row < (uint32_t)rows && end == row && (begin != row || before != row || k == 0)) h = far == row && beyond == k + 1 + LONG_JOIN ? ~(int64_t)row : (int64_t)row;
        }
        head[threadIdx.x] = h;
        const uint64_t here = __ballot(h >= 0 && h != NONE), reaching = __ballot(h < 0);
        if (threadIdx.x == 0) shorts = here, longs = reaching;
    }
    __syncthreads();
    const int groups = 256 / lanes, group = threadIdx.x / lanes;
    const int32_t at_column = (blockIdx.y * lanes + threadIdx.x % lanes) * P::W, c = P::column(at_column, width);
    const bool there = at_column < width;
    auto load = [&](int64_t at) {
        P p;
#pragma unroll
        for (int w = 0; w < P::W; ++w) p.x[w] = part[at * part_width + c + w];
        return p;
    };
    if (there)
        for (int h = group; h < many; h += groups) {
            if (!(shorts >> h & 1)) continue;
            const int64_t row = head[h];
            P sum = load(2 * (first + h) + 1);                  // what this run left for the row behind its end, and the first sums of those behind
            for (int64_t j = first + h + 1, more = 1; more; j += U) {
                uint32_t key[U];
                P p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t at = min(j + u, runs - 1);
                    key[u] = pair[at * run].x;
                    p[u] = load(2 * at);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    more = more && j + u < runs && key[u] == (uint32_t)row;
                    if (more) sum.add(p[u]);
                }
            }
            sum.scale(scale);
            sum.store(dtable + row * ld_dtable + c);
        }
    for (uint64_t those = longs; those; those &= those - 1) {   // the same for the whole workgroup
        const int h = __ffsll((unsigned long long)those) - 1;
        const int64_t row = ~head[h], k = first + h;
        int64_t low = k + 1, high = runs;                       // the last run that begins with the row: 256 places at a time
        while (high - low > 1) {
            const int64_t step = (high - low + 255) / 256, at = low + threadIdx.x * step;
            if (threadIdx.x == 0) equal = 0;
            __syncthreads();
            const uint64_t with = __ballot(at < high && pair[min(at, runs - 1) * run].x == (uint32_t)row);
            if (threadIdx.x % WAVE_LANES == 0) atomicAdd(&equal, (unsigned)__popcll(with));
            __syncthreads();
            const int64_t found = equal;                        // at least one: low itself
            high = min(high, low + found * step);
            low += (found - 1) * step;
            __syncthreads();
        }
        const int64_t count = low - k, each = (count + groups - 1) / groups, begin = min(count, group * each), end = min(count, begin + each);
        P sum;
        sum.fill(0.f);
        if (there) {
            if (group == 0) sum = load(2 * k + 1);
            for (int64_t j = begin; j < end; j += U) {
                P p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) p[u] = load(2 * (k + 1 + min(j + u, end - 1)));
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (j + u < end) sum.add(p[u]);
            }
        }
#pragma unroll
        for (int w = 0; w < P::W; ++w) shared[w * 256 + threadIdx.x] = sum.x[w];
        __syncthreads();
        for (int half = groups / 2; half > 0; half /= 2) {
            if (group < half)
#pragma unroll
                for (int w = 0; w < P::W; ++w) shared[w * 256 + threadIdx.x] += shared[w * 256 + half * lanes + threadIdx.x];
            __syncthreads();
        }
        if (group == 0 && there) {
#pragma unroll
            for (int w = 0; w < P::W; ++w) sum.x[w] = shared[w * 256 + threadIdx.x];
            sum.scale(scale);
            sum.store(dtable + row * ld_dtable + c);
        }
        __syncthreads();
    }
}

struct Layout {                     // lanes of a row, rows of workgroups for what is wider
    int lanes;
    unsigned slices;
};
Layout layout(int32_t width, int piece) {
    const int32_t pieces = width / piece + (width % piece != 0);
    int lanes = 1;
    while (lanes < WAVE_LANES && lanes < pieces) lanes *= 2;
    return {lanes, (unsigned)((pieces + lanes - 1) / lanes)};
}

// As many workgroups as the compute units hold at once, as long as their rows can be told apart in one pass: two for each, one where a
// workgroup has LDS for more than half of the most ids.
int64_t owned_rows(int64_t n, int64_t rows) {
    const int64_t owners = n <= OWNER_MAX_IDS / 2 ? 512 : 256;
    return std::min<int64_t>(std::max<int64_t>((rows + owners - 1) / owners, 1), OWNER_ROWS);
}
// Every owner reads all ids: they come out of the L2s, at some 10 TB/s, so 2^24 of them cost about as much as the launches of the sort.
bool few_ids(int64_t n, int64_t rows) { return n <= OWNER_MAX_IDS && n * ((rows + OWNER_ROWS - 1) / OWNER_ROWS) <= 1 << 24; }

struct BackwardWork {
    uint2 *pair[2];
    int32_t *count, *totals;
    float *part;
    int32_t run, part_width;
    int64_t runs;
    size_t bytes;
};

// Runs of 8 to 64 pairs: short enough for 2^18 threads of eight elements each, so that loads are in flight on every compute unit.
BackwardWork backward_work(void *base, int64_t n, int64_t rows, int32_t width) {
    BackwardWork w{};
    if (few_ids(n, rows)) return w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *p = reinterpret_cast<char *>(base) + at;
        at += (bytes + 255) / 256 * 256;
        return p;
    };
    w.run = 8;
    while (w.run < 64 && n / w.run * std::min((width + 7) / 8, 64) > 1 << 18) w.run *= 2;
    w.runs = (n + w.run - 1) / w.run;
    w.part_width = (width + 7) / 8 * 8;
    for (uint2 *&p : w.pair) p = (uint2 *)take((size_t)n * sizeof(uint2));
    w.count = (int32_t *)take((size_t)DIGITS * SORT_BLOCKS * 4);
    w.totals = (int32_t *)take(DIGITS * 4);
    w.part = (float *)take((size_t)w.runs * 2 * w.part_width * 4);
    w.bytes = at;
    return w;
}

constexpr int32_t MOST_WIDTH = 1 << 21;      // slices of 64 lanes are the second dimension of a launch

int backward_shape(int64_t n, int64_t rows, int32_t width) {
    if (n < 0 || rows < 0 || width < 1) return LIBRA_ERR_SHAPE;
    if (n > INT32_MAX || rows >= INT32_MAX) return LIBRA_ERR_TOO_LARGE;
    if (width > MOST_WIDTH) return LIBRA_ERR_UNSUPPORTED;
    return LIBRA_OK;
}

// f(T, how lanes may move the rows of two arrays)
template <class F> int for_rows(int dtype, const void *p, int64_t ld_p, const void *q, int64_t ld_q, int32_t width, F &&f) {
    const int piece = 16 / (int)dtype_bytes(dtype);
    const bool aligned = aligned_to(p, 16) && aligned_to(q, 16) && ld_p % piece == 0 && ld_q % piece == 0 && width % piece == 0;
    return for_dtype(dtype, [&](auto tag) {
        if (aligned) return f(tag, std::integral_constant<int, ALIGNED>{});
        if (width >= piece) return f(tag, std::integral_constant<int, ANYWHERE>{});
        return f(tag, std::integral_constant<int, ELEMENTS>{});
    });
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
    return for_rows(dtype, table, ld_table, out, ld_out, width, [&](auto tag, auto access) {
        typedef decltype(tag) T;
        constexpr int ACCESS = decltype(access)::value;
        const int lanes = layout(width, Piece<T, ACCESS>::W).lanes;
        const int64_t each = 256 / lanes * LOOKUP_ROWS;
        hipLaunchKernelGGL((embedding_kernel<T, ACCESS>), dim3((unsigned)std::min<int64_t>((n + each - 1) / each, 1 << 20)), dim3(256), 0, (hipStream_t)stream,
                           (const T *)table, rows, width, ld_table, index, index_type, n, scale, (T *)out, ld_out, lanes);
        return last_launch();
    });
}

extern "C" int libra_embedding_backward_workspace(int64_t n, int64_t rows, int32_t width, size_t *bytes) {
    if (!bytes) return LIBRA_ERR_NULL;
    if (int rc = backward_shape(n, rows, width)) return rc;
    *bytes = backward_work(nullptr, n, rows, width).bytes;
    return LIBRA_OK;
}

extern "C" int libra_embedding_backward(const void *dout, int64_t ld_dout, int dtype, const void *index, int index_type, int64_t n, int64_t rows, int32_t width, float scale,
                                        void *dtable, int64_t ld_dtable, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = backward_shape(n, rows, width)) return rc;
    if (ld_dout < width || ld_dtable < width) return LIBRA_ERR_SHAPE;
    if (!known_dtype(dtype)) return LIBRA_ERR_DTYPE;
    if (!known_index(index_type)) return LIBRA_ERR_OPTION;
    if (rows == 0) return LIBRA_OK;
    const BackwardWork w = backward_work(workspace, n, rows, width);
    if (!dtable || ((!dout || !index) && n > 0) || (!workspace && w.bytes > 0)) return LIBRA_ERR_NULL;
    if (!aligned_to(dout, dtype_bytes(dtype)) || !aligned_to(dtable, dtype_bytes(dtype)) || !aligned_to(index, index_bytes(index_type))) return LIBRA_ERR_BUFFER;
    if (w.bytes > 0 && (workspace_bytes < w.bytes || !aligned_to(workspace, 256))) return LIBRA_ERR_BUFFER;
    hipStream_t s = (hipStream_t)stream;
    if (few_ids(n, rows)) return for_rows(dtype, dout, ld_dout, dtable, ld_dtable, width, [&](auto tag, auto access) {
        typedef decltype(tag) T;
        constexpr int ACCESS = decltype(access)::value;
        const Layout l = layout(width, Piece<T, ACCESS>::W);
        const int64_t owned = owned_rows(n, rows);
        int row_bits = 1;
        while (1 << row_bits < owned) ++row_bits;
        const dim3 grid((unsigned)((rows + owned - 1) / owned), l.slices);
        auto launch = [&](auto most) {
            hipLaunchKernelGGL((owner_kernel<T, ACCESS, decltype(most)::value>), grid, dim3(OWNER_THREADS), 0, s, (const T *)dout, ld_dout, index, index_type, (int32_t)n, rows, width,
                               (int32_t)owned, row_bits, scale, (T *)dtable, ld_dtable, l.lanes);
        };
        if (n <= OWNER_MAX_IDS / 2) launch(std::integral_constant<int, OWNER_MAX_IDS / 2>{});
        else launch(std::integral_constant<int, OWNER_MAX_IDS>{});
        return last_launch();
    });
    int bits = 1;
    while (rows >> bits) ++bits;
    const int passes = (bits + DIGIT_BITS - 1) / DIGIT_BITS;
    const int64_t tiles = (n + SORT_TILE - 1) / SORT_TILE, per = (tiles + SORT_BLOCKS - 1) / SORT_BLOCKS, each = per * SORT_TILE;
    const unsigned blocks = (unsigned)((tiles + per - 1) / per);
    const bool scan = blocks > 32;              // every block of the next launch can add the counts of so few up by itself: 3 us less
    Keys in{index, index_type, rows, nullptr};
    const size_t size = dtype_bytes(dtype);
    for (int p = 0, shift = 0; p < passes; ++p) {
        const int digit = (bits - shift + passes - p - 1) / (passes - p);
        Zeros zeros{(char *)dtable, rows, (int64_t)width * (int64_t)size, ld_dtable * (int64_t)size, 1024, 2 * p, 2 * passes};
        hipLaunchKernelGGL(sort_count_kernel, dim3(blocks + zeros.blocks), dim3(SORT_THREADS), 0, s, in, n, each, shift, digit, blocks, w.count, zeros);
        if (scan) hipLaunchKernelGGL(sort_scan_kernel, dim3((unsigned)((1 << digit) + SCAN_DIGITS - 1) / SCAN_DIGITS), dim3(1024), 0, s, w.count, (int)blocks, w.totals);
        zeros.blocks = 256;
        zeros.share = 2 * p + 1;
        hipLaunchKernelGGL(sort_place_kernel, dim3(blocks + zeros.blocks), dim3(PLACE_THREADS), 0, s, in, n, each, shift, digit, blocks, w.count, scan ? w.totals : nullptr,
                           w.pair[p & 1], zeros);
        in.pair = w.pair[p & 1];
        shift += digit;
    }
    return for_rows(dtype, dout, ld_dout, dtable, ld_dtable, width, [&](auto tag, auto access) {
        typedef decltype(tag) T;
        constexpr int ACCESS = decltype(access)::value;
        const Layout l = layout(width, Piece<T, ACCESS>::W);
        const int groups = 256 / l.lanes;
        hipLaunchKernelGGL((run_sums_kernel<T, ACCESS>), dim3((unsigned)((w.runs + groups - 1) / groups), l.slices), dim3(256), 0, s, (const T *)dout, ld_dout, in.pair, n, w.run, rows,
                           width, scale, (T *)dtable, ld_dtable, w.part, w.part_width, l.lanes);
        hipLaunchKernelGGL((join_runs_kernel<T, ACCESS>), dim3((unsigned)((w.runs + join_runs(l.lanes) - 1) / join_runs(l.lanes)), l.slices), dim3(256), 0, s, in.pair, n, w.run, w.runs, rows, width,
                           scale, (T *)dtable, ld_dtable, w.part, w.part_width, l.lanes);
        return last_launch();
    });
}
