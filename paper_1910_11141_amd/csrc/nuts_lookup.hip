// Rows of a table by class, and the gradient of that: sums of rows class by class.
//
//   rows[i, :] = s T[id_i, :]                 dT[v, :] = s sum_{i: id_i = v} dRows[i, :]
//
// Both only move data: the first reads the distinct rows asked for and writes n, the second reads n and writes the table's.
// The gradient must not depend on the order in which workgroups come to run, so nothing is added with atomics: the
// positions i are sorted by class (stably, i ascending within a class), and every class's rows are added in that order, in
// pieces of a fixed length that are joined in order.
#include "nuts_cat.h"

#include <algorithm>

namespace nuts {
namespace {

constexpr int kThreads = 256;

// ---- lookup ---------------------------------------------------------------------------------------------------------

struct LookupArgs {
    const void* table;
    const void* ids;
    void* rows;
    long first_block, n_ids, n_classes, dim, table_stride, row_stride;
    float scale;
    int id_type, lane_bits;
};

// A group of 2^lane_bits threads copies kRows rows, 16 bytes a thread at a time: kRows classes are read first and then as many
// rows are in flight, for what a row costs is the wait for its class and then for its bytes.
template <typename T, int kRows>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1);
    const long first = ((a.first_block + blockIdx.x) * (kThreads >> a.lane_bits) + (threadIdx.x >> a.lane_bits)) * kRows;
    const T* table = static_cast<const T*>(a.table);
    T* rows = static_cast<T*>(a.rows);
    int id[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) id[r] = first + r < a.n_ids ? class_at(a.ids, a.id_type, first + r, a.n_classes) : -2;
    for (long c = (long)lane * kN; c < a.dim; c += (long)lanes * kN) {
        if (c + kN <= a.dim) {
            Pack<T, kN> in[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (id[r] >= 0) in[r] = load_pack<T, kN>(table + id[r] * a.table_stride + c);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                if (id[r] == -2) continue;
                Pack<T, kN> out;
#pragma unroll
                for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(id[r] >= 0 ? to_float(in[r].v[e]) * a.scale : 0.f);
                store_pack(rows + (first + r) * a.row_stride + c, out);
            }
        } else {
            for (int r = 0; r < kRows; ++r) {
                if (id[r] == -2) continue;
                for (long e = c; e < a.dim; ++e)
                    rows[(first + r) * a.row_stride + e] = rounded<T>(id[r] >= 0 ? to_float(table[id[r] * a.table_stride + e]) * a.scale : 0.f);
            }
        }
    }
}

// ---- gradient: common ------------------------------------------------------------------------------------------------

struct GradArgs {
    const void* rows;
    const void* ids;
    void* table;
    long n_ids, n_classes, dim, table_stride, row_stride;
    float scale;
    int id_type, accumulate, lane_bits;
};

template <typename T, int kN>
__device__ __forceinline__ void load_columns(const T* p, int left, float (&x)[kN])
{
    if (left >= kN) {
        const Pack<T, kN> in = load_pack<T, kN>(p);
#pragma unroll
        for (int e = 0; e < kN; ++e) x[e] = to_float(in.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) x[e] = e < left ? to_float(p[e]) : 0.f;
    }
}

// A class's finished sum to its row of the table's gradient.
template <typename T, int kN>
__device__ __forceinline__ void finish_columns(const GradArgs& a, T* p, int left, const float (&sum)[kN])
{
    if (left >= kN) {
        Pack<T, kN> out;
        if (a.accumulate) {
            const Pack<T, kN> old = load_pack<T, kN>(p);
#pragma unroll
            for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(__builtin_fmaf(a.scale, sum[e], to_float(old.v[e])));
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(a.scale * sum[e]);
        }
        store_pack(p, out);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (e < left) p[e] = rounded<T>(a.accumulate ? __builtin_fmaf(a.scale, sum[e], to_float(p[e])) : a.scale * sum[e]);
    }
}

template <typename T, int kN>
__device__ __forceinline__ void zero_columns(T* p, int left)
{
    if (left >= kN) {
        Pack<T, kN> out;
#pragma unroll
        for (int e = 0; e < kN; ++e) out.v[e] = static_cast<T>(0.f);
        store_pack(p, out);
    } else {
        for (int e = 0; e < left; ++e) p[e] = static_cast<T>(0.f);
    }
}

// ---- gradient of few rows: one launch --------------------------------------------------------------------------------

constexpr int kFew = 1024;     // positions that a workgroup looks through by itself
constexpr int kFewRows = 64;   // at most so many classes a workgroup (an occupancy mask is one word)

// A workgroup owns `classes` neighbouring rows of the table: it finds the positions of theirs among all n (few, from
// cache), in ascending order, and adds them up.
template <typename T>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(GradArgs a, int classes, long first_block)
{
    constexpr int kN = 16 / sizeof(T);
    __shared__ int position[kFew];
    __shared__ unsigned char of_class[kFew];
    __shared__ int found[kThreads / 64];
    __shared__ unsigned occupied_half[2];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const long v0 = (first_block + blockIdx.x) * classes;
    const int own = (int)min((long)classes, a.n_classes - v0);
    if (threadIdx.x < 2) occupied_half[threadIdx.x] = 0u;
    __syncthreads();
    int count = 0;
    for (int base = 0; base < a.n_ids; base += kThreads) {
        const int i = base + threadIdx.x;
        const int id = i < a.n_ids ? class_at(a.ids, a.id_type, i, a.n_classes) : -1;
        const bool hit = id >= v0 && id < v0 + own;
        const unsigned long long hits = __ballot(hit);
        if (lane == 0) found[wave] = __popcll(hits);
        __syncthreads();
        int at = count;
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) at += found[w];
            count += found[w];
        }
        if (hit) {
            at += __popcll(hits & ((1ull << lane) - 1));
            position[at] = i;
            of_class[at] = (unsigned char)(id - v0);
            atomicOr(&occupied_half[(id - v0) >> 5], 1u << ((id - v0) & 31));
        }
        __syncthreads();
    }
    const unsigned long long occupied = occupied_half[0] | (unsigned long long)occupied_half[1] << 32;
    const long packs = (a.dim + kN - 1) / kN;
    T* table = static_cast<T*>(a.table);
    const T* rows = static_cast<const T*>(a.rows);
    // groups of 64 or of all threads go through the classes, a thread through its columns
    const int lanes = 1 << a.lane_bits, group = threadIdx.x >> a.lane_bits;
    for (int r = group; r < own; r += kThreads >> a.lane_bits) {
        const bool any = occupied >> r & 1;
        if (!any && a.accumulate) continue;
        for (long p = threadIdx.x & (lanes - 1); p < packs; p += lanes) {
            const long c = p * kN;
            const int left = (int)min((long)kN, a.dim - c);
            T* to = table + (v0 + r) * a.table_stride + c;
            if (!any) {
                zero_columns<T, kN>(to, left);
                continue;
            }
            float sum[kN];
#pragma unroll
            for (int e = 0; e < kN; ++e) sum[e] = 0.f;
            for (int m = 0; m < count; m += 4) {  // four rows in flight
                float x[4][kN];
                bool mine[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    mine[u] = m + u < count && of_class[m + u] == r;
                    if (mine[u]) load_columns<T, kN>(rows + (long)position[m + u] * a.row_stride + c, left, x[u]);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (mine[u]) {
#pragma unroll
                        for (int e = 0; e < kN; ++e) sum[e] += x[u][e];
                    }
            }
            finish_columns<T, kN>(a, to, left, sum);
        }
    }
}

// ---- gradient: sorting the positions by class ------------------------------------------------------------------------
//
// A stable radix sort, digit by digit from the lowest: every workgroup counts the digits of its tile of positions, one
// workgroup turns the counts into places, and every workgroup puts its tile's there.  Classes that are none get the key n_classes and
// end up last.

constexpr int kMaxDigitBits = 11;
constexpr int kWaves = kThreads / 64;

struct SortArgs {
    const void* ids;          // first digit: the classes themselves; else keys_in, pos_in
    const unsigned* keys_in;
    const unsigned* pos_in;
    unsigned* keys_out;
    unsigned* pos_out;
    unsigned* counts;         // [tile][digit], then places within the digit
    unsigned* starts;         // [digit]
    unsigned char* present;   // [n_classes]: 1 where a class comes
    long n_ids, n_classes;
    int id_type, shift, digit_bits, tile, tiles;
};

template <bool kFirst>
__device__ __forceinline__ unsigned key_at(const SortArgs& a, long i)
{
    if (!kFirst) return a.keys_in[i];
    const int id = class_at(a.ids, a.id_type, i, a.n_classes);
    return id < 0 ? (unsigned)a.n_classes : (unsigned)id;
}

template <bool kFirst>
__global__ __launch_bounds__(kThreads) void count_kernel(SortArgs a)
{
    __shared__ unsigned count[1 << kMaxDigitBits];
    const int digits = 1 << a.digit_bits;
    for (int d = threadIdx.x; d < digits; d += kThreads) count[d] = 0;
    __syncthreads();
    const long begin = (long)blockIdx.x * a.tile, end = min(begin + a.tile, a.n_ids);
    for (long i = begin + threadIdx.x; i < end; i += kThreads) atomicAdd(&count[key_at<kFirst>(a, i) >> a.shift & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kThreads) a.counts[(long)blockIdx.x * digits + d] = count[d];
    if (kFirst && a.present) {  // nothing is present yet
        const long words = (a.n_classes + 15) / 16;
        uint4* p = reinterpret_cast<uint4*>(a.present);
        for (long w = (long)blockIdx.x * kThreads + threadIdx.x; w < words; w += (long)gridDim.x * kThreads) p[w] = uint4{0, 0, 0, 0};
    }
}

__global__ __launch_bounds__(1024) void places_kernel(SortArgs a)
{
    __shared__ unsigned total[1 << kMaxDigitBits];
    const int digits = 1 << a.digit_bits;
    for (int d = threadIdx.x; d < digits; d += 1024) {
        unsigned sum = 0;
        int t = 0;
        for (; t + 8 <= a.tiles; t += 8) {  // eight reads in flight
            unsigned c[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] = a.counts[(long)(t + u) * digits + d];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                a.counts[(long)(t + u) * digits + d] = sum;
                sum += c[u];
            }
        }
        for (; t < a.tiles; ++t) {
            const unsigned c = a.counts[(long)t * digits + d];
            a.counts[(long)t * digits + d] = sum;
            sum += c;
        }
        total[d] = sum;
    }
    __syncthreads();
    if (threadIdx.x < 64) {  // one wave turns the totals into starts, 64 digits at a time
        unsigned before = 0;
        for (int d = threadIdx.x; d < ((digits + 63) & ~63); d += 64) {
            const unsigned own = d < digits ? total[d] : 0;
            unsigned sum = own;
            for (int step = 1; step < 64; step *= 2) {
                const unsigned other = __shfl_up(sum, step);
                if ((int)threadIdx.x >= step) sum += other;
            }
            if (d < digits) a.starts[d] = before + sum - own;
            before += __shfl(sum, 63);
        }
    }
}

// A wave places its run of the tile 64 positions at a time: lanes that hold the same digit find each other by a ballot for each bit.
template <bool kFirst>
__global__ __launch_bounds__(kThreads) void place_kernel(SortArgs a)
{
    extern __shared__ unsigned next[];  // [wave][digit]
    const int digits = 1 << a.digit_bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    for (int d = threadIdx.x; d < kWaves * digits; d += kThreads) next[d] = 0;
    __syncthreads();
    const long tile_begin = (long)blockIdx.x * a.tile, run = a.tile / kWaves;
    const long begin = tile_begin + wave * run, end = min(begin + run, a.n_ids);
    unsigned* own = next + wave * digits;
    for (long i = begin + lane; i < end; i += 64) atomicAdd(&own[key_at<kFirst>(a, i) >> a.shift & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kThreads) {
        unsigned at = a.starts[d] + a.counts[(long)blockIdx.x * digits + d];
        for (int w = 0; w < kWaves; ++w) {
            const unsigned c = next[w * digits + d];
            next[w * digits + d] = at;
            at += c;
        }
    }
    __syncthreads();
    for (long base = begin; base < end; base += 64) {
        const long i = base + lane;
        const bool valid = i < end;
        const unsigned key = valid ? key_at<kFirst>(a, i) : 0u;
        const unsigned digit = key >> a.shift & (digits - 1);
        unsigned long long same = __ballot(valid);
        for (int b = 0; b < a.digit_bits; ++b) {
            const bool set = digit >> b & 1;
            const unsigned long long with = __ballot(set);
            same &= set ? with : ~with;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const unsigned start = valid ? own[digit] : 0u;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid && before == 0) own[digit] = start + (unsigned)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid) {
            a.keys_out[start + before] = key;
            a.pos_out[start + before] = kFirst ? (unsigned)i : a.pos_in[i];
            if (kFirst && a.present && key < (unsigned long)a.n_classes) a.present[key] = 1;
        }
    }
}

// ---- gradient: adding up sorted rows ---------------------------------------------------------------------------------

struct SumArgs {
    GradArgs g;
    const unsigned* keys;
    const unsigned* pos;
    const unsigned char* present;  // NULL: no rows to clear
    float* part;                   // [chunk][2][dim]
    long chunks, sum_blocks;       // (of the first column block)
    int chunk;                     // positions in a chunk
};

// A group of 2^lane_bits threads adds the rows of one chunk of the sorted positions, a thread 16 bytes of columns.  A class that
// lies wholly in the chunk is finished; what belongs to one that began before goes to the chunk's part 0, to one that begins
// here and goes on to part 1.  The workgroups behind the last chunk's clear the rows of classes that do not come.
template <typename T>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    constexpr int kFlight = 8;
    const int lanes = 1 << a.g.lane_bits, groups = kThreads >> a.g.lane_bits;
    T* table = static_cast<T*>(a.g.table);
    const long c = ((long)blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * kN;
    if (c >= a.g.dim) return;
    const int left = (int)min((long)kN, a.g.dim - c);
    if ((long)blockIdx.x >= a.sum_blocks) {
        const long step = ((long)gridDim.x - a.sum_blocks) * groups;
        for (long v = ((long)blockIdx.x - a.sum_blocks) * groups + (threadIdx.x >> a.g.lane_bits); v < a.g.n_classes; v += step)
            if (!a.present[v]) zero_columns<T, kN>(table + v * a.g.table_stride + c, left);
        return;
    }
    const long q = (long)blockIdx.x * groups + (threadIdx.x >> a.g.lane_bits);
    if (q >= a.chunks) return;
    const long begin = q * a.chunk, end = min(begin + a.chunk, a.g.n_ids);
    const T* rows = static_cast<const T*>(a.g.rows);
    const unsigned none = (unsigned)a.g.n_classes;
    const unsigned before = begin > 0 ? a.keys[begin - 1] : none, after = end < a.g.n_ids ? a.keys[end] : none;
    float sum[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) sum[e] = 0.f;
    unsigned current = a.keys[begin];
    bool entered = current == before;  // the class began in an earlier chunk
    auto flush = [&](bool open) {
        if (current == none) return;
        if (entered || open) {
            float* to = a.part + (q * 2 + (entered ? 0 : 1)) * a.g.dim + c;
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < left) to[e] = sum[e];
        } else {
            finish_columns<T, kN>(a.g, table + current * a.g.table_stride + c, left, sum);
        }
    };
    for (long i = begin; i < end; i += kFlight) {
        unsigned key[kFlight];
        float x[kFlight][kN];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            key[u] = i + u < end ? a.keys[i + u] : none;
            if (key[u] != none) load_columns<T, kN>(rows + (long)a.pos[i + u] * a.g.row_stride + c, left, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            if (key[u] == none) continue;  // (no class: such keys are the last)
            if (key[u] != current) {
                flush(false);
                current = key[u];
                entered = false;
#pragma unroll
                for (int e = 0; e < kN; ++e) sum[e] = x[u][e];
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e) sum[e] += x[u][e];
            }
        }
    }
    flush(current == after);
}

// Classes that reach over chunks: the group of the chunk in which one begins joins its parts, in order.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(SumArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    constexpr int kFlight = 8;
    const int lanes = 1 << a.g.lane_bits, groups = kThreads >> a.g.lane_bits;
    const long c = ((long)blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * kN;
    const long q = (long)blockIdx.x * groups + (threadIdx.x >> a.g.lane_bits);
    if (c >= a.g.dim || q + 1 >= a.chunks) return;  // (the last chunk's classes end in it)
    const int left = (int)min((long)kN, a.g.dim - c);
    const unsigned none = (unsigned)a.g.n_classes;
    const long begin = q * a.chunk, end = begin + a.chunk;
    const unsigned key = a.keys[end - 1];
    if (key == none || a.keys[end] != key) return;
    if (begin > 0 && a.keys[begin - 1] == key) return;  // it began earlier
    long low = end, high = a.g.n_ids;  // the first position behind the class: in (low, high]
    while (high - low > 1) {
        const long mid = (low + high) / 2;
        (a.keys[mid] == key ? low : high) = mid;
    }
    const long last = low / a.chunk;
    float sum[kN];
    const float* part = a.part + c;
#pragma unroll
    for (int e = 0; e < kN; ++e) sum[e] = e < left ? part[(q * 2 + 1) * a.g.dim + e] : 0.f;
    for (long r = q + 1; r <= last; r += kFlight) {
        float x[kFlight][kN];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (r + u <= last) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[u][e] = e < left ? part[(r + u) * 2 * a.g.dim + e] : 0.f;
            }
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (r + u <= last) {
#pragma unroll
                for (int e = 0; e < kN; ++e) sum[e] += x[u][e];
            }
    }
    finish_columns<T, kN>(a.g, static_cast<T*>(a.g.table) + key * a.g.table_stride + c, left, sum);
}

// ---- host -----------------------------------------------------------------------------------------------------------

int check_lookup(const nuts_lookup_desc* d, const char* who)
{
    if (!d) return api_fail(NUTS_E_INVALID_ARG, "%s: desc must not be NULL", who);
    if (!cat_dtype_known(d->dtype)) return api_fail(NUTS_E_INVALID_ARG, "%s: dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16", who);
    if (d->id_type != NUTS_I32 && d->id_type != NUTS_I64) return api_fail(NUTS_E_INVALID_ARG, "%s: id_type must be NUTS_I32 or NUTS_I64", who);
    if (d->n_ids < 0 || d->n_ids > INT32_MAX - 1) return api_fail(NUTS_E_INVALID_ARG, "%s: n_ids must be in [0, 2^31 - 2]", who);
    if (d->n_classes < 1 || d->n_classes > INT32_MAX - 1) return api_fail(NUTS_E_INVALID_ARG, "%s: n_classes must be in [1, 2^31 - 2]", who);
    if (d->dim < 1 || d->dim > (1 << 24)) return api_fail(NUTS_E_INVALID_ARG, "%s: dim must be in [1, 2^24]", who);
    if (d->table_stride < d->dim || d->row_stride < d->dim) return api_fail(NUTS_E_INVALID_ARG, "%s: a stride is smaller than dim", who);
    if (d->table_stride > INT64_MAX / 8 / d->n_classes || (d->n_ids > 0 && d->row_stride > INT64_MAX / 8 / d->n_ids))
        return api_fail(NUTS_E_INVALID_ARG, "%s: a stride is too large", who);
    if (!std::isfinite(d->scale) || !std::isfinite((float)d->scale)) return api_fail(NUTS_E_INVALID_ARG, "%s: scale must be finite", who);
    if (d->accumulate != 0 && d->accumulate != 1) return api_fail(NUTS_E_INVALID_ARG, "%s: accumulate must be 0 or 1", who);
    return NUTS_OK;
}

// Threads of a group that works on one row: a power of two, enough for 16 bytes each, no more than a workgroup.
int lane_bits_of(int64_t dim, int dtype, int least)
{
    const int64_t packs = ceil_div(dim, 16 / (int64_t)cat_size(dtype));
    int bits = least;
    while (bits < 8 && (1 << bits) < packs) ++bits;
    return bits;
}

struct GradPlan {
    bool few;
    int few_classes;
    int digit_bits, passes, tile, tiles;
    int chunk;
    long chunks;
    // offsets into the workspace
    size_t counts, starts, keys[2], pos[2], present, part, bytes;
};

GradPlan plan_grad(const nuts_lookup_desc* d)
{
    GradPlan p{};
    p.few = d->n_ids <= kFew;
    if (p.few) {
        // about a thousand workgroups where the table has so many rows: each looks through all positions again
        p.few_classes = (int)std::clamp<int64_t>(d->n_classes / 1024, 4, kFewRows);
        return p;
    }
    int bits = 1;
    while (d->n_classes >> bits) ++bits;  // n_classes itself is a key
    p.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    p.digit_bits = (bits + p.passes - 1) / p.passes;
    p.tile = d->n_ids <= (1 << 17) ? 2048 : 8192;
    p.tiles = (int)ceil_div(d->n_ids, p.tile);
    // chunks: short enough that there are thousands, long enough that a class over many of them is joined from few parts
    p.chunk = 32;
    while (d->n_ids / p.chunk > 4096) p.chunk *= 2;
    p.chunks = ceil_div(d->n_ids, p.chunk);
    auto take = [&](size_t bytes) {
        const size_t at = p.bytes;
        p.bytes += (bytes + 255) & ~(size_t)255;
        return at;
    };
    p.counts = take((size_t)p.tiles * sizeof(unsigned) << p.digit_bits);
    p.starts = take(sizeof(unsigned) << p.digit_bits);
    for (int s = 0; s < 2; ++s) {
        p.keys[s] = take(sizeof(unsigned) * d->n_ids);
        p.pos[s] = take(sizeof(unsigned) * d->n_ids);
    }
    p.present = take((size_t)d->n_classes + 16);
    p.part = take((size_t)p.chunks * 2 * d->dim * sizeof(float));
    return p;
}

}  // namespace
}  // namespace nuts

using namespace nuts;

extern "C" {

int nuts_lookup(const nuts_lookup_desc* d, const void* table, const void* ids, void* rows)
{
    if (int rc = check_lookup(d, "nuts_lookup")) return rc;
    if (d->n_ids == 0) return NUTS_OK;
    if (!table || !ids || !rows) return api_fail(NUTS_E_INVALID_ARG, "nuts_lookup: null pointer");
    if (int rc = api_have_device()) return rc;
    LookupArgs a{table, ids, rows, 0, (long)d->n_ids, (long)d->n_classes, (long)d->dim, (long)d->table_stride, (long)d->row_stride,
                 (float)d->scale, d->id_type, lane_bits_of(d->dim, d->dtype, 0)};
    const int groups = kThreads >> a.lane_bits;
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        // several rows a group where that leaves the chip more workgroups than it holds at once (2048)
        const bool several = d->n_ids >= 4 * 2048 * (int64_t)groups;
        for (const long blocks = (long)ceil_div(d->n_ids, (several ? 4 : 1) * groups); a.first_block < blocks; a.first_block += kMaxBlocks)
            hipLaunchKernelGGL((several ? lookup_kernel<T, 4> : lookup_kernel<T, 1>), dim3((unsigned)std::min(blocks - a.first_block, kMaxBlocks)),
                               dim3(kThreads), 0, api_stream(), a);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_lookup_grad_workspace(const nuts_lookup_desc* d, int64_t* bytes)
{
    if (int rc = check_lookup(d, "nuts_lookup_grad_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_lookup_grad_workspace: bytes must not be NULL");
    *bytes = (int64_t)plan_grad(d).bytes;
    return NUTS_OK;
}

int nuts_lookup_grad(const nuts_lookup_desc* d, const void* grad_rows, const void* ids, void* grad_table, void* workspace,
                     int64_t workspace_bytes)
{
    if (int rc = check_lookup(d, "nuts_lookup_grad")) return rc;
    if (!grad_table || (d->n_ids > 0 && (!grad_rows || !ids))) return api_fail(NUTS_E_INVALID_ARG, "nuts_lookup_grad: null pointer");
    const GradPlan p = plan_grad(d);
    if ((int64_t)p.bytes > 0 && (!workspace || workspace_bytes < (int64_t)p.bytes))
        return api_fail(NUTS_E_INVALID_ARG, "nuts_lookup_grad: needs a workspace of %zu bytes", p.bytes);
    if (reinterpret_cast<uintptr_t>(workspace) % 256 && p.bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_lookup_grad: workspace must be aligned to 256 bytes");
    if (int rc = api_have_device()) return rc;
    hipStream_t stream = api_stream();
    SumArgs a{};
    a.g = GradArgs{grad_rows, ids, grad_table, (long)d->n_ids, (long)d->n_classes, (long)d->dim, (long)d->table_stride, (long)d->row_stride,
                   (float)d->scale, d->id_type, d->accumulate, 0};
    if (p.few) {
        a.g.lane_bits = lane_bits_of(d->dim, d->dtype, 6) > 6 ? 8 : 6;
        by_dtype(d->dtype, [&](auto t) {
            for (long first = 0, blocks = (long)ceil_div(d->n_classes, p.few_classes); first < blocks; first += kMaxBlocks)
                hipLaunchKernelGGL(few_rows_kernel<decltype(t)>, dim3((unsigned)std::min(blocks - first, kMaxBlocks)), dim3(kThreads), 0, stream, a.g,
                                   p.few_classes, first);
        });
        NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
        return NUTS_OK;
    }
    char* w = static_cast<char*>(workspace);
    unsigned char* present = d->accumulate ? nullptr : reinterpret_cast<unsigned char*>(w + p.present);
    for (int k = 0; k < p.passes; ++k) {
        SortArgs s{ids, reinterpret_cast<unsigned*>(w + p.keys[(k + 1) & 1]), reinterpret_cast<unsigned*>(w + p.pos[(k + 1) & 1]),
                   reinterpret_cast<unsigned*>(w + p.keys[k & 1]), reinterpret_cast<unsigned*>(w + p.pos[k & 1]),
                   reinterpret_cast<unsigned*>(w + p.counts), reinterpret_cast<unsigned*>(w + p.starts), present,
                   (long)d->n_ids, (long)d->n_classes, d->id_type, k * p.digit_bits, p.digit_bits, p.tile, p.tiles};
        const size_t lds = (size_t)kWaves * sizeof(unsigned) << p.digit_bits;
        hipLaunchKernelGGL(k == 0 ? count_kernel<true> : count_kernel<false>, dim3(p.tiles), dim3(kThreads), 0, stream, s);
        hipLaunchKernelGGL(places_kernel, dim3(1), dim3(1024), 0, stream, s);
        hipLaunchKernelGGL(k == 0 ? place_kernel<true> : place_kernel<false>, dim3(p.tiles), dim3(kThreads), lds, stream, s);
    }
    a.keys = reinterpret_cast<unsigned*>(w + p.keys[(p.passes - 1) & 1]);
    a.pos = reinterpret_cast<unsigned*>(w + p.pos[(p.passes - 1) & 1]);
    a.present = present;
    a.part = reinterpret_cast<float*>(w + p.part);
    a.chunks = p.chunks;
    a.chunk = p.chunk;
    a.g.lane_bits = lane_bits_of(d->dim, d->dtype, 0);
    const int groups = kThreads >> a.g.lane_bits;
    const int64_t columns = (int64_t)(16 / cat_size(d->dtype)) << a.g.lane_bits;
    a.sum_blocks = (long)ceil_div(p.chunks, groups);
    const unsigned clear = present ? (unsigned)std::min<int64_t>(ceil_div(d->n_classes, groups), 4096) : 0u;
    const unsigned slices = (unsigned)ceil_div(d->dim, columns);
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(sum_kernel<T>, dim3((unsigned)a.sum_blocks + clear, slices), dim3(kThreads), 0, stream, a);
        hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)a.sum_blocks, slices), dim3(kThreads), 0, stream, a);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
