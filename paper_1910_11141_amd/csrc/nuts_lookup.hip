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
#include <type_traits>

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
    int id_type, lane_bits, streamed;
};

// A group of 2^lane_bits threads copies a row, 16 bytes a thread at a time: a wave a row where there are enough rows to fill the chip,
// which then waits for some of them while it writes others.  Bound by its reads and writes: 65536 rows of 4 KB 72 us, 6.9 TB/s of
// them, with stores past the caches; with plain ones 89 us (then also: with a workgroup a row 99 us, four 16-byte pieces of a row under
// way a thread 94 us, two or four rows a workgroup at once 95 and 104 us).  64 rows take 2.5 us, less than their launch.
template <typename T>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1);
    const long row = (a.first_block + blockIdx.x) * (kThreads >> a.lane_bits) + (threadIdx.x >> a.lane_bits);
    if (row >= a.n_ids) return;
    const int id = class_at(a.ids, a.id_type, row, a.n_classes);
    const T* from = static_cast<const T*>(a.table) + max(id, 0) * a.table_stride;
    T* to = static_cast<T*>(a.rows) + row * a.row_stride;
    for (long first = (long)lane * kN; first < a.dim; first += (long)lanes * kN) {
        const long c = max(0l, min(first, a.dim - kN));  // (a ragged row's last columns: 16 bytes that end with the row)
        if (c + kN <= a.dim) {
            Pack<T, kN> x;
            if (id >= 0) x = load_pack<T, kN>(from + c);
            Pack<T, kN> out;
#pragma unroll
            for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(id >= 0 ? to_float(x.v[e]) * a.scale : 0.f);
            a.streamed ? stream_pack(to + c, out) : store_pack(to + c, out);
        } else {
            for (long e = c; e < a.dim; ++e) to[e] = rounded<T>(id >= 0 ? to_float(from[e]) * a.scale : 0.f);
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
    int id_type, accumulate, lane_bits, streamed;
};

// The columns of the pack that begins at column `first`: where nothing is accumulated, the last pack of a ragged row ends with the
// row and shares columns with the one before, which has the same sums.
template <typename T, int kN>
struct Columns {
    long c;
    int left;  // columns from c on, at most kN; 0 behind the row
    __device__ Columns(const GradArgs& a, long first)
    {
        c = a.accumulate || a.dim < kN ? first : min(first, a.dim - kN);
        left = first < a.dim ? (int)min((long)kN, a.dim - c) : 0;
    }
};

// kN columns of a row; fewer, and zeros behind them, for the threads at a row's ragged end (kWhole = false).  Which of both a
// thread does is settled outside of its loops: loads on two ways that meet would be waited for one by one.
template <typename T, int kN, bool kWhole>
__device__ __forceinline__ Pack<T, kN> load_part(const T* p, int left)
{
    if (kWhole) return load_pack<T, kN>(p);
    Pack<T, kN> x;
#pragma unroll
    for (int e = 0; e < kN; ++e) x.v[e] = e < left ? p[e] : static_cast<T>(0.f);
    return x;
}
template <typename F>
__device__ __forceinline__ void by_width(bool whole, F f)
{
    if (whole) f(std::true_type{});
    else f(std::false_type{});
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
        if (sizeof(out) == 16 && a.streamed) stream_pack(p, *reinterpret_cast<const Pack<T, 16 / sizeof(T)>*>(&out));
        else store_pack(p, out);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (e < left) p[e] = rounded<T>(a.accumulate ? __builtin_fmaf(a.scale, sum[e], to_float(p[e])) : a.scale * sum[e]);
    }
}

template <typename T, int kN>
__device__ __forceinline__ void zero_columns(const GradArgs& a, T* p, int left)
{
    if (left >= kN) {
        Pack<T, kN> out;
#pragma unroll
        for (int e = 0; e < kN; ++e) out.v[e] = static_cast<T>(0.f);
        a.streamed ? stream_pack(p, out) : store_pack(p, out);
    } else {
        for (int e = 0; e < left; ++e) p[e] = static_cast<T>(0.f);
    }
}

// Threads that go together over the pieces of neighbouring rows: piece `first` of all rows' and every step-th behind it, without a
// division at each.
struct Steps {
    long row;
    int piece;
    const int pieces, piece_step;
    const long row_step;
    __device__ Steps(long first, long step, int n) : row(first / n), piece((int)(first % n)), pieces(n), piece_step((int)(step % n)), row_step(step / n) {}
    __device__ void next()
    {
        row += row_step;
        piece += piece_step;
        if (piece >= pieces) {
            piece -= pieces;
            ++row;
        }
    }
};

// ---- gradient of few rows: one launch --------------------------------------------------------------------------------

constexpr int kFewEach = 4;                    // positions of a thread
constexpr int kFew = kFewEach * kThreads;      // positions that a workgroup looks through by itself
constexpr int kFewRows = 64;                   // at most so many classes a workgroup (an occupancy mask is one word)

// A workgroup owns `classes` neighbouring rows of the table, or a slice of their columns: it finds the positions of theirs among all
// n (few, from cache) and adds them up.  What bounds it is the wait for memory, twice at least, and again for every 32 rows or so of
// the class that comes most often: 1000 positions, 5000 classes of 100 in binary32 9 us (13 where the frequent classes are neighbours).
// Slices: 1000 positions, 1000 classes of 2048 in binary32 16 us, 76 without; up to 4096 workgroups: 100 positions, 4168 classes of 1842,
// binary32 14 us, 23 with 2048 and 19 with 16384.  Sorting the positions first, as is done with more of them, takes three launches: 15 us
// for 1100 positions where this takes 11 for 1000.  Only a table that has to be cleared and is too large for the caches is cleared
// faster beside a sort (100003 classes of 2048 in bfloat16, 1000 positions: 77 us so, 92 by this kernel).
template <typename T>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(GradArgs a, int classes, long slice_packs, long first_block)
{
    constexpr int kN = 16 / sizeof(T);
    constexpr int kFlight = 8;
    __shared__ int position[kFew];
    __shared__ unsigned char of_class[kFew];
    __shared__ int found[kFewEach][kThreads / 64];
    __shared__ unsigned occupied_half[2];
    __shared__ int mine[kThreads / 64][64];    // a wave's class's among 64 positions
    __shared__ float sums[kThreads / 64][kN][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const long v0 = (first_block + blockIdx.x) * classes;
    const int own = (int)min((long)classes, a.n_classes - v0);
    if (threadIdx.x < 2) occupied_half[threadIdx.x] = 0u;
    int id[kFewEach];
    unsigned long long hits[kFewEach];
#pragma unroll
    for (int u = 0; u < kFewEach; ++u) {
        const int i = u * kThreads + (int)threadIdx.x;
        id[u] = i < a.n_ids ? class_at(a.ids, a.id_type, i, a.n_classes) : -1;
    }
#pragma unroll
    for (int u = 0; u < kFewEach; ++u) {
        hits[u] = __ballot(id[u] >= v0 && id[u] < v0 + own);
        if (lane == 0) found[u][wave] = __popcll(hits[u]);
    }
    __syncthreads();
    int count = 0;
#pragma unroll
    for (int u = 0; u < kFewEach; ++u)
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w == wave && (hits[u] >> lane & 1)) {
                const int at = count + __popcll(hits[u] & ((1ull << lane) - 1)), c = (int)(id[u] - v0);
                position[at] = u * kThreads + (int)threadIdx.x;
                of_class[at] = (unsigned char)c;
                atomicOr(&occupied_half[c >> 5], 1u << (c & 31));
            }
            count += found[u][w];
        }
    __syncthreads();
    const unsigned long long occupied = occupied_half[0] | (unsigned long long)occupied_half[1] << 32;
    const int first = (int)(blockIdx.y * slice_packs), packs = (int)min(slice_packs, (a.dim + kN - 1) / kN - first);
    T* table = static_cast<T*>(a.table) + v0 * a.table_stride;
    const T* rows = static_cast<const T*>(a.rows);
    if (!a.accumulate)
        for (Steps at(threadIdx.x, kThreads, packs); at.row < own; at.next()) {
            const Columns<T, kN> at_row(a, (long)(first + at.piece) * kN);
            if (!(occupied >> at.row & 1)) zero_columns<T, kN>(a, table + at.row * a.table_stride + at_row.c, at_row.left);
        }
    // Each class is added up by the whole workgroup: a row is read by 2^lane_bits lanes of a wave (or by a wave in several
    // turns), and every wave has a list of the class's positions for itself, of which its groups of lanes take turns.
    const int lanes = 1 << a.lane_bits, workers = kThreads >> a.lane_bits, worker = threadIdx.x >> a.lane_bits;
    for (unsigned long long rest = occupied; rest; rest &= rest - 1) {
        const int r = __builtin_ctzll(rest);
        for (int p = lane & (lanes - 1); p < ((packs + lanes - 1) & -lanes); p += lanes) {
            const Columns<T, kN> columns(a, (long)(first + p) * kN);
            const long c = columns.c;
            const int left = p < packs ? columns.left : 0;
            float sum[kN];
#pragma unroll
            for (int e = 0; e < kN; ++e) sum[e] = 0.f;
            for (int m = 0; m < count; m += 64) {
                const bool hit = m + lane < count && of_class[m + lane] == r;
                const unsigned long long all = __ballot(hit);
                if (hit) mine[wave][__popcll(all & ((1ull << lane) - 1))] = position[m + lane];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                const int n = left > 0 ? __popcll(all) : 0;
                by_width(left >= kN, [&](auto whole) {
                    for (int q = worker; q < n; q += workers * kFlight) {
                        Pack<T, kN> x[kFlight];
#pragma unroll
                        for (int u = 0; u < kFlight; ++u)  // (one row again where there are no more)
                            x[u] = load_part<T, kN, decltype(whole)::value>(rows + (long)mine[wave][q + u * workers < n ? q + u * workers : q] * a.row_stride + c, left);
#pragma unroll
                        for (int u = 0; u < kFlight; ++u)
                            if (q + u * workers < n) {
#pragma unroll
                                for (int e = 0; e < kN; ++e) sum[e] += to_float(x[u].v[e]);
                            }
                    }
                });
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            for (int step = lanes; step < 64; step *= 2)
#pragma unroll
                for (int e = 0; e < kN; ++e) sum[e] += __shfl_xor(sum[e], step);
#pragma unroll
            for (int e = 0; e < kN; ++e) sums[wave][e][lane] = sum[e];
            __syncthreads();
            if (wave == 0 && lane < lanes && left > 0) {
#pragma unroll
                for (int e = 0; e < kN; ++e) sum[e] = (sums[0][e][lane] + sums[1][e][lane]) + (sums[2][e][lane] + sums[3][e][lane]);
                finish_columns<T, kN>(a, table + r * a.table_stride + c, left, sum);
            }
            __syncthreads();
        }
    }
}

// ---- gradient: clearing the rows of classes that do not come -------------------------------------------------------------

constexpr int kClear = 16;        // neighbouring classes that a wave or workgroup looks at to clear them
constexpr int64_t kLongRow = 1024;  // bytes

struct ClearArgs {
    const unsigned char* present;  // NULL: every row is cleared
    char* table;
    long stride, bytes;            // of a row
    long from, to;                 // classes; from: a multiple of kClear
    int first_block, together, streamed;
};

// 16 bytes of a row of zeros, the last of them up to its end; shorter rows element by element.
__device__ __forceinline__ void clear_piece(const ClearArgs& a, long row, int piece)
{
    char* to = a.table + row * a.stride;
    const Pack<f16, 8> zeros{};
    if (a.bytes >= 16) {
        f16* p = reinterpret_cast<f16*>(to + min(piece * 16l, a.bytes - 16));
        a.streamed ? stream_pack(p, zeros) : store_pack(p, zeros);
    } else {
        for (int b = 0; b < a.bytes; b += 2) *reinterpret_cast<f16*>(to + b) = static_cast<f16>(0.f);
    }
}

// Workgroups of a kernel from first_block on.  Where not all rows are cleared, a wave looks at 16 classes at once, or, where rows are
// long, a workgroup (100003 rows of 4 KB, 65536 positions: 152 us with waves, 148 with workgroups).
__device__ void clear_rows(const ClearArgs& a)
{
    const int pieces = (int)((a.bytes + 15) / 16);
    const long block = (long)blockIdx.x - a.first_block, blocks = (long)gridDim.x - a.first_block;
    if (!a.present) {
        for (Steps at(block * blockDim.x + threadIdx.x, blocks * blockDim.x, pieces); a.from + at.row < a.to; at.next())
            clear_piece(a, a.from + at.row, at.piece);
        return;
    }
    const int team = a.together ? blockDim.x : 64, teams = blockDim.x / team, member = threadIdx.x % team;
    for (long v = a.from + (block * teams + threadIdx.x / team) * kClear; v < a.to; v += blocks * teams * kClear) {
        const uint4 flags = *reinterpret_cast<const uint4*>(a.present + v);  // (padded to whole words)
        unsigned absent = 0;
#pragma unroll
        for (int r = 0; r < kClear; ++r) {
            const unsigned word = r < 4 ? flags.x : r < 8 ? flags.y : r < 12 ? flags.z : flags.w;
            absent |= (unsigned)!(word >> r % 4 * 8 & 0xff) << r;
        }
        const long rows = min((long)kClear, a.to - v);
        for (Steps at(member, team, pieces); at.row < rows; at.next())
            if (absent >> at.row & 1) clear_piece(a, v + at.row, at.piece);
    }
}

// ---- gradient: sorting the positions by class ------------------------------------------------------------------------
//
// A stable radix sort, digit by digit from the lowest: every workgroup counts the digits of its tile of positions, the counts are turned
// into places, and every workgroup puts its tile's there.  Classes that are none get the key n_classes and end up last.
//
// Places are found by every workgroup for itself while the counts are few (kFewCounts), else by one workgroup in a launch of its
// own, which takes 8 us and the launch (the whole gradient, 32000 positions, 50000 classes of 512, binary32: 63 us so, 52 without;
// 65536 positions, 100003 classes of 2048, bfloat16: 156 and 152).

constexpr int kMaxDigitBits = 11;
constexpr int kWaves = kThreads / 64;
// rounds of a tile: short tiles while the counts of all of them are little work for one workgroup
constexpr int kFewRounds = 4, kManyRounds = 16;
constexpr long kManyIds = 1l << 17;
constexpr long kFewCounts = 1l << 16;  // tiles x digits: 256 KB, which each workgroup reads from cache

struct SortArgs {
    const void* ids;          // first digit: the classes themselves; else keys_in, pos_in
    const unsigned* keys_in;
    const unsigned* pos_in;
    unsigned* keys_out;
    unsigned* pos_out;
    unsigned* counts;         // [tile][digit], then places within the digit
    unsigned* starts;         // [digit]; NULL: counts are counts, and every workgroup finds its places itself
    unsigned char* present;   // [n_classes]: 1 where a class comes
    long n_ids, n_classes;
    int id_type, shift, digit_bits, tile, tiles;
    ClearArgs clear;          // what the workgroups behind those of the tiles do: small kernels leave the chip to that
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
    if (!kFirst && (int)blockIdx.x >= a.tiles) return clear_rows(a.clear);
    __shared__ unsigned count[1 << kMaxDigitBits];
    const int digits = 1 << a.digit_bits;
    for (int d = threadIdx.x; d < digits; d += kThreads) count[d] = 0;
    __syncthreads();
    const long begin = (long)blockIdx.x * a.tile, end = min(begin + a.tile, a.n_ids);
    for (long i = begin + threadIdx.x; i < end; i += 4 * kThreads) {
        unsigned key[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kThreads < end) key[u] = key_at<kFirst>(a, i + u * kThreads);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kThreads < end) atomicAdd(&count[key[u] >> a.shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kThreads) a.counts[(long)blockIdx.x * digits + d] = count[d];
    if (kFirst && a.present) {  // nothing is present yet
        const long words = (a.n_classes + 15) / 16;
        uint4* p = reinterpret_cast<uint4*>(a.present);
        for (long w = (long)blockIdx.x * kThreads + threadIdx.x; w < words; w += (long)a.tiles * kThreads) p[w] = uint4{0, 0, 0, 0};
    }
}

__global__ __launch_bounds__(1024) void places_kernel(SortArgs a)
{
    if (blockIdx.x >= 1) return clear_rows(a.clear);
    __shared__ unsigned total[1 << kMaxDigitBits];
    const int digits = 1 << a.digit_bits;
    for (int d = threadIdx.x; d < digits; d += 1024) {
        unsigned sum = 0;
        int t = 0;
        for (; t + 16 <= a.tiles; t += 16) {  // sixteen reads in flight
            unsigned c[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) c[u] = a.counts[(long)(t + u) * digits + d];
#pragma unroll
            for (int u = 0; u < 16; ++u) {
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

// A wave places its run of the tile, kRounds times 64 positions: lanes that hold the same digit find each other by a ballot for each bit.
// 65536 positions, 512 digits: 11 us, after 5 for the counts; waits for memory and LDS, one behind the other.
template <bool kFirst, int kRounds>
__global__ __launch_bounds__(kThreads) void place_kernel(SortArgs a)
{
    if (!kFirst && (int)blockIdx.x >= a.tiles) return clear_rows(a.clear);
    extern __shared__ unsigned next[];  // [wave][digit], [digit]
    const int digits = 1 << a.digit_bits, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const long begin = (long)blockIdx.x * a.tile + wave * kRounds * 64 + lane;
    unsigned key[kRounds], pos[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (begin + r * 64 < a.n_ids) {
            key[r] = key_at<kFirst>(a, begin + r * 64);
            pos[r] = kFirst ? (unsigned)(begin + r * 64) : a.pos_in[begin + r * 64];
        }
    for (int d = threadIdx.x; d < kWaves * digits; d += kThreads) next[d] = 0;
    __syncthreads();
    unsigned* own = next + wave * digits;
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (begin + r * 64 < a.n_ids) atomicAdd(&own[key[r] >> a.shift & (digits - 1)], 1u);
    unsigned* starts = next + kWaves * digits;
    constexpr int kEach = (1 << kMaxDigitBits) / kThreads;
    unsigned before[kEach];  // in the tiles before this one
    if (a.starts) {
#pragma unroll
        for (int u = 0; u < kEach; ++u)
            if (const int d = u * kThreads + (int)threadIdx.x; d < digits) {
                starts[d] = a.starts[d];
                before[u] = a.counts[(long)blockIdx.x * digits + d];
            }
    } else {
        constexpr int kFlight = 32;
#pragma unroll
        for (int u = 0; u < kEach; ++u)
            if (const int d = u * kThreads + (int)threadIdx.x; d < digits) {
                unsigned sum = 0, own_sum = 0;
                for (int t = 0; t < a.tiles; t += kFlight) {
                    unsigned c[kFlight];
#pragma unroll
                    for (int v = 0; v < kFlight; ++v) c[v] = a.counts[(long)min(t + v, a.tiles - 1) * digits + d];
#pragma unroll
                    for (int v = 0; v < kFlight; ++v) {
                        if (t + v == (int)blockIdx.x) own_sum = sum;
                        sum += t + v < a.tiles ? c[v] : 0u;
                    }
                }
                before[u] = own_sum;
                starts[d] = sum;
            }
        // the sums of the digits below: a thread's `each` digits, the threads of its wave below it, the waves below
        __shared__ unsigned of_wave[kWaves];
        __syncthreads();
        const int each = max(1, digits / kThreads), first = (int)threadIdx.x * each;
        unsigned own_sum = 0;
        for (int d = first; d < min(first + each, digits); ++d) own_sum += starts[d];
        unsigned sum = own_sum;
        for (int step = 1; step < 64; step *= 2) {
            const unsigned other = __shfl_up(sum, step);
            if (lane >= step) sum += other;
        }
        if (lane == 63) of_wave[wave] = sum;
        __syncthreads();
        unsigned at = sum - own_sum;
        for (int w = 0; w < wave; ++w) at += of_wave[w];
        for (int d = first; d < min(first + each, digits); ++d) {
            const unsigned c = starts[d];
            starts[d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int d = u * kThreads + (int)threadIdx.x;
        if (d >= digits) continue;
        unsigned at = starts[d] + before[u];
        for (int w = 0; w < kWaves; ++w) {
            const unsigned c = next[w * digits + d];
            next[w * digits + d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const bool valid = begin + r * 64 < a.n_ids;
        const unsigned digit = valid ? key[r] >> a.shift & (digits - 1) : 0u;
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
            a.keys_out[start + before] = key[r];
            a.pos_out[start + before] = pos[r];
            if (kFirst && a.present && key[r] < (unsigned long)a.n_classes) a.present[key[r]] = 1;
        }
    }
}

// Not too many positions are sorted in one launch: a position's place is the number of those of lower classes and of those before it
// of its own.  A workgroup finds the places of 16 positions, each of its 512 threads counts for all of them among every 512th: n^2 / 64
// comparisons of a wave, which bound it.  2000 positions take 6 us, where the launches of the digits' sort take 25 us together.  The whole
// gradient of 1000 classes of 25 (one digit), binary32: 10000 positions 28 us so, as long as 16000 by digits; of 50000 classes of 512 (two
// digits) 10000 positions 37 us and 16384 54, 16385 by digits 46; of 100003 classes of 2048, bfloat16, cleared beside the sort, 102
// and 119.  1000 classes of 25, 10000 positions with 256 threads 30 us, with 1024 33.
constexpr int kRanked = 16, kRankThreads = 512;
constexpr long kRankedIds = 10240, kRankedIdsOfMany = 12288, kRankedIdsBesideClearing = 16384;  // one digit; more; a table past the caches

struct RankArgs {
    const void* ids;
    unsigned* keys;
    unsigned* pos;
    long n_ids, n_classes;
    int id_type, blocks;
    ClearArgs clear;  // of the workgroups behind `blocks`
};

__global__ __launch_bounds__(kRankThreads) void rank_kernel(RankArgs a)
{
    if ((int)blockIdx.x >= a.blocks) return clear_rows(a.clear);
    constexpr int kFlight = 8, kLanes = kRankThreads / kRanked;
    __shared__ int own_keys[kRanked];
    __shared__ int counts[kRanked][kRankThreads + 1];
    const int n = (int)a.n_ids, first = (int)blockIdx.x * kRanked, last = min(first + kRanked, n);
    auto key_of = [&](int i) {
        const int id = class_at(a.ids, a.id_type, i, a.n_classes);
        return id < 0 ? (int)a.n_classes : id;
    };
    // Before its own position equal keys count too: those keys are taken one less.
    int key[kFlight];
    auto load = [&](int at) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int j = at + u * kRankThreads;
            key[u] = j < n ? key_of(j) - (j < first) : INT32_MAX;
        }
    };
    int at = threadIdx.x;
    load(at);
    if (threadIdx.x < kRanked) own_keys[threadIdx.x] = key_of(min(first + (int)threadIdx.x, n - 1));
    __syncthreads();
    int own[kRanked], count[kRanked];
#pragma unroll
    for (int o = 0; o < kRanked; ++o) {
        own[o] = __builtin_amdgcn_readfirstlane(own_keys[o]);
        count[o] = 0;
    }
    for (;;) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            if (__builtin_amdgcn_readfirstlane(at) + u * kRankThreads >= n) break;  // (for the whole wave)
#pragma unroll
            for (int o = 0; o < kRanked; ++o) count[o] += key[u] < own[o] ? 1 : 0;
        }
        at += kFlight * kRankThreads;
        if (at >= n) break;
        load(at);
    }
    if ((int)threadIdx.x < last - first) {
        const int mine = own_keys[threadIdx.x];
#pragma unroll
        for (int o = 0; o < kRanked; ++o) count[o] += (int)threadIdx.x < o && mine == own[o] ? 1 : 0;
    }
#pragma unroll
    for (int o = 0; o < kRanked; ++o) counts[o][threadIdx.x] = count[o];
    __syncthreads();
    const int o = threadIdx.x / kLanes, member = threadIdx.x % kLanes;
    int place = 0;
    for (int t = member; t < kRankThreads; t += kLanes) place += counts[o][t];
    for (int step = kLanes / 2; step; step /= 2) place += __shfl_xor(place, step);
    if (member == 0 && first + o < last) {
        a.keys[place] = (unsigned)own_keys[o];
        a.pos[place] = (unsigned)(first + o);
    }
}

// ---- gradient: adding up sorted rows ---------------------------------------------------------------------------------

struct SumArgs {
    GradArgs g;
    const unsigned* keys;
    const unsigned* pos;
    ClearArgs clear;               // of the workgroups behind sum_blocks
    float* part;                   // [chunk][2][part_stride]
    long chunks, sum_blocks, part_stride;
    int chunk;                     // positions in a chunk
};

constexpr int kBatch = 32;         // positions whose keys are read at once; a chunk is a multiple
// Where the whole call waits for single groups, chunks are shorter (1000 classes of 25, binary32: 1100 positions 20 us with 32 in a
// chunk, 17 with 16, 15 with 8; of 2048, bfloat16, 4000 positions 22 us with 16, 24 with 8, and 10000 41 and 46).
constexpr int kFewChunk = 8;
constexpr long kFewChunkIds = 4096;
constexpr int kLeastLanes = 3;     // groups of 8 threads and more: at most 32 in a workgroup

// A group of 2^lane_bits threads adds the rows of one chunk of the sorted positions, a thread 16 bytes of columns.  A class that
// lies wholly in the chunk is finished; what belongs to one that began before goes to the chunk's part 0, to one that begins
// here and goes on to part 1.  Bound by its reads and writes (65536 rows of 4 KB in 64 us: 405 MB at 6.3 TB/s).
template <typename T>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    constexpr int kFlight = 8;
    __shared__ unsigned keys[kThreads >> kLeastLanes][kBatch], positions[kThreads >> kLeastLanes][kBatch];
    const int lanes = 1 << a.g.lane_bits, groups = kThreads >> a.g.lane_bits, group = threadIdx.x >> a.g.lane_bits;
    const int lane = threadIdx.x & (lanes - 1);
    T* table = static_cast<T*>(a.g.table);
    const Columns<T, kN> columns(a.g, ((long)blockIdx.y * lanes + lane) * kN);
    const long c = columns.c;
    const int left = columns.left;
    if ((long)blockIdx.x >= a.sum_blocks) {
        if (blockIdx.y == 0) clear_rows(a.clear);
        return;
    }
    const long q = (long)blockIdx.x * groups + group;
    const long begin = min(q * a.chunk, a.g.n_ids), end = min(begin + a.chunk, a.g.n_ids);
    const T* rows = static_cast<const T*>(a.g.rows) + c;
    const unsigned none = (unsigned)a.g.n_classes;
    const unsigned before = begin > 0 ? a.keys[begin - 1] : none, after = end < a.g.n_ids ? a.keys[end] : none;
    float sum[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) sum[e] = 0.f;
    unsigned current = none;
    bool entered = false;  // the class began in an earlier chunk
    auto flush = [&](bool open) {
        if (current == none || left == 0) return;
        if (entered || open) {  // (parts are padded to whole packs)
            float* to = a.part + (q * 2 + (entered ? 0 : 1)) * a.part_stride + c;
#pragma unroll
            for (int e = 0; e < kN; e += 4) store_pack(to + e, Pack<float, 4>{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]});
        } else {
            finish_columns<T, kN>(a.g, table + current * a.g.table_stride + c, left, sum);
        }
    };
    for (int batch = 0; batch < a.chunk; batch += kBatch) {
        const long first = begin + batch;
        for (int i = lane; i < kBatch; i += lanes) {
            keys[group][i] = first + i < end ? a.keys[first + i] : none;
            positions[group][i] = first + i < end ? a.pos[first + i] : 0u;
        }
        __syncthreads();
        if (batch == 0) {
            current = keys[group][0];
            entered = current == before;
        }
        if (left > 0)
            by_width(left >= kN, [&](auto whole) {
                for (int i = 0; i < kBatch && keys[group][i] != none; i += kFlight) {  // (no class: such keys are the last)
                    Pack<T, kN> x[kFlight];
#pragma unroll
                    for (int u = 0; u < kFlight; ++u)  // (a row of no class is read and not used)
                        x[u] = load_part<T, kN, decltype(whole)::value>(rows + (long)positions[group][i + u] * a.g.row_stride, left);
#pragma unroll
                    for (int u = 0; u < kFlight; ++u) {
                        const unsigned key = keys[group][i + u];
                        if (key == none) break;
                        if (key != current) {
                            flush(false);
                            current = key;
                            entered = false;
#pragma unroll
                            for (int e = 0; e < kN; ++e) sum[e] = 0.f;
                        }
#pragma unroll
                        for (int e = 0; e < kN; ++e) sum[e] += to_float(x[u].v[e]);
                    }
                }
            });
        __syncthreads();
    }
    flush(current == after);
}

// Classes that reach over chunks: the workgroups of the chunk in which one begins join its parts.  Each of the four waves adds every
// fourth part, in order, four columns a thread; then the waves' sums are added in order.  Bound by the wait for the parts of the class
// that comes most often, 32 at a time (9 us where it comes 3600 times, with 64 positions in a chunk).
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(SumArgs a)
{
    constexpr int kFlight = 8;
    __shared__ int over[kThreads / 64];
    __shared__ float4 sums[kThreads / 64][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const long q = blockIdx.x, begin = q * a.chunk, end = begin + a.chunk;  // (the last chunk's classes end in it and have no workgroup)
    const unsigned none = (unsigned)a.g.n_classes;
    const unsigned key = a.keys[end - 1], next = a.keys[end], before = begin > 0 ? a.keys[begin - 1] : none;
    if (key == none || next != key || before == key) return;
    // the chunks behind this one that the class goes on beyond: all of the first, and then none
    long more = 0;
    for (long first = q + 1;; first += kThreads) {
        const long r = first + threadIdx.x;
        const bool goes_on = (r + 1) * a.chunk < a.g.n_ids && a.keys[(r + 1) * a.chunk] == key;
        const unsigned long long all = __ballot(goes_on);
        if (lane == 0) over[wave] = __popcll(all);
        __syncthreads();
        int here = 0;
        for (int w = 0; w < kThreads / 64; ++w) here += over[w];
        __syncthreads();
        more += here;
        if (here < kThreads) break;
    }
    const long parts = more + 2;  // this chunk's, those of the chunks that it goes on beyond, that of the one where it ends
    const long c = ((long)blockIdx.y * 64 + lane) * 4;
    const float* part = a.part + q * 2 * a.part_stride + min(c, a.part_stride - 4);
    float4 sum{0.f, 0.f, 0.f, 0.f};
    for (long r = wave; r < parts; r += kThreads / 64 * kFlight) {
        float4 x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const long at = min(r + u * (kThreads / 64), parts - 1);  // (one part again where there are no more)
            x[u] = *reinterpret_cast<const float4*>(part + (at * 2 + (at == 0 ? 1 : 0)) * a.part_stride);
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
            if (r + u * (kThreads / 64) < parts) {
                sum.x += x[u].x;
                sum.y += x[u].y;
                sum.z += x[u].z;
                sum.w += x[u].w;
            }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= a.g.dim) return;
    float total[4] = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < kThreads / 64; ++w) {
        const float4 x = sums[w][lane];
        total[0] += x.x;
        total[1] += x.y;
        total[2] += x.z;
        total[3] += x.w;
    }
    finish_columns<T, 4>(a.g, static_cast<T*>(a.g.table) + key * a.g.table_stride + c, (int)min(4l, a.g.dim - c), total);
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
    bool few, ranked;
    int few_classes;
    long slice_packs;
    int digit_bits, passes, tile, tiles;
    int chunk;
    long chunks, part_stride;
    // offsets into the workspace
    size_t counts, starts, keys[2], pos[2], present, part, bytes;
};

GradPlan plan_grad(const nuts_lookup_desc* d)
{
    GradPlan p{};
    const bool large = !d->accumulate && d->n_classes * d->dim * (int64_t)cat_size(d->dtype) >= kStreamed;
    p.few = d->n_ids <= kFew && !large;
    if (p.few) {
        // about a thousand workgroups where the table has so many rows: each looks through all positions again; else the columns
        // are shared out too
        p.few_classes = (int)std::clamp<int64_t>(d->n_classes / 1024, 4, kFewRows);
        const int64_t packs = ceil_div(d->dim, 16 / (int64_t)cat_size(d->dtype)), lanes = 1 << std::min(6, lane_bits_of(d->dim, d->dtype, 0));
        const int64_t slices = std::clamp<int64_t>(4096 / ceil_div(d->n_classes, p.few_classes), 1, ceil_div(packs, lanes));
        p.slice_packs = (long)(ceil_div(ceil_div(packs, lanes), slices) * lanes);
        return p;
    }
    int bits = 1;
    while (d->n_classes >> bits) ++bits;  // n_classes itself is a key
    p.ranked = d->n_ids <= (large ? kRankedIdsBesideClearing : bits > kMaxDigitBits ? kRankedIdsOfMany : kRankedIds);
    p.passes = p.ranked ? 0 : (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    p.digit_bits = p.ranked ? 0 : (bits + p.passes - 1) / p.passes;
    p.tile = (d->n_ids <= kManyIds ? kFewRounds : kManyRounds) * kThreads;
    p.tiles = (int)ceil_div(d->n_ids, p.tile);
    // chunks: short enough that there are a thousand workgroups, long enough that a class over many of them is joined from few parts
    p.chunk = d->n_ids <= kFewChunkIds ? kFewChunk : p.ranked ? 2 * kFewChunk : kBatch;
    while (d->n_ids / (p.chunk * 2) >= 1024 * (int64_t)(kThreads >> lane_bits_of(d->dim, d->dtype, kLeastLanes))) p.chunk *= 2;
    p.chunks = ceil_div(d->n_ids, p.chunk);
    auto take = [&](size_t bytes) {
        const size_t at = p.bytes;
        p.bytes += (bytes + 255) & ~(size_t)255;
        return at;
    };
    for (int s = 0; s < std::min(2, std::max(1, p.passes)); ++s) {
        p.keys[s] = take(sizeof(unsigned) * d->n_ids);
        p.pos[s] = take(sizeof(unsigned) * d->n_ids);
    }
    if (!p.ranked) {
        p.counts = take((size_t)p.tiles * sizeof(unsigned) << p.digit_bits);
        p.starts = take(sizeof(unsigned) << p.digit_bits);
        p.present = take((size_t)d->n_classes + kClear);
    }
    p.part_stride = (long)(ceil_div(d->dim, 8) * 8);
    p.part = take((size_t)p.chunks * 2 * p.part_stride * sizeof(float));
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
                 (float)d->scale, d->id_type, std::min(d->n_ids >= 2048 ? 6 : 8, lane_bits_of(d->dim, d->dtype, 0)),
                 d->n_ids * d->dim * (int64_t)cat_size(d->dtype) >= kStreamed};
    const int groups = kThreads >> a.lane_bits;
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        for (const long blocks = (long)ceil_div(d->n_ids, groups); a.first_block < blocks; a.first_block += kMaxBlocks)
            hipLaunchKernelGGL(lookup_kernel<T>, dim3((unsigned)std::min(blocks - a.first_block, kMaxBlocks)), dim3(kThreads), 0, api_stream(), a);
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
                   (float)d->scale, d->id_type, d->accumulate, 0, d->n_classes * d->dim * (int64_t)cat_size(d->dtype) >= kStreamed};
    if (p.few) {
        a.g.lane_bits = std::min(6, lane_bits_of(d->dim, d->dtype, 0));
        by_dtype(d->dtype, [&](auto t) {
            constexpr int64_t kN = 16 / sizeof(decltype(t));
            const unsigned slices = (unsigned)ceil_div(ceil_div(d->dim, kN), p.slice_packs);
            for (long first = 0, blocks = (long)ceil_div(d->n_classes, p.few_classes); first < blocks; first += kMaxBlocks)
                hipLaunchKernelGGL(few_rows_kernel<decltype(t)>, dim3((unsigned)std::min(blocks - first, kMaxBlocks), slices), dim3(kThreads), 0, stream,
                                   a.g, p.few_classes, p.slice_packs, first);
        });
        NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
        return NUTS_OK;
    }
    char* w = static_cast<char*>(workspace);
    unsigned char* present = d->accumulate ? nullptr : reinterpret_cast<unsigned char*>(w + p.present);
    // The rows to clear are known when the first digit has been placed: what is left of the sort, two or three small kernels a digit,
    // clears them in equal shares beside it (with one digit the kernel of the sums does).
    const int64_t size = (int64_t)cat_size(d->dtype);
    const bool few_counts = (int64_t)p.tiles << p.digit_bits <= kFewCounts;
    const int shares = std::max(1, (few_counts ? 2 : 3) * (p.passes - 1));
    const int64_t share = ceil_div(ceil_div(d->n_classes, shares), kClear) * kClear;
    int shared_out = 0;
    auto next_share = [&](int first_block, int waves, unsigned* more) {
        ClearArgs c{present, static_cast<char*>(grad_table), (long)(d->table_stride * size), (long)(d->dim * size),
                    (long)std::min(d->n_classes, share * shared_out), (long)std::min(d->n_classes, share * (shared_out + 1)), first_block,
                    d->dim * size >= kLongRow, a.g.streamed};
        ++shared_out;
        *more = present ? (unsigned)std::min<int64_t>(ceil_div(c.to - c.from, (c.together ? 1 : waves) * kClear), 1 << 16) : 0u;
        return c;
    };
    unsigned more = 0;
    if (p.ranked) {
        // So few positions' rows cost less to write twice than to find out about beforehand: all are cleared, 8 pieces a thread.
        RankArgs r{ids, reinterpret_cast<unsigned*>(w + p.keys[0]), reinterpret_cast<unsigned*>(w + p.pos[0]), (long)d->n_ids, (long)d->n_classes,
                   d->id_type, (int)ceil_div(d->n_ids, kRanked), ClearArgs{}};
        r.clear = ClearArgs{nullptr, static_cast<char*>(grad_table), (long)(d->table_stride * size), (long)(d->dim * size), 0, (long)d->n_classes,
                            r.blocks, 0, a.g.streamed};
        if (!d->accumulate) more = (unsigned)std::min<int64_t>(ceil_div(d->n_classes * ceil_div(d->dim * size, 16), 8 * kRankThreads), 1 << 16);
        hipLaunchKernelGGL(rank_kernel, dim3(r.blocks + more), dim3(kRankThreads), 0, stream, r);
    }
    for (int k = 0; k < p.passes; ++k) {
        SortArgs s{ids, reinterpret_cast<unsigned*>(w + p.keys[(k + 1) & 1]), reinterpret_cast<unsigned*>(w + p.pos[(k + 1) & 1]),
                   reinterpret_cast<unsigned*>(w + p.keys[k & 1]), reinterpret_cast<unsigned*>(w + p.pos[k & 1]),
                   reinterpret_cast<unsigned*>(w + p.counts), few_counts ? nullptr : reinterpret_cast<unsigned*>(w + p.starts), present,
                   (long)d->n_ids, (long)d->n_classes, d->id_type, k * p.digit_bits, p.digit_bits, p.tile, p.tiles, ClearArgs{}};
        const size_t lds = (size_t)(kWaves + 1) * sizeof(unsigned) << p.digit_bits;
        if (k > 0) s.clear = next_share(p.tiles, kWaves, &more);
        hipLaunchKernelGGL(k == 0 ? count_kernel<true> : count_kernel<false>, dim3(p.tiles + more), dim3(kThreads), 0, stream, s);
        if (!few_counts) {
            if (k > 0) s.clear = next_share(1, 1024 / 64, &more);
            hipLaunchKernelGGL(places_kernel, dim3(1 + more), dim3(1024), 0, stream, s);
        }
        void (*place)(SortArgs) = d->n_ids <= kManyIds ? (k == 0 ? place_kernel<true, kFewRounds> : place_kernel<false, kFewRounds>)
                                                       : (k == 0 ? place_kernel<true, kManyRounds> : place_kernel<false, kManyRounds>);
        if (k > 0) s.clear = next_share(p.tiles, kWaves, &more);
        hipLaunchKernelGGL(place, dim3(p.tiles + more), dim3(kThreads), lds, stream, s);
    }
    const int sorted = p.ranked ? 0 : (p.passes - 1) & 1;
    a.keys = reinterpret_cast<unsigned*>(w + p.keys[sorted]);
    a.pos = reinterpret_cast<unsigned*>(w + p.pos[sorted]);
    a.part = reinterpret_cast<float*>(w + p.part);
    a.chunks = p.chunks;
    a.chunk = p.chunk;
    a.part_stride = p.part_stride;
    a.g.lane_bits = lane_bits_of(d->dim, d->dtype, kLeastLanes);
    const int groups = kThreads >> a.g.lane_bits;
    const int64_t columns = (int64_t)(16 / cat_size(d->dtype)) << a.g.lane_bits;
    a.sum_blocks = (long)ceil_div(p.chunks, groups);
    const unsigned slices = (unsigned)ceil_div(d->dim, columns);
    more = 0;
    if (p.passes == 1) a.clear = next_share((int)a.sum_blocks, kWaves, &more);
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        if (p.chunks > 0) hipLaunchKernelGGL(sum_kernel<T>, dim3((unsigned)a.sum_blocks + more, slices), dim3(kThreads), 0, stream, a);
        if (p.chunks > 1)
            hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)(p.chunks - 1), (unsigned)ceil_div(d->dim, 256)), dim3(kThreads), 0, stream, a);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
