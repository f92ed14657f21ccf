// Logits adjusted by what was said before, by biases and by masks, and the gradient of that.
//
//   z = x > 0 ? x / r : x r  where v was seen,   z -= f count_v + q [count_v > 0],   z += bias_v,   -infinity where v is not allowed
//   dx_v = g_v (seen_v ? (x > 0 ? 1 / r : r) : 1),   dbias_v = sum over rows of g_v,   0 where v is not allowed
#include "nuts_cat.h"

#include <algorithm>
#include <type_traits>

namespace nuts {
namespace {

// A workgroup's threads, and the classes that it has a counter for in LDS: a slice.  Each slice looks through the whole history.
struct Usual {
    static constexpr int kThreads = 512, kSlice = 4096;
};
struct Wide {
    static constexpr int kThreads = 1024, kSlice = 16384;
};
constexpr int kJoinThreads = 1024;
constexpr int kLong = 2048, kFull = 256;  // of wide slices: places of a history (binary32), workgroups
// Workgroups of rows that go together: what the chip has at a time (4096 rows, forward and gradient: 120 and 268 us; with twice as many 121 and
// 296, with two thirds of them 150 and 315).
constexpr int kGroups = 1024, kGradGroups = 768;
// Rows whose gradients are added up, at least: 1000 of 1000 binary32, joins included, 15.5 us with 2, 16.1 with 1 and with 4.
constexpr int64_t kBiasRows = 2;
// Rows that a workgroup adds up one behind the other, at most: sums of some thousands in binary32 lose three places (4 million rows on 768 workgroups: 7e-5 of a
// sum, which becomes 2e-6 with 128).  There are more workgroups then, for as many whole rounds of them as it takes (200000 rows of 1000 bfloat16 545 us, 633 with 768
// workgroups; binary32 717 and 709); and groups that are joined at a time, where there are more in two launches.
constexpr int64_t kBiasRun = 128, kJoined = 1024;
// Classes up to which 16 of them are joined by a workgroup, and not 64: 1000 classes 4.0 us and 5.7, 4000 3.5 and 3.7, 16384 5.7 and 4.1.
constexpr int kNarrow = 4096;

// A class's counter: how often it was said behind the prompt; whether it was in the prompt; whether it has a bias of its own, or several.
constexpr unsigned kPrompt = 1u << 31, kBiased = 1u << 30, kAgain = 1u << 29, kCount = kAgain - 1, kSeen = kPrompt | kCount;
constexpr unsigned kPlace = NUTS_CAT_MAX_BIAS - 1;  // of the bias that stands for a class

struct PenaltyArgs {
    const void* logits;
    const void* history;
    const int32_t* lengths;
    const int32_t* prompts;
    const float* repetition;
    const float* frequency;
    const float* presence;
    const float* bias;
    const void* bias_ids;
    const float* bias_values;
    const uint32_t* allowed;
    const void* grad_out;
    void* out;
    float* grad_bias;  // of groups of rows
    long first_block, row_stride, out_stride, grad_stride, allowed_stride, bias_stride, history_stride, n_rows;
    float r, f, q;
    int n_classes, id_type, history_len, n_bias, slices, rows_each, streamed;
};

// What all threads read at a place that no thread of the launch writes: by way of the scalar cache, whose loads nobody waits for who waits for a row.
template <typename V>
__device__ __forceinline__ V uniform(const V* p)
{
#ifdef __HIP_DEVICE_COMPILE__
    return *(const __attribute__((address_space(4))) V*)p;
#else
    return *p;
#endif
}

__device__ __forceinline__ long id_at(const void* ids, int id_type, long i)
{
    return id_type == NUTS_I64 ? static_cast<const int64_t*>(ids)[i] : (long)static_cast<const int32_t*>(ids)[i];
}

__device__ __forceinline__ int clamped(const int32_t* lengths, long row, int most, int otherwise)
{
    return lengths ? min(max(uniform(lengths + row), 0), most) : otherwise;
}

// Calls `see` for the places from .. to - 1 of a history that hold one of the classes begin .. begin + n - 1, thread by thread.
template <typename W, typename Id, typename See>
__device__ __forceinline__ void look_through(const Id* history, int from, int to, int begin, int n, See see)
{
    constexpr int kEach = 16 / sizeof(Id), kStep = W::kThreads * kEach, kFlight = 4;
    auto look = [&](Id id, int i) {
        const uint64_t v = (uint64_t)(int64_t)id - (uint64_t)begin;
        if (v < (uint64_t)n) see(i, (int)v);
    };
    long i = from + (long)threadIdx.x * kEach;
    for (; i + (kFlight - 1) * kStep + kEach <= to; i += kFlight * kStep) {
        Pack<Id, kEach> in[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) in[u] = load_pack<Id, kEach>(history + i + u * kStep);
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
#pragma unroll
            for (int e = 0; e < kEach; ++e) look(in[u].v[e], (int)i + u * kStep + e);
    }
    for (; i < to; i += kStep) {
        if (i + kEach <= to) {
            const Pack<Id, kEach> in = load_pack<Id, kEach>(history + i);
#pragma unroll
            for (int e = 0; e < kEach; ++e) look(in.v[e], (int)i + e);
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (i + e < to) look(history[i + e], (int)i + e);
        }
    }
}
template <typename W, typename See>
__device__ __forceinline__ void look_through(const PenaltyArgs& a, long row, int from, int to, int begin, int n, See see)
{
    if (a.id_type == NUTS_I64) look_through<W>(static_cast<const int64_t*>(a.history) + row * a.history_stride, from, to, begin, n, see);
    else look_through<W>(static_cast<const int32_t*>(a.history) + row * a.history_stride, from, to, begin, n, see);
}

// The class at a place of a row's history, as one of the slice, or -1: the same for all threads.
__device__ __forceinline__ int class_in(const PenaltyArgs& a, long row, int i, int begin, int n)
{
    const long at = row * a.history_stride + i;
    const long id = a.id_type == NUTS_I64 ? (long)uniform(static_cast<const int64_t*>(a.history) + at) : (long)uniform(static_cast<const int32_t*>(a.history) + at);
    const uint64_t v = (uint64_t)id - (uint64_t)begin;
    return v < (uint64_t)n ? (int)v : -1;
}

// A row's history: how long it is, and how much of it is prompt.
struct Seen {
    int length, prompt;
};
__device__ __forceinline__ Seen seen_of(const PenaltyArgs& a, long row)
{
    return Seen{clamped(a.lengths, row, a.history_len, a.history_len), clamped(a.prompts, row, a.history_len, 0)};
}

// The counters of a thread's classes: those of its packs, of which pack u begins at class (u threads + thread) kN of the slice.
template <typename T>
constexpr int kPackN = 16 / sizeof(T);
template <typename W, typename T>
constexpr int kPacks = W::kSlice / W::kThreads / kPackN<T>;
template <typename W, typename T>
__device__ __forceinline__ int class_of_pack(int u)
{
    return (u * W::kThreads + (int)threadIdx.x) * kPackN<T>;
}
template <typename W, typename T>
struct Counters {
    unsigned c[kPacks<W, T>][kPackN<T>];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u)
#pragma unroll
            for (int e = 0; e < kPackN<T>; ++e) c[u][e] = 0;
    }
    __device__ __forceinline__ unsigned any(int u) const
    {
        unsigned all = 0;
#pragma unroll
        for (int e = 0; e < kPackN<T>; ++e) all |= c[u][e];
        return all;
    }
    __device__ __forceinline__ void read(const unsigned* shared)
    {
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u)
#pragma unroll
            for (int e = 0; e < kPackN<T>; e += 4) {
                const uint4 in = *reinterpret_cast<const uint4*>(&shared[class_of_pack<W, T>(u) + e]);
                c[u][e] = in.x, c[u][e + 1] = in.y, c[u][e + 2] = in.z, c[u][e + 3] = in.w;
            }
    }
    // One class of the slice (or none) was said, or what was counted as said is prompt.  (A wave whose it is not goes on at once; the one whose it is has no
    // branches, which the compiler would make an index into memory.)
    __device__ __forceinline__ void said(int v, bool prompt, bool again)
    {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) {
            const unsigned off = (unsigned)(v - class_of_pack<W, T>(u));
            if (!__builtin_amdgcn_ballot_w64(off < (unsigned)kPackN<T>)) continue;
#pragma unroll
            for (int e = 0; e < kPackN<T>; ++e) {
                const unsigned hit = off == (unsigned)e;
                c[u][e] = prompt ? (c[u][e] - (hit & (unsigned)again)) | hit << 31 : c[u][e] + hit;
            }
        }
#endif
    }
};

// What single classes have as biases of their own: the row's, in their order, those of other slices with no class.  One of a class's biases stands
// for it in the end: its value is their sum, its count what was counted, and the class's counter is its place.
struct Biases {
    uint16_t v[NUTS_CAT_MAX_BIAS];
    float value[NUTS_CAT_MAX_BIAS];
    unsigned count[NUTS_CAT_MAX_BIAS];

    static constexpr uint16_t kNone = 0xffff;
    static_assert(Wide::kSlice < kNone && Usual::kSlice < kNone, "classes of 16 bits");

    template <typename W>
    __device__ __forceinline__ void read(const PenaltyArgs& a, long row, int begin, int n)
    {
        for (int k = threadIdx.x; k < a.n_bias; k += W::kThreads) {
            const uint64_t at = (uint64_t)id_at(a.bias_ids, a.id_type, row * a.n_bias + k) - (uint64_t)begin;
            v[k] = at < (uint64_t)n ? (uint16_t)at : kNone;
            value[k] = a.bias_values[row * a.n_bias + k];
        }
    }
    // While others count: the counters' bits do not touch.  Returns a bit for each of this thread's biases that is to stand for its class.
    template <typename W>
    __device__ __forceinline__ unsigned mark(const PenaltyArgs& a, unsigned* shared) const
    {
        unsigned mine = 0, bit = 1;
        for (int k = threadIdx.x; k < a.n_bias; k += W::kThreads, bit *= 2) {
            if (v[k] == kNone) continue;
            if (atomicOr(&shared[v[k]], kBiased) & kBiased) atomicOr(&shared[v[k]], kAgain);
            else mine |= bit;
        }
        return mine;
    }
    // Behind a barrier.  Classes of several values are added up by whole waves, one class after the other: the values of a class are read by one wave,
    // which then writes one of them.  (1000 rows of 8000 with 1000 biases each at random: 41 us, 178 with a thread for each class that looks through all;
    // 64 rows of 128000 with 300: 11.5, 19.9; 4096 rows of 1000 with 300: 68, 73.)
    template <typename W>
    __device__ __forceinline__ void add_up(const PenaltyArgs& a, unsigned mine, unsigned* shared)
    {
#ifdef __HIP_DEVICE_COMPILE__
        constexpr int kFlight = 4;
        static_assert(NUTS_CAT_MAX_BIAS % (kFlight * 64) == 0, "what is read and not a bias is not behind the arrays");
        const int lane = (int)threadIdx.x % 64;
        for (int first = __builtin_amdgcn_readfirstlane((int)threadIdx.x - lane); first < a.n_bias; first += W::kThreads, mine /= 2) {
            const int k = first + lane;
            const bool stands = mine & 1;
            const int own = stands ? v[k] : kNone;
            const unsigned c = stands ? shared[own] : 0;
            for (uint64_t several = __builtin_amdgcn_ballot_w64(c & kAgain); several; several &= several - 1) {
                const int leader = __builtin_ctzll(several), its = __builtin_amdgcn_readlane(own, leader);
                float sum = -0.f;  // (which adds nothing to anything)
                for (int from = 0; from < a.n_bias; from += kFlight * 64) {
                    int at[kFlight], x[kFlight];
#pragma unroll
                    for (int u = 0; u < kFlight; ++u) at[u] = v[from + u * 64 + lane], x[u] = __float_as_int(value[from + u * 64 + lane]);
#pragma unroll
                    for (int u = 0; u < kFlight; ++u)
                        for (uint64_t hits = __builtin_amdgcn_ballot_w64(at[u] == its && from + u * 64 + lane < a.n_bias); hits; hits &= hits - 1)
                            sum += __int_as_float(__builtin_amdgcn_readlane(x[u], __builtin_ctzll(hits)));
                }
                if (lane == leader) value[k] = sum;
            }
            if (stands) {
                count[k] = c & kSeen;
                shared[own] = kBiased | (unsigned)k;
            }
        }
#endif
    }
};

// The counters of a slice from a row's history, in LDS, where adding whole numbers in any order gives the same.
template <typename W, typename T, typename B>
__device__ __forceinline__ void count(const PenaltyArgs& a, long row, int begin, int n, const Seen& now, unsigned* shared, B&& biases, Counters<W, T>& counters)
{
    constexpr bool kBiases = std::is_same_v<B, Biases&>;
    if constexpr (kBiases) biases.template read<W>(a, row, begin, n);
    else __syncthreads();  // (a row before this one may still be read)
    for (int i = (int)threadIdx.x * 4; i < (n + 7) / 8 * 8; i += W::kThreads * 4) *reinterpret_cast<uint4*>(&shared[i]) = uint4{0, 0, 0, 0};
    __syncthreads();
    unsigned mine = 0;
    if constexpr (kBiases) mine = biases.template mark<W>(a, shared);
    look_through<W>(a, row, 0, now.length, begin, n, [&](int i, int v) {
        if (i >= now.prompt) atomicAdd(&shared[v], 1u);
        else atomicOr(&shared[v], kPrompt);
    });
    __syncthreads();
    if constexpr (kBiases) {
        biases.template add_up<W>(a, mine, shared);
        __syncthreads();
    }
    counters.read(shared);
}

// Places of a history that a row has more than the one before and that each thread looks at by itself.
constexpr int kFew = 16;

// Where all rows have one history and a row has seen a little more of it than the one before, the counters stay in registers and what is new is added
// to them: rows of one text wait for no one then.  False: it is not so.  (Gradient of 4096 rows of 50001: 362 us with counters in LDS and barriers
// before and behind each row, 308 so, 284 with what is the same for all threads read by way of the scalar cache.)
template <typename W, typename T>
__device__ __forceinline__ bool count_on(const PenaltyArgs& a, long row, int begin, int n, const Seen& done, const Seen& now, Counters<W, T>& counters)
{
    const int more = now.length - done.length, less = now.prompt - done.prompt;
    if (more < 0 || less < 0 || more > kFew || less > kFew) return false;
    for (int i = done.prompt; i < min(now.prompt, done.length); ++i) counters.said(class_in(a, row, i, begin, n), true, true);
    for (int i = done.length; i < now.length; ++i) counters.said(class_in(a, row, i, begin, n), i < now.prompt, false);
    return true;
}

struct RowFactors {
    float r, by_r, f, q;
};
// Without branches: of 64 lanes one has a class that was seen nearly always.  (A product with 1 / r is a unit in the last place off x / r at most,
// and a quotient ten instructions more.)
__device__ __forceinline__ float penalised(float x, unsigned count, const RowFactors& p)
{
    const float z = x * (count & kSeen ? (x > 0.f ? p.by_r : p.r) : 1.f);
    const unsigned said = count & kCount;
    return z - (said ? __builtin_fmaf(p.f, (float)said, p.q) : 0.f);
}

// The pack at class v of a slice of n, which begins at `row`.  Where there are fewer numbers left, the last ones of the row up to there, which `unpack`
// puts in their places: one load without a branch, for a wave that would merge several has to wait for them.  (Rows that are shorter than a
// pack are read one by one.)  kOnce: past the caches, as far as they let it, for what nobody reads again.
template <bool kOnce, typename T>
__device__ __forceinline__ Pack<T, kPackN<T>> load_some(const T* row, int v, int n, int n_classes)
{
    constexpr int kN = kPackN<T>;
    Pack<T, kN> in{};
    if (n_classes >= kN) {
        if (v < n) {
            const T* at = row + min(v, n - kN);
            if (!kOnce) return load_pack<T, kN>(at);
            const typename Pack<T, kN>::Value words = __builtin_nontemporal_load(reinterpret_cast<const typename Pack<T, kN>::Words*>(at));
            __builtin_memcpy(&in, &words, sizeof(in));
        }
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (v + e < n) in.v[e] = row[v + e];
    }
    return in;
}
template <typename T>
__device__ __forceinline__ void unpack(const Pack<T, kPackN<T>>& in, int v, int n, int n_classes, float (&x)[kPackN<T>])
{
    constexpr int kN = kPackN<T>;
#pragma unroll
    for (int e = 0; e < kN; ++e) x[e] = to_float(in.v[e]);
    const int early = v + kN - n;  // numbers in front of v
    if (early > 0 && n_classes >= kN) {
#pragma unroll
        for (int step = kN / 2; step >= 1; step /= 2)
#pragma unroll
            for (int e = 0; e < kN; ++e) x[e] = early & step ? (e + step < kN ? x[e + step] : 0.f) : x[e];
    }
}
template <typename W, typename T>
struct Slice {
    Pack<T, kPackN<T>> pack[kPacks<W, T>];
    template <bool kOnce>
    __device__ __forceinline__ void fetch(const T* row, int n, int n_classes)
    {
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) pack[u] = load_some<kOnce>(row, class_of_pack<W, T>(u), n, n_classes);
    }
};
template <typename T>
__device__ __forceinline__ void write_pack(T* to, const float (&x)[kPackN<T>], int v, int n, bool streamed)
{
    Pack<T, kPackN<T>> out;
#pragma unroll
    for (int e = 0; e < kPackN<T>; ++e) out.v[e] = rounded<T>(x[e]);
    if (v + kPackN<T> <= n) {
        streamed ? stream_pack(to + v, out) : store_pack(to + v, out);
    } else {
#pragma unroll
        for (int e = 0; e < kPackN<T>; ++e)
            if (v + e < n) to[v + e] = out.v[e];
    }
}
template <int kN>
__device__ __forceinline__ void read_bias(const float* bias, int v, int n, float (&b)[kN])
{
    if (v + kN <= n) {
#pragma unroll
        for (int e = 0; e < kN; e += 4) {
            const Pack<float, 4> in = load_pack<float, 4>(bias + v + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) b[e + k] = in.v[k];
        }
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) b[e] = v + e < n ? bias[v + e] : 0.f;
    }
}
// A bit for each class of a pack that may come.
template <int kN>
__device__ __forceinline__ unsigned allowed_of(const uint32_t* allowed, int v, int n)
{
    constexpr unsigned kAll = (1u << kN) - 1;
    return allowed && v < n ? reinterpret_cast<const unsigned char*>(allowed)[v >> 3] >> (v & 7) & kAll : kAll;
}

// A workgroup a slice of one row, or (kShared) of `rows_each` rows that have one history.  Bound by its reads and writes: 4096 rows of 32001 bfloat16
// with one history and biases 112 us, 4.7 TB/s (120 with stores that the caches keep, 119 with loads that they do, 135 with registers enough for all of it and fewer waves), 500 rows of 128000 with histories
// of their own 56 us (68 with loads that the caches keep), 4.6 TB/s.  64 such rows with masks and 32 biases each take 13 us: a length, a history and
// the counters, waited for one behind the other.  4096 rows of 32001 binary32 216 us, 4.9 TB/s, though a lane keeps 56 bytes in scratch memory.  (With one
// history and 16 bits it is 44, else 24 at most; registers enough and fewer waves are slower, see above.)
template <typename W, typename T, bool kShared, bool kBiases>
__global__ __launch_bounds__(W::kThreads, 8) void penalties_kernel(PenaltyArgs a)
{
    constexpr int kN = kPackN<T>;
    __shared__ __attribute__((aligned(16))) unsigned shared[W::kSlice];
    __shared__ std::conditional_t<kBiases, Biases, int> biases;
    const long block = a.first_block + blockIdx.x, group = block / a.slices;
    const int begin = (int)(block % a.slices) * W::kSlice, n = min(W::kSlice, a.n_classes - begin);
    const bool sparse = a.logits == a.out && !a.bias;  // what nothing changes is left alone
    long row = group * a.rows_each;
    const long end = min(row + a.rows_each, a.n_rows);
    const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride + begin;
    Slice<W, T> next;
    if (!sparse) next.template fetch<true>(x_row, n, a.n_classes);
    Counters<W, T> counters;
    counters.clear();
    float bias[kPacks<W, T>][kN];
    unsigned may[kPacks<W, T>];
    auto prepare = [&]() {  // what may be the same for all rows
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) {
            if (a.bias) read_bias<kN>(a.bias + row * a.bias_stride + begin, class_of_pack<W, T>(u), n, bias[u]);
            may[u] = allowed_of<kN>(a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr, class_of_pack<W, T>(u), n);
        }
    };
    prepare();
    auto finish_row = [&](const Slice<W, T>& own) {
        const float r = a.repetition ? uniform(a.repetition + row) : a.r;
        const RowFactors p{r, 1.f / r, a.frequency ? uniform(a.frequency + row) : a.f, a.presence ? uniform(a.presence + row) : a.q};
        T* to = static_cast<T*>(a.out) + row * a.out_stride + begin;
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) {
            const int v = class_of_pack<W, T>(u);
            if (v >= n) break;
            const unsigned any = counters.any(u);
            Pack<T, kN> in = own.pack[u];
            if (sparse) {
                if (!any && may[u] == (1u << kN) - 1) continue;
                in = load_some<true>(x_row, v, n, a.n_classes);
            }
            float x[kN];
            unpack(in, v, n, a.n_classes, x);
            if (any) {
#pragma unroll
                for (int e = 0; e < kN; ++e) {
                    unsigned c = counters.c[u][e];
                    if constexpr (kBiases) c = c & kBiased ? biases.count[c & kPlace] : c;
                    x[e] = penalised(x[e], c, p);
                }
            }
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[e] += bias[u][e];
            }
            if constexpr (kBiases) {
                if (any & kBiased) {
#pragma unroll
                    for (int e = 0; e < kN; ++e)
                        if (counters.c[u][e] & kBiased) x[e] += biases.value[counters.c[u][e] & kPlace];
                }
            }
            if (a.allowed) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[e] = may[u] >> e & 1 ? x[e] : -INFINITY;
            }
            write_pack(to, x, v, n, a.streamed);
        }
    };
    if constexpr (!kShared) {
        count(a, row, begin, n, seen_of(a, row), shared, biases, counters);
        finish_row(next);
    } else {
        while (row < end) {
            Seen done = seen_of(a, row);
            if (a.history_len > 0) count(a, row, begin, n, done, shared, 0, counters);
            while (true) {
                const Slice<W, T> own = next;
                if (!sparse && row + 1 < end) next.template fetch<true>(x_row + a.row_stride, n, a.n_classes);
                finish_row(own);
                ++row;
                x_row += a.row_stride;
                if (row >= end) break;
                if (a.bias_stride || a.allowed_stride) prepare();
                const Seen now = seen_of(a, row);
                if (!count_on(a, row, begin, n, done, now, counters)) break;
                done = now;
            }
        }
    }
}

// A workgroup a slice of `rows_each` rows, whose gradients it adds up.  kShared: they have one history.  Bound by its reads and writes: 4096 rows of 50001
// bfloat16 255 us, 4.5 TB/s with some 320 MB of logits, for most lines of memory have a class that was seen; 177 us, 4.6 TB/s without a
// history.  (Asking for the next row's logits a row earlier changes nothing.)  Of binary32 a lane keeps 36 to 56 bytes in scratch memory, which is most of what
// few classes write: 1000 rows of 1000 with histories of their own and a bias 13 us and 19 MB written for 6 MB of results.  Histories of their own are counted row
// by row between barriers: 500 rows of 50001 bfloat16 with 16384 places each 75 us, 84 with a bias's gradient, 47 with that and 100 places.
template <typename W, typename T, bool kShared>
__global__ __launch_bounds__(W::kThreads, 6) void penalties_grad_kernel(PenaltyArgs a)
{
    constexpr int kN = kPackN<T>;
    __shared__ __attribute__((aligned(16))) unsigned shared[W::kSlice];
    const long block = a.first_block + blockIdx.x, group = block / a.slices;
    const int begin = (int)(block % a.slices) * W::kSlice, n = min(W::kSlice, a.n_classes - begin);
    const bool sparse = a.grad_out == a.out && !a.grad_bias, counting = a.out && a.history_len > 0;
    long row = group * a.rows_each;
    const long end = min(row + a.rows_each, a.n_rows);
    const T* g_row = static_cast<const T*>(a.grad_out) + row * a.grad_stride + begin;
    float sum[kPacks<W, T>][kN] = {};
    Slice<W, T> next;
    if (!sparse) next.template fetch<false>(g_row, n, a.n_classes);
    Counters<W, T> counters;
    counters.clear();
    unsigned may[kPacks<W, T>];
    auto prepare = [&]() {
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) may[u] = allowed_of<kN>(a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr, class_of_pack<W, T>(u), n);
    };
    prepare();
    auto finish_row = [&]() {
        const Slice<W, T> own = next;
        const float r = a.repetition ? uniform(a.repetition + row) : a.r, by_r = 1.f / r;
        const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride + begin;
        T* to = a.out ? static_cast<T*>(a.out) + row * a.out_stride + begin : nullptr;
        // (loads come back in their order: what this row waits for goes before what the next one does)
        Slice<W, T> logits{};
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) {
            const int v = class_of_pack<W, T>(u);
            if (counters.any(u)) logits.pack[u] = load_some<false>(x_row, v, n, a.n_classes);
        }
        if (!sparse && row + 1 < end) next.template fetch<false>(g_row + a.grad_stride, n, a.n_classes);
#pragma unroll
        for (int u = 0; u < kPacks<W, T>; ++u) {
            const int v = class_of_pack<W, T>(u);
            if (v >= n) break;
            const unsigned any = counters.any(u);
            Pack<T, kN> in = own.pack[u];
            if (sparse) {
                if (!any && may[u] == (1u << kN) - 1) continue;
                in = load_some<false>(g_row, v, n, a.n_classes);
            }
            float g[kN];
            unpack(in, v, n, a.n_classes, g);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                if (a.allowed) g[e] = may[u] >> e & 1 ? g[e] : 0.f;
                sum[u][e] += g[e];
            }
            if (!to) continue;
            if (any) {
                float x[kN];
                unpack(logits.pack[u], v, n, a.n_classes, x);
#pragma unroll
                for (int e = 0; e < kN; ++e) g[e] *= counters.c[u][e] && (may[u] >> e & 1) ? (x[e] > 0.f ? by_r : r) : 1.f;
            }
            write_pack(to, g, v, n, a.streamed);
        }
    };
    auto seen = [&]() { return Seen{clamped(a.lengths, row, a.history_len, a.history_len), 0}; };
    while (row < end) {
        Seen done = seen();
        if (counting) count(a, row, begin, n, done, shared, 0, counters);
        while (true) {
            finish_row();
            ++row;
            g_row += a.grad_stride;
            if (row >= end) break;
            if (a.allowed_stride) prepare();
            if constexpr (!kShared) {
                if (counting) break;
            } else {
                const Seen now = seen();
                if (counting && !count_on(a, row, begin, n, done, now, counters)) break;
                done = now;
            }
        }
    }
    if (!a.grad_bias) return;
#pragma unroll
    for (int u = 0; u < kPacks<W, T>; ++u) {
        const int v = class_of_pack<W, T>(u);
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (v + e < n) a.grad_bias[group * a.n_classes + begin + v + e] = sum[u][e];
    }
}

// Groups' sums as those of all rows, or of each `each` groups: kColumns classes a workgroup, the groups divided between 1024 / kColumns rows of threads.
template <int kColumns>
__global__ __launch_bounds__(kJoinThreads) void join_bias_kernel(const float* part, float* grad_bias, long n_groups, long each, int n_classes, long first_block)
{
    constexpr int kParts = kJoinThreads / kColumns;
    __shared__ float shared[kParts][kColumns];
    const long v = (first_block + blockIdx.x) * kColumns + threadIdx.x % kColumns;
    const int own = threadIdx.x / kColumns;
    const long begin = blockIdx.y * each, end = min(begin + each, n_groups);
    float sum = 0.f;
    if (v < n_classes) {
#pragma unroll 4
        for (long k = begin + own; k < end; k += kParts) sum += part[k * n_classes + v];
    }
    shared[own][threadIdx.x % kColumns] = sum;
    __syncthreads();
    for (int half = kParts / 2; half >= 1; half /= 2) {
        if (own < half) shared[own][threadIdx.x % kColumns] += shared[own + half][threadIdx.x % kColumns];
        __syncthreads();
    }
    if (own == 0 && v < n_classes) grad_bias[(long)blockIdx.y * n_classes + v] = shared[0][threadIdx.x];
}

// ---- host -----------------------------------------------------------------------------------------------------------

int check_penalties(const nuts_penalties_desc* d, const char* who)
{
    if (!d) return api_fail(NUTS_E_INVALID_ARG, "%s: desc must not be NULL", who);
    if (!cat_dtype_known(d->dtype)) return api_fail(NUTS_E_INVALID_ARG, "%s: dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16", who);
    if (d->id_type != NUTS_I32 && d->id_type != NUTS_I64) return api_fail(NUTS_E_INVALID_ARG, "%s: id_type must be NUTS_I32 or NUTS_I64", who);
    if (d->n_rows < 0 || d->n_rows > INT32_MAX - 1) return api_fail(NUTS_E_INVALID_ARG, "%s: n_rows must be in [0, 2^31 - 2]", who);
    if (d->n_classes < 1 || d->n_classes > INT32_MAX - (1 << 18)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_classes must be in [1, 2^31 - 2^18)", who);
    const int64_t most = INT64_MAX / 8 / std::max<int64_t>(1, d->n_rows);
    if (d->row_stride < d->n_classes || d->row_stride > most) return api_fail(NUTS_E_INVALID_ARG, "%s: row_stride is smaller than n_classes or too large", who);
    if (d->out_stride < d->n_classes || d->out_stride > most) return api_fail(NUTS_E_INVALID_ARG, "%s: out_stride is smaller than n_classes or too large", who);
    if (d->allowed_stride < 0 || (d->allowed_stride > 0 && d->allowed_stride < ceil_div(d->n_classes, 32)) || d->allowed_stride > most)
        return api_fail(NUTS_E_INVALID_ARG, "%s: allowed_stride must be 0 or at least n_classes / 32 words", who);
    if (d->bias_stride < 0 || (d->bias_stride > 0 && d->bias_stride < d->n_classes) || d->bias_stride > most)
        return api_fail(NUTS_E_INVALID_ARG, "%s: bias_stride must be 0 or at least n_classes", who);
    if (d->history_len < 0 || d->history_len > (int64_t)kCount) return api_fail(NUTS_E_INVALID_ARG, "%s: history_len must be in [0, 2^29)", who);
    if (d->history_stride < 0 || (d->history_stride > 0 && d->history_stride < d->history_len) || d->history_stride > most)
        return api_fail(NUTS_E_INVALID_ARG, "%s: history_stride must be 0 or at least history_len", who);
    if (d->n_bias < 0 || d->n_bias > NUTS_CAT_MAX_BIAS) return api_fail(NUTS_E_INVALID_ARG, "%s: n_bias must be in [0, %d]", who, NUTS_CAT_MAX_BIAS);
    const float r = (float)d->repetition;
    if (!std::isfinite(r) || !(r > 0.f)) return api_fail(NUTS_E_INVALID_ARG, "%s: repetition must be finite and > 0", who);
    if (!std::isfinite((float)d->frequency) || !std::isfinite((float)d->presence))
        return api_fail(NUTS_E_INVALID_ARG, "%s: frequency and presence must be finite", who);
    return NUTS_OK;
}

PenaltyArgs args_of(const nuts_penalties_desc* d)
{
    PenaltyArgs a{};
    a.row_stride = (long)d->row_stride;
    a.out_stride = (long)d->out_stride;
    a.allowed_stride = (long)d->allowed_stride;
    a.bias_stride = (long)d->bias_stride;
    a.history_stride = (long)d->history_stride;
    a.n_rows = (long)d->n_rows;
    a.r = (float)d->repetition;
    a.f = (float)d->frequency;
    a.q = (float)d->presence;
    a.n_classes = (int)d->n_classes;
    a.id_type = d->id_type;
    a.history_len = (int)d->history_len;
    a.n_bias = (int)d->n_bias;
    a.streamed = d->n_rows * d->n_classes * (int64_t)cat_size(d->dtype) >= kStreamed;
    return a;
}

bool shares(const nuts_penalties_desc* d) { return d->history_len == 0 || d->history_stride == 0; }
// Where rows have histories of their own wide slices look through them less often, and their threads have more on their way: 500 rows of 128000 bfloat16
// with histories of 256 56 us (usual ones 66), of 8000 73 (100); binary32 45 (43) and 53 (58).  Not where a wide slice would be half empty
// (3000 rows of 5000: 29, 24) and for too few workgroups, and not for gradients, whose rows keep their sums in registers (500 rows of
// 50001: 98, 54).
bool wants_wide(const nuts_penalties_desc* d)
{
    return !shares(d) && d->n_classes >= Wide::kSlice / 2 && (d->dtype != NUTS_F32 || d->history_len >= kLong) &&
           d->n_rows * ceil_div(d->n_classes, Wide::kSlice) >= kFull;
}
// Rows of a workgroup, for a launch of `groups` workgroups, but at least `least`.
int64_t rows_of_group(const nuts_penalties_desc* d, int64_t groups, int64_t least)
{
    return std::max<int64_t>(1, std::min(std::max(ceil_div(d->n_rows * ceil_div(d->n_classes, Usual::kSlice), groups), least), d->n_rows));
}
// Rows go together where they have one history, whose counts are carried on, and where their gradients are added up.
int64_t rows_each(const nuts_penalties_desc* d) { return shares(d) && d->n_bias == 0 ? rows_of_group(d, kGroups, 1) : 1; }
int64_t grad_rows_each(const nuts_penalties_desc* d, bool bias)
{
    if (!bias) return shares(d) ? rows_of_group(d, kGradGroups, 1) : 1;
    const int64_t rounds = ceil_div(rows_of_group(d, kGradGroups, kBiasRows), kBiasRun);
    return std::min(rows_of_group(d, kGradGroups * rounds, kBiasRows), kBiasRun);
}
// Rows of the workspace: groups' sums, and where there are many those of each kJoined of them.
int64_t grad_groups(const nuts_penalties_desc* d) { return ceil_div(d->n_rows, grad_rows_each(d, true)); }
int64_t grad_joined(const nuts_penalties_desc* d) { return grad_groups(d) > kJoined ? ceil_div(grad_groups(d), kJoined) : 0; }
int64_t grad_bytes(const nuts_penalties_desc* d) { return (grad_groups(d) + grad_joined(d)) * d->n_classes * (int64_t)sizeof(float); }

// The sums of each `each` of n_groups rows of `part`, as rows of `to`.
void join_groups(const float* part, float* to, int64_t n_groups, int64_t each, int n_classes)
{
    const bool narrow = n_classes <= kNarrow;  // (few classes: more workgroups for them)
    const int64_t rows = std::max<int64_t>(1, ceil_div(n_groups, each));
    const long most = std::max<long>(1, kMaxBlocks * 512 / kJoinThreads / rows);
    for (long first = 0, blocks = (long)ceil_div(n_classes, narrow ? 16 : 64); first < blocks; first += most)
        hipLaunchKernelGGL(narrow ? join_bias_kernel<16> : join_bias_kernel<64>, dim3((unsigned)std::min(blocks - first, most), (unsigned)rows), dim3(kJoinThreads), 0,
                           api_stream(), part, to, (long)n_groups, (long)each, n_classes, first);
}

template <typename W>
void launch(void (*kernel)(PenaltyArgs), PenaltyArgs a)
{
    a.slices = (int)ceil_div(a.n_classes, W::kSlice);
    constexpr long kMost = kMaxBlocks * 512 / W::kThreads;
    for (const long blocks = (long)ceil_div(a.n_rows, a.rows_each) * a.slices; a.first_block < blocks; a.first_block += kMost)
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(blocks - a.first_block, kMost)), dim3(W::kThreads), 0, api_stream(), a);
}

}  // namespace
}  // namespace nuts

using namespace nuts;

extern "C" {

int nuts_penalties(const nuts_penalties_desc* d, const void* logits, const void* history, const int32_t* lengths, const int32_t* prompts,
                   const float* repetition, const float* frequency, const float* presence, const float* bias, const void* bias_ids,
                   const float* bias_values, const uint32_t* allowed, void* out)
{
    if (int rc = check_penalties(d, "nuts_penalties")) return rc;
    if (d->n_rows == 0) return NUTS_OK;
    if (!logits || !out) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties: null pointer");
    if (d->history_len > 0 && !history) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties: history must not be NULL");
    if (d->n_bias > 0 && (!bias_ids || !bias_values)) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties: n_bias needs bias_ids and bias_values");
    if (logits == out && d->row_stride != d->out_stride && d->n_rows > 1)
        return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties: in place row_stride and out_stride must be the same");
    if (int rc = api_have_device()) return rc;
    PenaltyArgs a = args_of(d);
    a.logits = logits;
    a.history = history;
    a.lengths = lengths;
    a.prompts = prompts;
    a.repetition = repetition;
    a.frequency = frequency;
    a.presence = presence;
    a.bias = bias;
    a.bias_ids = bias_ids;
    a.bias_values = bias_values;
    a.allowed = allowed;
    a.out = out;
    a.rows_each = (int)rows_each(d);
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        if (wants_wide(d)) launch<Wide>(d->n_bias > 0 ? penalties_kernel<Wide, T, false, true> : penalties_kernel<Wide, T, false, false>, a);
        else if (d->n_bias > 0) launch<Usual>(penalties_kernel<Usual, T, false, true>, a);
        else launch<Usual>(shares(d) ? penalties_kernel<Usual, T, true, false> : penalties_kernel<Usual, T, false, false>, a);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_penalties_grad_workspace(const nuts_penalties_desc* d, int64_t* bytes)
{
    if (int rc = check_penalties(d, "nuts_penalties_grad_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad_workspace: bytes must not be NULL");
    *bytes = grad_bytes(d);
    return NUTS_OK;
}

int nuts_penalties_grad(const nuts_penalties_desc* d, const void* grad_out, int64_t grad_stride, const void* logits, const void* history,
                        const int32_t* lengths, const float* repetition, const uint32_t* allowed, void* grad_logits, float* grad_bias,
                        void* workspace, int64_t workspace_bytes)
{
    if (int rc = check_penalties(d, "nuts_penalties_grad")) return rc;
    if (grad_stride < d->n_classes || grad_stride > INT64_MAX / 8 / std::max<int64_t>(1, d->n_rows))
        return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: grad_stride is smaller than n_classes or too large");
    if (!grad_logits && !grad_bias) return NUTS_OK;
    if (d->n_rows > 0) {
        if (!grad_out || (grad_logits && !logits)) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: null pointer");
        if (grad_logits && d->history_len > 0 && !history) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: history must not be NULL");
        if (grad_logits == logits && grad_logits) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: the gradient must not overlap the logits");
        if (grad_logits == grad_out && grad_stride != d->out_stride && d->n_rows > 1)
            return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: in place grad_stride and out_stride must be the same");
    }
    const int64_t groups = grad_groups(d), joined = grad_joined(d);
    if (grad_bias && groups > 0) {
        const int64_t bytes = grad_bytes(d);
        if (!workspace || workspace_bytes < bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: needs a workspace of %lld bytes", (long long)bytes);
        if (reinterpret_cast<uintptr_t>(workspace) % 256) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad: workspace must be aligned to 256 bytes");
    }
    if (d->n_rows == 0 && !grad_bias) return NUTS_OK;
    if (int rc = api_have_device()) return rc;
    PenaltyArgs a = args_of(d);
    a.logits = logits;
    a.history = history;
    a.lengths = lengths;
    a.repetition = repetition;
    a.allowed = allowed;
    a.grad_out = grad_out;
    a.grad_stride = (long)grad_stride;
    a.out = grad_logits;
    a.grad_bias = grad_bias ? static_cast<float*>(workspace) : nullptr;
    a.rows_each = (int)grad_rows_each(d, grad_bias != nullptr);
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        launch<Usual>(shares(d) ? penalties_grad_kernel<Usual, T, true> : penalties_grad_kernel<Usual, T, false>, a);
    });
    if (grad_bias) {
        const float* part = static_cast<const float*>(workspace);
        if (joined > 0) {
            float* to = static_cast<float*>(workspace) + groups * d->n_classes;
            join_groups(part, to, groups, kJoined, (int)d->n_classes);
            part = to;
        }
        const int64_t left = joined > 0 ? joined : groups;
        join_groups(part, grad_bias, left, std::max<int64_t>(1, left), (int)d->n_classes);
    }
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
