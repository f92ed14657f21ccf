// Log-probabilities of given classes from rows of logits, with the rows' entropies and most probable classes, and the
// gradient of that.
//
//   z = s x,  lse = log sum e^z,  logprob = z_y - lse,  entropy = lse - sum p z,  p = e^(z - lse)
//   dx_v = s (g_lp ([v = y] - p_v) + g_lse p_v - g_H p_v (log p_v + H))
#include "nuts_softmax.h"

#include <algorithm>

namespace nuts {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kCandidates = 1024;  // alternatives that are put in order at once
constexpr int kJoinKeys = 4096;    // alternatives of a row's parts that are joined: no more than 16 a thread

struct LogitsArgs {
    const void* logits;
    const void* targets;
    const uint32_t* allowed;
    float* logprob;
    float* lse;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    float4* part_stats;               // [row][part]: m, S, T
    unsigned long long* part_keys;    // [row][part][n_top]
    long first_block, row_stride, allowed_stride;
    float scale;
    int n_classes, id_type, n_top, parts, part_len;
};

// The order of alternatives as whole numbers: larger logit first, NaN before all, the lower class first of equal ones.  0 is none.
__device__ __forceinline__ unsigned long long key_of(float x, int v)
{
    const unsigned bits = __float_as_uint(x + 0.f);  // (-0 is 0)
    const unsigned order = x != x ? ~0u : bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return (unsigned long long)order << 32 | (unsigned)~v;
}
__device__ __forceinline__ int class_of(unsigned long long key) { return key ? (int)~(unsigned)key : -1; }
__device__ __forceinline__ float logit_of(unsigned long long key)
{
    const unsigned order = (unsigned)(key >> 32);
    return order == ~0u ? NAN : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}

__device__ __forceinline__ bool may_come(const uint32_t* allowed, int v) { return !allowed || (allowed[v >> 5] >> (v & 31) & 1); }

// The logits v .. v + kN - 1 of a row, as many of them as there are (`end`); those that may not come as -infinity.
// Returns a bit for each that may.  v is a multiple of kN, and kN divides 8.
template <typename T, int kN, bool kMask>
__device__ __forceinline__ unsigned load_logits(const T* row, const uint32_t* allowed, int v, int end, float (&x)[kN])
{
    unsigned may = (1u << kN) - 1;
    if (v + kN <= end) {
        const Pack<T, kN> in = load_pack<T, kN>(row + v);
#pragma unroll
        for (int e = 0; e < kN; ++e) x[e] = to_float(in.v[e]);
    } else {
        may = (1u << (end - v)) - 1;
#pragma unroll
        for (int e = 0; e < kN; ++e) x[e] = v + e < end ? to_float(row[v + e]) : -INFINITY;
    }
    if (kMask) {
        may &= reinterpret_cast<const unsigned char*>(allowed)[v >> 3] >> (v & 7);
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (!(may >> e & 1)) x[e] = -INFINITY;
    }
    return may;
}

// The n_top largest of a workgroup's logits, sorted: `collect(least, see)` goes through those of them that are `least` or more (or
// NaN) and `every(see)` through all, thread by thread, in any order.  `best`: the largest of this thread's, NaNs aside.
// Four threads' best make a group's, of which there are 64, and the n_top-th largest of these is no larger than the n_top-th
// largest logit: what is below it need not be looked at twice.  A few logits more than n_top are left and get
// their ranks by counting.  Rows with very many equal ones (or fewer finite ones than groups) leave too many: then the largest
// is looked for n_top times.
template <typename Collect, typename Every>
__device__ void select_top(int n_top, float best, unsigned long long* sorted, Collect collect, Every every)
{
    __shared__ __attribute__((aligned(16))) unsigned long long candidate[kCandidates];
    __shared__ __attribute__((aligned(16))) float bests[64];
    __shared__ unsigned long long most[kWaves];
    __shared__ int count;
    float group = fmaxf(best, __shfl_xor(best, 1));
    group = fmaxf(group, __shfl_xor(group, 2));
    if (threadIdx.x % 4 == 0) bests[threadIdx.x / 4] = group;
    if (threadIdx.x == 0) count = 0;
    if (threadIdx.x < (unsigned)n_top) sorted[threadIdx.x] = 0;
    __syncthreads();
    const int lane = threadIdx.x % 64;
    const float own = bests[lane];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < 64; i += 4) {
        const float4 other = *reinterpret_cast<const float4*>(&bests[i]);
        rank += (other.x > own || (other.x == own && i < lane)) + (other.y > own || (other.y == own && i + 1 < lane)) +
                (other.z > own || (other.z == own && i + 2 < lane)) + (other.w > own || (other.w == own && i + 3 < lane));
    }
    const float least = __shfl(own, __builtin_ctzll(__ballot(rank == n_top - 1)));
    collect(least, [&](float x, int v) {
        if (x >= least || x != x) {
            const int at = atomicAdd(&count, 1);
            if (at < kCandidates) candidate[at] = key_of(x, v);
        }
    });
    __syncthreads();
    const int n = count;
    if (n <= kCandidates) {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const unsigned long long key = candidate[i];
            int r = 0;
#pragma unroll 8
            for (int k = 0; k < n; ++k) r += candidate[k] > key;
            if (r < n_top) sorted[r] = key;
        }
    } else {
        unsigned long long last = ~0ull;
        for (int r = 0; r < n_top; ++r) {
            unsigned long long next = 0;
            every([&](float x, int v) {
                const unsigned long long key = key_of(x, v);
                if (key < last && key > next) next = key;
            });
#pragma unroll
            for (int step = 32; step >= 1; step /= 2) next = max(next, (unsigned long long)__shfl_xor(next, step));
            if (lane == 0) most[threadIdx.x / 64] = next;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) next = max(next, most[w]);
            if (threadIdx.x == 0) sorted[r] = next;
            __syncthreads();
            if (next == 0) break;
            last = next;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ void write_top(const LogitsArgs& a, long row, const Row& r, const unsigned long long* sorted)
{
    if (threadIdx.x >= (unsigned)a.n_top) return;
    const unsigned long long key = sorted[threadIdx.x];
    if (a.top_ids) a.top_ids[row * a.n_top + threadIdx.x] = class_of(key);
    if (a.top_logprobs) a.top_logprobs[row * a.n_top + threadIdx.x] = key ? logprob_of(r, logit_of(key), a.scale) : -INFINITY;
}

// Thread 0 asks for the row's target before the row is read, for its logit behind that, and writes the results.
struct Target {
    long id;
    int y;
    float x;
};
__device__ __forceinline__ void ask_target(const LogitsArgs& a, long row, Target& t)
{
    t = Target{-1, -1, -INFINITY};
    if (threadIdx.x == 0 && a.targets && a.logprob)
        t.id = a.id_type == NUTS_I64 ? static_cast<const int64_t*>(a.targets)[row] : static_cast<const int32_t*>(a.targets)[row];
}
template <typename T>
__device__ __forceinline__ void ask_logit(const LogitsArgs& a, long row, Target& t)
{
    if (t.id < 0 || t.id >= a.n_classes) return;
    t.y = (int)t.id;
    if (may_come(a.allowed ? a.allowed + row * a.allowed_stride : nullptr, t.y)) t.x = to_float(static_cast<const T*>(a.logits)[row * a.row_stride + t.y]);
}
__device__ __forceinline__ void write_row(const LogitsArgs& a, long row, const Row& r, const Target& t)
{
    if (threadIdx.x != 0) return;
    if (a.lse) a.lse[row] = r.lse;
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.logprob) a.logprob[row] = t.y >= 0 ? logprob_of(r, t.x, a.scale) : 0.f;
}

// kCount packs of a thread, kThreads packs apart, from `at` on; none behind `end`.
template <typename T, int kN, bool kMask, int kCount>
struct Packs {
    float x[kCount * kN];
    unsigned may[kCount];
    __device__ __forceinline__ void load(const T* row, const uint32_t* allowed, int at, int end)
    {
#pragma unroll
        for (int u = 0; u < kCount; ++u) {
            const int v = at + u * kThreads * kN;
            float(&to)[kN] = *reinterpret_cast<float(*)[kN]>(&x[u * kN]);
            may[u] = 0;
            if (v < end) {
                may[u] = load_logits<T, kN, kMask>(row, allowed, v, end, to);
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e) to[e] = -INFINITY;
            }
        }
    }
};

// One workgroup a row, or a part of one where there are few rows (kWhole = false: join_rows_kernel ends them).  One pass, bound by its
// reads where there are many rows: 4096 x 32001 bfloat16 with 5 alternatives 63 us, 4.7 TB/s of them; of few rows by the wait for one
// read of memory and the alternatives' exchange through LDS: 8 x 128000, masked, with 20 alternatives 9 us and 7 for join_rows_kernel.
template <typename T, bool kMask, bool kTop, bool kWhole>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogitsArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    __shared__ Stats shared[kWaves];
    __shared__ unsigned long long sorted[NUTS_CAT_MAX_TOP];
    const long row = kWhole ? a.first_block + blockIdx.x : (long)(blockIdx.x / (unsigned)a.parts);
    const int part = kWhole ? 0 : (int)(blockIdx.x % (unsigned)a.parts);
    const int begin = part * a.part_len, end = kWhole ? a.n_classes : min(begin + a.part_len, a.n_classes);
    const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride;
    const uint32_t* allowed = kMask ? a.allowed + row * a.allowed_stride : nullptr;
    const float c = a.scale * kLog2e;
    Target target;
    if (kWhole) ask_target(a, row, target);
    Stats v{-INFINITY, 0.f, 0.f};
    // Two packs of a thread at a time, the next two under way while these are added up; the maximum is settled once for all of them.
    // (Four took registers that further rows of a compute unit could use while this one names its alternatives: 4096 rows of 32001
    // with five 75 us, with two packs 67 us; workgroups of 128 or 512 threads 68 and 88 us.)
    constexpr int kFlight = 2, kStep = kFlight * kThreads * kN;
    int at = begin + (int)threadIdx.x * kN;
    const int last = end - (kFlight - 1) * kThreads * kN - kN;  // where two whole packs still fit
    if (at <= last) {
        Pack<T, kN> next[kFlight];
        unsigned may[kFlight];
        auto fetch = [&](int from) {
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                const int i = from + u * kThreads * kN;
                next[u] = load_pack<T, kN>(x_row + i);
                if (kMask) may[u] = reinterpret_cast<const unsigned char*>(allowed)[i >> 3] >> (i & 7);
            }
        };
        fetch(at);
        while (true) {
            float x[kFlight * kN];
#pragma unroll
            for (int u = 0; u < kFlight; ++u)
#pragma unroll
                for (int e = 0; e < kN; ++e) x[u * kN + e] = kMask && !(may[u] >> e & 1) ? -INFINITY : to_float(next[u].v[e]);
            at += kStep;
            const bool more = at <= last;
            if (more) fetch(at);
            add_logits<kFlight * kN>(v, x, c);
            if (!more) break;
        }
    }
    if (at < end) {
        Packs<T, kN, kMask, kFlight> rest;
        rest.load(x_row, allowed, at, end);
        add_logits<kFlight * kN>(v, rest.x, c);
    }
    if (kWhole) ask_logit<T>(a, row, target);
    const float best = v.m;
    const bool has_nan = v.s != v.s;
    const Stats all = join_block(v, c, shared);
    if (kTop) {
        // all logits of the threads in `mine` (of this wave): each thread its own, or, where few are asked for, a thread's by the whole wave
        auto look = [&](unsigned long long mine, auto see) {
            const int each = (end - begin + kThreads * kN - 1) / (kThreads * kN);  // packs of a thread
            const int lane = threadIdx.x % 64;
            auto see_pack = [&](int i) {
                float x[kN];
                const unsigned may = load_logits<T, kN, kMask>(x_row, allowed, i, end, x);
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (may >> e & 1) see(x[e], i + e);
            };
            if (__popcll(mine) * ((each + 63) / 64) <= (each + kFlight - 1) / kFlight) {
                for (; mine; mine &= mine - 1) {
                    const int thread = (int)(threadIdx.x & ~63u) + __builtin_ctzll(mine);
                    for (int i = begin + (thread + lane * kThreads) * kN; i < end; i += 64 * kThreads * kN) see_pack(i);
                }
            } else if (mine >> lane & 1) {
                for (int i = begin + (int)threadIdx.x * kN; i < end; i += kStep) {
                    Packs<T, kN, kMask, kFlight> packs;
                    packs.load(x_row, allowed, i, end);
#pragma unroll
                    for (int u = 0; u < kFlight; ++u)
#pragma unroll
                        for (int e = 0; e < kN; ++e)
                            if (packs.may[u] >> e & 1) see(packs.x[u * kN + e], i + u * kThreads * kN + e);
                }
            }
        };
        select_top(a.n_top, best, sorted, [&](float least, auto see) { look(__ballot(best >= least || has_nan), see); },
                   [&](auto see) {
                       for (int i = begin + (int)threadIdx.x * kN; i < end; i += kThreads * kN) {
                           float x[kN];
                           const unsigned may = load_logits<T, kN, kMask>(x_row, allowed, i, end, x);
#pragma unroll
                           for (int e = 0; e < kN; ++e)
                               if (may >> e & 1) see(x[e], i + e);
                       }
                   });
    }
    if (kWhole) {
        const Row r = finish(all, a.scale);
        write_row(a, row, r, target);
        if (kTop) write_top(a, row, r, sorted);
    } else {
        if (threadIdx.x == 0) a.part_stats[blockIdx.x] = float4{all.m, all.s, all.t, 0.f};
        if (kTop && threadIdx.x < (unsigned)a.n_top) a.part_keys[(long)blockIdx.x * a.n_top + threadIdx.x] = sorted[threadIdx.x];
    }
}

template <typename T, bool kTop>
__global__ __launch_bounds__(kThreads) void join_rows_kernel(LogitsArgs a)
{
    __shared__ Stats shared[kWaves];
    __shared__ unsigned long long sorted[NUTS_CAT_MAX_TOP];
    const long row = blockIdx.x;
    const float c = a.scale * kLog2e;
    Target target;
    ask_target(a, row, target);
    // (a thread's keys stay in registers)
    constexpr int kKeys = kTop ? kJoinKeys / kThreads : 1;
    unsigned long long keys[kKeys];
    const int n = a.parts * a.n_top;
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const int i = k * kThreads + (int)threadIdx.x;
        keys[k] = kTop && i < n ? a.part_keys[row * n + i] : 0;
    }
    Stats v{-INFINITY, 0.f, 0.f};
    for (int p = threadIdx.x; p < a.parts; p += kThreads) {
        const float4 s = a.part_stats[row * a.parts + p];
        v = join(v, Stats{s.x, s.y, s.z}, c);
    }
    ask_logit<T>(a, row, target);
    const Row r = finish(join_block(v, c, shared), a.scale);
    write_row(a, row, r, target);
    if (kTop) {
        float best = -INFINITY;
        auto every = [&](auto see) {
#pragma unroll
            for (int k = 0; k < kKeys; ++k)
                if (keys[k]) see(logit_of(keys[k]), class_of(keys[k]));
        };
        every([&](float x, int) { best = fmaxf(best, x); });
        select_top(a.n_top, best, sorted, [&](float, auto see) { every(see); }, every);
        write_top(a, row, r, sorted);
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------------

struct GradArgs {
    const void* logits;
    const void* targets;
    const uint32_t* allowed;
    const float* lse;
    const float* entropy;
    const float* grad_logprob;
    const float* grad_lse;
    const float* grad_entropy;
    void* grad;
    long first_block, row_stride, allowed_stride, grad_stride;
    float scale;
    int n_classes, id_type, parts, streamed;
};

constexpr int kGradPacks = 4;  // of a thread
constexpr float kOffOne = 1e-4f;  // more than what lse's rounding and the order of its sum can put the sum of p off 1

// A workgroup a part of a row.  Bound by its reads and writes: one exponential an element; 4096 x 50001 bfloat16 with entropies
// 139 us one after the other, 144 in turn with the forward pass, 833 MB at 5.8 TB/s; with a mask 155.  A large gradient is written past the
// caches, which then keep the logits that the forward pass left there (both passes on 4096 x 50001 bfloat16: 252 us with plain
// stores, 231 us so).
//
// p = e^(z - lse) takes half a unit in the last place of lse as an error.  In binary32 that is more than all else is off by, and a row
// that a workgroup holds in its registers is divided by the sum of its p, which without that error is 1 (8000 x 4000: 41 us, 39
// without), unless that is far off: then lse is that of a longer row.  Far from 0 (kFar) each of the row's workgroups goes through all
// of it for its maximum and sum, from the caches (4096 x 50001 bfloat16 490 us where lse is enough for 140; to leave such rows to one
// workgroup each takes 250, and registers that cost all others 3 %).
template <typename T, bool kMask, bool kEntropy>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(GradArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    __shared__ Stats shared[kWaves];
    const long row = (a.first_block + blockIdx.x) / a.parts;
    const int begin = (int)((a.first_block + blockIdx.x) % a.parts) * (kGradPacks * kThreads * kN) + (int)threadIdx.x * kN;
    const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride;
    T* to = static_cast<T*>(a.grad) + row * a.grad_stride;
    const uint32_t* allowed = kMask ? a.allowed + row * a.allowed_stride : nullptr;
    float x[kGradPacks][kN];
    unsigned may[kGradPacks];
#pragma unroll
    for (int u = 0; u < kGradPacks; ++u) {
        const int v = begin + u * kThreads * kN;
        if (v < a.n_classes) may[u] = load_logits<T, kN, kMask>(x_row, allowed, v, a.n_classes, x[u]);
    }
    const int y = a.targets ? class_at(a.targets, a.id_type, row, a.n_classes) : -1;
    const float lse = a.lse[row];
    const bool empty = lse == -INFINITY, far = far_from_0<T>(lse);
    const float g_lp = a.grad_logprob && y >= 0 && !empty ? a.grad_logprob[row] * a.scale : 0.f;
    const float g_p = (a.grad_lse ? a.grad_lse[row] * a.scale : 0.f) - g_lp;
    const float g_h = kEntropy ? -a.grad_entropy[row] * a.scale : 0.f, entropy = kEntropy ? a.entropy[row] : 0.f;
    // p = e^(s (x - base) - shift) / sum
    float base = 0.f, shift = empty ? INFINITY : lse, one_by_sum = 1.f, ln_sum = 0.f;
    if (far) {
        Stats v{-INFINITY, 0.f, 0.f};
        for (int i = threadIdx.x * kN; i < a.n_classes; i += kThreads * kN) {  // (a pack at a time: x is in registers, too)
            float some[kN];
            load_logits<T, kN, kMask>(x_row, allowed, i, a.n_classes, some);
            add_logits<kN>(v, some, a.scale * kLog2e);
        }
        v = join_block(v, a.scale * kLog2e, shared);
        // (lse - s m has fewer digits than ln S, and is to be taken where it is another number: lse is that of a longer row)
        if (v.m > -INFINITY) {
            base = v.m;
            shift = logf(v.s);
            const float given = __builtin_fmaf(-v.m, a.scale, lse);
            if (__builtin_fabsf(given - shift) > __builtin_fmaf(__builtin_fabsf(lse), 0x1p-22f, kOffOne)) shift = given;
        }
    } else if (sizeof(T) == 4 && a.parts == 1 && !empty) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < kGradPacks; ++u)
            if (begin + u * kThreads * kN < a.n_classes) {
#pragma unroll
                for (int e = 0; e < kN; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][e], a.scale, -lse) * kLog2e);
            }
#pragma unroll
        for (int step = 32; step >= 1; step /= 2) sum += __shfl_xor(sum, step);
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64].s = sum;
        __syncthreads();
        sum = (shared[0].s + shared[1].s) + (shared[2].s + shared[3].s);
        if (__builtin_fabsf(sum - 1.f) <= kOffOne) {
            one_by_sum = 1.f / sum;
            ln_sum = logf(sum);
        }
    }
#pragma unroll
    for (int u = 0; u < kGradPacks; ++u) {
        const int v = begin + u * kThreads * kN;
        if (v >= a.n_classes) break;
        float g[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const float w = __builtin_fmaf(x[u][e] - base, a.scale, -shift), p = __builtin_amdgcn_exp2f(w * kLog2e) * one_by_sum;
            // (where p is 0 there is no gradient, however far below log p is and whatever comes in)
            g[e] = p == 0.f ? 0.f : p * (kEntropy ? __builtin_fmaf(g_h, fmaxf(w - ln_sum, kNothing) + entropy, g_p) : g_p);
            if (kMask && !(may[u] >> e & 1)) g[e] = 0.f;  // (also where the row has no lse, or no finite gradient)
        }
        if (y >= v && y < v + kN) {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (v + e == y && (may[u] >> e & 1)) g[e] += g_lp;
        }
        Pack<T, kN> out;
#pragma unroll
        for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(g[e]);
        if (v + kN <= a.n_classes) {
            a.streamed ? stream_pack(to + v, out) : store_pack(to + v, out);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (v + e < a.n_classes) to[v + e] = out.v[e];
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------

int check_logits(const nuts_logits_desc* d, const char* who)
{
    if (!d) return api_fail(NUTS_E_INVALID_ARG, "%s: desc must not be NULL", who);
    if (!cat_dtype_known(d->dtype)) return api_fail(NUTS_E_INVALID_ARG, "%s: dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16", who);
    if (d->id_type != NUTS_I32 && d->id_type != NUTS_I64) return api_fail(NUTS_E_INVALID_ARG, "%s: id_type must be NUTS_I32 or NUTS_I64", who);
    if (d->n_rows < 0 || d->n_rows > INT32_MAX - 1) return api_fail(NUTS_E_INVALID_ARG, "%s: n_rows must be in [0, 2^31 - 2]", who);
    // (indexes of classes are 32 bits, and the next that a thread would look at may lie 2^17 behind the last)
    if (d->n_classes < 1 || d->n_classes > INT32_MAX - (1 << 18)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_classes must be in [1, 2^31 - 2^18)", who);
    if (d->row_stride < d->n_classes) return api_fail(NUTS_E_INVALID_ARG, "%s: row_stride is smaller than n_classes", who);
    if (d->n_rows > 0 && d->row_stride > INT64_MAX / 8 / d->n_rows) return api_fail(NUTS_E_INVALID_ARG, "%s: row_stride is too large", who);
    if (d->allowed_stride < 0 || (d->allowed_stride > 0 && d->allowed_stride < ceil_div(d->n_classes, 32)))
        return api_fail(NUTS_E_INVALID_ARG, "%s: allowed_stride must be 0 or at least n_classes / 32 words", who);
    const float scale = (float)d->scale;
    if (!std::isfinite(scale) || !(scale > 0.f)) return api_fail(NUTS_E_INVALID_ARG, "%s: scale must be finite and > 0", who);
    if (d->n_top < 0 || d->n_top > NUTS_CAT_MAX_TOP) return api_fail(NUTS_E_INVALID_ARG, "%s: n_top must be in [0, %d]", who, NUTS_CAT_MAX_TOP);
    return NUTS_OK;
}

struct LogitsPlan {
    int parts, part_len;
    size_t keys, bytes;
};

// Rows are divided where they are fewer than four workgroups a compute unit, down to 16 bytes a thread.
LogitsPlan plan_logits(const nuts_logits_desc* d)
{
    LogitsPlan p{1, (int)d->n_classes, 0, 0};
    const int64_t least = kThreads * (16 / (int64_t)cat_size(d->dtype));
    int64_t parts = d->n_rows > 0 ? ceil_div(1024, d->n_rows) : 1;
    parts = std::min(parts, ceil_div(d->n_classes, least));
    if (d->n_top > 0) parts = std::min<int64_t>(parts, kJoinKeys / d->n_top);
    if (parts > 1) {
        p.part_len = (int)(ceil_div(ceil_div(d->n_classes, parts), least) * least);
        p.parts = (int)ceil_div(d->n_classes, p.part_len);
    }
    if (p.parts > 1) {
        p.keys = ((size_t)d->n_rows * p.parts * sizeof(float4) + 255) & ~(size_t)255;
        p.bytes = p.keys + (size_t)d->n_rows * p.parts * d->n_top * sizeof(unsigned long long);
    }
    return p;
}

template <typename T, bool kMask, bool kTop>
void launch_logprobs(LogitsArgs a, long n_rows, hipStream_t stream)
{
    if (a.parts == 1) {
        for (; a.first_block < n_rows; a.first_block += kMaxBlocks)
            hipLaunchKernelGGL((logprobs_kernel<T, kMask, kTop, true>), dim3((unsigned)std::min(n_rows - a.first_block, kMaxBlocks)), dim3(kThreads), 0, stream, a);
    } else {
        hipLaunchKernelGGL((logprobs_kernel<T, kMask, kTop, false>), dim3((unsigned)(n_rows * a.parts)), dim3(kThreads), 0, stream, a);
        hipLaunchKernelGGL((join_rows_kernel<T, kTop>), dim3((unsigned)n_rows), dim3(kThreads), 0, stream, a);
    }
}

}  // namespace
}  // namespace nuts

using namespace nuts;

extern "C" {

int nuts_logprobs_workspace(const nuts_logits_desc* d, int64_t* bytes)
{
    if (int rc = check_logits(d, "nuts_logprobs_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_workspace: bytes must not be NULL");
    *bytes = (int64_t)plan_logits(d).bytes;
    return NUTS_OK;
}

int nuts_logprobs(const nuts_logits_desc* d, const void* logits, const void* targets, const uint32_t* allowed, float* logprob,
                  float* lse, float* entropy, int32_t* top_ids, float* top_logprobs, void* workspace, int64_t workspace_bytes)
{
    if (int rc = check_logits(d, "nuts_logprobs")) return rc;
    if (d->n_rows == 0) return NUTS_OK;
    if (!logits) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs: logits must not be NULL");
    const LogitsPlan p = plan_logits(d);
    if (p.bytes > 0 && (!workspace || workspace_bytes < (int64_t)p.bytes))
        return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs: needs a workspace of %zu bytes", p.bytes);
    if (p.bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % 256) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs: workspace must be aligned to 256 bytes");
    if (int rc = api_have_device()) return rc;
    const bool top = d->n_top > 0 && (top_ids || top_logprobs);
    char* w = static_cast<char*>(workspace);
    LogitsArgs a{logits, targets, allowed, logprob, lse, entropy, top_ids, top_logprobs,
                 reinterpret_cast<float4*>(w), p.parts > 1 ? reinterpret_cast<unsigned long long*>(w + p.keys) : nullptr,
                 0, (long)d->row_stride, (long)d->allowed_stride, (float)d->scale,
                 (int)d->n_classes, d->id_type, d->n_top, p.parts, p.part_len};
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        hipStream_t s = api_stream();
        const long n = (long)d->n_rows;
        if (allowed) top ? launch_logprobs<T, true, true>(a, n, s) : launch_logprobs<T, true, false>(a, n, s);
        else top ? launch_logprobs<T, false, true>(a, n, s) : launch_logprobs<T, false, false>(a, n, s);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_logprobs_grad(const nuts_logits_desc* d, const void* logits, const void* targets, const uint32_t* allowed, const float* lse,
                       const float* entropy, const float* grad_logprob, const float* grad_lse, const float* grad_entropy,
                       void* grad_logits, int64_t grad_stride)
{
    if (int rc = check_logits(d, "nuts_logprobs_grad")) return rc;
    if (grad_stride < d->n_classes) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_grad: grad_stride is smaller than n_classes");
    if (d->n_rows > 0 && grad_stride > INT64_MAX / 8 / d->n_rows) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_grad: grad_stride is too large");
    if (d->n_rows == 0) return NUTS_OK;
    if (!logits || !lse || !grad_logits) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_grad: null pointer");
    if (grad_entropy && !entropy) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_grad: grad_entropy needs the entropy");
    if (grad_logits == logits) return api_fail(NUTS_E_INVALID_ARG, "nuts_logprobs_grad: the gradient must not overlap the logits");
    const int64_t parts = ceil_div(d->n_classes, (int64_t)kGradPacks * kThreads * (16 / (int64_t)cat_size(d->dtype)));
    if (int rc = api_have_device()) return rc;
    GradArgs a{logits, targets, allowed, lse, entropy, grad_logprob, grad_lse, grad_entropy, grad_logits, 0, (long)d->row_stride,
               (long)d->allowed_stride, (long)grad_stride, (float)d->scale, (int)d->n_classes, d->id_type, (int)parts,
               d->n_rows * d->n_classes * (int64_t)cat_size(d->dtype) >= kStreamed};
    by_dtype(d->dtype, [&](auto t) {
        using T = decltype(t);
        void (*kernel)(GradArgs) = allowed ? (grad_entropy ? logprobs_grad_kernel<T, true, true> : logprobs_grad_kernel<T, true, false>)
                                           : (grad_entropy ? logprobs_grad_kernel<T, false, true> : logprobs_grad_kernel<T, false, false>);
        for (const long blocks = (long)(d->n_rows * parts); a.first_block < blocks; a.first_block += kMaxBlocks)
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(blocks - a.first_block, kMaxBlocks)), dim3(kThreads), 0, api_stream(), a);
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
