// Logits adjusted by what was said before, by biases and by masks, and the gradient of that.
//
//   z = x > 0 ? x / r : x r  where v was seen,   z -= f count_v + q [count_v > 0],   z += bias_v,   -infinity where v is not allowed
//   dx_v = g_v (seen_v ? (x > 0 ? 1 / r : r) : 1),   dbias_v = sum over rows of g_v,   0 where v is not allowed
#include "nuts_cat.h"

#include <algorithm>
#include <climits>

namespace nuts {
namespace {

constexpr int kThreads = 512;
constexpr int kSlice = 4096;        // classes of a workgroup, with a counter each in LDS
constexpr int kColumns = 64;        // of a workgroup that joins the biases' gradients
constexpr int kJoinThreads = 1024;
constexpr int kGroups = 1024;       // workgroups that the rows are divided between where they are added up

// A class's counter: how often it was said behind the prompt; whether it has a bias of its own; whether it was in the prompt.
constexpr unsigned kPrompt = 1u << 31, kBiased = 1u << 30, kCount = kBiased - 1, kSeen = kPrompt | kCount;

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

__device__ __forceinline__ long id_at(const void* ids, int id_type, long i)
{
    return id_type == NUTS_I64 ? static_cast<const int64_t*>(ids)[i] : (long)static_cast<const int32_t*>(ids)[i];
}

__device__ __forceinline__ int clamped(const int32_t* lengths, long row, int most, int otherwise)
{
    return lengths ? min(max(lengths[row], 0), most) : otherwise;
}

// What a workgroup's counters hold: the places 0 .. length - 1 of a row's history, the first `prompt` as prompt.
struct Counted {
    int length, prompt;
};

__device__ __forceinline__ bool may_come(const uint32_t* allowed, int v) { return !allowed || (allowed[v >> 5] >> (v & 31) & 1); }

// Calls `see` for the places from .. to - 1 of a history that hold one of the classes begin .. begin + n - 1, thread by thread.
template <typename Id, typename See>
__device__ __forceinline__ void look_through(const Id* history, int from, int to, int begin, int n, See see)
{
    constexpr int kEach = 4, kN = 16 / sizeof(Id);
    for (int i = from + (int)threadIdx.x * kEach; i < to; i += kThreads * kEach) {
        Id id[kEach];
        if (i + kEach <= to) {
#pragma unroll
            for (int u = 0; u < kEach; u += kN) {
                const Pack<Id, kN> in = load_pack<Id, kN>(history + i + u);
#pragma unroll
                for (int e = 0; e < kN; ++e) id[u + e] = in.v[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) id[e] = i + e < to ? history[i + e] : (Id)-1;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint64_t v = (uint64_t)(int64_t)id[e] - (uint64_t)begin;
            if (v < (uint64_t)n && i + e < to) see(i + e, (int)v);
        }
    }
}
template <typename See>
__device__ __forceinline__ void look_through(const PenaltyArgs& a, long row, int from, int to, int begin, int n, See see)
{
    if (a.id_type == NUTS_I64) look_through(static_cast<const int64_t*>(a.history) + row * a.history_stride, from, to, begin, n, see);
    else look_through(static_cast<const int32_t*>(a.history) + row * a.history_stride, from, to, begin, n, see);
}

// Counters for the next row of a workgroup.  Where all rows have one history and the row has seen no less of it than the one before, they
// are carried on: 4096 rows of one text of 4096 classes are counted once by each workgroup, not once by each row.  No
// thread may still be reading them; the caller waits before they are read.
__device__ __forceinline__ void count_on(const PenaltyArgs& a, long row, int begin, int n, Counted& done, const Counted& now, unsigned* count)
{
    if (a.history_stride != 0 || now.length < done.length || now.prompt < done.prompt) {
        for (int i = (int)threadIdx.x * 4; i < n; i += kThreads * 4) *reinterpret_cast<uint4*>(&count[i]) = uint4{0, 0, 0, 0};  // (kSlice is a multiple of 4)
        done = Counted{0, 0};
        __syncthreads();
    }
    if (now.prompt > done.prompt && done.prompt < done.length)
        look_through(a, row, done.prompt, min(now.prompt, done.length), begin, n, [&](int, int v) {
            atomicSub(&count[v], 1u);
            atomicOr(&count[v], kPrompt);
        });
    look_through(a, row, done.length, now.length, begin, n, [&](int i, int v) {
        if (i >= now.prompt) atomicAdd(&count[v], 1u);
        else atomicOr(&count[v], kPrompt);
    });
    done = now;
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

// The packs of a thread in a slice: pack u begins at class (u kThreads + thread) kN.
template <typename T>
constexpr int kPackN = 16 / sizeof(T);
template <typename T>
constexpr int kPacks = kSlice / kThreads / kPackN<T>;

template <typename T>
struct Slice {
    Pack<T, kPackN<T>> pack[kPacks<T>];
    // whole packs only: what is behind them is read one by one
    __device__ __forceinline__ void fetch(const T* row, int n)
    {
#pragma unroll
        for (int u = 0; u < kPacks<T>; ++u) {
            const int v = (u * kThreads + (int)threadIdx.x) * kPackN<T>;
            if (v + kPackN<T> <= n) pack[u] = load_pack<T, kPackN<T>>(row + v);
        }
    }
};
template <typename T>
__device__ __forceinline__ void unpack(const Pack<T, kPackN<T>>& in, const T* row, int v, int n, float (&x)[kPackN<T>])
{
#pragma unroll
    for (int e = 0; e < kPackN<T>; ++e) x[e] = v + kPackN<T> <= n ? to_float(in.v[e]) : v + e < n ? to_float(row[v + e]) : 0.f;
}
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
// The counters of a pack, and all of them together.
template <int kN>
__device__ __forceinline__ unsigned read_counts(const unsigned* count, unsigned (&c)[kN])
{
    unsigned any = 0;
#pragma unroll
    for (int e = 0; e < kN; e += 4) {
        const uint4 in = *reinterpret_cast<const uint4*>(&count[e]);
        c[e] = in.x, c[e + 1] = in.y, c[e + 2] = in.z, c[e + 3] = in.w;
        any |= in.x | in.y | in.z | in.w;
    }
    return any;
}
// A bit for each class of a pack that may come.
template <int kN>
__device__ __forceinline__ unsigned allowed_of(const uint32_t* allowed, int v, int n)
{
    constexpr unsigned kAll = (1u << kN) - 1;
    return allowed && v < n ? reinterpret_cast<const unsigned char*>(allowed)[v >> 3] >> (v & 7) & kAll : kAll;
}

// A workgroup a slice of `rows_each` rows.  The history's counts are made in LDS, where adding whole numbers in any order gives the same.
template <typename T>
__global__ __launch_bounds__(kThreads, 8) void penalties_kernel(PenaltyArgs a)
{
    constexpr int kN = kPackN<T>;
    __shared__ __attribute__((aligned(16))) unsigned count[kSlice];
    __shared__ int biased[NUTS_CAT_MAX_BIAS];
    const long block = a.first_block + blockIdx.x, group = block / a.slices;
    const int begin = (int)(block % a.slices) * kSlice, n = min(kSlice, a.n_classes - begin);
    const bool sparse = a.logits == a.out && !a.bias;  // what nothing changes is left alone
    const bool counting = a.history_len > 0 || a.n_bias > 0;
    Counted done{INT_MAX, INT_MAX};  // (nothing yet: the first row begins anew)
    const long end = min((group + 1) * a.rows_each, a.n_rows);
    const T* x_row = static_cast<const T*>(a.logits) + group * a.rows_each * a.row_stride + begin;
    for (long row = group * a.rows_each; row < end; ++row, x_row += a.row_stride) {
        T* to = static_cast<T*>(a.out) + row * a.out_stride + begin;
        const float* bias = a.bias ? a.bias + row * a.bias_stride + begin : nullptr;
        const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr;
        const float r = a.repetition ? a.repetition[row] : a.r;
        const RowFactors p{r, 1.f / r, a.frequency ? a.frequency[row] : a.f, a.presence ? a.presence[row] : a.q};
        Slice<T> own;  // on its way while the history is counted
        if (!sparse) own.fetch(x_row, n);
        if (counting) {
            for (int i = threadIdx.x; i < a.n_bias; i += kThreads) {
                const long v = id_at(a.bias_ids, a.id_type, row * a.n_bias + i) - begin;
                biased[i] = v >= 0 && v < n ? (int)v : -1;
            }
            count_on(a, row, begin, n, done, Counted{clamped(a.lengths, row, a.history_len, a.history_len), clamped(a.prompts, row, a.history_len, 0)}, count);
            for (int i = threadIdx.x; i < a.n_bias; i += kThreads)
                if (biased[i] >= 0) atomicOr(&count[biased[i]], kBiased);
            __syncthreads();
        }
        // classes with biases of their own: by the thread that has the first of them
        for (int i = threadIdx.x; i < a.n_bias; i += kThreads) {
            const int v = biased[i];
            if (v < 0) continue;
            bool first = true;
            for (int k = 0; k < i; ++k) first &= biased[k] != v;
            if (!first) continue;
            float sum = a.bias_values[row * a.n_bias + i];
            for (int k = i + 1; k < a.n_bias; ++k)
                if (biased[k] == v) sum += a.bias_values[row * a.n_bias + k];
            float z = penalised(to_float(x_row[v]), count[v], p);
            if (bias) z += bias[v];
            z += sum;
            to[v] = rounded<T>(may_come(allowed, v) ? z : -INFINITY);
        }
#pragma unroll
        for (int u = 0; u < kPacks<T>; ++u) {
            const int v = (u * kThreads + (int)threadIdx.x) * kN;
            if (v >= n) break;
            unsigned c[kN] = {};
            const unsigned any = counting ? read_counts<kN>(&count[v], c) : 0;
            const unsigned may = allowed_of<kN>(allowed, v, n);
            if (sparse) {
                if (!any && may == (1u << kN) - 1) continue;
                if (v + kN <= n) own.pack[u] = load_pack<T, kN>(x_row + v);
            }
            float x[kN];
            unpack(own.pack[u], x_row, v, n, x);
            if (any) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[e] = penalised(x[e], c[e], p);
            }
            if (bias) {
#pragma unroll
                for (int e = 0; e < kN; e += 4) {
                    if (v + kN <= n) {
                        const Pack<float, 4> b = load_pack<float, 4>(bias + v + e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[e + k] += b.v[k];
                    } else {
#pragma unroll
                        for (int k = e; k < e + 4; ++k)
                            if (v + k < n) x[k] += bias[v + k];
                    }
                }
            }
            if (allowed) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[e] = may >> e & 1 ? x[e] : -INFINITY;
            }
            if (any & kBiased) {
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (v + e < n && !(c[e] & kBiased)) to[v + e] = rounded<T>(x[e]);
            } else {
                write_pack(to, x, v, n, a.streamed);
            }
        }
        if (counting && row + 1 < end) {
            __syncthreads();
            if (a.n_bias > 0) {  // the next row's biases are others
                for (int i = threadIdx.x; i < a.n_bias; i += kThreads)
                    if (biased[i] >= 0) atomicAnd(&count[biased[i]], ~kBiased);
                __syncthreads();
            }
        }
    }
}

// A workgroup a slice of `rows_each` rows, whose gradients it adds up.
template <typename T>
__global__ __launch_bounds__(kThreads, 8) void penalties_grad_kernel(PenaltyArgs a)
{
    constexpr int kN = kPackN<T>;
    __shared__ __attribute__((aligned(16))) unsigned count[kSlice];
    const long block = a.first_block + blockIdx.x, group = block / a.slices;
    const int begin = (int)(block % a.slices) * kSlice, n = min(kSlice, a.n_classes - begin);
    const bool sparse = a.grad_out == a.out && !a.grad_bias, counting = a.out && a.history_len > 0;
    Counted done{INT_MAX, INT_MAX};
    const long end = min((group + 1) * a.rows_each, a.n_rows);
    const T* g_row = static_cast<const T*>(a.grad_out) + group * a.rows_each * a.grad_stride + begin;
    float sum[kPacks<T>][kN] = {};
    for (long row = group * a.rows_each; row < end; ++row, g_row += a.grad_stride) {
        const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride + begin;
        T* to = a.out ? static_cast<T*>(a.out) + row * a.out_stride + begin : nullptr;
        const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr;
        const float r = a.repetition ? a.repetition[row] : a.r, by_r = 1.f / r;
        Slice<T> own;
        if (!sparse) own.fetch(g_row, n);
        if (counting) {
            count_on(a, row, begin, n, done, Counted{clamped(a.lengths, row, a.history_len, a.history_len), 0}, count);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kPacks<T>; ++u) {
            const int v = (u * kThreads + (int)threadIdx.x) * kN;
            if (v >= n) break;
            unsigned c[kN] = {};
            const unsigned any = counting ? read_counts<kN>(&count[v], c) : 0;
            const unsigned may = allowed_of<kN>(allowed, v, n);
            if (sparse) {
                if (!any && may == (1u << kN) - 1) continue;
                if (v + kN <= n) own.pack[u] = load_pack<T, kN>(g_row + v);
            }
            float g[kN];
            unpack(own.pack[u], g_row, v, n, g);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                if (!(may >> e & 1)) g[e] = 0.f;
                sum[u][e] += g[e];
            }
            if (!to) continue;
            if (any) {
                Pack<T, kN> logits{};
                if (v + kN <= n) logits = load_pack<T, kN>(x_row + v);
                float x[kN];
                unpack(logits, x_row, v, n, x);
#pragma unroll
                for (int e = 0; e < kN; ++e) g[e] *= c[e] && (may >> e & 1) ? (x[e] > 0.f ? by_r : r) : 1.f;
            }
            write_pack(to, g, v, n, a.streamed);
        }
        if (counting && row + 1 < end) __syncthreads();
    }
    if (!a.grad_bias) return;
#pragma unroll
    for (int u = 0; u < kPacks<T>; ++u) {
        const int v = (u * kThreads + (int)threadIdx.x) * kN;
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (v + e < n) a.grad_bias[group * a.n_classes + begin + v + e] = sum[u][e];
    }
}

// Groups' sums as those of all rows: 64 classes a workgroup, the groups divided between its 16 waves.
__global__ __launch_bounds__(kJoinThreads) void join_bias_kernel(const float* part, float* grad_bias, long n_groups, int n_classes, long first_block)
{
    constexpr int kParts = kJoinThreads / kColumns;
    __shared__ float shared[kParts][kColumns];
    const long v = (first_block + blockIdx.x) * kColumns + threadIdx.x % kColumns;
    const int own = threadIdx.x / kColumns;
    float sum = 0.f;
    if (v < n_classes)
        for (long k = own; k < n_groups; k += kParts) sum += part[k * n_classes + v];
    shared[own][threadIdx.x % kColumns] = sum;
    __syncthreads();
    if (own != 0 || v >= n_classes) return;
    for (int k = 1; k < kParts; ++k) sum += shared[k][threadIdx.x];
    grad_bias[v] = sum;
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
    if (d->history_len < 0 || d->history_len > (1 << 30) - 1) return api_fail(NUTS_E_INVALID_ARG, "%s: history_len must be in [0, 2^30)", who);
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
    a.slices = (int)ceil_div(d->n_classes, kSlice);
    a.rows_each = 1;
    a.streamed = d->n_rows * d->n_classes * (int64_t)cat_size(d->dtype) >= kStreamed;
    return a;
}

// Rows of a workgroup: for a launch of about kGroups, which is what the chip has at a time, but at least `least`.
int64_t rows_of_group(const nuts_penalties_desc* d, int64_t least)
{
    return std::max<int64_t>(1, std::min(std::max(ceil_div(d->n_rows * ceil_div(d->n_classes, kSlice), kGroups), least), d->n_rows));
}
// Rows go together where they have one history, whose counts are carried on.
int64_t rows_of_group_sharing(const nuts_penalties_desc* d) { return d->history_len > 0 && d->history_stride == 0 ? rows_of_group(d, 1) : 1; }
constexpr int64_t kBiasRows = 4;  // that are added up: their sums are stored

void launch(void (*kernel)(PenaltyArgs), PenaltyArgs a)
{
    for (const long blocks = (long)ceil_div(a.n_rows, a.rows_each) * a.slices; a.first_block < blocks; a.first_block += kMaxBlocks)
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(blocks - a.first_block, kMaxBlocks)), dim3(kThreads), 0, api_stream(), a);
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
    a.rows_each = (int)rows_of_group_sharing(d);
    by_dtype(d->dtype, [&](auto t) { launch(penalties_kernel<decltype(t)>, a); });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_penalties_grad_workspace(const nuts_penalties_desc* d, int64_t* bytes)
{
    if (int rc = check_penalties(d, "nuts_penalties_grad_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad_workspace: bytes must not be NULL");
    *bytes = ceil_div(d->n_rows, rows_of_group(d, kBiasRows)) * d->n_classes * (int64_t)sizeof(float);
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
    const int64_t rows_each = rows_of_group(d, kBiasRows), groups = ceil_div(d->n_rows, rows_each);
    if (grad_bias && groups > 0) {
        const int64_t bytes = groups * d->n_classes * (int64_t)sizeof(float);
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
    a.rows_each = grad_bias ? (int)rows_each : (int)rows_of_group_sharing(d);
    by_dtype(d->dtype, [&](auto t) { launch(penalties_grad_kernel<decltype(t)>, a); });
    if (grad_bias) {
        constexpr long kMost = kMaxBlocks / (kJoinThreads / kThreads);
        for (long first = 0, blocks = (long)ceil_div(d->n_classes, kColumns); first < blocks; first += kMost)
            hipLaunchKernelGGL(join_bias_kernel, dim3((unsigned)std::min(blocks - first, kMost)), dim3(kJoinThreads), 0, api_stream(),
                               static_cast<const float*>(workspace), grad_bias, (long)groups, (int)d->n_classes, first);
    }
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
