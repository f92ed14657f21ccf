// Logits adjusted by what was said before, by biases and by masks, and the gradient of that.
//
//   z = x > 0 ? x / r : x r  where v was seen,   z -= f count_v + q [count_v > 0],   z += bias_v,   -infinity where v is not allowed
//   dx_v = g_v (seen_v ? (x > 0 ? 1 / r : r) : 1),   dbias_v = sum over rows of g_v,   0 where v is not allowed
#include "nuts_cat.h"

#include <algorithm>

namespace nuts {
namespace {

constexpr int kThreads = 512;
constexpr int kSlice = 8192;        // classes of a workgroup, with a counter each in LDS
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

// Counters of the classes begin .. begin + kSlice - 1 from the places from .. to - 1 of a history.
__device__ __forceinline__ void count_history(const PenaltyArgs& a, long row, int begin, int n, int from, int to, int prompt, unsigned* count)
{
    const long at = row * a.history_stride;
    for (int i = from + (int)threadIdx.x; i < to; i += kThreads) {
        const long v = id_at(a.history, a.id_type, at + i) - begin;
        if (v < 0 || v >= n) continue;
        if (i >= prompt) atomicAdd(&count[v], 1u);
        else atomicOr(&count[v], kPrompt);
    }
}

__device__ __forceinline__ bool may_come(const uint32_t* allowed, int v) { return !allowed || (allowed[v >> 5] >> (v & 31) & 1); }

struct RowFactors {
    float r, f, q;
};
__device__ __forceinline__ float penalised(float x, unsigned count, const RowFactors& p)
{
    if (!(count & kSeen)) return x;
    float z = x > 0.f ? x / p.r : x * p.r;
    const unsigned said = count & kCount;
    if (said) z -= p.f * (float)said + p.q;
    return z;
}

// A workgroup a slice of a row.  The history's counts are made in LDS, where adding whole numbers in any order gives the same.
template <typename T>
__global__ __launch_bounds__(kThreads) void penalties_kernel(PenaltyArgs a)
{
    __shared__ __attribute__((aligned(16))) unsigned count[kSlice];
    __shared__ int biased[NUTS_CAT_MAX_BIAS];
    const long block = a.first_block + blockIdx.x, row = block / a.slices;
    const int begin = (int)(block % a.slices) * kSlice, n = min(kSlice, a.n_classes - begin);
    const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride + begin;
    T* to = static_cast<T*>(a.out) + row * a.out_stride + begin;
    const float* bias = a.bias ? a.bias + row * a.bias_stride + begin : nullptr;
    const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr;
    const bool in_place = a.logits == a.out;
    const RowFactors p{a.repetition ? a.repetition[row] : a.r, a.frequency ? a.frequency[row] : a.f, a.presence ? a.presence[row] : a.q};
    for (int i = threadIdx.x; i < kSlice; i += kThreads) count[i] = 0;
    for (int i = threadIdx.x; i < a.n_bias; i += kThreads) {
        const long v = id_at(a.bias_ids, a.id_type, row * a.n_bias + i) - begin;
        biased[i] = v >= 0 && v < n ? (int)v : -1;
    }
    __syncthreads();
    const int length = clamped(a.lengths, row, a.history_len, a.history_len), prompt = clamped(a.prompts, row, a.history_len, 0);
    count_history(a, row, begin, n, 0, length, prompt, count);
    for (int i = threadIdx.x; i < a.n_bias; i += kThreads)
        if (biased[i] >= 0) atomicOr(&count[biased[i]], kBiased);
    __syncthreads();
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
    for (int v = threadIdx.x; v < n; v += kThreads) {
        const unsigned c = count[v];
        if (c & kBiased) continue;
        const bool may = may_come(allowed, v);
        if (in_place && may && !c && !bias) continue;
        float z = -INFINITY;
        if (may) {
            z = penalised(to_float(x_row[v]), c, p);
            if (bias) z += bias[v];
        }
        to[v] = rounded<T>(z);
    }
}

// A workgroup a slice of `rows_each` rows, whose gradients it adds up.
template <typename T>
__global__ __launch_bounds__(kThreads) void penalties_grad_kernel(PenaltyArgs a)
{
    constexpr int kEach = kSlice / kThreads;
    __shared__ __attribute__((aligned(16))) unsigned count[kSlice];
    const long block = a.first_block + blockIdx.x, group = block / a.slices;
    const int begin = (int)(block % a.slices) * kSlice, n = min(kSlice, a.n_classes - begin);
    float sum[kEach] = {};
    for (long row = group * a.rows_each; row < min((group + 1) * a.rows_each, a.n_rows); ++row) {
        const T* x_row = static_cast<const T*>(a.logits) + row * a.row_stride + begin;
        const T* g_row = static_cast<const T*>(a.grad_out) + row * a.grad_stride + begin;
        T* to = a.out ? static_cast<T*>(a.out) + row * a.out_stride + begin : nullptr;
        const uint32_t* allowed = a.allowed ? a.allowed + row * a.allowed_stride + begin / 32 : nullptr;
        const float r = a.repetition ? a.repetition[row] : a.r;
        if (to) {
            for (int i = threadIdx.x; i < kSlice; i += kThreads) count[i] = 0;
            __syncthreads();
            count_history(a, row, begin, n, 0, clamped(a.lengths, row, a.history_len, a.history_len), 0, count);
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int v = (int)threadIdx.x + e * kThreads;
            if (v >= n) break;
            float g = may_come(allowed, v) ? to_float(g_row[v]) : 0.f;
            sum[e] += g;
            if (!to) continue;
            if (count[v]) g = to_float(x_row[v]) > 0.f ? g / r : g * r;
            to[v] = rounded<T>(may_come(allowed, v) ? g : 0.f);
        }
        __syncthreads();
    }
    if (!a.grad_bias) return;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int v = (int)threadIdx.x + e * kThreads;
        if (v < n) a.grad_bias[group * a.n_classes + begin + v] = sum[e];
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

// Rows that a workgroup adds up, for a launch of about kGroups.
int64_t rows_of_group(const nuts_penalties_desc* d)
{
    return std::max<int64_t>(1, std::min(ceil_div(d->n_rows * ceil_div(d->n_classes, kSlice), kGroups), d->n_rows));
}

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
    by_dtype(d->dtype, [&](auto t) { launch(penalties_kernel<decltype(t)>, a); });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_penalties_grad_workspace(const nuts_penalties_desc* d, int64_t* bytes)
{
    if (int rc = check_penalties(d, "nuts_penalties_grad_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_penalties_grad_workspace: bytes must not be NULL");
    *bytes = ceil_div(d->n_rows, rows_of_group(d)) * d->n_classes * (int64_t)sizeof(float);
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
    const int64_t rows_each = rows_of_group(d), groups = ceil_div(d->n_rows, rows_each);
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
    a.rows_each = grad_bias ? (int)rows_each : 1;
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
