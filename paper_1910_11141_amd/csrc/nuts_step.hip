// Steps over many tensors at once: the norm of all their numbers, and AdamW with moments of 32 or 8 bits.
//
//   norm = sqrt(sum x^2),   factor = min(1, max_norm / norm)
//   g = s factor grad,   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   p = p (1 - lr d) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
//
// The tensors' table goes to a launch among its arguments, which captured launches keep: nothing is copied to the device.
#include "nuts_cat.h"
#include "nuts_rng.h"

#include <algorithm>
#include <cmath>

namespace nuts {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kLongest = (int64_t)1 << 40;

// The tensor that a workgroup belongs to: the last whose first workgroup is no later.
template <int kTensors>
__device__ __forceinline__ int tensor_of(const int (&first)[kTensors], int block)
{
    int t = 0;
    for (int k = 1; k < kTensors; ++k) t += first[k] <= block;
    return t;
}

// ---- norm -----------------------------------------------------------------------------------------------------------

constexpr int kNormTensors = 120;
constexpr int kNormBlocks = 2048;   // about so many workgroups in all
constexpr int kNormLeast = 8192;    // numbers of a workgroup, at least

struct NormArgs {
    const void* data[kNormTensors];
    long n[kNormTensors];
    int first[kNormTensors];
    unsigned char dtype[kNormTensors];
    double* part;
    long each;
};
static_assert(sizeof(NormArgs) <= 4096, "the arguments of a launch");

__device__ __forceinline__ double block_sum(double v, double* shared, int n_waves)
{
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v += __shfl_xor(v, step);
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < n_waves; ++w) v += shared[w];
    return v;
}

template <typename T>
__device__ __forceinline__ double squares(const T* x, long n)
{
    double sum = 0;
    for (long i = threadIdx.x; i < n; i += kThreads) {
        const double v = (double)to_float(x[i]);
        sum = fma(v, v, sum);
    }
    return sum;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a)
{
    __shared__ double shared[kThreads / 64];
    const int t = tensor_of(a.first, (int)blockIdx.x);
    const long begin = (long)((int)blockIdx.x - a.first[t]) * a.each, n = min(a.each, a.n[t] - begin);
    double sum;
    if (a.dtype[t] == NUTS_F32) sum = squares(static_cast<const float*>(a.data[t]) + begin, n);
    else if (a.dtype[t] == NUTS_BF16) sum = squares(static_cast<const bf16*>(a.data[t]) + begin, n);
    else sum = squares(static_cast<const f16*>(a.data[t]) + begin, n);
    sum = block_sum(sum, shared, kThreads / 64);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void join_norm_kernel(const double* part, long n, double max_norm, float* norm, float* factor)
{
    __shared__ double shared[kThreads / 64];
    double sum = 0;
    for (long i = threadIdx.x; i < n; i += kThreads) sum += part[i];
    sum = block_sum(sum, shared, kThreads / 64);
    if (threadIdx.x != 0) return;
    const double root = sqrt(sum);
    if (norm) *norm = (float)root;
    if (factor) *factor = !(root < INFINITY) ? NAN : root > max_norm ? (float)(max_norm / root) : 1.f;
}

// Numbers of a workgroup: a multiple of 2048, so that kNormBlocks or so (and one for each tensor) do.
int64_t norm_each(const nuts_tensor* tensors, int64_t n)
{
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) total += tensors[i].n;
    return std::max<int64_t>(kNormLeast, ceil_div(ceil_div(total, kNormBlocks), 2048) * 2048);
}

int check_norm(const nuts_tensor* tensors, int64_t n, const char* who)
{
    if (n < 0 || n > (1 << 20)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_tensors must be in [0, 2^20]", who);
    if (n > 0 && !tensors) return api_fail(NUTS_E_INVALID_ARG, "%s: tensors must not be NULL", who);
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (!cat_dtype_known(tensors[i].dtype)) return api_fail(NUTS_E_INVALID_ARG, "%s: dtype of tensor %lld must be NUTS_F32, NUTS_BF16 or NUTS_F16", who, (long long)i);
        if (tensors[i].n < 0 || tensors[i].n > kLongest) return api_fail(NUTS_E_INVALID_ARG, "%s: n of tensor %lld must be in [0, 2^40]", who, (long long)i);
        if (tensors[i].n > 0 && !tensors[i].data) return api_fail(NUTS_E_INVALID_ARG, "%s: data of tensor %lld must not be NULL", who, (long long)i);
        total += tensors[i].n;
    }
    if (total > kLongest) return api_fail(NUTS_E_INVALID_ARG, "%s: more than 2^40 numbers", who);
    return NUTS_OK;
}

int64_t norm_blocks(const nuts_tensor* tensors, int64_t n)
{
    const int64_t each = norm_each(tensors, n);
    int64_t blocks = 0;
    for (int64_t i = 0; i < n; ++i) blocks += ceil_div(tensors[i].n, each);
    return blocks;
}

// ---- AdamW ----------------------------------------------------------------------------------------------------------

constexpr int kStepTensors = 48;
constexpr int kChunk = 8192;  // numbers of a workgroup

struct StepArgs {
    nuts_adamw_tensor tensor[kStepTensors];
    int first[kStepTensors];
    const int64_t* step;
    const float* lr_at;
    const float* factor;
    double log_beta1, log_beta2, lr, decay;
    float beta1, rest1, beta2, rest2, eps, scale;
    float keep, size, root_scale;  // 1 - lr d, lr / (1 - b1^t), 1 / sqrt(1 - b2^t), where neither t nor lr is on the device
    unsigned t, k0, k1, first_tensor;
    long first_block;
    int64_t host_step;
    int copy_dtype;
};
static_assert(sizeof(StepArgs) <= 4096, "the arguments of a launch");

struct Factors {
    float scale, keep, size, root_scale;
    unsigned t;
};

__device__ __forceinline__ Factors factors_of(const StepArgs& a, float factor)
{
    Factors f{a.scale * factor, a.keep, a.size, a.root_scale, a.t};
    if (a.step || a.lr_at) {
        const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
        const int64_t t = a.step ? max(*a.step, (int64_t)1) : a.host_step;
        f.keep = (float)(1.0 - lr * a.decay);
        f.size = (float)(lr / -expm1((double)t * a.log_beta1));
        f.root_scale = (float)(1.0 / sqrt(-expm1((double)t * a.log_beta2)));
        f.t = (unsigned)t;
    }
    return f;
}

// Four numbers next to each other, as many of them as there are.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, float (&x)[4])
{
    if (n >= 4) {
        const Pack<T, 4> in = load_pack<T, 4>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = to_float(in.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < n ? to_float(p[e]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int n, const float (&x)[4])
{
    Pack<T, 4> out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out.v[e] = rounded<T>(x[e]);
    if (n >= 4) {
        store_pack(p, out);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) p[e] = out.v[e];
    }
}

// To bfloat16, up with the probability of what is cut off: 12 random bits and a half.
__device__ __forceinline__ float rounded_at_random(float x, unsigned word)
{
    const unsigned bits = __float_as_uint(x);
    if ((bits & 0x7f800000u) == 0x7f800000u) return x;
    return __uint_as_float((bits + (word >> 20 << 4 | 8u)) & 0xffff0000u);
}

__device__ __forceinline__ float chance(unsigned bits) { return ((float)(bits & 1023u) + 0.5f) * (1.f / 1024.f); }

// Codes of 8 bits.  x is in units of the scale: 127^2 or 254^2 at a block's largest.
__device__ __forceinline__ float m_value(int code, float scale) { return code == -128 ? NAN : (float)(code * abs(code)) * scale; }
__device__ __forceinline__ float root_value(unsigned code, float scale) { return code == 255 ? NAN : (float)(code * code) * scale; }
__device__ __forceinline__ int m_code(float m, float scale, unsigned word)
{
    if (!(__builtin_fabsf(m) < INFINITY)) return -128;
    const float x = scale > 0.f ? __builtin_fabsf(m) / scale : 0.f;
    float c = fminf(floorf(sqrtf(x)), 126.f);
    if (x - c * c > (2.f * c + 1.f) * chance(word)) c += 1.f;
    return m < 0.f ? -(int)c : (int)c;
}
__device__ __forceinline__ unsigned v_code(float root, float scale, unsigned word)
{
    if (!(root < INFINITY)) return 255;
    const float x = scale > 0.f ? root / scale : 0.f;
    float c = fminf(floorf(sqrtf(x)), 253.f);
    const float below = c * c, above = (c + 1.f) * (c + 1.f);
    if (x * x - below * below > (above - below) * (above + below) * chance(word >> 10)) c += 1.f;
    if (root > 0.f) c = fmaxf(c, 1.f);
    return (unsigned)c;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = fmaxf(v, __shfl_xor(v, step));
    return v;
}
__device__ __forceinline__ float if_finite(float v) { return __builtin_fabsf(v) < INFINITY ? __builtin_fabsf(v) : 0.f; }

// A workgroup kChunk numbers of a tensor, a wave 256 of them at a time: a block of the moments of 8 bits.
template <typename P, typename G, bool kEight>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs a)
{
    const float factor = a.factor ? *a.factor : 1.f;
    if (factor != factor) return;
    const Factors f = factors_of(a, factor);
    const int k = tensor_of(a.first, (int)blockIdx.x);
    const nuts_adamw_tensor& t = a.tensor[k];
    const long begin = (a.first_block + (long)((int)blockIdx.x - a.first[k])) * kChunk, end = min(begin + kChunk, (long)t.n);
    const int lane = threadIdx.x % 64;
    for (long block = begin + threadIdx.x / 64 * 256; block < end; block += kThreads * 4) {
        const long i = block + lane * 4;
        const int n = (int)max(min(end - i, 4l), 0l);
        float p[4], g[4], m[4], v[4], root[4];
        load4(static_cast<const P*>(t.param) + i, n, p);
        load4(static_cast<const G*>(t.grad) + i, n, g);
        if (kEight) {
            const float m_scale = t.m_scale[block / 256], v_scale = t.v_scale[block / 256];
            const int8_t* m_at = static_cast<const int8_t*>(t.m) + i;
            const uint8_t* v_at = static_cast<const uint8_t*>(t.v) + i;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = e < n ? m_value(m_at[e], m_scale) : 0.f;
                root[e] = e < n ? root_value(v_at[e], v_scale) : 0.f;
                v[e] = root[e] * root[e];
            }
        } else {
            load4(static_cast<const float*>(t.m) + i, n, m);
            load4(static_cast<const float*>(t.v) + i, n, v);
        }
        Words4 w{0, 0, 0, 0};
        if (kEight || sizeof(P) == 2) w = philox4x32_10((unsigned)(i / 4), 6u | (unsigned)(i / 4 >> 32) << 8, f.t, a.first_tensor + k, a.k0, a.k1);
        const unsigned words[4] = {w.w0, w.w1, w.w2, w.w3};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = g[e] * f.scale;
            m[e] = m[e] * a.beta1 + x * a.rest1;
            v[e] = v[e] * a.beta2 + x * x * a.rest2;
            root[e] = sqrtf(v[e]);
            p[e] = p[e] * f.keep - f.size * m[e] / (root[e] * f.root_scale + a.eps);
            if (sizeof(P) == 2) p[e] = rounded_at_random(p[e], words[e]);
        }
        store4(static_cast<P*>(t.param) + i, n, p);
        if (t.copy) a.copy_dtype == NUTS_BF16 ? store4(static_cast<bf16*>(t.copy) + i, n, p) : store4(static_cast<f16*>(t.copy) + i, n, p);
        if (kEight) {
            float m_top = 0.f, v_top = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) {
                    m_top = fmaxf(m_top, if_finite(m[e]));
                    v_top = fmaxf(v_top, if_finite(root[e]));
                }
            const float m_scale = wave_max(m_top) * (1.f / (127.f * 127.f)), v_scale = wave_max(v_top) * (1.f / (254.f * 254.f));
            int8_t* m_at = static_cast<int8_t*>(t.m) + i;
            uint8_t* v_at = static_cast<uint8_t*>(t.v) + i;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) {
                    m_at[e] = (int8_t)m_code(m[e], m_scale, words[e]);
                    v_at[e] = (uint8_t)v_code(root[e], v_scale, words[e]);
                }
            if (lane == 0) {
                t.m_scale[block / 256] = m_scale;
                t.v_scale[block / 256] = v_scale;
            }
        } else {
            store4(static_cast<float*>(t.m) + i, n, m);
            store4(static_cast<float*>(t.v) + i, n, v);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void values_kernel(StepArgs a)
{
    const int k = tensor_of(a.first, (int)blockIdx.x);
    const nuts_adamw_tensor& t = a.tensor[k];
    const long begin = (a.first_block + (long)((int)blockIdx.x - a.first[k])) * kChunk, end = min(begin + kChunk, (long)t.n);
    for (long i = begin + (long)threadIdx.x * 4; i < end; i += kThreads * 4) {
        const int n = (int)min(end - i, 4l);
        float m[4], v[4];
        const int8_t* m_at = static_cast<const int8_t*>(t.m) + i;
        const uint8_t* v_at = static_cast<const uint8_t*>(t.v) + i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = e < n ? m_value(m_at[e], t.m_scale[i / 256]) : 0.f;
            const float root = e < n ? root_value(v_at[e], t.v_scale[i / 256]) : 0.f;
            v[e] = root * root;
        }
        if (t.param) store4(static_cast<T*>(t.param) + i, n, m);
        if (t.copy) store4(static_cast<T*>(t.copy) + i, n, v);
    }
}

// Calls `go` for as many tensors at a time as a launch takes, and as many workgroups as it takes.
template <typename Wanted, typename Go>
void by_tables(StepArgs& a, const nuts_adamw_tensor* tensors, int64_t n, Wanted wanted, Go go)
{
    int64_t at = 0;
    while (at < n) {
        int64_t blocks = 0;
        int used = 0;
        a.first_tensor = (unsigned)at;
        a.first_block = 0;
        for (; used < kStepTensors && at < n; ++used, ++at) {
            const int64_t own = wanted(tensors[at]) ? ceil_div(tensors[at].n, kChunk) : 0;
            if (blocks + own > kMaxBlocks) {
                if (used > 0) break;
                // a tensor of more workgroups than a launch has: alone, in several
                a.tensor[0] = tensors[at];
                for (int k = 0; k < kStepTensors; ++k) a.first[k] = k ? INT32_MAX : 0;
                for (int64_t done = 0; done < own; done += kMaxBlocks) {
                    a.first_block = (long)done;
                    go((unsigned)std::min<int64_t>(own - done, kMaxBlocks));
                }
                blocks = 0;
                used = 0;
                ++at;
                break;
            }
            a.tensor[used] = tensors[at];
            a.first[used] = (int)blocks;
            blocks += own;
        }
        if (blocks == 0) continue;
        for (int k = used; k < kStepTensors; ++k) a.first[k] = INT32_MAX;
        go((unsigned)blocks);
    }
}

int check_tensors(const nuts_adamw_tensor* tensors, int64_t n, const char* who)
{
    if (n < 0 || n > (1 << 20)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_tensors must be in [0, 2^20]", who);
    if (n > 0 && !tensors) return api_fail(NUTS_E_INVALID_ARG, "%s: tensors must not be NULL", who);
    for (int64_t i = 0; i < n; ++i)
        if (tensors[i].n < 0 || tensors[i].n > kLongest) return api_fail(NUTS_E_INVALID_ARG, "%s: n of tensor %lld must be in [0, 2^40]", who, (long long)i);
    return NUTS_OK;
}

template <typename P, typename G>
void (*step_kernel(int bits))(StepArgs)
{
    return bits == 8 ? adamw_kernel<P, G, true> : adamw_kernel<P, G, false>;
}

}  // namespace
}  // namespace nuts

using namespace nuts;

extern "C" {

int nuts_norm_workspace(const nuts_tensor* tensors, int64_t n_tensors, int64_t* bytes)
{
    if (int rc = check_norm(tensors, n_tensors, "nuts_norm_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_norm_workspace: bytes must not be NULL");
    *bytes = norm_blocks(tensors, n_tensors) * (int64_t)sizeof(double);
    return NUTS_OK;
}

int nuts_norm(const nuts_tensor* tensors, int64_t n_tensors, double max_norm, float* norm, float* factor, void* workspace,
              int64_t workspace_bytes)
{
    if (int rc = check_norm(tensors, n_tensors, "nuts_norm")) return rc;
    if (!std::isfinite(max_norm) || !(max_norm > 0)) return api_fail(NUTS_E_INVALID_ARG, "nuts_norm: max_norm must be finite and > 0");
    if (!norm && !factor) return NUTS_OK;
    const int64_t blocks = norm_blocks(tensors, n_tensors), bytes = blocks * (int64_t)sizeof(double);
    if (bytes > 0 && (!workspace || workspace_bytes < bytes)) return api_fail(NUTS_E_INVALID_ARG, "nuts_norm: needs a workspace of %lld bytes", (long long)bytes);
    if (bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % 256) return api_fail(NUTS_E_INVALID_ARG, "nuts_norm: workspace must be aligned to 256 bytes");
    if (int rc = api_have_device()) return rc;
    NormArgs a{};
    a.each = (long)norm_each(tensors, n_tensors);
    double* part = static_cast<double*>(workspace);
    for (int64_t at = 0; at < n_tensors;) {
        int64_t own = 0;
        int used = 0;
        for (; used < kNormTensors && at < n_tensors; ++used, ++at) {
            a.data[used] = tensors[at].data;
            a.n[used] = (long)tensors[at].n;
            a.dtype[used] = (unsigned char)tensors[at].dtype;
            a.first[used] = (int)own;
            own += ceil_div(tensors[at].n, a.each);
        }
        for (; used < kNormTensors; ++used) a.first[used] = INT32_MAX;
        a.part = part;
        if (own > 0) hipLaunchKernelGGL(norm_kernel, dim3((unsigned)own), dim3(kThreads), 0, api_stream(), a);
        part += own;
    }
    hipLaunchKernelGGL(join_norm_kernel, dim3(1), dim3(kThreads), 0, api_stream(), static_cast<const double*>(workspace), (long)blocks, max_norm, norm, factor);
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_adamw(const nuts_adamw_desc* d, const nuts_adamw_tensor* tensors, int64_t n_tensors, const int64_t* step, const float* lr,
               const float* factor)
{
    if (!d) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: desc must not be NULL");
    if (d->param_dtype != NUTS_F32 && d->param_dtype != NUTS_BF16) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: param_dtype must be NUTS_F32 or NUTS_BF16");
    if (!cat_dtype_known(d->grad_dtype)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: grad_dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16");
    if (d->copy_dtype != NUTS_BF16 && d->copy_dtype != NUTS_F16) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: copy_dtype must be NUTS_BF16 or NUTS_F16");
    if (d->state_bits != 32 && d->state_bits != 8) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: state_bits must be 32 or 8");
    if (!std::isfinite((float)d->lr)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: lr must be finite");
    // (as the kernels have them: 32 bits)
    if (!(d->beta1 >= 0) || !((float)d->beta1 < 1.f) || !(d->beta2 >= 0) || !((float)d->beta2 < 1.f)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: beta1 and beta2 must be in [0, 1)");
    if (!std::isfinite((float)d->eps) || !(d->eps >= 0)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: eps must be finite and >= 0");
    if (!std::isfinite((float)d->weight_decay)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: weight_decay must be finite");
    if (!std::isfinite((float)d->scale)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: scale must be finite");
    if (d->step < 1) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: step must be at least 1");
    if (int rc = check_tensors(tensors, n_tensors, "nuts_adamw")) return rc;
    int64_t total = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const nuts_adamw_tensor& t = tensors[i];
        if (t.n == 0 || !t.grad) continue;
        if (!t.param || !t.m || !t.v || (d->state_bits == 8 && (!t.m_scale || !t.v_scale)))
            return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw: null pointer in tensor %lld", (long long)i);
        total += t.n;
    }
    if (total == 0) return NUTS_OK;
    if (int rc = api_have_device()) return rc;
    StepArgs a{};
    a.step = step;
    a.lr_at = lr;
    a.factor = factor;
    a.log_beta1 = std::log(d->beta1);
    a.log_beta2 = std::log(d->beta2);
    a.lr = d->lr;
    a.decay = d->weight_decay;
    a.beta1 = (float)d->beta1;
    a.rest1 = (float)(1.0 - d->beta1);
    a.beta2 = (float)d->beta2;
    a.rest2 = (float)(1.0 - d->beta2);
    a.eps = (float)d->eps;
    a.scale = (float)d->scale;
    a.keep = (float)(1.0 - d->lr * d->weight_decay);
    a.size = (float)(d->lr / -std::expm1((double)d->step * a.log_beta1));
    a.root_scale = (float)(1.0 / std::sqrt(-std::expm1((double)d->step * a.log_beta2)));
    a.t = (unsigned)d->step;
    a.host_step = d->step;
    a.k0 = (unsigned)d->seed;
    a.k1 = (unsigned)(d->seed >> 32);
    a.copy_dtype = d->copy_dtype;
    void (*kernel)(StepArgs) = nullptr;
    by_dtype(d->grad_dtype, [&](auto g) {
        using G = decltype(g);
        kernel = d->param_dtype == NUTS_F32 ? step_kernel<float, G>(d->state_bits) : step_kernel<bf16, G>(d->state_bits);
    });
    by_tables(a, tensors, n_tensors, [](const nuts_adamw_tensor& t) { return t.grad != nullptr; },
              [&](unsigned blocks) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, api_stream(), a); });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_adamw_values(const nuts_adamw_tensor* tensors, int64_t n_tensors, int32_t dtype)
{
    if (!cat_dtype_known(dtype)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw_values: dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16");
    if (int rc = check_tensors(tensors, n_tensors, "nuts_adamw_values")) return rc;
    int64_t total = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const nuts_adamw_tensor& t = tensors[i];
        if (t.n == 0 || (!t.param && !t.copy)) continue;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw_values: null pointer in tensor %lld", (long long)i);
        total += t.n;
    }
    if (total == 0) return NUTS_OK;
    if (int rc = api_have_device()) return rc;
    StepArgs a{};
    by_dtype(dtype, [&](auto t) {
        by_tables(a, tensors, n_tensors, [](const nuts_adamw_tensor& x) { return x.param || x.copy; },
                  [&](unsigned blocks) { hipLaunchKernelGGL(values_kernel<decltype(t)>, dim3(blocks), dim3(kThreads), 0, api_stream(), a); });
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
