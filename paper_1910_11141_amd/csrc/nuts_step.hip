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

// The tensor that a workgroup belongs to: the last whose first workgroup is no later.  A lane looks at every 64th.
template <int kTensors>
__device__ __forceinline__ int tensor_of(const int (&first)[kTensors], int block)
{
    int t = -1;
#ifdef __HIP_DEVICE_COMPILE__
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int k = 0; k < kTensors; k += 64) t += __popcll(__builtin_amdgcn_ballot_w64(k + lane < kTensors && first[min(k + lane, kTensors - 1)] <= block));
#endif
    return t;
}

// ---- norm -----------------------------------------------------------------------------------------------------------

// A pass over all numbers, bound by its reads: 200 million bfloat16 in 150 tensors 72 us, 5.6 TB/s, and 2 for joining the workgroups' sums.  The sums are binary64,
// which hold the squares of all types and cost nothing here: two instructions a number.
constexpr int kNormTensors = 190;
constexpr int kNormBlocks = 2048;   // about so many workgroups in all
constexpr int kNormLeast = 8192;    // numbers of a workgroup, at least
constexpr int kNormThreads = 1024;  // of the workgroup that joins theirs
// Numbers of a part of a tensor, which a wave of one workgroup takes at a time, and parts up to which that workgroup does all of it alone.  48 parts take it
// 4.1 to 5.9 us and two launches 4.6, for which the host has 14.8 us to do where one needs 10.6 (16 parts: 3.3 us, 64: 6.9).
constexpr int kNormPart = 2048;
constexpr int kNormSmall = 48;

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

// The squares of n numbers that lie next to each other, by kCount threads, of which this is one.
template <typename T, int kCount>
__device__ __forceinline__ double squares(const T* x, long n, int thread)
{
    constexpr int kN = 16 / sizeof(T), kFlight = 4;
    double sum[kFlight] = {};
    long i = (long)thread * kN;
    for (; i + (kFlight - 1) * kCount * kN + kN <= n; i += kFlight * kCount * kN) {
        Pack<T, kN> in[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) in[u] = load_pack<T, kN>(x + i + u * kCount * kN);
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const double v = (double)to_float(in[u].v[e]);
                sum[u] = fma(v, v, sum[u]);
            }
    }
    for (; i < n; i += kCount * kN) {
        Pack<T, kN> in{};
        if (i + kN <= n) {
            in = load_pack<T, kN>(x + i);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (i + e < n) in.v[e] = x[i + e];
        }
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const double v = (double)to_float(in.v[e]);
            sum[e % kFlight] = fma(v, v, sum[e % kFlight]);
        }
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
template <int kCount>
__device__ __forceinline__ double squares(const void* data, int dtype, long begin, long n, int thread)
{
    if (dtype == NUTS_F32) return squares<float, kCount>(static_cast<const float*>(data) + begin, n, thread);
    if (dtype == NUTS_BF16) return squares<bf16, kCount>(static_cast<const bf16*>(data) + begin, n, thread);
    return squares<f16, kCount>(static_cast<const f16*>(data) + begin, n, thread);
}

__device__ __forceinline__ void write_norm(double sum, double max_norm, float* norm, float* factor)
{
    if (threadIdx.x != 0) return;
    const double root = sqrt(sum);
    if (norm) *norm = (float)root;
    if (factor) *factor = !(root < INFINITY) ? NAN : root > max_norm ? (float)(max_norm / root) : 1.f;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a)
{
    __shared__ double shared[kThreads / 64];
    const int t = tensor_of(a.first, (int)blockIdx.x);
    const long begin = (long)((int)blockIdx.x - a.first[t]) * a.each, n = min(a.each, a.n[t] - begin);
    const double sum = block_sum(squares<kThreads>(a.data[t], a.dtype[t], begin, n, (int)threadIdx.x), shared, kThreads / 64);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kNormThreads) void join_norm_kernel(const double* part, long n, double max_norm, float* norm, float* factor)
{
    __shared__ double shared[kNormThreads / 64];
    double sum = 0;
#pragma unroll 4
    for (long i = threadIdx.x; i < n; i += kNormThreads) sum += part[i];
    write_norm(block_sum(sum, shared, kNormThreads / 64), max_norm, norm, factor);
}

// All of it by one workgroup, where there is little: one launch in place of two.  Each wave its parts, one after the other.
__global__ __launch_bounds__(kNormThreads) void small_norm_kernel(NormArgs a, int n_parts, double max_norm, float* norm, float* factor)
{
    __shared__ double shared[kNormThreads / 64];
    double sum = 0;
    for (int part = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64); part < n_parts; part += kNormThreads / 64) {
        const int t = tensor_of(a.first, part);
        const long begin = (long)(part - a.first[t]) * kNormPart, n = min((long)kNormPart, a.n[t] - begin);
        sum += squares<64>(a.data[t], a.dtype[t], begin, n, (int)threadIdx.x % 64);
    }
    write_norm(block_sum(sum, shared, kNormThreads / 64), max_norm, norm, factor);
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

bool norm_is_small(const nuts_tensor* tensors, int64_t n)
{
    int64_t parts = 0;
    for (int64_t i = 0; i < n && parts <= kNormSmall; ++i) parts += ceil_div(tensors[i].n, kNormPart);
    return n <= kNormTensors && parts <= kNormSmall;
}

int64_t norm_blocks(const nuts_tensor* tensors, int64_t n)
{
    if (norm_is_small(tensors, n)) return 0;
    const int64_t each = norm_each(tensors, n);
    int64_t blocks = 0;
    for (int64_t i = 0; i < n; ++i) blocks += ceil_div(tensors[i].n, each);
    return blocks;
}

// ---- AdamW ----------------------------------------------------------------------------------------------------------

// Numbers of a workgroup: 256 a wave at a time, eight times in large calls; in small ones as few times as kStepBlocks workgroups allow (16000
// numbers: 8.4 us with eight times, 3.8 with one).
constexpr int64_t kChunkLeast = 1024, kChunkMost = 8192, kStepBlocks = 1024;

// What a launch knows of its tensors.  Addresses and counts of 48 bits, so that there are more tensors: 300 of 100 numbers 26 us, 37 with 56 tensors a launch.
template <bool kEight>
struct StepArgs {
    static constexpr int kPlaces = kEight ? 8 : 6, kTensors = kEight ? 75 : 98;
    unsigned tensor[kTensors][kPlaces * 3 / 2];
    int first[kTensors];
    unsigned t, k0, k1, first_tensor;
    const int64_t* step;
    const float* lr_at;
    const float* factor;
    double log_beta1, log_beta2, lr, decay;
    float beta1, rest1, beta2, rest2, eps, scale;
    float keep, size, root_scale;  // 1 - lr d, lr / (1 - b1^t), 1 / sqrt(1 - b2^t), where neither t nor lr is on the device
    int chunk;
    long first_block;
    int64_t host_step;
    int copy_dtype;
    // What the reciprocal takes is below 2^-126 (and counts as 0), or it gives such a number (and 0), only for an eps that is not in [2^-100, 2^100]: sqrt(v) times its
    // factor is 2^77 at most.  Then m and the denominator are moved by 2^64.
    int usual_eps;
};
static_assert(sizeof(StepArgs<false>) <= 4096 && sizeof(StepArgs<true>) <= 4096, "the arguments of a launch");

// A tensor's addresses and count, two in three words.
template <bool kEight>
void pack_tensor(const nuts_adamw_tensor& t, unsigned* words)
{
    const uint64_t place[8] = {(uint64_t)t.n,          (uint64_t)(uintptr_t)t.param, (uint64_t)(uintptr_t)t.grad,    (uint64_t)(uintptr_t)t.copy,
                               (uint64_t)(uintptr_t)t.m, (uint64_t)(uintptr_t)t.v,     (uint64_t)(uintptr_t)t.m_scale, (uint64_t)(uintptr_t)t.v_scale};
    for (int k = 0; k < StepArgs<kEight>::kPlaces; k += 2, words += 3) {
        words[0] = (unsigned)place[k];
        words[1] = (unsigned)(place[k] >> 32 & 0xffff) | (unsigned)place[k + 1] << 16;
        words[2] = (unsigned)(place[k + 1] >> 16);
    }
}
// (of the device's memory, which an address alone does not say)
__device__ __forceinline__ void* global(uint64_t address)
{
#ifdef __HIP_DEVICE_COMPILE__
    return (void*)(__attribute__((address_space(1))) void*)address;
#else
    return reinterpret_cast<void*>(address);
#endif
}
template <bool kEight>
__device__ __forceinline__ nuts_adamw_tensor unpack_tensor(const unsigned* words)
{
    uint64_t place[8] = {};
#pragma unroll
    for (int k = 0; k < StepArgs<kEight>::kPlaces; k += 2) {
        const unsigned *w = words + k * 3 / 2, middle = w[1];
        place[k] = (uint64_t)(middle & 0xffffu) << 32 | w[0];
        place[k + 1] = (uint64_t)w[2] << 16 | middle >> 16;
    }
    nuts_adamw_tensor t;
    t.n = (int64_t)place[0];
    t.param = global(place[1]);
    t.grad = global(place[2]);
    t.copy = global(place[3]);
    t.m = global(place[4]);
    t.v = global(place[5]);
    t.m_scale = static_cast<float*>(global(place[6]));
    t.v_scale = static_cast<float*>(global(place[7]));
    return t;
}

struct Factors {
    float scale, keep, size, root_scale;
    unsigned t;
};

template <bool kEight>
__device__ __forceinline__ Factors factors_of(const StepArgs<kEight>& a, float factor)
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

template <typename T, int kN>
__device__ __forceinline__ void store_some(T* p, int n, const Pack<T, kN>& out)
{
    if (n == kN) {
#pragma unroll
        for (int e = 0; e < kN; e += 16 / sizeof(T)) {
            Pack<T, 16 / sizeof(T)> part;
            __builtin_memcpy(&part, &out.v[e], 16);
            store_pack(p + e, part);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
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

// philox4x32_10 of nuts_rng.h with the halves of a product from one instruction and exclusive ors of three from another.
__device__ __forceinline__ void random_words(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1, unsigned (&words)[4])
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
#ifdef __HIP_DEVICE_COMPILE__
        c0 = __builtin_amdgcn_bitop3_b32((unsigned)(p1 >> 32), c1, k0, 0x96);
        c2 = __builtin_amdgcn_bitop3_b32((unsigned)(p0 >> 32), c3, k1, 0x96);
#endif
        c1 = (unsigned)p1;
        c3 = (unsigned)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    words[0] = c0, words[1] = c1, words[2] = c2, words[3] = c3;
}

// 1024 times a chance of 10 bits and a half: (2^23 + bits) - (2^23 - 1/2).
__device__ __forceinline__ float chance(unsigned bits) { return __uint_as_float((bits & 1023u) | 0x4b000000u) - 8388607.5f; }

// Codes of 8 bits.  x is what they stand for in units of the scale: 127^2, or 254^2, at a block's largest.  The code below x is the whole part of
// its root, and where that comes out one too high or too low for a last place (or is the last code) the comparison makes up for it: these
// square roots need not be exact.  All else is rounded as single operations are, so that a step has the same codes wherever it is made.
__device__ __forceinline__ float m_value(float code, float scale) { return code * __builtin_fabsf(code) * scale; }
__device__ __forceinline__ float root_value(float code, float scale) { return code * code * scale; }
struct Scale {
    float of, by;  // by = 1 / of, 0 for 0
};
// x / scale, rounded once: a product that is at most a unit in the last place off, and its remainder (Markstein, 1990).
__device__ __forceinline__ float in_units(float x, const Scale& s)
{
    const float q = x * s.by;
    return __builtin_fmaf(__builtin_fmaf(-q, s.of, x), s.by, q);
}
__device__ __forceinline__ Scale scale_of(float top, float last)  // top / last^2
{
    // (a scale with fewer than 24 places is taken as 0)
    const float of = top * (1.f / (last * last));
    if (!(of >= 0x1p-126f)) return Scale{0.f, 0.f};
    const float by = __builtin_amdgcn_rcpf(of);
    return Scale{of, __builtin_fmaf(__builtin_fmaf(-of, by, 1.f), by, by)};
}
__device__ __forceinline__ float m_code(float m, const Scale& scale, unsigned word)
{
    const float x = in_units(__builtin_fabsf(m), scale), c = floorf(__builtin_amdgcn_sqrtf(x));
    const float gap = __builtin_fmaf(c, 2.f / 1024.f, 1.f / 1024.f);  // ((c + 1)^2 - c^2) / 1024
    const bool up = __builtin_fmaf(-c, c, x) > gap * chance(word);
    return __builtin_copysignf(up ? c + 1.f : c, m);
}
// For a code c of v: c^4, and ((c + 1)^4 - c^4) / 1024.  A table in LDS, for the vector units have the most to do here.
constexpr int kSteps = 256;
__device__ __forceinline__ float2 v_step(float c)
{
    const float below = c * c, gap = __builtin_fmaf(2.f, c, 1.f);  // (c + 1)^2 - c^2
    return float2{below * below, gap * __builtin_fmaf(2.f / 1024.f, below, gap * (1.f / 1024.f))};
}
__device__ __forceinline__ unsigned v_code(float root, const Scale& scale, unsigned word, const float2* steps)
{
    const float x = in_units(root, scale);
    const unsigned c = (unsigned)__builtin_amdgcn_sqrtf(x);  // 254 at most: x is 254^2 and a unit in its last place at most
    const float2 step = steps[c];
    const unsigned code = c + (x * x - step.x > step.y * chance(word >> 10));
    return max(code, (unsigned)(x > 0.f));  // (1 at least, where there is anything)
}
// The square root of a number of 24 places, rounded once: from one that is a unit or two in the last place off, and the remainder of its square.
// (Of a v below 2^-100 the remainder has fewer places: a unit off then.)
__device__ __forceinline__ float exact_root(float v)
{
    const float y = __builtin_amdgcn_rsqf(v), s = v * y;
    return __builtin_fmaf(__builtin_fmaf(-s, s, v), 0.5f * y, s);
}

// The root that a step divides by: of moments of 32 bits the instruction's, a unit in the last place off at most; of 8 bits, whose codes follow
// from it, rounded once.
template <bool kExact>
__device__ __forceinline__ float root_of(float v)
{
    const float s = __builtin_amdgcn_sqrtf(v);
    return kExact && __builtin_isnormal(v) ? exact_root(v) : s;
}

// The largest of a wave's numbers that are 0 or more, in all of its lanes.
__device__ __forceinline__ float wave_max(float x)
{
    unsigned v = __float_as_uint(x);  // (which rises as they do)
#ifdef __HIP_DEVICE_COMPILE__
#define NUTS_MAX_STEP(control, rows) v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, control, rows, 0xf, rows == 0xf))
    NUTS_MAX_STEP(0xb1, 0xf);   // quads: neighbours, then pairs
    NUTS_MAX_STEP(0x4e, 0xf);
    NUTS_MAX_STEP(0x141, 0xf);  // rows of 16: mirrored halves, then mirrored
    NUTS_MAX_STEP(0x140, 0xf);
    NUTS_MAX_STEP(0x142, 0xa);  // rows 1 and 3: the last lane of the row before
    NUTS_MAX_STEP(0x143, 0xc);  // the upper half: lane 31
#undef NUTS_MAX_STEP
    v = (unsigned)__builtin_amdgcn_readlane((int)v, 63);
#endif
    return __uint_as_float(v);
}
__device__ __forceinline__ float largest(const float (&x)[4])
{
    return wave_max(fmaxf(fmaxf(__builtin_fabsf(x[0]), __builtin_fabsf(x[1])), fmaxf(__builtin_fabsf(x[2]), __builtin_fabsf(x[3]))));
}
// Whether any lane says so.
__device__ __forceinline__ bool any_lane(bool is)
{
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_ballot_w64(is) != 0;
#else
    return is;
#endif
}

// The codes of four numbers in a word, as many of them as there are.
__device__ __forceinline__ unsigned load_codes(const void* codes, long i, int n)
{
    const uint8_t* at = static_cast<const uint8_t*>(codes) + i;
    if (n >= 4) {
        const Pack<uint8_t, 4> in = load_pack<uint8_t, 4>(at);
        unsigned word;
        __builtin_memcpy(&word, &in, 4);
        return word;
    }
    unsigned word = 0;
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) word |= (unsigned)at[e] << 8 * e;
    return word;
}
__device__ __forceinline__ void store_codes(void* codes, long i, int n, unsigned word)
{
    uint8_t* at = static_cast<uint8_t*>(codes) + i;
    if (n >= 4) {
        Pack<uint8_t, 4> out;
        __builtin_memcpy(&out, &word, 4);
        store_pack(at, out);
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) at[e] = (uint8_t)(word >> 8 * e);
}
__device__ __forceinline__ unsigned zero_bytes(unsigned word) { return (word - 0x01010101u) & ~word & 0x80808080u; }  // 0: there is none

// What four codes stand for: m, and the root of v.  Returns whether a lane has one that counts as NaN.
__device__ __forceinline__ bool decode(unsigned m_word, unsigned v_word, float m_scale, float v_scale, float (&m)[4], float (&root)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m[e] = m_value((float)(int8_t)(m_word >> 8 * e), m_scale);
        root[e] = root_value((float)(uint8_t)(v_word >> 8 * e), v_scale);
    }
    const bool lost = any_lane((zero_bytes(m_word ^ 0x80808080u) | zero_bytes(~v_word)) != 0);
    if (lost) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((m_word >> 8 * e & 255u) == 128u) m[e] = NAN;
            if ((v_word >> 8 * e & 255u) == 255u) root[e] = NAN;
        }
    }
    return lost;
}

// A block's moments, four in each lane, as codes and scales.  lost: some may not be finite.
__device__ __forceinline__ void encode(const nuts_adamw_tensor& t, long block, long i, int n, bool lost, float (&m)[4], float (&root)[4],
                                       const unsigned (&words)[4], const float2* steps)
{
    unsigned m_lost = 0, v_lost = 0;
    if (lost) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!(__builtin_fabsf(m[e]) < INFINITY)) {
                m[e] = 0.f;
                m_lost |= 255u << 8 * e;
            }
            if (!(root[e] < INFINITY)) {
                root[e] = 0.f;
                v_lost |= 255u << 8 * e;
            }
        }
    }
    const Scale m_scale = scale_of(largest(m), 127.f), v_scale = scale_of(largest(root), 254.f);
    unsigned m_word = 0, v_word = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m_word |= ((unsigned)(int)m_code(m[e], m_scale, words[e]) & 255u) << 8 * e;
        v_word |= v_code(root[e], v_scale, words[e], steps) << 8 * e;
    }
    store_codes(t.m, i, n, lost ? (m_word & ~m_lost) | (m_lost & 0x80808080u) : m_word);
    store_codes(t.v, i, n, v_word | v_lost);
    if (threadIdx.x % 64 == 0) {
        t.m_scale[block] = m_scale.of;
        t.v_scale[block] = v_scale.of;
    }
}

// Four numbers of each lane, from i on; kWhole: every lane has four.
template <typename P, typename G, bool kEight, bool kWhole>
__device__ __forceinline__ void step_block(const StepArgs<kEight>& a, const Factors& f, const nuts_adamw_tensor& t, unsigned tensor, long at, long end, const float2* steps)
{
    const long i = at + threadIdx.x % 64 * 4, block = at / 256;
    const int n = kWhole ? 4 : (int)max(min(end - i, 4l), 0l);
    float p[4], g[4], m[4], v[4], root[4];
    bool lost = false;
    load4(static_cast<const P*>(t.param) + i, n, p);
    load4(static_cast<const G*>(t.grad) + i, n, g);
    if (kEight) {
        lost = decode(load_codes(t.m, i, n), load_codes(t.v, i, n), t.m_scale[block], t.v_scale[block], m, root);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = root[e] * root[e];
    } else {
        load4(static_cast<const float*>(t.m) + i, n, m);
        load4(static_cast<const float*>(t.v) + i, n, v);
    }
    unsigned words[4] = {};
    if (kEight || sizeof(P) == 2) random_words((unsigned)((uint64_t)at >> 2) + threadIdx.x % 64, 6u | (unsigned)((uint64_t)at >> 34) << 8, f.t, tensor, a.k0, a.k1, words);
    bool usual = true;  // (not below 2^-126, not infinity, not NaN)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x = g[e] * f.scale;
        m[e] = m[e] * a.beta1 + x * a.rest1;
        v[e] = v[e] * a.beta2 + x * x * a.rest2;
        usual &= __builtin_isnormal(v[e]);
    }
    if (any_lane(!usual)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool low = v[e] < 0x1p-126f;  // (of which the root's instruction makes 0)
            root[e] = root_of<kEight>(low ? v[e] * 0x1p64f : v[e]);
            if (low) root[e] *= 0x1p-32f;
            if (kEight) lost |= !(v[e] < INFINITY);
        }
        if (kEight) lost = any_lane(lost);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) root[e] = kEight ? exact_root(v[e]) : __builtin_amdgcn_sqrtf(v[e]);
    }
    if (a.usual_eps) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            // (a reciprocal a unit in the last place off at most)
            p[e] = __builtin_fmaf(-f.size * m[e], __builtin_amdgcn_rcpf(__builtin_fmaf(root[e], f.root_scale, a.eps)), p[e] * f.keep);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float under = __builtin_fmaf(root[e], f.root_scale, a.eps), move = under < 0x1p-60f ? 0x1p64f : under > 0x1p100f ? 0x1p-64f : 1.f;
            p[e] = __builtin_fmaf(-f.size * (m[e] * move), __builtin_amdgcn_rcpf(under * move), p[e] * f.keep);
        }
    }
    if (sizeof(P) == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = rounded_at_random(p[e], words[e]);
    }
    store4(static_cast<P*>(t.param) + i, n, p);
    if (t.copy) a.copy_dtype == NUTS_BF16 ? store4(static_cast<bf16*>(t.copy) + i, n, p) : store4(static_cast<f16*>(t.copy) + i, n, p);
    if (kEight) {
        encode(t, block, i, n, lost, m, root, words, steps);
    } else {
        store4(static_cast<float*>(t.m) + i, n, m);
        store4(static_cast<float*>(t.v) + i, n, v);
    }
}

// A workgroup `chunk` numbers of a tensor, a wave 256 of them at a time: a block of the moments of 8 bits.  One pass, each number read and written once.
//
// 32 bits: bound by memory.  102 million numbers, all binary32: 548 us, 5.2 TB/s; 120 million with gradients and copies of 16 bits in 150 tensors, two
// launches, 632 us, 5.3 TB/s.
// 8 bits: 200 million binary32 parameters with gradients and copies of 16 bits 657 us, 4.9 TB/s.  Instructions are as near: some 92 a number, of which
// the ten rounds of Philox are 10 and the two codes 36 (42 without the table of the codes' steps); 67 million bfloat16 parameters and gradients, 10 bytes a
// number, 177 us, 3.8 TB/s, are bound by them (183 without the table).  With library roots and quotients, lanes checked one by one and
// codes by bytes 200 million took 1290 us.
template <typename P, typename G, bool kEight>
__global__ __launch_bounds__(kThreads) void adamw_kernel(StepArgs<kEight> a)
{
    __shared__ float2 steps[kEight ? kSteps : 1];
    if (kEight) {
        static_assert(kThreads == kSteps, "a thread a step");
        steps[threadIdx.x] = v_step((float)threadIdx.x);
        __syncthreads();
    }
    const float factor = a.factor ? *a.factor : 1.f;
    if (factor != factor) return;
    const Factors f = factors_of(a, factor);
    const int k = tensor_of(a.first, (int)blockIdx.x);
    const nuts_adamw_tensor t = unpack_tensor<kEight>(a.tensor[k]);
    const long begin = (a.first_block + (long)((int)blockIdx.x - a.first[k])) * a.chunk, end = min(begin + a.chunk, (long)t.n);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    long at = begin + wave * 256;
    for (; at + 256 <= end; at += kThreads * 4) step_block<P, G, kEight, true>(a, f, t, a.first_tensor + k, at, end, steps);
    if (at < end) step_block<P, G, kEight, false>(a, f, t, a.first_tensor + k, at, end, steps);
}

// Eight numbers a thread.  Bound by memory: 200 million to bfloat16 234 us, 5.1 TB/s (285 with four numbers a thread).
template <typename T>
__global__ __launch_bounds__(kThreads) void values_kernel(StepArgs<true> a)
{
    constexpr int kEach = 8;
    const int k = tensor_of(a.first, (int)blockIdx.x);
    const nuts_adamw_tensor t = unpack_tensor<true>(a.tensor[k]);
    const long begin = (a.first_block + (long)((int)blockIdx.x - a.first[k])) * a.chunk, end = min(begin + a.chunk, (long)t.n);
    for (long at = begin; at < end; at += kThreads * kEach) {  // (whole waves)
        const long i = at + (long)threadIdx.x * kEach;
        const int n = (int)max(min(end - i, (long)kEach), 0l);
        unsigned m_word[2] = {}, v_word[2] = {};
        if (n == kEach) {
            const Pack<uint8_t, kEach> m_in = load_pack<uint8_t, kEach>(static_cast<const uint8_t*>(t.m) + i), v_in = load_pack<uint8_t, kEach>(static_cast<const uint8_t*>(t.v) + i);
            __builtin_memcpy(m_word, &m_in, kEach);
            __builtin_memcpy(v_word, &v_in, kEach);
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                m_word[q] = load_codes(t.m, i + 4 * q, max(min(n - 4 * q, 4), 0));
                v_word[q] = load_codes(t.v, i + 4 * q, max(min(n - 4 * q, 4), 0));
            }
        }
        const float m_scale = n > 0 ? t.m_scale[i / 256] : 0.f, v_scale = n > 0 ? t.v_scale[i / 256] : 0.f;
        Pack<T, kEach> m_out, v_out;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float m[4], root[4];
            decode(m_word[q], v_word[q], m_scale, v_scale, m, root);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m_out.v[4 * q + e] = rounded<T>(m[e]);
                v_out.v[4 * q + e] = rounded<T>(root[e] * root[e]);
            }
        }
        if (t.param) store_some(static_cast<T*>(t.param) + i, n, m_out);
        if (t.copy) store_some(static_cast<T*>(t.copy) + i, n, v_out);
    }
}

// Calls `go` for as many tensors at a time as a launch takes, and as many workgroups as it takes.
template <bool kEight, typename Wanted, typename Go>
void by_tables(StepArgs<kEight>& a, const nuts_adamw_tensor* tensors, int64_t n, Wanted wanted, Go go)
{
    constexpr int kTensors = StepArgs<kEight>::kTensors;
    int64_t at = 0, total = 0;
    for (int64_t i = 0; i < n; ++i) total += wanted(tensors[i]) ? tensors[i].n : 0;
    a.chunk = (int)std::clamp(ceil_div(ceil_div(total, kStepBlocks), kChunkLeast) * kChunkLeast, kChunkLeast, kChunkMost);
    while (at < n) {
        int64_t blocks = 0;
        int used = 0;
        a.first_tensor = (unsigned)at;
        a.first_block = 0;
        for (; used < kTensors && at < n; ++used, ++at) {
            const int64_t own = wanted(tensors[at]) ? ceil_div(tensors[at].n, a.chunk) : 0;
            if (blocks + own > kMaxBlocks) {
                if (used > 0) break;
                // a tensor of more workgroups than a launch has: alone, in several
                pack_tensor<kEight>(tensors[at], a.tensor[0]);
                for (int k = 0; k < kTensors; ++k) a.first[k] = k ? INT32_MAX : 0;
                for (int64_t done = 0; done < own; done += kMaxBlocks) {
                    a.first_block = (long)done;
                    go((unsigned)std::min<int64_t>(own - done, kMaxBlocks));
                }
                blocks = 0;
                used = 0;
                ++at;
                break;
            }
            pack_tensor<kEight>(tensors[at], a.tensor[used]);
            a.first[used] = (int)blocks;
            blocks += own;
        }
        if (blocks == 0) continue;
        for (int k = used; k < kTensors; ++k) a.first[k] = INT32_MAX;
        go((unsigned)blocks);
    }
}

// grads, scales: whether the call has to do with them.
int check_tensors(const nuts_adamw_tensor* tensors, int64_t n, bool grads, bool scales, const char* who)
{
    if (n < 0 || n > (1 << 20)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_tensors must be in [0, 2^20]", who);
    if (n > 0 && !tensors) return api_fail(NUTS_E_INVALID_ARG, "%s: tensors must not be NULL", who);
    for (int64_t i = 0; i < n; ++i) {
        const nuts_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > kLongest) return api_fail(NUTS_E_INVALID_ARG, "%s: n of tensor %lld must be in [0, 2^40]", who, (long long)i);
        // (a launch has 48 bits of an address, which all of the device's have)
        uint64_t any = (uintptr_t)t.param | (uintptr_t)t.copy | (uintptr_t)t.m | (uintptr_t)t.v;
        if (grads) any |= (uintptr_t)t.grad;
        if (scales) any |= (uintptr_t)t.m_scale | (uintptr_t)t.v_scale;
        if (any >> 48) return api_fail(NUTS_E_INVALID_ARG, "%s: tensor %lld has an address that is none of the device's", who, (long long)i);
    }
    return NUTS_OK;
}

// The workgroups' step for all tensors.
template <bool kEight>
void step_all(const nuts_adamw_desc* d, const nuts_adamw_tensor* tensors, int64_t n_tensors, const int64_t* step, const float* lr, const float* factor)
{
    StepArgs<kEight> a{};
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
    a.usual_eps = a.eps >= 0x1p-100f && a.eps <= 0x1p100f;
    a.scale = (float)d->scale;
    a.keep = (float)(1.0 - d->lr * d->weight_decay);
    a.size = (float)(d->lr / -std::expm1((double)d->step * a.log_beta1));
    a.root_scale = (float)(1.0 / std::sqrt(-std::expm1((double)d->step * a.log_beta2)));
    a.t = (unsigned)d->step;
    a.host_step = d->step;
    a.k0 = (unsigned)d->seed;
    a.k1 = (unsigned)(d->seed >> 32);
    a.copy_dtype = d->copy_dtype;
    void (*kernel)(StepArgs<kEight>) = nullptr;
    by_dtype(d->grad_dtype, [&](auto g) {
        using G = decltype(g);
        kernel = d->param_dtype == NUTS_F32 ? adamw_kernel<float, G, kEight> : adamw_kernel<bf16, G, kEight>;
    });
    by_tables(a, tensors, n_tensors, [](const nuts_adamw_tensor& t) { return t.grad != nullptr; },
              [&](unsigned blocks) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, api_stream(), a); });
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
    // A table from tensor `at` on, of parts of `each` numbers; returns how many they are.
    int64_t at = 0;
    auto next_table = [&](int64_t each) {
        int64_t parts = 0;
        int used = 0;
        for (; used < kNormTensors && at < n_tensors; ++used, ++at) {
            a.data[used] = tensors[at].data;
            a.n[used] = (long)tensors[at].n;
            a.dtype[used] = (unsigned char)tensors[at].dtype;
            a.first[used] = (int)parts;
            parts += ceil_div(tensors[at].n, each);
        }
        for (; used < kNormTensors; ++used) a.first[used] = INT32_MAX;
        return parts;
    };
    if (norm_is_small(tensors, n_tensors)) {
        const int parts = (int)next_table(kNormPart);
        hipLaunchKernelGGL(small_norm_kernel, dim3(1), dim3(kNormThreads), 0, api_stream(), a, parts, max_norm, norm, factor);
        NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
        return NUTS_OK;
    }
    a.each = (long)norm_each(tensors, n_tensors);
    double* part = static_cast<double*>(workspace);
    while (at < n_tensors) {
        const int64_t own = next_table(a.each);
        a.part = part;
        if (own > 0) hipLaunchKernelGGL(norm_kernel, dim3((unsigned)own), dim3(kThreads), 0, api_stream(), a);
        part += own;
    }
    hipLaunchKernelGGL(join_norm_kernel, dim3(1), dim3(kNormThreads), 0, api_stream(), static_cast<const double*>(workspace), (long)blocks, max_norm, norm, factor);
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
    if (int rc = check_tensors(tensors, n_tensors, true, d->state_bits == 8, "nuts_adamw")) return rc;
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
    d->state_bits == 8 ? step_all<true>(d, tensors, n_tensors, step, lr, factor) : step_all<false>(d, tensors, n_tensors, step, lr, factor);
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int nuts_adamw_values(const nuts_adamw_tensor* tensors, int64_t n_tensors, int32_t dtype)
{
    if (!cat_dtype_known(dtype)) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw_values: dtype must be NUTS_F32, NUTS_BF16 or NUTS_F16");
    if (int rc = check_tensors(tensors, n_tensors, false, true, "nuts_adamw_values")) return rc;
    int64_t total = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const nuts_adamw_tensor& t = tensors[i];
        if (t.n == 0 || (!t.param && !t.copy)) continue;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale) return api_fail(NUTS_E_INVALID_ARG, "nuts_adamw_values: null pointer in tensor %lld", (long long)i);
        total += t.n;
    }
    if (total == 0) return NUTS_OK;
    if (int rc = api_have_device()) return rc;
    StepArgs<true> a{};
    by_dtype(dtype, [&](auto t) {
        by_tables(a, tensors, n_tensors, [](const nuts_adamw_tensor& x) { return x.param || x.copy; },
                  [&](unsigned blocks) { hipLaunchKernelGGL(values_kernel<decltype(t)>, dim3(blocks), dim3(kThreads), 0, api_stream(), a); });
    });
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

}  // extern "C"
