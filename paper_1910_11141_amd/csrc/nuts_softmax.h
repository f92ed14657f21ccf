// Statistics of rows of logits: one pass, any order of the parts.
//
// The forward pass reads each logit once: every thread keeps the largest logit m that it has seen, the sum S of
// 2^w, w = (x - m) s log2(e), and the sum T of w 2^w; when m grows by d, S and T change to 2^-d S and 2^-d (T - d S).  With them
// lse = s m + ln S and entropy = ln S - ln2 T / S, which loses nothing to cancellation, as lse - sum p z does in rows of large
// logits.  It is the difference x - m that is multiplied: rows of the type's lowest value come out as any constant
// row does.
#pragma once
#include "nuts_cat.h"

namespace nuts {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNothing = -1000.f;  // 2^this is 0

struct Stats {
    float m, s, t;
};

// Two parts' statistics as those of both.  c = s log2(e).
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b, float c)
{
    const float m = fmaxf(a.m, b.m);
    const float wa = a.m == m ? 0.f : (a.m - m) * c, wb = b.m == m ? 0.f : (b.m - m) * c;
    const float fa = __builtin_amdgcn_exp2f(wa), fb = __builtin_amdgcn_exp2f(wb);
    // (a part that counts for nothing may be infinitely far away; a NaN stays one)
    const float ta = fa == 0.f ? 0.f : fa * __builtin_fmaf(wa, a.s, a.t), tb = fb == 0.f ? 0.f : fb * __builtin_fmaf(wb, b.s, b.t);
    return Stats{m, fa * a.s + fb * b.s, ta + tb};
}

template <int kN>
__device__ __forceinline__ void add_logits(Stats& a, const float (&x)[kN], float c)
{
    float m = x[0];
#pragma unroll
    for (int e = 1; e < kN; ++e) m = fmaxf(m, x[e]);
    if (m > a.m) {
        const float w = (a.m - m) * c, f = __builtin_amdgcn_exp2f(w);
        a.t = f == 0.f ? 0.f : f * __builtin_fmaf(w, a.s, a.t);
        a.s = f * a.s;
        a.m = m;
    }
    const float base = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        const float w = (x[e] - base) * c, p = __builtin_amdgcn_exp2f(w);
        a.s += p;
        a.t = __builtin_fmaf(fmaxf(w, kNothing), p, a.t);  // 0 where p is, also for w = -infinity
    }
}

// All threads get the workgroup's.
template <int kWaves>
__device__ __forceinline__ Stats join_block(Stats v, float c, Stats (&shared)[kWaves])
{
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = join(v, Stats{__shfl_xor(v.m, step), __shfl_xor(v.s, step), __shfl_xor(v.t, step)}, c);
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v = join(v, shared[w], c);
    return v;
}

// A row's results.  ln S and the row's largest logit stand for lse where a difference is wanted.
struct Row {
    float m, ln_s, lse, entropy;
    bool empty;  // every z is -infinity
};
__device__ __forceinline__ Row finish(const Stats& v, float scale)
{
    Row r;
    r.m = v.m;
    r.ln_s = logf(v.s);
    r.lse = __builtin_fmaf(v.m, scale, r.ln_s);
    if (v.s == 0.f || (v.s == v.s && v.m * scale == -INFINITY)) r.lse = -INFINITY;
    if (v.m * scale == INFINITY) r.lse = r.ln_s = NAN;
    r.empty = r.lse == -INFINITY;
    r.entropy = r.empty ? 0.f : r.ln_s - kLn2 * (v.t / v.s);
    if (r.ln_s != r.ln_s) r.entropy = NAN;
    return r;
}
__device__ __forceinline__ float logprob_of(const Row& r, float x, float scale)
{
    return r.empty ? -INFINITY : __builtin_fmaf(x - r.m, scale, -r.ln_s);
}

// Half a unit in the last place of lse is an error of p = e^(z - lse), relative to it: up to here 2^-19, or 2^-15 where gradients are rounded
// to 16 bits.  For rows farther from 0 they find maximum and sum themselves.
template <typename T>
constexpr float kFar = sizeof(T) == 4 ? 64.f : 1024.f;
template <typename T>
__device__ __forceinline__ bool far_from_0(float lse)
{
    return __builtin_fabsf(lse) > kFar<T> && lse != -INFINITY;  // (-infinity: an empty row)
}

}  // namespace nuts
