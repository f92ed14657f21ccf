// Shared by the categorical operators (lookup, log-probabilities, scores): element types, loads of several elements,
// reductions over a workgroup, and the host side's checks of arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <cstdarg>

#include "../../include/nuts.h"

namespace nuts {

// nuts_api.hip: the message of nuts_last_error() on this thread, and the stream of nuts_set_stream().
int api_fail(int code, const char* fmt, ...);
hipStream_t api_stream();
// NUTS_OK if there is a device to run on.
int api_have_device();

#define NUTS_CAT_TRY(expr, code)                                                                                    \
    do {                                                                                                            \
        hipError_t e_ = (expr);                                                                                     \
        if (e_ != hipSuccess) return ::nuts::api_fail((code), "%s failed: %s", #expr, hipGetErrorString(e_));       \
    } while (0)

inline size_t cat_size(int dtype) { return dtype == NUTS_F32 ? 4 : 2; }
inline bool cat_dtype_known(int dtype) { return dtype == NUTS_F32 || dtype == NUTS_BF16 || dtype == NUTS_F16; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups of one launch: a launch's threads are counted in 32 bits.  Larger grids go in several.
constexpr long kMaxBlocks = 1l << 22;

using bf16 = __bf16;
using f16 = _Float16;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float to_float(f16 v) { return static_cast<float>(v); }

// A binary32 result rounded to the element type.  (The compiler would make a product and its rounding to binary16 one
// instruction, which rounds once where the other types round the product first: the results of all types are binary32's.)
template <typename T>
__device__ __forceinline__ T rounded(float v)
{
    return static_cast<T>(v);
}
template <>
__device__ __forceinline__ f16 rounded<f16>(float v)
{
#ifdef __HIP_DEVICE_COMPILE__
    asm("" : "+v"(v));
#endif
    return static_cast<f16>(v);
}

// kN elements that lie next to each other, 4, 8 or 16 bytes, at any address that suits one element.  (Loads and stores need no more
// than the element's alignment here: rows of an odd number of 16-bit values are read as wide as all others.  They
// are written as those of words: as those of a structure of elements the compiler takes many apart again.)
template <typename T, int kN>
struct Pack {
    T v[kN];
    typedef __attribute__((ext_vector_type(sizeof(T) * kN / 4))) unsigned Value;
    typedef __attribute__((ext_vector_type(sizeof(T) * kN / 4), aligned(sizeof(T)))) unsigned Words;
};
template <typename T, int kN>
__device__ __forceinline__ Pack<T, kN> load_pack(const T* p)
{
    const typename Pack<T, kN>::Value words = *reinterpret_cast<const typename Pack<T, kN>::Words*>(p);
    Pack<T, kN> r;
    __builtin_memcpy(&r, &words, sizeof(r));
    return r;
}
template <typename T, int kN>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, kN>& r)
{
    typename Pack<T, kN>::Value words;
    __builtin_memcpy(&words, &r, sizeof(r));
    *reinterpret_cast<typename Pack<T, kN>::Words*>(p) = words;
}
// The same past the caches, for outputs that would push out of them what is still to be read (kStreamed).
template <typename T, int kN>
__device__ __forceinline__ void stream_pack(T* p, const Pack<T, kN>& r)
{
    typename Pack<T, kN>::Value words;
    __builtin_memcpy(&words, &r, sizeof(r));
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("");  // (where a plain store stands beside this one the compiler would make them one: a plain one)
#endif
    __builtin_nontemporal_store(words, reinterpret_cast<typename Pack<T, kN>::Words*>(p));
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("");
#endif
}

// Outputs of this many bytes and more go past the caches: half the last-level cache (256 MB).
constexpr int64_t kStreamed = (int64_t)1 << 27;

// A class as the kernels hold it: the id, or -1 where it is outside [0, n_classes).
__device__ __forceinline__ int class_at(const void* ids, int id_type, long i, long n_classes)
{
    const long id = id_type == NUTS_I64 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
    return id >= 0 && id < n_classes ? static_cast<int>(id) : -1;
}

// f with a value of the element type.
template <typename F>
void by_dtype(int dtype, F f)
{
    if (dtype == NUTS_F32) f(float{});
    else if (dtype == NUTS_BF16) f(bf16{});
    else f(f16{});
}

}  // namespace nuts
