// C = A B' on the matrix instructions: rows of A and rows of B lie along the contraction, binary32 or bfloat16, sums binary32.
//
// A workgroup makes a tile of kM x kN; its waves divide it.  Per step the workgroup takes 128 bytes of each of its rows of A
// and B from memory straight into LDS (no registers in between), kStages - 1 steps ahead.  A row's eight 16-byte pieces lie
// in LDS in the order piece ^ (row % 8), so that the 16 rows that a matrix instruction reads at one place of the
// contraction are in different banks.  What lies outside the matrices is read as zero by the bounds of the buffer
// descriptors: rows behind the last by their offset, and pieces behind the contraction's end by an offset that no
// buffer has.  (Rows have to begin at multiples of 16 bytes and to consist of whole pieces: others are copied first.)
//
// The first operand of an instruction is B: a lane then holds four neighbouring columns of one row of C, which are stored
// together, and most of a reduction along a row of C stays within lanes.
#pragma once
#include "nuts_softmax.h"

namespace nuts {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kStepBytes = 128;                   // of a row
constexpr unsigned kNowhere = 0x80000000u;        // an offset beyond every buffer
constexpr int64_t kMostBufferBytes = 0x7fffffff;  // of the kM (kN) rows of a tile

enum ProductKind { kScores, kSums, kOutput };

struct ProductArgs {
    const char* a;
    const char* b;
    long a_stride, b_stride;  // bytes
    int m, n, k_bytes;
    int tiles_m, tiles_n;
    int splits, split_steps;  // the contraction is divided: steps of a division
    // kSums: binary32 [split][m][n], added to what is there if `add`
    float* sums;
    int add;
    // kOutput, and kScores' logits (or NULL)
    void* c;
    long c_stride;  // elements
    // kScores
    float scale;
    const void* targets;
    int id_type;
    float4* stats;        // [row][tiles_n x waves along n]: m, S, T of z = scale C
    float* target_logit;  // [row]
};

__device__ __forceinline__ f32x4 multiply(const float (&b)[4], const float (&a)[4], f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[e], a[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4 multiply(const bf16x8& b, const bf16x8& a, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
}

template <typename T>
struct Piece;  // 16 bytes along the contraction
template <>
struct Piece<float> {
    float v[4];
    __device__ __forceinline__ static f32x4 multiply_add(const Piece& b, const Piece& a, f32x4 c) { return multiply(b.v, a.v, c); }
};
template <>
struct Piece<bf16> {
    bf16x8 v;
    __device__ __forceinline__ static f32x4 multiply_add(const Piece& b, const Piece& a, f32x4 c) { return multiply(b.v, a.v, c); }
};

// The tile of a workgroup: workgroups go to the eight dies in turn, each die gets neighbouring tiles (its own cache keeps
// what they share), four rows of tiles at a time.
__device__ __forceinline__ void tile_of(unsigned id, int tiles_m, int tiles_n, int& tm, int& tn)
{
    const unsigned total = (unsigned)tiles_m * tiles_n, die = id % 8, each = total / 8, more = total % 8;
    const unsigned t = die * each + min(die, more) + id / 8;
    const unsigned band = t / (4u * tiles_n), in_band = t % (4u * tiles_n);
    const unsigned rows = min(4u, tiles_m - band * 4);
    tm = (int)(band * 4 + in_band % rows);
    tn = (int)(in_band / rows);
}

template <int kOutstanding>
__device__ __forceinline__ void wait_and_meet()
{
    // all but the last kOutstanding loads have arrived and nothing is still read that will be overwritten, for the whole workgroup
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kOutstanding) : "memory");
}

template <typename T, int kM, int kN, int kWavesM, int kWavesN, int kStages, ProductKind kKind>
__global__ __launch_bounds__(64 * kWavesM * kWavesN) void product_kernel(ProductArgs p)
{
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass knows neither buffer descriptors nor loads to LDS)
    constexpr int kWaves = kWavesM * kWavesN;
    constexpr int kFM = kM / kWavesM / 16, kFN = kN / kWavesN / 16;
    constexpr int kLoadsA = kM / 8 / kWaves, kLoadsB = kN / 8 / kWaves;  // of a wave: 8 rows each
    constexpr int kStageBytes = (kM + kN) * kStepBytes;
    static_assert(kLoadsA * 8 * kWaves == kM && kLoadsB * 8 * kWaves == kN, "");
    __shared__ __attribute__((aligned(1024))) char stage[kStages][kStageBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    int tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    const int m0 = tm * kM, n0 = tn * kN;
    const int rows_a = min(kM, p.m - m0), rows_b = min(kN, p.n - n0);
    const int all_steps = (p.k_bytes + kStepBytes - 1) / kStepBytes;
    const int first = blockIdx.y * p.split_steps, steps = min(p.split_steps, all_steps - first);
    const __amdgpu_buffer_rsrc_t from_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.a + (long)m0 * p.a_stride), 0, (int)((rows_a - 1) * p.a_stride + p.k_bytes), 0x00027000);
    const __amdgpu_buffer_rsrc_t from_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.b + (long)n0 * p.b_stride), 0, (int)((rows_b - 1) * p.b_stride + p.k_bytes), 0x00027000);
    // this lane's piece of a step, and its place in each of the wave's loads
    const int piece = (lane % 8) ^ (lane / 8);
    unsigned at_a[kLoadsA], at_b[kLoadsB];
#pragma unroll
    for (int j = 0; j < kLoadsA; ++j) {
        const int row = (j * kWaves + wave) * 8 + lane / 8;
        at_a[j] = row < rows_a ? (unsigned)(row * p.a_stride + piece * 16) : kNowhere;
    }
#pragma unroll
    for (int j = 0; j < kLoadsB; ++j) {
        const int row = (j * kWaves + wave) * 8 + lane / 8;
        at_b[j] = row < rows_b ? (unsigned)(row * p.b_stride + piece * 16) : kNowhere;
    }
    // every step has the same number of loads, also those behind the last, which read nothing: waits count loads
    auto fetch = [&](int s) {
        char* to = stage[s % kStages];
        const int step = first + s;
        const unsigned skip = s >= steps || step * kStepBytes + piece * 16 >= p.k_bytes ? kNowhere : 0u;
        const int k = s < steps ? step * kStepBytes : 0;
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_a, (__attribute__((address_space(3))) void*)(to + (j * kWaves + wave) * 1024), 16, at_a[j] | skip, k, 0, 0);
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_b, (__attribute__((address_space(3))) void*)(to + kM * kStepBytes + (j * kWaves + wave) * 1024), 16, at_b[j] | skip, k, 0, 0);
    };
    const int wave_m = wave / kWavesN, wave_n = wave % kWavesN;
    f32x4 c[kFM][kFN];
#pragma unroll
    for (int i = 0; i < kFM; ++i)
#pragma unroll
        for (int j = 0; j < kFN; ++j) c[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(s);
    for (int s = 0; s < steps; ++s) {
        wait_and_meet<(kStages - 2) * (kLoadsA + kLoadsB)>();
        fetch(s + kStages - 1);
        const char* a_rows = stage[s % kStages] + (wave_m * kFM * 16 + lane % 16) * kStepBytes;
        const char* b_rows = stage[s % kStages] + (kM + wave_n * kFN * 16 + lane % 16) * kStepBytes;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int at = ((half * 4 + lane / 16) ^ (lane % 8)) * 16;
            Piece<T> a[kFM], b[kFN];
#pragma unroll
            for (int i = 0; i < kFM; ++i) a[i] = *reinterpret_cast<const Piece<T>*>(a_rows + i * 16 * kStepBytes + at);
#pragma unroll
            for (int j = 0; j < kFN; ++j) b[j] = *reinterpret_cast<const Piece<T>*>(b_rows + j * 16 * kStepBytes + at);
#pragma unroll
            for (int i = 0; i < kFM; ++i)
#pragma unroll
                for (int j = 0; j < kFN; ++j) c[i][j] = Piece<T>::multiply_add(b[j], a[i], c[i][j]);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (loads of nothing may still be under way to LDS)

    const int row0 = m0 + wave_m * kFM * 16 + lane % 16, col0 = n0 + wave_n * kFN * 16 + lane / 16 * 4;
    const bool whole = n0 + kN <= p.n;
    if (kKind == kSums) {
        float* sums = p.sums + (long)blockIdx.y * p.m * p.n;
#pragma unroll
        for (int i = 0; i < kFM; ++i)
#pragma unroll
            for (int j = 0; j < kFN; ++j) {
                const int row = row0 + i * 16, col = col0 + j * 16;
                if (row >= p.m) continue;
                float* to = sums + (long)row * p.n + col;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < p.n) to[e] = p.add ? to[e] + c[i][j][e] : c[i][j][e];
            }
    }
    if (kKind == kOutput) {
        T* out = static_cast<T*>(p.c);
#pragma unroll
        for (int i = 0; i < kFM; ++i)
#pragma unroll
            for (int j = 0; j < kFN; ++j) {
                const int row = row0 + i * 16, col = col0 + j * 16;
                if (row >= p.m) continue;
                Pack<T, 4> values;
#pragma unroll
                for (int e = 0; e < 4; ++e) values.v[e] = rounded<T>(c[i][j][e]);
                if (whole) {
                    store_pack(out + row * p.c_stride + col, values);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < p.n) out[row * p.c_stride + col + e] = values.v[e];
                }
            }
    }
    if (kKind == kScores) {
        const int parts = p.tiles_n * kWavesN;
#pragma unroll
        for (int i = 0; i < kFM; ++i) {
            const int row = row0 + i * 16;
            float z[kFN * 4];
#pragma unroll
            for (int j = 0; j < kFN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) z[j * 4 + e] = whole || col0 + j * 16 + e < p.n ? c[i][j][e] * p.scale : -INFINITY;
            if (p.stats) {
                Stats v{-INFINITY, 0.f, 0.f};
                float m = z[0];
#pragma unroll
                for (int e = 1; e < kFN * 4; ++e) m = fmaxf(m, z[e]);
                m = fmaxf(m, __shfl_xor(m, 16));
                v.m = fmaxf(m, __shfl_xor(m, 32));
                add_logits<kFN * 4>(v, z, kLog2e);
                v.s += __shfl_xor(v.s, 16);
                v.s += __shfl_xor(v.s, 32);
                v.t += __shfl_xor(v.t, 16);
                v.t += __shfl_xor(v.t, 32);
                if (lane < 16 && row < p.m) p.stats[(long)row * parts + tn * kWavesN + wave_n] = float4{v.m, v.s, v.t, 0.f};
                const int target = p.targets && row < p.m ? class_at(p.targets, p.id_type, row, p.n) : -1;
                const int away = target - col0;
                const bool here = target >= 0 && away >= 0 && away < kFN * 16 && away % 16 < 4;
                if (__ballot(here)) {
#pragma unroll
                    for (int j = 0; j < kFN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (here && away == j * 16 + e) p.target_logit[row] = z[j * 4 + e];
                }
            }
            if (p.c && row < p.m) {
                float* out = static_cast<float*>(p.c) + row * p.c_stride;
#pragma unroll
                for (int j = 0; j < kFN; ++j) {
                    const int col = col0 + j * 16;
                    if (whole) {
                        Pack<float, 4> values{{z[j * 4], z[j * 4 + 1], z[j * 4 + 2], z[j * 4 + 3]}};
                        store_pack(out + col, values);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < p.n) out[col + e] = z[j * 4 + e];
                    }
                }
            }
        }
    }
#endif
}

}  // namespace nuts
