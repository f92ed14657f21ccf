// C = A B' on the matrix instructions: binary32 or bfloat16, sums binary32.  A is m x k, B is n x k.
//
// A workgroup makes a tile of kM x kN; its waves divide it.  Per step along the contraction the workgroup takes 128 bytes for each row
// of its tile of A and of B from memory straight into LDS (no registers in between), kAhead (two) steps ahead.  Either
// matrix may lie in memory along its rows ("along": a row's elements, which are the contraction's, are neighbours) or across them
// (its transpose lies along: the elements that belong to one place of the contraction are neighbours); the tile in LDS lies as
// the memory does.
//
// Along: a row's eight 16-byte pieces lie in LDS in the order piece ^ (row % 8), so that the 16 rows that a matrix
// instruction reads at one place of the contraction are in different banks.  Across: a place's 16-byte pieces are exchanged
// likewise, 32 bytes (16 bfloat16 rows) at a time by bits 0, 1 and 3 of the place, or 64 bytes (16 binary32 rows) by bits 2 and 3;
// binary32 rows are read element by element, bfloat16 by the loads that transpose 4 x 16 elements.
//
// What lies outside the matrices is read as zero by the bounds of the buffer descriptors: rows behind the last by their
// offset, and pieces behind the contraction's end by an offset that no buffer has.  Rows have to begin at multiples of 4
// bytes (others are copied first).  A piece at the ragged end of a row holds the beginning of the next one too.  Across, that makes
// sums that are not stored; along, it is cleared in LDS before it is read (kRagged; or, dZ, it is zero beside lines that are: behind the
// contraction's end 0 times infinity would count).
//
// The first operand of an instruction is B: a lane then holds four neighbouring columns of one row of C, which are stored
// together, and most of a reduction along a row of C stays within lanes.
#pragma once
#include "nuts_softmax.h"

#include <type_traits>

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
    long a_stride, b_stride;  // bytes from row to row (across: from place to place of the contraction)
    int m, n, k;
    int tiles_m, tiles_n;
    int splits, split_steps;  // the contraction is divided: steps of a division
    // kSums: binary32 [split][m][n], added to what is there if `add`
    float* sums;
    int add;
    // kOutput, and kScores' logits (or NULL)
    void* c;
    long c_stride;  // elements
    int streamed;   // what is stored goes past the caches
    // kScores
    float scale;
    const void* targets;  // (and with `residual`)
    int id_type;
    // Of bfloat16 products with dZ, what its targets' entries lost when they were rounded, or NULL; of classes from `first_class` on
    const float* residual;  // [row]
    int first_class, n_classes;
    float4* stats;        // [row][tiles_n x waves along n]: m, S, T of z = scale C
    float* target_logit;  // [row]
    const float* lse;     // [row]: tiles without a row far from 0 are left out; or NULL: none is
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

#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass knows neither buffer descriptors nor loads to LDS)

// One operand's tile of kRows rows: its way from memory to LDS, and from there to the matrix instructions.
template <typename T, int kRows, bool kAcross, int kWaves>
struct Operand {
    static constexpr int kSize = sizeof(T), kPlaces = kStepBytes / kSize, kBytes = kRows * kStepBytes;
    static constexpr int kLoads = kBytes / 1024 / kWaves;                        // of a wave, 1024 bytes each
    static constexpr int kPieces = kAcross ? kRows * kSize / 16 : kStepBytes / 16;  // of a line in LDS
    static_assert(kLoads * 1024 * kWaves == kBytes, "");
    typedef __attribute__((ext_vector_type(4))) unsigned Descriptor;
    const char* from;
    long stride;
    int rows, k;       // of this tile; the contraction's length
    int piece;         // along: this lane's in each of its loads
    unsigned at[kLoads];

    __device__ __forceinline__ static int exchange(int place)
    {
        return (kSize == 4 ? (place >> 2 & 3) << 2 : ((place & 3) | (place >> 3 & 1) << 2) << 1) & (kPieces - 1);
    }

    __device__ __forceinline__ void begin(const char* matrix, long matrix_stride, int first_row, int all_rows, int all_k, int wave, int lane)
    {
        stride = matrix_stride;
        rows = min(kRows, all_rows - first_row);
        k = all_k;
        from = matrix + (kAcross ? (long)first_row * kSize : (long)first_row * stride);
        piece = (lane % 8) ^ (lane / 8);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int unit = (j * kWaves + wave) * 64 + lane, line = unit / kPieces;
            if (kAcross) at[j] = (unsigned)(line * stride + ((unit % kPieces) ^ exchange(line)) * 16);
            else at[j] = line < rows ? (unsigned)(line * stride + piece * 16) : kNowhere;
        }
    }

    // What a step's loads have in common.  Every step has the same number of them, also those behind the last (`none`), which read
    // nothing: waits count loads.
    struct Step {
        Descriptor buffer;
        unsigned skip, place, to;
    };
    __device__ __forceinline__ Step at_step(const char* to, int step, bool none, int wave) const
    {
        const int left = k - step * kPlaces;
        // (a buffer reads no part of a word)
        const int line = ((kAcross ? rows : k) * kSize + 3) & ~3;
        const int bytes = (int)((kAcross ? min(left, kPlaces) - 1 : rows - 1) * stride) + line;
        const unsigned long long base = (unsigned long long)(from + (kAcross && !none ? (long)step * kPlaces * stride : 0));
        return Step{Descriptor{(unsigned)base, (unsigned)(base >> 32), none ? 0u : (unsigned)bytes, 0x00027000u},
                    none || (!kAcross && piece * (16 / kSize) >= left) ? kNowhere : 0u, kAcross || none ? 0u : (unsigned)(step * kStepBytes),
                    (unsigned)(uintptr_t)(__attribute__((address_space(3))) const char*)to + wave * 1024u};
    }
    // Load j of a step.  (In assembly: of its own loads to LDS the compiler knows that they write there, and has some reads of other
    // places of LDS wait for them.  It has no result; who needs what it writes waits for it in wait_and_meet.)
    __device__ __forceinline__ void fetch(const Step& s, int j) const
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(s.to + j * (kWaves * 1024u)), "v"(at[j] | s.skip), "s"(s.buffer),
                     "s"(s.place)
                     : "m0");
    }

    // Along, a tile of the step in which the contraction ends inside a piece: the rest of that piece.
    __device__ __forceinline__ void clear_tail(char* tile, int step) const
    {
        static_assert(!kAcross, "");
        constexpr int kPer = 16 / kSize;
        const int left = k - step * kPlaces;
        for (int row = threadIdx.x; row < kRows; row += 64 * kWaves)
            for (int e = left % kPer; e < kPer; ++e) reinterpret_cast<T*>(tile + row * kStepBytes + (left / kPer ^ row % 8) * 16)[e] = static_cast<T>(0.f);
    }

    // Where a lane reads: its place in a tile, and what its row is exchanged by.
    struct Reader {
        unsigned at, swap;
    };
    __device__ __forceinline__ static Reader reader(int lane)
    {
        if constexpr (!kAcross) return Reader{(unsigned)(lane % 16 * kStepBytes), (unsigned)(lane % 8 * 16)};
        const int place = kSize == 4 ? lane / 16 * 4 : lane / 16 * 8 + lane % 16 / 4;
        return Reader{(unsigned)(place * kPieces * 16 + (kSize == 4 ? lane % 16 * 4 : lane % 4 * 8)), (unsigned)(exchange(place) * 16)};
    }
    // 16 rows from `row` on, half a step: lane l has row l % 16 and the places of its quarter l / 16.
    __device__ __forceinline__ static Piece<T> read(const char* tile, int row, int half, int lane, const Reader& r)
    {
        Piece<T> p;
        if constexpr (!kAcross) {
            p = *reinterpret_cast<const Piece<T>*>(tile + r.at + row * kStepBytes + ((half * 64 + lane / 16 * 16) ^ r.swap));
        } else if constexpr (kSize == 4) {
            const char* line = tile + r.at + half * 16 * kPieces * 16 + ((row * 4) ^ r.swap);
#pragma unroll
            for (int e = 0; e < 4; ++e) p.v[e] = *reinterpret_cast<const float*>(line + e * kPieces * 16);
        } else {
            typedef __attribute__((ext_vector_type(4))) short Four;
            const char* line = tile + r.at + half * 32 * kPieces * 16 + ((row * 2) ^ r.swap);
            struct {
                Four four[2];
            } both;
#pragma unroll
            for (int t = 0; t < 2; ++t)
                both.four[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)(line + t * 4 * kPieces * 16));
            p.v = __builtin_bit_cast(bf16x8, both);
        }
        return p;
    }
};

#endif

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

// kAhead steps are under way to LDS while one is multiplied; B has a buffer more than A, so that its loads are spread over the
// first half of a step and those of A over the second, behind the barrier at which all are done with the step before.
//
// Bound by the matrix instructions and, between them, by the rate at which the chip lets them run (kept busy with random
// numbers and nothing else they reach 2.0 PFLOP/s in bfloat16): 8192 x 32000 x 4096 in 1.56 ms with the statistics, 1.38 PFLOP/s, the
// instructions busy 75 % of the time; 4096 x 32001 x 2048 with z stored 482 us, 1.12 PFLOP/s, dX 422 us, dW 474 us (1.27 and
// 1.13).  binary32: 2048 x 16384 x 512 in 262 us, 131 TFLOP/s.  One row of x: the reads of the weights, 41 us for 262 MB.
template <typename T, int kM, int kN, int kWavesM, int kWavesN, int kAhead, bool kAcrossA, bool kAcrossB, bool kRagged, ProductKind kKind>
__global__ __launch_bounds__(64 * kWavesM * kWavesN) void product_kernel(ProductArgs p)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int kWaves = kWavesM * kWavesN;
    constexpr int kFM = kM / kWavesM / 16, kFN = kN / kWavesN / 16;
    using A = Operand<T, kM, kAcrossA, kWaves>;
    using B = Operand<T, kN, kAcrossB, kWaves>;
    constexpr int kColumns = kFN * 16, kOutSize = kKind == kOutput ? sizeof(T) : 4, kPitch = kColumns * kOutSize + 16;
    constexpr int kStages = kAhead * A::kBytes + (kAhead + 1) * B::kBytes, kStores = 16 * kPitch * kWaves;
    __shared__ __attribute__((aligned(1024))) char lds[kStages > kStores ? kStages : kStores];
    auto tile_a = [&](int s) { return lds + (s % kAhead) * A::kBytes; };
    auto tile_b = [&](int s) { return lds + kAhead * A::kBytes + (s % (kAhead + 1)) * B::kBytes; };
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const int wave_m = wave / kWavesN, wave_n = wave % kWavesN;
    int tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, tm, tn);
    const int m0 = tm * kM, n0 = tn * kN;
    if constexpr (kKind == kScores) {
        if (p.lse) {
            bool far = false;
            for (int r = lane; r < kM; r += 64) far |= m0 + r < p.m && far_from_0<T>(p.lse[m0 + r]);
            if (!__ballot(far)) return;  // (each wave has looked at all rows)
        }
    }
    const int all_steps = (p.k + A::kPlaces - 1) / A::kPlaces;
    const int first = blockIdx.y * p.split_steps, steps = min(p.split_steps, all_steps - first);
    A from_a;
    B from_b;
    from_a.begin(p.a, p.a_stride, m0, p.m, p.k, wave, lane);
    from_b.begin(p.b, p.b_stride, n0, p.n, p.k, wave, lane);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
        const typename B::Step step_b = from_b.at_step(tile_b(s), first + s, s >= steps, wave);
#pragma unroll
        for (int l = 0; l < B::kLoads; ++l) from_b.fetch(step_b, l);
        const typename A::Step step_a = from_a.at_step(tile_a(s), first + s, s >= steps, wave);
#pragma unroll
        for (int l = 0; l < A::kLoads; ++l) from_a.fetch(step_a, l);
    }
    f32x4 c[kFM][kFN];
#pragma unroll
    for (int i = 0; i < kFM; ++i)
#pragma unroll
        for (int j = 0; j < kFN; ++j) c[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    wait_and_meet<(kAhead - 1) * (A::kLoads + B::kLoads)>();
    const int ragged = first + steps == all_steps ? steps - 1 : -1;  // the step in which the contraction ends
    auto clear_tails = [&](int s) {
        if constexpr (kRagged) {
            if (s != ragged) return;
            from_a.clear_tail(tile_a(s), first + s);
            from_b.clear_tail(tile_b(s), first + s);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    };
    clear_tails(0);
    // A half step in kFN turns: a column of the products of this half, behind which the column's piece of the next half takes
    // the place of this one's, and with each a part of the rows' pieces of the next half and of the loads.
    typename A::Reader read_a = A::reader(lane);
    typename B::Reader read_b = B::reader(lane);
    Piece<T> a[2][kFM], b[kFN];
#pragma unroll
    for (int i = 0; i < kFM; ++i) a[0][i] = A::read(tile_a(0), (wave_m * kFM + i) * 16, 0, lane, read_a);
#pragma unroll
    for (int j = 0; j < kFN; ++j) b[j] = B::read(tile_b(0), (wave_n * kFN + j) * 16, 0, lane, read_b);
    auto half_step = [&](int half, int next, auto load, int loads) {
        const char* next_a = tile_a(next);
        const char* next_b = tile_b(next);
        // (across, addresses are made from these here, each where it is used: kept for all pieces they would take the registers of the sums)
        if constexpr (kAcrossA) asm volatile("" : "+v"(read_a.at), "+v"(read_a.swap));
        if constexpr (kAcrossB) asm volatile("" : "+v"(read_b.at), "+v"(read_b.swap));
#pragma unroll
        for (int j = 0; j < kFN; ++j) {
#pragma unroll
            for (int i = j * kFM / kFN; i < (j + 1) * kFM / kFN; ++i) a[1 - half][i] = A::read(next_a, (wave_m * kFM + i) * 16, 1 - half, lane, read_a);
#pragma unroll
            for (int l = j * loads / kFN; l < (j + 1) * loads / kFN; ++l) load(l);
#pragma unroll
            for (int i = 0; i < kFM; ++i) c[i][j] = Piece<T>::multiply_add(b[j], a[half][i], c[i][j]);
            b[j] = B::read(next_b, (wave_n * kFN + j) * 16, 1 - half, lane, read_b);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int s = 0; s < steps; ++s) {
        const typename B::Step step_b = from_b.at_step(tile_b(s + kAhead), first + s + kAhead, s + kAhead >= steps, wave);
        half_step(0, s, [&](int l) { from_b.fetch(step_b, l); }, B::kLoads);
        wait_and_meet<(kAhead - 1) * B::kLoads + (kAhead - 2) * A::kLoads>();
        clear_tails(s + 1);
        const typename A::Step step_a = from_a.at_step(tile_a(s + kAhead), first + s + kAhead, s + kAhead >= steps, wave);
        half_step(1, s + 1, [&](int l) { from_a.fetch(step_a, l); }, A::kLoads);
    }
    wait_and_meet<0>();  // (loads of nothing may still be under way to LDS, and other waves may still read there)

    const int own_row = lane % 16, own_col = lane / 16 * 4;
    // The entry of a row's target is most of dZ, and its rounding to 8 bits would be most of the error: what it lost is made up for.
    if constexpr (sizeof(T) == 2 && kAcrossB && !kAcrossA) {
        // dX: the lost part times the target's weights, in binary32
        if (p.residual && blockIdx.y == 0) {
#pragma unroll
            for (int i = 0; i < kFM; ++i) {
                const int row = m0 + (wave_m * kFM + i) * 16 + own_row;
                const int target = row < p.m ? class_at(p.targets, p.id_type, row, p.n_classes) - p.first_class : -1;
                if (target < 0 || target >= p.k) continue;
                const float lost = p.residual[row];
                const T* weights = reinterpret_cast<const T*>(p.b + (long)target * p.b_stride);
#pragma unroll
                for (int j = 0; j < kFN; ++j) {
                    const int col = n0 + (wave_n * kFN + j) * 16 + own_col;
                    if (col + 4 <= p.n) {
                        const Pack<T, 4> w = load_pack<T, 4>(weights + col);
#pragma unroll
                        for (int e = 0; e < 4; ++e) c[i][j][e] = __builtin_fmaf(lost, to_float(w.v[e]), c[i][j][e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (col + e < p.n) c[i][j][e] = __builtin_fmaf(lost, to_float(weights[col + e]), c[i][j][e]);
                    }
                }
            }
        }
    }
    if constexpr (sizeof(T) == 2 && kAcrossB && kAcrossA) {
        // dW: the places of this contraction whose targets are rows of this tile, as further steps: 64 of them at a time, A with the lost
        // parts in their targets' rows and nothing else, B with the places' features.
        if (p.residual) {
            constexpr int kThreads = 64 * kWaves, kEach = 8;
            int* list = reinterpret_cast<int*>(tile_b(1));             // place in the chunk << 8 | row
            int(*found)[kWaves] = reinterpret_cast<int(*)[kWaves]>(tile_b(2));
            static_assert(kThreads * kEach * 4 <= B::kBytes && kM <= 256 && kAhead == 2, "");
            const int last = min(p.k, (first + steps) * A::kPlaces);
            for (int chunk = first * A::kPlaces; chunk < last; chunk += kThreads * kEach) {
                int row[kEach];
                unsigned long long hits[kEach];
#pragma unroll
                for (int u = 0; u < kEach; ++u) {
                    const int place = chunk + u * kThreads + (int)threadIdx.x;
                    row[u] = place < last ? class_at(p.targets, p.id_type, place, p.n_classes) - p.first_class - m0 : -1;
                }
#pragma unroll
                for (int u = 0; u < kEach; ++u) {
                    hits[u] = __ballot(row[u] >= 0 && row[u] < from_a.rows);
                    if (lane == 0) found[u][wave] = __popcll(hits[u]);
                }
                __syncthreads();
                int count = 0;
                for (int u = 0; u < kEach; ++u)
                    for (int w = 0; w < kWaves; ++w) {
                        if (w == wave && (hits[u] >> lane & 1)) list[count + __popcll(hits[u] & ((1ull << lane) - 1))] = (u * kThreads + (int)threadIdx.x) << 8 | row[u];
                        count += found[u][w];
                    }
                __syncthreads();
                for (int g = 0; g < count; g += A::kPlaces) {
                    for (int at = threadIdx.x * 16; at < A::kBytes; at += kThreads * 16) *reinterpret_cast<uint4*>(tile_a(0) + at) = uint4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < B::kLoads; ++j) {
                        const int unit = (j * kWaves + wave) * 64 + lane, line = unit / B::kPieces, piece = unit % B::kPieces ^ B::exchange(line);
                        Pack<T, 8> x{};
                        if (g + line < count) {
                            const T* features = reinterpret_cast<const T*>(from_b.from + (long)(chunk + (list[g + line] >> 8)) * p.b_stride) + piece * 8;
                            if (piece * 8 + 8 <= from_b.rows) {
                                x = load_pack<T, 8>(features);
                            } else {
#pragma unroll
                                for (int e = 0; e < 7; ++e)
                                    if (piece * 8 + e < from_b.rows) x.v[e] = features[e];
                            }
                        }
                        *reinterpret_cast<Pack<T, 8>*>(__builtin_assume_aligned(tile_b(0) + unit * 16, 16)) = x;
                    }
                    __syncthreads();
                    if ((int)threadIdx.x < A::kPlaces && g + (int)threadIdx.x < count) {
                        const int line = threadIdx.x, entry = list[g + line], r = entry & 255;
                        *reinterpret_cast<T*>(tile_a(0) + line * A::kPieces * 16 + ((r / 8) ^ A::exchange(line)) * 16 + r % 8 * 2) = rounded<T>(p.residual[chunk + (entry >> 8)]);
                    }
                    __syncthreads();
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int i = 0; i < kFM; ++i) a[0][i] = A::read(tile_a(0), (wave_m * kFM + i) * 16, half, lane, read_a);
#pragma unroll
                        for (int j = 0; j < kFN; ++j) {
                            const Piece<T> x = B::read(tile_b(0), (wave_n * kFN + j) * 16, half, lane, read_b);
#pragma unroll
                            for (int i = 0; i < kFM; ++i) c[i][j] = Piece<T>::multiply_add(x, a[0][i], c[i][j]);
                        }
                    }
                    __syncthreads();
                }
            }
        }
    }

    // A wave stores 16 rows of its part of the tile at a time.  A lane has four neighbouring columns of one of them, which would
    // make stores of 32 or 64 bytes a row: the rows go through LDS and are stored whole.
    const int row0 = m0 + wave_m * kFM * 16, col0 = n0 + wave_n * kColumns;
    auto store_rows = [&](auto* to, long stride, int rows, const f32x4 (&values)[kFN], bool add) {
        using Out = std::remove_pointer_t<decltype(to)>;
        constexpr int kPack = 16 / sizeof(Out), kLanes = kColumns / kPack;  // kLanes: of a row
        static_assert(sizeof(Out) == kOutSize && kLanes >= 4 && kLanes <= 64, "");
        char* own = lds + wave * (16 * kPitch);
#pragma unroll
        for (int j = 0; j < kFN; ++j) {
            Pack<Out, 4> four;
#pragma unroll
            for (int e = 0; e < 4; ++e) four.v[e] = rounded<Out>(values[j][e]);
            *reinterpret_cast<Pack<Out, 4>*>(__builtin_assume_aligned(own + own_row * kPitch + (j * 16 + own_col) * sizeof(Out), 4 * sizeof(Out))) = four;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int col = lane % kLanes * kPack, left = p.n - col0 - col;
#pragma unroll
        for (int r = lane / kLanes; r < 16; r += 64 / kLanes) {
            if (r >= rows || left <= 0) continue;
            Pack<Out, kPack> pack = *reinterpret_cast<const Pack<Out, kPack>*>(__builtin_assume_aligned(own + r * kPitch + col * sizeof(Out), 16));
            Out* at = to + r * stride + col;
            if (left >= kPack) {
                if (add) {
                    const Pack<Out, kPack> old = load_pack<Out, kPack>(at);
#pragma unroll
                    for (int e = 0; e < kPack; ++e) pack.v[e] = rounded<Out>(to_float(pack.v[e]) + to_float(old.v[e]));
                }
                p.streamed ? stream_pack(at, pack) : store_pack(at, pack);
            } else {
#pragma unroll
                for (int e = 0; e < kPack; ++e)
                    if (e < left) at[e] = add ? rounded<Out>(to_float(pack.v[e]) + to_float(at[e])) : pack.v[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
#pragma unroll
    for (int i = 0; i < kFM; ++i) {
        const int row = row0 + i * 16, rows = p.m - row;
        if constexpr (kKind == kSums) store_rows(p.sums + ((long)blockIdx.y * p.m + row) * p.n + col0, p.n, rows, c[i], p.add != 0);
        if constexpr (kKind == kOutput) store_rows(static_cast<T*>(p.c) + row * p.c_stride + col0, p.c_stride, rows, c[i], false);
        if constexpr (kKind == kScores) {
            const int own = row + own_row, col = col0 + own_col;
            const bool whole = n0 + kN <= p.n;
#pragma unroll
            for (int j = 0; j < kFN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[i][j][e] = whole || col + j * 16 + e < p.n ? c[i][j][e] * p.scale : -INFINITY;
            if (p.stats) {
                float z[kFN * 4];
#pragma unroll
                for (int j = 0; j < kFN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[j * 4 + e] = c[i][j][e];
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
                if (lane < 16 && own < p.m) p.stats[(long)own * (p.tiles_n * kWavesN) + tn * kWavesN + wave_n] = float4{v.m, v.s, v.t, 0.f};
                const int target = p.targets && own < p.m ? class_at(p.targets, p.id_type, own, p.n) : -1;
                const int away = target - col;
                const bool here = target >= 0 && away >= 0 && away < kColumns && away % 16 < 4;
                if (__ballot(here)) {
#pragma unroll
                    for (int e = 0; e < kFN * 4; ++e)
                        if (here && away == e / 4 * 16 + e % 4) p.target_logit[own] = z[e];
                }
            }
            if (p.c) store_rows(static_cast<float*>(p.c) + row * p.c_stride + col0, p.c_stride, rows, c[i], false);
        }
    }
#endif
}

}  // namespace nuts
