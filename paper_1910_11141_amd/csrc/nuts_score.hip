// Log-probabilities of given classes from features and class weights, and the gradients of both.
//
//   z = s X W',  statistics of its rows as in nuts_softmax.h;   dX = dZ W,  dW = dZ' X,  dZ = s (g_lp ([v = y] - p) + ...)
//
// The work is matrix products (2 n V D operations forward, 4 n V D backward), which run on the matrix instructions
// (nuts_product.h).  Forward, a workgroup reduces its tile of z to each row's maximum, sum and weighted sum in
// registers and only those are stored; backward, dZ is made from binary32 z (kept, or computed again) and stored once, and the two
// products read it and the other operands along or across as they lie.  A large batch goes in pieces that bound the
// workspace: of rows forward, of classes backward.
#include "nuts_product.h"

#include <algorithm>

namespace nuts {
namespace {

constexpr int kThreads = 256;

// ---- small kernels --------------------------------------------------------------------------------------------------

struct PackArgs {
    const void* from[2];
    void* to[2];
    long stride[2], rows[2];
    int columns, to_stride;
};

// Rows at any place copied to rows of `to_stride` elements (whole 16 bytes), zeros behind their end: those of two matrices, one behind the other.
template <typename T>
__global__ __launch_bounds__(kThreads) void pack_rows_kernel(PackArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    const int packs = a.to_stride / kN;
    const long first = a.rows[0] * packs, all = first + a.rows[1] * packs;
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < all; i += (long)gridDim.x * kThreads) {
        const int which = i >= first;
        const long at = which ? i - first : i, row = at / packs;
        const int c = (int)(at % packs) * kN;
        const T* from = static_cast<const T*>(a.from[which]) + row * a.stride[which] + c;
        Pack<T, kN> x;
        if (c + kN <= a.columns) {
            x = load_pack<T, kN>(from);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) x.v[e] = c + e < a.columns ? from[e] : static_cast<T>(0.f);
        }
        store_pack(static_cast<T*>(a.to[which]) + row * a.to_stride + c, x);
    }
}

struct GradArgs {
    const float* z;     // of the classes [first, first + classes)
    const float4* far;  // [row]: statistics of rows far from 0 where z does not lie beside the rest of its row; or NULL
    const void* targets;
    const float* lse;
    const float* entropy;
    const float* grad_logprob;
    const float* grad_lse;
    const float* grad_entropy;
    void* dz;         // [rows][dz_stride], zeros behind the last class
    float* residual;  // [rows]: what the target's entry lost in its rounding, 0 where the piece has no target; or NULL
    long z_stride;
    int dz_stride, parts, first, classes, n_classes, id_type, streamed;
    float scale;
};

constexpr int kGradPacks = 4;  // of a thread

// dZ, rounded to the features' type: a workgroup a part of a row.  Bound by its reads and writes: 4096 x 32001, to bfloat16, 145 us, 789
// MB at 5.5 TB/s.  Of a row far from 0 (kFar) each of its workgroups goes through all of it for its maximum and sum (all rows of 4096 x
// 32001 far: 470 us).  Where z is made anew piece by piece, the tiles of such rows are multiplied once more before that, for their statistics
// (9000 x 40000 x 512 bfloat16 in two pieces: 2.07 ms, 2.52 with all rows far; 2.04 without the launches that ask which are).
template <typename T>
__global__ __launch_bounds__(kThreads) void dz_kernel(GradArgs a)
{
    constexpr int kN = 16 / sizeof(T);
    __shared__ Stats shared[kThreads / 64];
    const long row = blockIdx.x / (unsigned)a.parts;
    const int begin = (int)(blockIdx.x % (unsigned)a.parts) * (kGradPacks * kThreads * kN) + (int)threadIdx.x * kN;
    const float* z = a.z + row * a.z_stride;
    T* to = static_cast<T*>(a.dz) + row * a.dz_stride;
    float x[kGradPacks][kN];
#pragma unroll
    for (int u = 0; u < kGradPacks; ++u) {
        const int v = begin + u * kThreads * kN;
#pragma unroll
        for (int e = 0; e < kN; e += 4) {
            if (v + e + 4 <= a.classes) {
                const Pack<float, 4> four = load_pack<float, 4>(z + v + e);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[u][e + i] = four.v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[u][e + i] = v + e + i < a.classes ? z[v + e + i] : -INFINITY;
            }
        }
    }
    const int target = a.targets ? class_at(a.targets, a.id_type, row, a.n_classes) : -1;
    const int y = target >= a.first && target < a.first + a.classes ? target - a.first : -1;
    const float lse = a.lse[row];
    const bool empty = lse == -INFINITY;
    const float g_lp = a.grad_logprob && target >= 0 && !empty ? a.grad_logprob[row] * a.scale : 0.f;
    const float g_p = (a.grad_lse ? a.grad_lse[row] * a.scale : 0.f) - g_lp, g_h = a.grad_entropy ? -a.grad_entropy[row] * a.scale : 0.f;
    const float h = a.grad_entropy ? a.entropy[row] : 0.f;
    float base = 0.f, ln_s = empty ? INFINITY : lse;  // log p = (z - base) - ln_s
    if (far_from_0<T>(lse)) {
        Stats v{-INFINITY, 0.f, 0.f};
        if (a.far) {
            const float4 s = a.far[row];
            v = Stats{s.x, s.y, s.z};
        } else {
            const float* all = z - a.first;
            for (int i = threadIdx.x * 4; i < a.n_classes; i += kThreads * 4) {  // (four at a time: x is in registers, too)
                float some[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) some[e] = i + e < a.n_classes ? all[i + e] : -INFINITY;
                add_logits<4>(v, some, kLog2e);
            }
            v = join_block(v, kLog2e, shared);
        }
        if (v.m > -INFINITY) {
            base = v.m;
            ln_s = logf(v.s);
        }
    }
    if (a.residual && y < 0 && begin == 0) a.residual[row] = 0.f;
#pragma unroll
    for (int u = 0; u < kGradPacks; ++u) {
        const int v = begin + u * kThreads * kN;
        if (v >= a.dz_stride) break;
        float g[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const float log_p = (x[u][e] - base) - ln_s, p = __builtin_amdgcn_exp2f(log_p * kLog2e);
            g[e] = p == 0.f ? 0.f : p * __builtin_fmaf(g_h, fmaxf(log_p, kNothing) + h, g_p);  // (0 whatever comes in)
        }
        if (y >= v && y < v + kN) {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (v + e == y) {
                    g[e] += g_lp;
                    if (a.residual) {
                        const float lost = g[e] - to_float(rounded<T>(g[e]));
                        a.residual[row] = __builtin_fabsf(lost) < INFINITY ? lost : 0.f;
                    }
                }
        }
        Pack<T, kN> out;
#pragma unroll
        for (int e = 0; e < kN; ++e) out.v[e] = rounded<T>(g[e]);
        a.streamed ? stream_pack(to + v, out) : store_pack(to + v, out);
    }
}

// out[row][column] = scale * sum over the divisions of a contraction, in order, eight of them under way at a time, kN columns a thread.
// Bound by its reads and writes (2 divisions of 4096 x 2048, to bfloat16: 17 us, 84 MB at 5 TB/s; a column a thread 23 us).
template <typename T, int kN>
__global__ __launch_bounds__(kThreads) void add_up_kernel(const float* sums, int splits, long rows, int columns, float scale, T* out, long stride)
{
    constexpr int kFlight = 8;
    const long all = rows * columns;
    for (long i = ((long)blockIdx.x * kThreads + threadIdx.x) * kN; i < all; i += (long)gridDim.x * kThreads * kN) {
        float sum[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) sum[e] = 0.f;
        for (int s = 0; s < splits; s += kFlight) {
            Pack<float, kN> x[kFlight];
#pragma unroll
            for (int u = 0; u < kFlight; ++u)
                if (s + u < splits) x[u] = load_pack<float, kN>(sums + (s + u) * all + i);
#pragma unroll
            for (int u = 0; u < kFlight; ++u)
                if (s + u < splits) {
#pragma unroll
                    for (int e = 0; e < kN; ++e) sum[e] += x[u].v[e];
                }
        }
        T* to = out + i / columns * stride + i % columns;
        if constexpr (kN == 1) {
            *to = rounded<T>(sum[0] * scale);
        } else {
            Pack<T, kN> pack;
#pragma unroll
            for (int e = 0; e < kN; ++e) pack.v[e] = rounded<T>(sum[e] * scale);
            store_pack(to, pack);
        }
    }
}

struct FewArgs {
    const void* dz;         // [rows][dz_stride], rows padded with zeros to whole packs of kFewClasses
    const void* x;
    const void* targets;
    const float* residual;  // as in ProductArgs
    void* out;
    long x_stride, stride;
    int rows, dz_stride, dim, first, classes, n_classes, id_type, lane_bits, streamed;
};

template <typename T>
constexpr int kFewRows = 2 * sizeof(T);  // of x, which a thread's registers hold
constexpr int kFewClasses = 8;  // at a time
constexpr int64_t kFewGroups = 512;  // workgroups (62565 classes of 2262, bfloat16: 76 us, with 1024 90)

// dW of few rows: sums of so few products that it is all writing.  A thread has 16 bytes of columns of the rows of x in its registers and
// goes through the classes, eight at a time; workgroups are few, so that x is read for many classes.  dz and dW of 4 rows, bfloat16,
// 128000 classes of 4096: 205 us, 5.1 TB/s (341 by the product kernel, whose tiles begin and end for one step), 32000 of 1024 21 and 31;
// 8 rows, binary32, 50000 classes of 512: 24 and 39.  With 8 rows in bfloat16, which take twice the registers and additions, it is no faster than
// the product kernel.
template <typename T>
__global__ __launch_bounds__(kThreads) void few_rows_weights_kernel(FewArgs a)
{
    constexpr int kN = 16 / sizeof(T), kRows = kFewRows<T>;
    const int lanes = 1 << a.lane_bits, lane = threadIdx.x & (lanes - 1);
    const int begin = (int)(blockIdx.y * lanes + lane) * kN;
    if (begin >= a.dim) return;
    const int c = max(0, min(begin, a.dim - kN));  // (a ragged row's last columns: 16 bytes that end with the row)
    float x[kRows][kN], lost[kRows];
    int target[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const T* from = static_cast<const T*>(a.x) + i * a.x_stride + c;
        Pack<T, kN> pack{};
        if (i < a.rows) {
            if (a.dim >= kN) {
                pack = load_pack<T, kN>(from);
            } else {
#pragma unroll
                for (int e = 0; e < kN - 1; ++e)
                    if (e < a.dim) pack.v[e] = from[e];
            }
        }
#pragma unroll
        for (int e = 0; e < kN; ++e) x[i][e] = to_float(pack.v[e]);
        target[i] = a.residual && i < a.rows ? class_at(a.targets, a.id_type, i, a.n_classes) - a.first : -1;
        lost[i] = a.residual && i < a.rows ? a.residual[i] : 0.f;
    }
    const long step = (long)gridDim.x * (kThreads >> a.lane_bits) * kFewClasses;
    for (long v = ((long)blockIdx.x * (kThreads >> a.lane_bits) + (threadIdx.x >> a.lane_bits)) * kFewClasses; v < a.classes; v += step) {
        float dz[kRows][kFewClasses];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            Pack<T, kFewClasses> pack{};
            if (i < a.rows) pack = load_pack<T, kFewClasses>(static_cast<const T*>(a.dz) + (long)i * a.dz_stride + v);
#pragma unroll
            for (int r = 0; r < kFewClasses; ++r) dz[i][r] = to_float(pack.v[r]);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (target[i] >= v && target[i] < v + kFewClasses) {
#pragma unroll
                for (int r = 0; r < kFewClasses; ++r)
                    if (target[i] == v + r) dz[i][r] += lost[i];
            }
        T* to = static_cast<T*>(a.out) + v * a.stride + c;
#pragma unroll
        for (int r = 0; r < kFewClasses; ++r) {
            if (v + r >= a.classes) break;
            Pack<T, kN> out;
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kRows; ++i) sum = __builtin_fmaf(dz[i][r], x[i][e], sum);
                out.v[e] = rounded<T>(sum);
            }
            if (a.dim >= kN) {
                a.streamed ? stream_pack(to + r * a.stride, out) : store_pack(to + r * a.stride, out);
            } else {
#pragma unroll
                for (int e = 0; e < kN - 1; ++e)
                    if (e < a.dim) to[r * a.stride + e] = out.v[e];
            }
        }
    }
}

struct JoinArgs {
    const float4* stats;
    const float* target_logit;
    const void* targets;
    float* logprob;
    float* lse;
    float* entropy;
    long first_row, n_rows;  // of this piece of the batch
    int parts, n_classes, id_type;
};

// The statistics of a row's tiles joined, by a wave, or by four where there are few rows: 4 rows of 1000 parts 10 us with one and a load
// after the other, 3.8 with four and four loads each under way; 2047 rows of 250 parts 6.8 us with four, 4.8 with one; 8192 rows, 34
// MB, 8.3 us.
template <int kWaves>
__global__ __launch_bounds__(kThreads) void join_scores_kernel(JoinArgs a)
{
    constexpr int kFlight = 4, kTeam = 64 * kWaves, kRows = kThreads / kTeam;
    __shared__ Stats shared[kThreads / 64];
    const long row = (long)blockIdx.x * kRows + threadIdx.x / kTeam;
    const int member = threadIdx.x % kTeam;
    Stats v{-INFINITY, 0.f, 0.f};
    if (row < a.n_rows) {
        for (int p = member; p < a.parts; p += kTeam * kFlight) {
            float4 x[kFlight];
#pragma unroll
            for (int u = 0; u < kFlight; ++u) x[u] = p + u * kTeam < a.parts ? a.stats[row * a.parts + p + u * kTeam] : float4{-INFINITY, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < kFlight; ++u) v = join(v, Stats{x[u].x, x[u].y, x[u].z}, kLog2e);
        }
    }
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = join(v, Stats{__shfl_xor(v.m, step), __shfl_xor(v.s, step), __shfl_xor(v.t, step)}, kLog2e);
    if constexpr (kWaves > 1) {
        if (member % 64 == 0) shared[threadIdx.x / 64] = v;
        __syncthreads();
        for (int w = 1; w < kWaves; ++w) v = member == 0 ? join(v, shared[threadIdx.x / 64 + w], kLog2e) : v;
    }
    if (member != 0 || row >= a.n_rows) return;
    const Row r = finish(v, 1.f);
    const long at = a.first_row + row;
    if (a.lse) a.lse[at] = r.lse;
    if (a.entropy) a.entropy[at] = r.entropy;
    if (a.logprob) a.logprob[at] = a.targets && class_at(a.targets, a.id_type, at, a.n_classes) >= 0 ? logprob_of(r, a.target_logit[row], 1.f) : 0.f;
}

// The statistics of the rows far from 0, of a piece of the classes joined to those before it: a wave a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_far_kernel(const float4* stats, const float* lse, float4* far, int rows, int parts, int first)
{
    const int row = blockIdx.x * (kThreads / 64) + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (row >= rows || !far_from_0<T>(lse[row])) return;
    Stats v{-INFINITY, 0.f, 0.f};
    for (int p = lane; p < parts; p += 64) {
        const float4 x = stats[(long)row * parts + p];
        v = join(v, Stats{x.x, x.y, x.z}, kLog2e);
    }
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = join(v, Stats{__shfl_xor(v.m, step), __shfl_xor(v.s, step), __shfl_xor(v.t, step)}, kLog2e);
    if (lane != 0) return;
    if (first > 0) v = join(Stats{far[row].x, far[row].y, far[row].z}, v, kLog2e);
    far[row] = float4{v.m, v.s, v.t, 0.f};
}

constexpr int64_t kJoinedByOneWave = 1024;  // rows, from which on there are waves enough

// ---- which tiles ------------------------------------------------------------------------------------------------------

enum Tiles { kLarge, kMiddle, kSmall };
// What tiles cost, measured on products of whole rounds of workgroups: us for a step and for the rest, when a compute unit holds as
// many workgroups as it can.  (binary32 runs at the matrix instructions' rate in all of them.)
struct TileShape {
    int m, n, parts_n;    // parts_n: waves along the columns
    int per_cu;           // workgroups that a compute unit holds
    float step[2], rest;  // bfloat16, binary32
};
constexpr TileShape kShapes[] = {{256, 256, 2, 1, {1.5f, 7.5f}, 10.f}, {128, 128, 2, 2, {0.87f, 4.05f}, 6.f}, {32, 64, 2, 5, {0.62f, 1.33f}, 3.5f}};
constexpr float kLeastStep = 0.35f;  // us, however few workgroups a compute unit holds: the wait for memory
constexpr int kUnits = 256;          // compute units
constexpr int kLeastSteps = 4;       // of a division of a contraction

struct Choice {
    Tiles tiles;
    int tiles_m, tiles_n, splits, split_steps;
    int64_t groups() const { return (int64_t)tiles_m * tiles_n * splits; }
};

int steps_of(int64_t k, int dtype) { return (int)ceil_div(k * cat_size(dtype), kStepBytes); }

// us for so many workgroups of so many steps: whole rounds of them over the chip, and a last one that may leave room.
float time_of(const TileShape& s, int dtype, int64_t groups, int steps)
{
    const float step = s.step[dtype == NUTS_F32];
    const int64_t rounds = groups / (kUnits * s.per_cu), more = ceil_div(groups % (kUnits * s.per_cu), kUnits);
    return rounds * (step * steps + s.rest) + (more ? std::max(step * more / s.per_cu, kLeastStep) * steps + s.rest : 0.f);
}

// The tiles, and the divisions of the contraction (1, unless it may be divided), that take least time.
Choice choose(int64_t m, int64_t n, int64_t k, int dtype, bool may_split)
{
    Choice best{};
    float least = INFINITY;
    const int steps = std::max(1, steps_of(k, dtype));
    for (int t = kLarge; t <= kSmall; ++t) {
        const TileShape& s = kShapes[t];
        const int64_t tiles = ceil_div(m, s.m) * ceil_div(n, s.n), slots = (int64_t)kUnits * s.per_cu;
        const int most = may_split && tiles < slots ? (int)std::max<int64_t>(1, std::min<int64_t>(slots / tiles, steps / kLeastSteps)) : 1;
        for (int splits = 1; splits <= most; ++splits) {
            Choice c{(Tiles)t, (int)ceil_div(m, s.m), (int)ceil_div(n, s.n), 1, (int)ceil_div(steps, splits)};
            c.splits = (int)ceil_div(steps, c.split_steps);
            // the divisions' sums are stored, read and added up at 4 TB/s or so, in a launch of its own
            const float join = c.splits > 1 ? 4.f + 8e-6f * (float)(m * n) * c.splits / 4.f : 0.f;
            const float time = time_of(s, dtype, c.groups(), c.split_steps) + join;
            if (time < least) {
                least = time;
                best = c;
            }
        }
    }
    return best;
}

template <ProductKind kKind, bool kAcrossA, bool kAcrossB, typename T>
void launch_product(const Choice& c, ProductArgs p, hipStream_t stream)
{
    p.tiles_m = c.tiles_m;
    p.tiles_n = c.tiles_n;
    p.splits = c.splits;
    p.split_steps = c.split_steps;
    p.streamed = (int64_t)p.m * p.n * (kKind == kOutput ? sizeof(T) : sizeof(float) * c.splits) >= kStreamed;
    const dim3 grid((unsigned)c.tiles_m * c.tiles_n, c.splits);
    auto launch = [&](auto ragged) {  // (a kernel of its own: what it does beside the steps would cost the others 3 %)
        constexpr bool kRagged = decltype(ragged)::value;
        switch (c.tiles) {
        case kLarge: hipLaunchKernelGGL((product_kernel<T, 256, 256, 4, 2, 2, kAcrossA, kAcrossB, kRagged, kKind>), grid, dim3(512), 0, stream, p); break;
        case kMiddle: hipLaunchKernelGGL((product_kernel<T, 128, 128, 2, 2, 2, kAcrossA, kAcrossB, kRagged, kKind>), grid, dim3(256), 0, stream, p); break;
        case kSmall: hipLaunchKernelGGL((product_kernel<T, 32, 64, 2, 2, 2, kAcrossA, kAcrossB, kRagged, kKind>), grid, dim3(256), 0, stream, p); break;
        }
    };
    if constexpr (!kAcrossA && !kAcrossB) {
        if (p.k % (int)(16 / sizeof(T)) != 0) return launch(std::true_type{});
    }
    launch(std::false_type{});
}

// ---- host -------------------------------------------------------------------------------------------------------------

int check_score(const nuts_score_desc* d, const char* who)
{
    if (!d) return api_fail(NUTS_E_INVALID_ARG, "%s: desc must not be NULL", who);
    if (d->dtype != NUTS_F32 && d->dtype != NUTS_BF16) return api_fail(NUTS_E_INVALID_ARG, "%s: dtype must be NUTS_F32 or NUTS_BF16", who);
    if (d->id_type != NUTS_I32 && d->id_type != NUTS_I64) return api_fail(NUTS_E_INVALID_ARG, "%s: id_type must be NUTS_I32 or NUTS_I64", who);
    if (d->n_rows < 0 || d->n_rows > (1 << 20)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_rows must be in [0, 2^20]", who);
    if (d->n_classes < 1 || d->n_classes > (1 << 24)) return api_fail(NUTS_E_INVALID_ARG, "%s: n_classes must be in [1, 2^24]", who);
    if (d->dim < 1 || d->dim > (1 << 20)) return api_fail(NUTS_E_INVALID_ARG, "%s: dim must be in [1, 2^20]", who);
    if (d->x_stride < d->dim || d->weight_stride < d->dim || d->grad_x_stride < d->dim || d->grad_weight_stride < d->dim || d->logits_stride < d->n_classes)
        return api_fail(NUTS_E_INVALID_ARG, "%s: a stride is smaller than its rows", who);
    const int64_t most = INT64_MAX / 8 / (1 << 24);
    if (d->x_stride > most || d->weight_stride > most || d->grad_x_stride > most || d->grad_weight_stride > most || d->logits_stride > most)
        return api_fail(NUTS_E_INVALID_ARG, "%s: a stride is too large", who);
    const float scale = (float)d->scale;
    if (!std::isfinite(scale) || !(scale > 0.f)) return api_fail(NUTS_E_INVALID_ARG, "%s: scale must be finite and > 0", who);
    return NUTS_OK;
}

struct Space {
    size_t bytes = 0;
    size_t take(size_t n)
    {
        const size_t at = bytes;
        bytes += (n + 255) & ~(size_t)255;
        return at;
    }
};

int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Whether rows are read as they lie.  Rows that begin between 16 bytes touch a line of memory more each step, which costs less than
// to copy them, up to several thousand rows of x: with 2046 or 4094 bfloat16 features, 1000 rows' gradients of 32001 classes 530 us
// and 597 with copies, 4096 rows' 1593 and 1610, but 8192 rows' scores of 32000 classes 1785 and 1675.
constexpr int64_t kCopiedRows = 6144;
bool rows_fit(const nuts_score_desc* d, int64_t stride)
{
    const int64_t bytes = stride * (int64_t)cat_size(d->dtype);
    return bytes <= kMostBufferBytes / 256 && (bytes % 16 == 0 || (bytes % 4 == 0 && d->n_rows < kCopiedRows));
}
bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

constexpr int64_t kMostStats = (int64_t)1 << 28;     // bytes of statistics of one piece of a batch
constexpr int64_t kMostPiece = (int64_t)1 << 28;     // logits of one piece of the classes
constexpr int64_t kSeparateGroups = 128;             // fewer workgroups than this, and the contraction is divided

// Forward.  Where few tiles would have a long contraction each, the products are divided along it and z is stored; nuts_logprobs
// then goes over it (it is small).
struct ScorePlan {
    int64_t dim_pad;  // of packed rows
    bool separate;
    Choice choice;
    int64_t piece;    // rows of x at a time
    int parts;
    nuts_logits_desc logits;
    size_t x, weight, stats, target_logit, sums, z, logprobs;
    int64_t logprobs_bytes;
    Space space;
};

ScorePlan plan_score(const nuts_score_desc* d)
{
    ScorePlan p{};
    const size_t size = cat_size(d->dtype);
    p.dim_pad = round_up(d->dim, 64);
    p.choice = choose(d->n_rows, d->n_classes, d->dim, d->dtype, false);
    p.separate = p.choice.groups() < kSeparateGroups && steps_of(d->dim, d->dtype) >= 4 * kLeastSteps;
    p.x = p.space.take(rows_fit(d, d->x_stride) ? 0 : (size_t)d->n_rows * p.dim_pad * size);
    p.weight = p.space.take(rows_fit(d, d->weight_stride) ? 0 : (size_t)d->n_classes * p.dim_pad * size);
    if (p.separate) {
        p.choice = choose(d->n_rows, d->n_classes, d->dim, d->dtype, true);
        p.piece = d->n_rows;
        p.logits = nuts_logits_desc{NUTS_F32, d->id_type, d->n_rows, d->n_classes, round_up(d->n_classes, 4), 0, 1.0, 0, 0};
        p.sums = p.space.take((size_t)p.choice.splits * d->n_rows * d->n_classes * sizeof(float));
        p.z = p.space.take((size_t)d->n_rows * p.logits.row_stride * sizeof(float));
        nuts_logits_desc any = p.logits;  // (the caller's own logits may have any stride)
        nuts_logprobs_workspace(&any, &p.logprobs_bytes);
        p.logprobs = p.space.take((size_t)p.logprobs_bytes);
    } else {
        p.parts = p.choice.tiles_n * kShapes[p.choice.tiles].parts_n;
        p.piece = std::max<int64_t>(256, kMostStats / ((int64_t)p.parts * sizeof(float4)) / 256 * 256);
        p.piece = std::min(p.piece, d->n_rows);
        p.stats = p.space.take((size_t)p.piece * p.parts * sizeof(float4));
        p.target_logit = p.space.take((size_t)p.piece * sizeof(float));
    }
    return p;
}

// x and weight as the products read them: as they lie, or (`room`) copied to rows that begin at multiples of 16 bytes.
struct Matrices {
    const void *x, *weight;
    int64_t x_stride, weight_stride;
    int64_t dim;  // with the zeros behind rows of whole pieces
};
template <typename T>
Matrices pack(const nuts_score_desc* d, const void* x, const void* weight, bool want_x, bool want_weight, char* x_room, char* weight_room, int64_t dim_pad,
              hipStream_t stream)
{
    Matrices m{x, weight, d->x_stride, d->weight_stride, d->dim};
    PackArgs a{{x, weight}, {x_room, weight_room}, {(long)d->x_stride, (long)d->weight_stride}, {0, 0}, (int)d->dim, (int)dim_pad};
    if (want_x && !rows_fit(d, d->x_stride)) {
        a.rows[0] = (long)d->n_rows;
        m.x = x_room;
        m.x_stride = dim_pad;
    }
    if (want_weight && !rows_fit(d, d->weight_stride)) {
        a.rows[1] = (long)d->n_classes;
        m.weight = weight_room;
        m.weight_stride = dim_pad;
    }
    if (a.rows[0] && a.rows[1]) m.dim = round_up(d->dim, 16 / sizeof(T));
    const int64_t packs = (a.rows[0] + a.rows[1]) * (dim_pad * (int64_t)sizeof(T) / 16);
    if (packs > 0) hipLaunchKernelGGL(pack_rows_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(packs, kThreads), 1 << 16)), dim3(kThreads), 0, stream, a);
    return m;
}

template <typename T>
void add_up(const float* sums, int splits, int64_t rows, int64_t columns, float scale, void* out, int64_t stride, hipStream_t stream)
{
    const int each = columns % 4 == 0 ? 4 : 1;
    hipLaunchKernelGGL((each == 4 ? add_up_kernel<T, 4> : add_up_kernel<T, 1>), dim3((unsigned)std::min<int64_t>(ceil_div(rows * columns, kThreads * each), 16384)),
                       dim3(kThreads), 0, stream, sums, splits, (long)rows, (int)columns, scale, static_cast<T*>(out), (long)stride);
}

template <typename T>
int score(const nuts_score_desc* d, const ScorePlan& p, const void* x, const void* weight, const void* targets, float* logprob, float* lse,
          float* entropy, float* logits, char* w)
{
    hipStream_t stream = api_stream();
    const size_t size = sizeof(T);
    const Matrices m = pack<T>(d, x, weight, true, true, w + p.x, w + p.weight, p.dim_pad, stream);
    ProductArgs a{};
    a.a = static_cast<const char*>(m.x);
    a.b = static_cast<const char*>(m.weight);
    a.a_stride = (long)(m.x_stride * size);
    a.b_stride = (long)(m.weight_stride * size);
    a.n = (int)d->n_classes;
    a.k = (int)m.dim;
    if (p.separate) {
        a.m = (int)d->n_rows;
        a.sums = reinterpret_cast<float*>(w + p.sums);
        launch_product<kSums, false, false, T>(p.choice, a, stream);
        float* z = logits ? logits : reinterpret_cast<float*>(w + p.z);
        nuts_logits_desc l = p.logits;
        if (logits) l.row_stride = d->logits_stride;
        add_up<float>(a.sums, p.choice.splits, d->n_rows, d->n_classes, (float)d->scale, z, l.row_stride, stream);
        NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
        return nuts_logprobs(&l, z, targets, nullptr, logprob, lse, entropy, nullptr, nullptr, w + p.logprobs, p.logprobs_bytes);
    }
    const bool wanted = logprob || lse || entropy;
    for (int64_t row = 0; row < d->n_rows; row += p.piece) {
        const int64_t rows = std::min(p.piece, d->n_rows - row);
        a.a = static_cast<const char*>(m.x) + row * a.a_stride;
        a.m = (int)rows;
        a.c = logits ? logits + row * d->logits_stride : nullptr;
        a.c_stride = (long)d->logits_stride;
        a.scale = (float)d->scale;
        a.targets = !targets ? nullptr : static_cast<const char*>(targets) + row * (d->id_type == NUTS_I64 ? 8 : 4);
        a.id_type = d->id_type;
        a.stats = wanted ? reinterpret_cast<float4*>(w + p.stats) : nullptr;
        a.target_logit = reinterpret_cast<float*>(w + p.target_logit);
        Choice c = p.choice;
        c.tiles_m = (int)ceil_div(rows, kShapes[c.tiles].m);
        launch_product<kScores, false, false, T>(c, a, stream);
        if (wanted) {
            const JoinArgs j{a.stats, a.target_logit, targets, logprob, lse, entropy, (long)row, (long)rows, p.parts, (int)d->n_classes, d->id_type};
            if (rows < kJoinedByOneWave) hipLaunchKernelGGL(join_scores_kernel<4>, dim3((unsigned)rows), dim3(kThreads), 0, stream, j);
            else hipLaunchKernelGGL(join_scores_kernel<1>, dim3((unsigned)ceil_div(rows, kThreads / 64)), dim3(kThreads), 0, stream, j);
        }
    }
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

// Backward: pieces of the classes.  dX reads the class weights across (classes are the contraction), dW both dZ and the features.
struct ScoreGradPlan {
    int64_t dim_pad, piece, piece_pad, pieces;
    Choice scores, grad_x, grad_weight;
    size_t x, weight, z, dz, residual, far, sums_x, sums_weight;
    Space space;
};

ScoreGradPlan plan_score_grad(const nuts_score_desc* d)
{
    ScoreGradPlan p{};
    const size_t size = cat_size(d->dtype);
    const int64_t n = std::max<int64_t>(d->n_rows, 1);
    p.dim_pad = round_up(d->dim, 64);
    p.piece = std::clamp<int64_t>(kMostPiece / n / 256 * 256, 256, 1 << 20);
    p.piece = std::min(p.piece, d->n_classes);
    p.pieces = ceil_div(d->n_classes, p.piece);
    p.piece_pad = round_up(p.piece, 64);
    p.scores = choose(n, p.piece, d->dim, d->dtype, false);
    p.grad_x = choose(n, d->dim, p.piece, d->dtype, true);
    p.grad_weight = choose(p.piece, d->dim, n, d->dtype, true);
    // (whether z is computed again is the call's)
    p.x = p.space.take(rows_fit(d, d->x_stride) ? 0 : (size_t)d->n_rows * p.dim_pad * size);
    p.weight = p.space.take(rows_fit(d, d->weight_stride) ? 0 : (size_t)d->n_classes * p.dim_pad * size);
    p.z = p.space.take((size_t)d->n_rows * p.piece_pad * sizeof(float));
    p.dz = p.space.take((size_t)d->n_rows * p.piece_pad * size);
    p.residual = p.space.take((size_t)d->n_rows * sizeof(float));
    p.far = p.space.take(p.pieces > 1 ? (size_t)d->n_rows * sizeof(float4) : 0);
    p.sums_x = p.space.take(p.grad_x.splits > 1 || p.pieces > 1 ? (size_t)p.grad_x.splits * d->n_rows * d->dim * sizeof(float) : 0);
    p.sums_weight = p.space.take(p.grad_weight.splits > 1 ? (size_t)p.grad_weight.splits * p.piece * d->dim * sizeof(float) : 0);
    return p;
}

template <typename T>
int score_grad(const nuts_score_desc* d, const ScoreGradPlan& p, const void* x, const void* weight, const void* targets, const float* logits,
               const float* lse, const float* entropy, const float* grad_logprob, const float* grad_lse, const float* grad_entropy,
               void* grad_x, void* grad_weight, char* w)
{
    hipStream_t stream = api_stream();
    const int64_t size = sizeof(T), n = d->n_rows, dim = d->dim;
    const Matrices m = pack<T>(d, x, weight, n > 0 && (grad_weight || !logits), n > 0 && (grad_x || !logits), w + p.x, w + p.weight, p.dim_pad, stream);
    float* residual = targets && grad_logprob && size == 2 ? reinterpret_cast<float*>(w + p.residual) : nullptr;
    // z of the classes [first, first + classes), or their statistics in the rows far from 0
    auto scores = [&](int64_t first, int64_t classes, float4* stats) {
        ProductArgs a{};
        a.a = static_cast<const char*>(m.x);
        a.b = static_cast<const char*>(m.weight) + first * m.weight_stride * size;
        a.a_stride = (long)(m.x_stride * size);
        a.b_stride = (long)(m.weight_stride * size);
        a.m = (int)n;
        a.n = (int)classes;
        a.k = (int)m.dim;
        a.c = stats ? nullptr : w + p.z;
        a.c_stride = (long)p.piece_pad;
        a.scale = (float)d->scale;
        a.stats = stats;
        a.lse = stats ? lse : nullptr;
        Choice c = p.scores;
        c.tiles_n = (int)ceil_div(classes, kShapes[c.tiles].n);
        launch_product<kScores, false, false, T>(c, a, stream);
        return c.tiles_n * kShapes[c.tiles].parts_n;
    };
    float4* far = !logits && p.pieces > 1 ? reinterpret_cast<float4*>(w + p.far) : nullptr;
    for (int64_t first = 0; far && n > 0 && first < d->n_classes; first += p.piece) {
        float4* stats = reinterpret_cast<float4*>(w + p.dz);  // (16 bytes for 32 columns and more; dZ comes later)
        const int parts = scores(first, std::min(p.piece, d->n_classes - first), stats);
        hipLaunchKernelGGL(join_far_kernel<T>, dim3((unsigned)ceil_div(n, kThreads / 64)), dim3(kThreads), 0, stream, stats, lse, far, (int)n, parts, (int)first);
    }
    for (int64_t first = 0; first < d->n_classes; first += p.piece) {
        const int64_t classes = std::min(p.piece, d->n_classes - first);
        const char* own_weight = static_cast<const char*>(m.weight) + first * m.weight_stride * size;
        const float* z = logits ? logits + first : nullptr;
        int64_t z_stride = d->logits_stride;
        if (!logits && n > 0) {
            scores(first, classes, nullptr);
            z = reinterpret_cast<const float*>(w + p.z);
            z_stride = p.piece_pad;
        }
        if (n > 0) {
            const int parts = (int)ceil_div(p.piece_pad, kGradPacks * kThreads * (16 / size));
            const GradArgs g{z, far, targets, lse, entropy, grad_logprob, grad_lse, grad_entropy, w + p.dz, residual, (long)z_stride, (int)p.piece_pad, parts, (int)first,
                             (int)classes, (int)d->n_classes, d->id_type, n * p.piece_pad * size >= kStreamed, (float)d->scale};
            hipLaunchKernelGGL(dz_kernel<T>, dim3((unsigned)(n * parts)), dim3(kThreads), 0, stream, g);
        }
        if (grad_x && n > 0) {
            ProductArgs a{};
            a.a = w + p.dz;
            a.b = own_weight;
            a.a_stride = (long)(p.piece_pad * size);
            a.b_stride = (long)(m.weight_stride * size);
            a.m = (int)n;
            a.n = (int)dim;
            a.k = (int)classes;
            a.sums = reinterpret_cast<float*>(w + p.sums_x);
            a.add = first > 0;
            a.c = grad_x;
            a.c_stride = (long)d->grad_x_stride;
            a.targets = targets;
            a.id_type = d->id_type;
            a.residual = residual;
            a.first_class = (int)first;
            a.n_classes = (int)d->n_classes;
            if (p.grad_x.splits > 1 || p.pieces > 1) launch_product<kSums, false, true, T>(p.grad_x, a, stream);
            else launch_product<kOutput, false, true, T>(p.grad_x, a, stream);
        }
        if (grad_weight && n > 0 && n <= kFewRows<T>) {
            int lane_bits = 0;
            while (lane_bits < 8 && (1 << lane_bits) * (16 / size) < dim) ++lane_bits;
            const FewArgs a{w + p.dz, m.x, targets, residual, static_cast<char*>(grad_weight) + first * d->grad_weight_stride * size, (long)m.x_stride,
                            (long)d->grad_weight_stride, (int)n, (int)p.piece_pad, (int)dim, (int)first, (int)classes, (int)d->n_classes, d->id_type,
                            lane_bits, classes * dim * size >= kStreamed};
            const int64_t groups = ceil_div(ceil_div(classes, kFewClasses), kThreads >> lane_bits);
            const int64_t slices = ceil_div(dim, (int64_t)(16 / size) << lane_bits);
            const dim3 grid((unsigned)std::min<int64_t>(groups, ceil_div(kFewGroups, slices)), (unsigned)slices);
            hipLaunchKernelGGL(few_rows_weights_kernel<T>, grid, dim3(kThreads), 0, stream, a);
        } else if (grad_weight) {
            ProductArgs a{};
            a.a = w + p.dz;
            a.b = static_cast<const char*>(m.x);
            a.a_stride = (long)(p.piece_pad * size);
            a.b_stride = (long)(m.x_stride * size);
            a.m = (int)classes;
            a.n = (int)dim;
            a.k = (int)n;
            a.sums = reinterpret_cast<float*>(w + p.sums_weight);
            a.c = static_cast<char*>(grad_weight) + first * d->grad_weight_stride * size;
            a.c_stride = (long)d->grad_weight_stride;
            a.targets = targets;
            a.id_type = d->id_type;
            a.residual = n > 0 ? residual : nullptr;
            a.first_class = (int)first;
            a.n_classes = (int)d->n_classes;
            Choice c = p.grad_weight;
            c.tiles_m = (int)ceil_div(classes, kShapes[c.tiles].m);
            if (c.splits > 1) {
                launch_product<kSums, true, true, T>(c, a, stream);
                add_up<T>(a.sums, c.splits, classes, dim, 1.f, a.c, d->grad_weight_stride, stream);
            } else {
                launch_product<kOutput, true, true, T>(c, a, stream);
            }
        }
    }
    if (grad_x && n > 0 && (p.grad_x.splits > 1 || p.pieces > 1))
        add_up<T>(reinterpret_cast<const float*>(w + p.sums_x), p.grad_x.splits, n, dim, 1.f, grad_x, d->grad_x_stride, stream);
    NUTS_CAT_TRY(hipGetLastError(), NUTS_E_DEVICE);
    return NUTS_OK;
}

int check_workspace(const char* who, const void* workspace, int64_t given, size_t bytes)
{
    if (bytes > 0 && (!workspace || given < (int64_t)bytes)) return api_fail(NUTS_E_INVALID_ARG, "%s: needs a workspace of %zu bytes", who, bytes);
    if (bytes > 0 && reinterpret_cast<uintptr_t>(workspace) % 256) return api_fail(NUTS_E_INVALID_ARG, "%s: workspace must be aligned to 256 bytes", who);
    return NUTS_OK;
}

}  // namespace
}  // namespace nuts

using namespace nuts;

extern "C" {

int nuts_score_workspace(const nuts_score_desc* d, int64_t* bytes)
{
    if (int rc = check_score(d, "nuts_score_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_score_workspace: bytes must not be NULL");
    *bytes = d->n_rows == 0 ? 0 : (int64_t)plan_score(d).space.bytes;
    return NUTS_OK;
}

int nuts_score(const nuts_score_desc* d, const void* x, const void* weight, const void* targets, float* logprob, float* lse, float* entropy,
               float* logits, void* workspace, int64_t workspace_bytes)
{
    if (int rc = check_score(d, "nuts_score")) return rc;
    if (d->n_rows == 0) return NUTS_OK;
    if (!x || !weight) return api_fail(NUTS_E_INVALID_ARG, "nuts_score: null pointer");
    if (!aligned(x) || !aligned(weight)) return api_fail(NUTS_E_INVALID_ARG, "nuts_score: x and weight must begin at multiples of 16 bytes");
    const ScorePlan p = plan_score(d);
    if (int rc = check_workspace("nuts_score", workspace, workspace_bytes, p.space.bytes)) return rc;
    if (int rc = api_have_device()) return rc;
    char* w = static_cast<char*>(workspace);
    return d->dtype == NUTS_F32 ? score<float>(d, p, x, weight, targets, logprob, lse, entropy, logits, w)
                                : score<bf16>(d, p, x, weight, targets, logprob, lse, entropy, logits, w);
}

int nuts_score_grad_workspace(const nuts_score_desc* d, int64_t* bytes)
{
    if (int rc = check_score(d, "nuts_score_grad_workspace")) return rc;
    if (!bytes) return api_fail(NUTS_E_INVALID_ARG, "nuts_score_grad_workspace: bytes must not be NULL");
    *bytes = (int64_t)plan_score_grad(d).space.bytes;
    return NUTS_OK;
}

int nuts_score_grad(const nuts_score_desc* d, const void* x, const void* weight, const void* targets, const float* logits, const float* lse,
                    const float* entropy, const float* grad_logprob, const float* grad_lse, const float* grad_entropy, void* grad_x,
                    void* grad_weight, void* workspace, int64_t workspace_bytes)
{
    if (int rc = check_score(d, "nuts_score_grad")) return rc;
    if (d->n_rows > 0 && (!x || !weight || !lse)) return api_fail(NUTS_E_INVALID_ARG, "nuts_score_grad: null pointer");
    if (!aligned(x) || !aligned(weight)) return api_fail(NUTS_E_INVALID_ARG, "nuts_score_grad: x and weight must begin at multiples of 16 bytes");
    if (grad_entropy && !entropy) return api_fail(NUTS_E_INVALID_ARG, "nuts_score_grad: grad_entropy needs the entropy");
    if (!grad_x && !grad_weight) return NUTS_OK;
    const ScoreGradPlan p = plan_score_grad(d);
    if (int rc = check_workspace("nuts_score_grad", workspace, workspace_bytes, p.space.bytes)) return rc;
    if (int rc = api_have_device()) return rc;
    char* w = static_cast<char*>(workspace);
    return d->dtype == NUTS_F32
               ? score_grad<float>(d, p, x, weight, targets, logits, lse, entropy, grad_logprob, grad_lse, grad_entropy, grad_x, grad_weight, w)
               : score_grad<bf16>(d, p, x, weight, targets, logits, lse, entropy, grad_logprob, grad_lse, grad_entropy, grad_x, grad_weight, w);
}

}  // extern "C"
