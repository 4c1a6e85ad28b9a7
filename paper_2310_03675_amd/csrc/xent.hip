// Softmax cross entropy of a linear classifier over N classes, in pieces of the classes (gfx950):
//   z = X W + b,  lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,target(i)  (0 where the target is to be ignored)
//   dz_ij = g_i (exp(z_ij - lse_i) - [j = target(i)]),  dX = dz W^T,  dW = X^T dz,  db = sum_i dz_ij
// Forward, every tile of the product leaves the largest logit of a row and the sum of exponentials relative to it; a
// second launch joins a row's pairs.  Backward, the logits of a piece of the classes are multiplied again and become dz in
// the workspace, from which the three gradients are taken; dX is added up over the pieces in 32 bits.
//
// The matrix pipe bounds large problems: four products of 2 M K N operations forward and backward, of which three are what the
// gradients need and one is what not keeping the logits costs.  8192 x 4096 x 128000 in bfloat16: 28.2 ms, the products 6.9 to
// 7.4 each, 1170 to 1240 TFLOP/s, where a large library product reaches 1160 to 1525 by orientation; 4096 x 2048 x 50257 3.1 ms,
// 1110, of it 0.11 for W, whose rows are no whole 16 bytes.  fp32 (six products of planes; a step keeps the logits where the classes are
// one piece): 777 x 320 x 10007 155 us of which the three products take 124, 120 TFLOP/s of 32 bits, 720 of bfloat16; the library's
// large fp32 product has 154.
// dz is rounded to bfloat16 where the problem is, by 2^-8 of each at most: the matrix cores' bfloat16 products take it, at sixteen times
// the rate of 32-bit ones and a third of the memory of planes, and the error is of the size of the operands' own; db is summed in
// front of that rounding.  Small problems (below) wait for launches and memory, not for the matrix pipe.
#include "bf16_product.hpp"

namespace hdqt {

namespace {

using bf16::kAlong;
using bf16::kDown;
using bf16::v16f;

constexpr int kThreads = 256;

__device__ __forceinline__ float any_load(const void* p, int dtype, int64_t i)
{
    return dtype == kBf16 ? load_as<kBf16>(p, i) : load_as<kF32>(p, i);
}

// exp(t) for t <= 0 up to rounding.  EXACT: the product with log2 e in two parts, for results in 32 bits; else its rounding
// is |t| 2^-24 of the result, at most 2^-25 of the row's largest one: far below dz's own rounding to bfloat16, and as much as any
// rounding in a row's sum.
template <bool EXACT>
__device__ __forceinline__ float exp_of(float t)
{
    constexpr float kLog2e = 1.44269504f, kRest = 1.92596303e-8f;       // log2 e - kLog2e
    const float h = t * kLog2e;
    if (!EXACT) return __builtin_amdgcn_exp2f(h);
    const float low = fmaf(t, kLog2e, -h) + t * kRest;
    const float e = __builtin_amdgcn_exp2f(h);
    return h < -160.0f ? e : fmaf(e, low * 0.693147181f, e);
}

// (largest, sum of exponentials relative to it) of two parts together
__device__ __forceinline__ void join(float& m, float& l, float om, float ol)
{
    const float top = fmaxf(m, om), base = top == -INFINITY ? 0.0f : top;
    l = l * exp_of<true>(m - base) + ol * exp_of<true>(om - base);
    m = top;
}

// ---- operands as the products take them: rows of whole 16 bytes, in planes where they are fp32 ----

struct PackArgs {
    const void* src;
    int64_t rows, cols, ld;
    uint16_t* dst;
    int64_t step;
    uint32_t across, groups;            // workgroups side by side, and of this operand
};

__device__ __forceinline__ void split(float x, uint32_t (&part)[3])
{
    uint32_t top = to_bf16(x);
    if ((top & 0x7FFFu) == 0x7F80u) top = __float_as_uint(x) >> 16;     // (rounded to infinity: cut instead)
    part[0] = top;
    const float rest = __builtin_isfinite(x) ? x - from_bf16(top) : 0.0f;
    part[1] = to_bf16(rest);
    part[2] = to_bf16(rest - from_bf16(part[1]));
}

// A thread has two columns of kPackRows rows, all of whose loads are in flight.  Two operands in one launch, or one.
constexpr int kPackRows = 8;
template <int DT>
__global__ __launch_bounds__(kThreads) void xent_pack_kernel(PackArgs one, PackArgs other)
{
    const bool second = blockIdx.x >= one.groups;
    const PackArgs a = second ? other : one;
    const uint32_t group = blockIdx.x - (second ? one.groups : 0), down = group / a.across;
    const int64_t c = 2 * ((int64_t)(group - down * a.across) * kThreads + threadIdx.x), row0 = (int64_t)down * kPackRows;
    if (c >= (DT == kBf16 ? a.step : a.step / 3)) return;
    float x[kPackRows], y[kPackRows];
#pragma unroll
    for (int i = 0; i < kPackRows; ++i) {
        const int64_t from = (row0 + i) * a.ld + c;
        x[i] = row0 + i < a.rows && c < a.cols ? load_as<DT>(a.src, from) : 0.0f;
        y[i] = row0 + i < a.rows && c + 1 < a.cols ? load_as<DT>(a.src, from + 1) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kPackRows; ++i) {
        if (row0 + i >= a.rows) break;
        uint32_t* to = reinterpret_cast<uint32_t*>(a.dst + (row0 + i) * a.step + (DT == kBf16 ? c : c / 32 * 96 + c % 32));
        if (DT == kBf16) {
            *to = __float_as_uint(x[i]) >> 16 | (__float_as_uint(y[i]) & 0xFFFF0000u);
        } else {
            uint32_t p[3], q[3];
            split(x[i], p);
            split(y[i], q);
#pragma unroll
            for (int k = 0; k < 3; ++k) to[16 * k] = p[k] | q[k] << 16;
        }
    }
}

// ---- logits, and what becomes of them ----

struct RowArgs {
    const void* bias;                   // of the piece's first class
    int bias_dtype;
    int64_t classes, first_class;       // of the piece
    const int64_t* target;
    int64_t ignore, M;
    float2* pairs;                      // [tiles of classes][M]: largest logit, sum of exponentials
    float* picked;                      // [M]: the target's logit
    const float *saved, *dloss;
    int each;                           // rows have a factor of their own
    uint16_t* dz;                       // [M][step], zeros behind the classes
    int64_t step;
    float* column;                      // [tiles of rows][classes]: dz's sums over a tile's rows, or over kRowsOfDz; null: not wanted
    int eights;                         // the latter
    float* z;                           // [M][z_step]: the logits, for a step's gradients; null: not kept
    int64_t z_step;
};

__device__ __forceinline__ float larger_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// over eight lanes side by side, and over lanes 0 .. 31 and lanes 32 .. 63, in every one of them
__device__ __forceinline__ float sum_of_8(float v)
{
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true));        // lane ^ 1
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, true));        // lane ^ 2
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, true));       // the other four of eight
    return v;
}
__device__ __forceinline__ float sum_of_32(float v)
{
    v = sum_of_8(v);
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, true));       // the other eight of sixteen
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A large tile's workgroup has a compute unit to itself, a small one's shares it with another: two waves to a SIMD either way.
#define HDQT_TILE_KERNEL(WA, WB) __global__ __launch_bounds__(64 * WA * WB) __attribute__((amdgpu_waves_per_eu(2, 2))) void

// two stages of P planes' operands in LDS, each an object of its own
#define HDQT_STAGES(P, TA, TB)                                                    \
    constexpr int kA = (P == 1 ? 128 : 192) * TA, kB = (P == 1 ? 128 : 192) * TB; \
    __shared__ __align__(1024) uint8_t a0[kA], a1[kA], b0[kB], b1[kB];            \
    const bf16::Stages stages{{a0, a1}, {b0, b1}};

// Rows whose dz is added up for dbias first where a step keeps the logits: the same, to the bit, when a backward call of that size
// multiplies them again.  (Where no step does, a tile's rows: a sum for eight rows is 0.5 bytes a logit, 40000 x 32 x 4321 backward
// 1117 us and 1323.)
constexpr int kRowsOfDz = 8;

// Lines of A are classes (W, read down), lines of B rows (X): a lane then holds sums of one row of the logits, and the
// maximum and the sum over classes stay inside it but for one exchange between the wave's halves.
template <bool GRAD, int P, int TA, int TB, int WA, int WB>
HDQT_TILE_KERNEL(WA, WB) xent_logits_kernel(bf16::Args g, RowArgs r)
{
    constexpr int NA = TA / WA / 32, NB = TB / WB / 32;
    constexpr bool kExact = P == 3;
    HDQT_STAGES(P, TA, TB);
    __shared__ __align__(16) float bias[TA];
    __shared__ float2 halves[GRAD ? 1 : WA][GRAD ? 1 : TB];
    __shared__ float columns[GRAD ? WB : 1][GRAD ? TA : 1];
    const bf16::Place p = bf16::place_of(g);
    if (!p.there) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int t = threadIdx.x; t < TA; t += 64 * WA * WB) {
        const int64_t c = (int64_t)p.at * TA + t;
        bias[t] = c >= r.classes ? -INFINITY : r.bias ? any_load(r.bias, r.bias_dtype, c) : 0.0f;
    }
    v16f acc[NA][NB] = {};
    bf16::multiply<P, kDown, kAlong, TA, TB, WA, WB>(g, p, stages, wave, lane, acc);

    const int class0 = (wave / WB) * (TA / WA), row0 = (wave % WB) * (TB / WB);
    auto column = [&](auto jj) {
        constexpr int j = decltype(jj)::value;
        const int64_t row = (int64_t)p.bt * TB + row0 + 32 * j + (lane & 31);
        const bool there = row < r.M;
        const int64_t target = there ? r.target[row] : -1;
        // the target's place among this lane's classes; of another lane or none: negative or beyond
        const int64_t away = target - r.first_class - ((int64_t)p.at * TA + class0 + 4 * (lane >> 5));
        const int at = away >= 0 && away < TA / WA && (away & 4) == 0 ? (int)away : -1;
        const bool any = __any(at >= 0);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 b = *reinterpret_cast<const float4*>(&bias[class0 + 32 * i + 8 * q + 4 * (lane >> 5)]);
                const float add[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z = acc[i][j][4 * q + e] + add[e];
                    acc[i][j][4 * q + e] = z;
                    if (!GRAD) top = fmaxf(top, z);
                }
            }
        if constexpr (!GRAD) {
            if (any) {
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (at == 32 * i + 8 * (e >> 2) + (e & 3)) r.picked[row] = acc[i][j][e];
            }
            if (P == 3 && r.z && there) {
                float* to = r.z + row * r.z_step + (int64_t)p.at * TA + class0 + 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<float4*>(to + 32 * i + 8 * q) =
                            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
            }
            top = larger_half(top);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += exp_of<kExact>(acc[i][j][e] - base);
            sum = sum_halves(sum);
            if (lane < 32) halves[wave / WB][row0 + 32 * j + lane] = make_float2(top, sum);
        } else {
            const bool counted = there && target != r.ignore;
            const float lse = there ? r.saved[row] : 0.0f, base = lse == -INFINITY ? 0.0f : lse;
            const float each = r.each && counted ? (r.dloss ? r.dloss[row] : 1.0f) : 1.0f;
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = exp_of<kExact>(acc[i][j][e] - base);
            if (any) {
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (at == 32 * i + 8 * (e >> 2) + (e & 3)) acc[i][j][e] -= 1.0f;
            }
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = counted ? acc[i][j][e] * each : 0.0f;
            if (there) {
                uint16_t* to = r.dz + row * r.step + P * ((int64_t)p.at * TA + class0) + 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                        if constexpr (P == 3) {
                            uint32_t s[4][3];
#pragma unroll
                            for (int e = 0; e < 4; ++e) split(v[e], s[e]);
#pragma unroll
                            for (int k = 0; k < 3; ++k)
                                *reinterpret_cast<uint2*>(to + 96 * i + 32 * k + 8 * q) =
                                    make_uint2(s[0][k] | s[1][k] << 16, s[2][k] | s[3][k] << 16);
                        } else {
                            *reinterpret_cast<uint2*>(to + 32 * i + 8 * q) =
                                make_uint2(to_bf16(v[0]) | to_bf16(v[1]) << 16, to_bf16(v[2]) | to_bf16(v[3]) << 16);
                        }
                    }
            }
        }
    };
    column(std::integral_constant<int, 0>{});
    if constexpr (NB > 1) column(std::integral_constant<int, 1>{});
    static_assert(NB <= 2, "a call for each");
    if constexpr (P == 3 && GRAD) {
        if (r.column && r.eights) {
            // a class's sums over eight rows, where a stage was; lines eight words longer, so that the four of a block lie in other banks
            constexpr int kLine = TA + 8;
            static_assert(TB / kRowsOfDz * kLine * sizeof(float) <= sizeof a0, "room for them");
            float* eights = reinterpret_cast<float*>(a0);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float s = sum_of_8(acc[i][j][e]);
                        if ((lane & 7) == 0)
                            eights[((row0 + 32 * j + (lane & 31)) >> 3) * kLine + class0 + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)] = s;
                    }
            __syncthreads();
            for (int t = threadIdx.x; t < TB / kRowsOfDz * TA; t += 64 * WA * WB) {
                const int64_t c = (int64_t)p.at * TA + t % TA, eight = (int64_t)p.bt * (TB / kRowsOfDz) + t / TA;
                if (c < r.classes && eight * kRowsOfDz < r.M) r.column[eight * r.classes + c] = eights[t / TA * kLine + t % TA];
            }
            return;
        }
    }
    if constexpr (!GRAD) {
        __syncthreads();
        for (int t = threadIdx.x; t < TB; t += 64 * WA * WB) {
            const int64_t row = (int64_t)p.bt * TB + t;
            if (row >= r.M) continue;
            float2 v = halves[0][t];
            for (int w = 1; w < WA; ++w) join(v.x, v.y, halves[w][t].x, halves[w][t].y);
            r.pairs[(int64_t)p.at * r.M + row] = v;
        }
    } else if (r.column) {
        // a class's sum over the tile's rows: this wave's, over the lanes of either half, then the waves side by side
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float s = acc[i][0][e];
#pragma unroll
                for (int j = 1; j < NB; ++j) s += acc[i][j][e];
                s = sum_of_32(s);
                if ((lane & 31) == 0) columns[wave % WB][class0 + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)] = s;
            }
        __syncthreads();
        for (int t = threadIdx.x; t < TA; t += 64 * WA * WB) {
            const int64_t c = (int64_t)p.at * TA + t;
            if (c >= r.classes) continue;
            float s = columns[0][t];
            for (int w = 1; w < WB; ++w) s += columns[w][t];
            r.column[(int64_t)p.bt * r.classes + c] = s;
        }
    }
}

// dz in planes from the logits that a step has kept: a workgroup has kRowsOfDz rows of 1024 classes, a thread four classes.  Memory
// bounds it: 4 bytes read and 6 written for a logit, 777 x 10007 in 15 us (5.2 TB/s, out of the memory-side cache), where the
// logits' product takes 45.
__global__ __launch_bounds__(kThreads) void xent_dz_kernel(RowArgs r)
{
    const int64_t c = 4 * ((int64_t)blockIdx.y * kThreads + threadIdx.x), row0 = (int64_t)blockIdx.x * kRowsOfDz;
    if (c >= r.step / 3) return;
    float column[4] = {};
#pragma unroll 1
    for (int half = 0; half < kRowsOfDz; half += 4) {
        float v[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t row = row0 + half + k, at_row = row < r.M ? row : r.M - 1;
            const int64_t target = r.target[at_row], at = target - r.first_class - c;
            const bool counted = row < r.M && target != r.ignore;
            const float lse = r.saved[at_row], base = lse == -INFINITY ? 0.0f : lse;
            const float each = r.each && counted ? (r.dloss ? r.dloss[at_row] : 1.0f) : 1.0f;
            // (behind the last class there is no logit in memory that anyone has written)
            const float4 q = c < r.z_step ? *reinterpret_cast<const float4*>(r.z + at_row * r.z_step + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            const float z[4] = {q.x, q.y, q.z, q.w};
            uint32_t s[4][3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = exp_of<true>(z[e] - base) - (at == e ? 1.0f : 0.0f);
                v[k][e] = counted && c + e < r.classes ? d * each : 0.0f;
                split(v[k][e], s[e]);
            }
            if (row >= r.M) continue;
            uint16_t* to = r.dz + row * r.step + c / 32 * 96 + c % 32;
#pragma unroll
            for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(to + 32 * p) = make_uint2(s[0][p] | s[1][p] << 16, s[2][p] | s[3][p] << 16);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) column[e] += (v[0][e] + v[1][e]) + (v[2][e] + v[3][e]);      // (in pairs, as lanes add them)
    }
    if (!r.column) return;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < r.classes) r.column[(int64_t)blockIdx.x * r.classes + c + e] = column[e];
}

// ---- gradients: dX (lines of A rows, of B features) and dW (lines of A features, of B classes) ----
//
// dX reads dz and W along their rows, dW both down theirs: no transposed copy of either.  8192 x 4096 x 128000 in bfloat16,
// sixteen pieces: dX 7.0 ms, dW 6.9 (1230 and 1250 TFLOP/s).

struct OutArgs {
    void* out;
    int64_t step;
    int dtype;
    const float *share, *dloss;         // factors of all, or null
    float* slices;                      // [part of the contraction][RA][RB]: added up by another launch, and over the pieces kept
    uint32_t parts;
    int first_piece, last_piece;
};

__device__ __forceinline__ float factor_of(const OutArgs& o) { return (o.share ? *o.share : 1.0f) * (o.dloss ? *o.dloss : 1.0f); }

// sum <- f(sum, descriptor, element) for a wave's sums and where they belong in memory: `to` is its first line's and column's place,
// lines are `step` apart.  A block of 32 lines has a descriptor of its own, which ends with the matrix: what lies behind the last
// line is left out by its range check, columns by an offset outside.
template <int NA, int NB, class T, class F>
__device__ __forceinline__ void each_sum(v16f (&acc)[NA][NB], int64_t lines, int64_t columns, int lane, T* to, int64_t step, F f)
{
    uint32_t at[NB];                // elements
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int col = 32 * j + (lane & 31);
        at[j] = col < columns ? 4 * (lane >> 5) * (uint32_t)step + col : bf16::kOutside / 4;
    }
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        const int64_t rows = lines - 32 * i < 32 ? lines - 32 * i : 32;
        const int64_t bytes = rows <= 0 ? 0 : (int64_t)sizeof(T) * ((rows - 1) * step + columns);
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(to + 32 * i * step, 0, bytes <= 0 ? 0 : (int)bytes, 0x00020000);
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j][e] = f(acc[i][j][e], rs, at[j] + (8 * (e >> 2) + (e & 3)) * (uint32_t)step);
    }
}

template <int P, int MODE, int TA, int TB, int WA, int WB>
HDQT_TILE_KERNEL(WA, WB) xent_gradient_kernel(bf16::Args g, OutArgs o)
{
    constexpr int NA = TA / WA / 32, NB = TB / WB / 32;
    HDQT_STAGES(P, TA, TB);
    const bf16::Place p = bf16::place_of(g);
    if (!p.there) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    v16f acc[NA][NB] = {};
    bf16::multiply<P, MODE, MODE, TA, TB, WA, WB>(g, p, stages, wave, lane, acc);
    const int64_t i0 = (int64_t)p.at * TA + (wave / WB) * (TA / WA), j0 = (int64_t)p.bt * TB + (wave % WB) * (TB / WB);
    const bool several = o.parts > 1;
    float* part = o.slices + (int64_t)p.part * g.RA * g.RB;
    if (!o.first_piece)
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, part + i0 * g.RB + j0, g.RB, [](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
            return v + __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, 4 * at, 0, 0));
        });
    if (several || !o.last_piece) {
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, part + i0 * g.RB + j0, g.RB, [](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rs, 4 * at, 0, 0);
            return v;
        });
        return;
    }
    const float factor = factor_of(o);
    if (o.dtype == kBf16)
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, static_cast<uint16_t*>(o.out) + i0 * o.step + j0, o.step,
                         [factor](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
                             // (outside in elements is outside in units of 2 bytes only with the bit above)
                             const uint32_t to = at >= bf16::kOutside / 4 ? bf16::kOutside : 2 * at;
                             __builtin_amdgcn_raw_buffer_store_b16((short)to_bf16(v * factor), rs, to, 0, 0);
                             return v;
                         });
    else
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, static_cast<float*>(o.out) + i0 * o.step + j0, o.step,
                         [factor](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
                             __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v * factor), rs, 4 * at, 0, 0);
                             return v;
                         });
}

// (four neighbours at a time where rows come in whole 16 bytes)
template <int V>
__global__ __launch_bounds__(kThreads) void xent_add_parts_kernel(OutArgs o, int64_t RA, int64_t RB)
{
    const float factor = factor_of(o);
    const int64_t j = V * ((int64_t)blockIdx.x * kThreads + threadIdx.x), size = RA * RB;
    if (j >= RB) return;
    for (int64_t i = blockIdx.y; i < RA; i += gridDim.y) {
        const float* from = o.slices + i * RB + j;
        float v[V] = {};
#pragma unroll 4
        for (uint32_t k = 0; k < o.parts; ++k) {
            if constexpr (V == 4) {
                const float4 q = *reinterpret_cast<const float4*>(from + k * size);
                v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
            } else {
                v[0] += from[k * size];
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (o.dtype == kBf16) store_as<kBf16>(o.out, i * o.step + j + e, v[e] * factor);
            else store_as<kF32>(o.out, i * o.step + j + e, v[e] * factor);
        }
    }
}

// ---- sums over rows ----

// A row's pairs joined, by `lanes` threads to a row: its log of the sum of exponentials and its loss, in the first of them.
struct Row {
    float lse, loss;
    bool counted;
};
__device__ __forceinline__ Row row_of(const XentArgs& a, const float2* pairs, int64_t tiles, const float* picked, int64_t row, int lane,
                                      int lanes)
{
    float m = -INFINITY, l = 0.0f, z = 0.0f;
    int64_t target = 0;
    if (row < a.M) {
        target = a.target[row];         // (on their way at once; of a row whose target is no class no one has written z)
        z = picked[row];
#pragma unroll 4
        for (int64_t i = lane; i < tiles; i += lanes) {
            const float2 p = pairs[i * a.M + row];
            join(m, l, p.x, p.y);
        }
    }
    for (int k = 1; k < lanes; k <<= 1) {
        const float om = __shfl_xor(m, k), ol = __shfl_xor(l, k);
        join(m, l, om, ol);
    }
    Row r{0.0f, 0.0f, false};
    if (row >= a.M || lane) return r;
    // (no class left: minus infinity; a logit of plus infinity: no probabilities)
    r.lse = m == INFINITY ? NAN : l > 0.0f ? m + logf(l) : l != l ? l : m;
    r.counted = target != a.ignore;
    if (r.counted) {
        const bool none = target < 0 || target >= a.N;          // (no class: seen in the loss and the gradients)
        if (none) r.lse = z = NAN;
        r.loss = z == -INFINITY && r.lse == r.lse ? INFINITY : r.lse - z;
    }
    return r;
}

// A row's share in the loss, in every thread, from each thread's sum and number of rows; `write`: that and the loss.
__device__ __forceinline__ float total_of(const XentArgs& a, double s, int n, bool write)
{
    __shared__ double sums[16];
    __shared__ int counts[16];
    s = wave_sum(s);
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = s; counts[threadIdx.x >> 6] = n; }
    __syncthreads();
    s = 0.0;
    n = 0;
    for (uint32_t w = 0; w < blockDim.x / kWave; ++w) { s += sums[w]; n += counts[w]; }
    const double share = a.reduction == kMean ? 1.0 / (double)(n > 0 ? n : 1) : 1.0;
    if (write && threadIdx.x == 0) {
        a.saved[a.M] = (float)share;
        if (a.reduction != kNone) a.loss[0] = (float)(s * share);
    }
    return (float)share;
}

// Where one workgroup has all rows (alone) it adds them up as well.
constexpr int kAlone = 512;
__global__ __launch_bounds__(kAlone) void xent_rows_kernel(XentArgs a, const float2* pairs, int64_t tiles, const float* picked, float* rows,
                                                           int lanes, int alone)
{
    const int lane = threadIdx.x & (lanes - 1), per = blockDim.x / lanes;
    double sum = 0.0;
    int count = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < a.M; row0 += (int64_t)gridDim.x * per) {
        const int64_t row = row0 + threadIdx.x / lanes;
        const Row r = row_of(a, pairs, tiles, picked, row, lane, lanes);
        if (row >= a.M || lane) continue;
        a.saved[row] = r.lse;
        if (!alone || a.reduction == kNone) rows[row] = r.loss;
        sum += (double)r.loss;
        count += r.counted;
    }
    if (alone) total_of(a, sum, count, true);
}

// one workgroup: the loss over all rows and a row's share in it
__global__ __launch_bounds__(1024) void xent_total_kernel(XentArgs a, const float* rows)
{
    double s = 0.0;
    int n = 0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < a.M; i += 1024) {
        s += (double)rows[i];
        n += a.target[i] != a.ignore;
    }
    total_of(a, s, n, true);
}

// db of a piece's classes: the tiles' sums of a class, sixteen threads to it (a launch more, 2 us, and dz is not read again)
__global__ __launch_bounds__(kThreads) void xent_dbias_kernel(const float* column, int64_t tiles, int64_t classes, void* dbias, OutArgs o)
{
    __shared__ float sums[16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + x;
    float s = 0.0f;
    if (c < classes)
#pragma unroll 4
        for (int64_t i = y; i < tiles; i += 16) s += column[i * classes + c];
    sums[y][x] = s;
    __syncthreads();
    if (y || c >= classes) return;
    for (int w = 1; w < 16; ++w) s += sums[w][x];
    s *= factor_of(o);
    if (o.dtype == kBf16) store_as<kBf16>(dbias, c, s);
    else store_as<kF32>(dbias, c, s);
}

// ---- small problems: straight from the operands, in 32 bits ----
//
// Packing, and products whose few tiles walk along the contraction one stage after the other, are most of what a small problem
// takes (128 x 512 x 100: 110 us, of it 13 packing, 80 in two products of one tile).  Here a workgroup of eight waves has
// 32 x 32 outputs, the waves share the contraction, sixteen bytes or four single elements a lane straight from memory, and
// the 32-bit matrix instructions multiply.  The logits stay in the workspace (kSmallLogits at most), and the gradients'
// products make dz from them as they read it: three launches forward and backward.

constexpr int kSmallWaves = 8, kSmallTile = 32;
constexpr int kSmallAhead = 4;                      // steps of eight of the contraction, four to a half of a wave's lanes, in flight
constexpr int kSmallSpan = 8 * kSmallAhead;         // of the contraction, side by side: a whole line of memory in fp32
constexpr int kSmallRound = kSmallSpan * kSmallWaves;
constexpr int kJoined = 2048;                       // rows, and pairs of them, that every workgroup of the gradients joins for itself
static_assert(kAlone == 64 * kSmallWaves, "sums in the same order as the rows' own launch");

struct SmallArgs {
    float* z;                           // [M][step], null: not wanted
    int64_t step;
    float2* pairs;                      // [tiles of classes][M]; null: not wanted
    float* picked;
    float* rows;                        // gradients that join the pairs: the rows' losses, where they are wanted
    int lanes;                          // and threads to a row
    uint32_t x_tiles, x_parts;          // gradients: tiles of dX, parts of its contraction; dW's tiles behind them
    uint32_t x_across, w_across;        // tiles side by side of dX (features), of the logits and dW (classes)
    uint32_t w_first;                   // first tile down of dW (where only db is wanted: the one with the line of ones)
    uint32_t w_tiles, w_parts;
    float *slices, *w_slices;           // of dX, of dW and db in parts: [part][M][K], [part][K + 1][N]
};

// four neighbours in memory, those from `left` on zero
template <int DT, bool VEC>
__device__ __forceinline__ void load4(const void* p, int64_t at, int64_t left, float (&v)[4])
{
    if constexpr (VEC) {                // (left is a multiple of four)
        if (left <= 0) {
            v[0] = v[1] = v[2] = v[3] = 0.0f;
        } else if (DT == kBf16) {
            const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
            v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
            v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
        } else {
            const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? load_as<DT>(p, at + e) : 0.0f;
    }
}

// The waves' sums of a 32 x 32 block added up: f(register, its number in this wave, sum) for the registers of this wave, in order
// of the waves.
template <class F>
__device__ __forceinline__ void join_waves(const v16f& acc, float (*lds)[16][64], int wave, int lane, F f)
{
#pragma unroll
    for (int e = 0; e < 16; ++e) lds[wave][e][lane] = acc[e];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16 / kSmallWaves; ++k) {
        const int e = wave * (16 / kSmallWaves) + k;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) s += lds[w][e][lane];
        f(e, k, s);
    }
}

// Lines of A are classes, of B rows, as in the large products.
template <int DT, bool VEC>
__global__ __launch_bounds__(64 * kSmallWaves) void xent_small_logits_kernel(XentArgs a, SmallArgs k)
{
    __shared__ float lds[kSmallWaves][16][64];
    __shared__ float z[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = lane & 31, half = lane >> 5;
    const uint32_t down = blockIdx.x / k.w_across, across = blockIdx.x - down * k.w_across;
    const int64_t class0 = (int64_t)across * kSmallTile, row0 = (int64_t)down * kSmallTile;
    const int64_t c = class0 + line, row = row0 + line;
    const bool class_there = c < a.N, row_there = row < a.M;
    const int64_t target = row_there ? a.target[row] : -1;
    float bias[16 / kSmallWaves];           // of the sums that this wave joins
#pragma unroll
    for (int q = 0; q < 16 / kSmallWaves; ++q) {
        const int e = wave * (16 / kSmallWaves) + q;
        const int64_t of = class0 + 8 * (e >> 2) + 4 * half + (e & 3);
        bias[q] = a.bias && of < a.N ? any_load(a.bias, a.bias_dtype, of) : 0.0f;
    }
    v16f acc = {};
    for (int64_t base = kSmallSpan * wave; base < a.K; base += kSmallRound) {
        float x[kSmallAhead][4], w[kSmallAhead][4];
#pragma unroll
        for (int u = 0; u < kSmallAhead; ++u) {
            const int64_t at = base + 8 * u + 4 * half;
            load4<DT, VEC>(a.X, row * a.ldx + at, row_there ? a.K - at : 0, x[u]);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[u][e] = class_there && at + e < a.K ? load_as<DT>(a.W, (at + e) * a.ldw + c) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kSmallAhead; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(w[u][e], x[u][e], acc, 0, 0, 0);
    }
    join_waves(acc, lds, wave, lane, [&](int e, int q, float s) {
        const int64_t of = class0 + 8 * (e >> 2) + 4 * half + (e & 3);
        z[e][lane] = of >= a.N ? -INFINITY : s + bias[q];
    });
    __syncthreads();
    if (wave) return;
    float v[16], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        v[e] = z[e][lane];
        top = fmaxf(top, v[e]);
        if (k.pairs && row_there && target == class0 + 8 * (e >> 2) + 4 * half + (e & 3)) k.picked[row] = v[e];
    }
    if (k.z && row_there)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (class0 + 8 * q + 4 * half < a.N)
                *reinterpret_cast<float4*>(k.z + row * k.step + class0 + 8 * q + 4 * half) =
                    make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    if (!k.pairs) return;
    top = larger_half(top);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += exp_of<true>(v[e] - base);
    sum = sum_halves(sum);
    if (row_there && half == 0) k.pairs[(int64_t)across * a.M + row] = make_float2(top, sum);
}

// dz of a logit
__device__ __forceinline__ float small_dz(float z, int64_t c, int64_t target, float lse, float factor)
{
    const float base = lse == -INFINITY ? 0.0f : lse;
    return (exp_of<true>(z - base) - (c == target ? 1.0f : 0.0f)) * factor;
}
// a part of a contraction: whole rounds of all waves
struct Share {
    int64_t begin, end;
};
__device__ __forceinline__ Share share_of(int64_t length, uint32_t part, uint32_t parts)
{
    const int64_t rounds = (length + kSmallRound - 1) / kSmallRound, per = (rounds + parts - 1) / parts * kSmallRound, begin = part * per;
    return {begin < length ? begin : length, begin + per < length ? begin + per : length};
}
__device__ __forceinline__ float row_factor(const XentArgs& a, int64_t row)
{
    return a.reduction == kNone && a.dloss ? a.dloss[row] : 1.0f;
}

// dX: lines of A are rows, of B features.  dW: lines of A features, and one of ones behind them, whose products are db; of B
// classes.
// JOIN: the forward pass has left the rows' pairs as they are.  Every workgroup joins all rows' for itself, and the first one
// writes what the forward pass owes: a launch less (1 x 561 x 11 16.8 us in three launches, 14.1 in two; 128 x 512 x 100 17.6 and
// 14.4).  Kernels this short wait for their own instructions: with the next round's loads in flight beside the products
// (half as much code again) they take 16.4 and 16.7, and large ones no less (32 x 256 x 64000 in fp32 by these kernels 405 us, without 217).
template <int DT, bool VEC, bool JOIN>
__global__ __launch_bounds__(64 * kSmallWaves) void xent_small_gradients_kernel(XentArgs a, SmallArgs k)
{
    __shared__ float lds[kSmallWaves][16][64];
    __shared__ float joined[JOIN ? kJoined : 1];
    float factor = a.reduction == kNone || !a.dloss ? 1.0f : *a.dloss;
    if constexpr (JOIN) {
        const int at = threadIdx.x & (k.lanes - 1), per = kAlone / k.lanes;
        double sum = 0.0;
        int count = 0;
        for (int64_t row0 = 0; row0 < a.M; row0 += per) {
            const int64_t row = row0 + threadIdx.x / k.lanes;
            const Row r = row_of(a, k.pairs, k.w_across, k.picked, row, at, k.lanes);
            if (row >= a.M || at) continue;
            joined[row] = r.lse;
            if (blockIdx.x == 0) {
                a.saved[row] = r.lse;
                if (a.reduction == kNone) k.rows[row] = r.loss;
            }
            sum += (double)r.loss;
            count += r.counted;
        }
        factor *= total_of(a, sum, count, blockIdx.x == 0);             // (its barrier stands before the first reader)
    } else {
        factor *= a.saved[a.M];
    }
    auto lse_of = [&](int64_t row) { return JOIN ? joined[row] : a.saved[row]; };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, line = lane & 31, half = lane >> 5;
    v16f acc = {};
    if (blockIdx.x < k.x_tiles * k.x_parts) {
        const uint32_t part = blockIdx.x / k.x_tiles, tile = blockIdx.x - part * k.x_tiles, down = tile / k.x_across;
        const int64_t row0 = (int64_t)down * kSmallTile, f0 = (int64_t)(tile - down * k.x_across) * kSmallTile;
        const int64_t row = row0 + line, f = f0 + line;
        const bool row_there = row < a.M, f_there = f < a.K;
        const int64_t target = row_there ? a.target[row] : -1;
        const bool counted = row_there && target != a.ignore;
        const float lse = row_there ? lse_of(row) : 0.0f, each = counted ? row_factor(a, row) : 0.0f;
        const Share share = share_of(a.N, part, k.x_parts);
        for (int64_t base = share.begin + kSmallSpan * wave; base < share.end; base += kSmallRound) {
            float z[kSmallAhead][4], w[kSmallAhead][4];
#pragma unroll
            for (int u = 0; u < kSmallAhead; ++u) {
                const int64_t at = base + 8 * u + 4 * half;
                load4<kF32, true>(k.z, row * k.step + at, counted && at < share.end ? 4 : 0, z[u]);
                load4<DT, VEC>(a.W, f * a.ldw + at, f_there ? share.end - at : 0, w[u]);
            }
#pragma unroll
            for (int u = 0; u < kSmallAhead; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t c = base + 8 * u + 4 * half + e;
                    const float d = counted && c < share.end ? small_dz(z[u][e], c, target, lse, each) : 0.0f;
                    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(d, w[u][e], acc, 0, 0, 0);
                }
        }
        join_waves(acc, lds, wave, lane, [&](int e, int, float s) {
            const int64_t i = row0 + 8 * (e >> 2) + 4 * half + (e & 3);
            if (i >= a.M || !f_there) return;
            if (k.x_parts > 1) k.slices[((int64_t)part * a.M + i) * a.K + f] = s;
            else store_as<DT>(a.dX, i * a.K + f, s * factor);
        });
        return;
    }
    const uint32_t at_w = blockIdx.x - k.x_tiles * k.x_parts, part = at_w / k.w_tiles, tile = at_w - part * k.w_tiles;
    const uint32_t down = k.w_first + tile / k.w_across;
    const int64_t f0 = (int64_t)down * kSmallTile, c0 = (int64_t)(tile % k.w_across) * kSmallTile;
    const int64_t f = f0 + line, c = c0 + line;
    const bool c_there = c < a.N;
    const Share share = share_of(a.M, part, k.w_parts);
    const bool each = a.reduction == kNone && a.dloss;
    for (int64_t base = share.begin + kSmallSpan / 2 * wave; base < share.end; base += kSmallRound / 2) {
        float x[kSmallAhead / 2][4], z[kSmallAhead / 2][4], lse[kSmallAhead / 2][4], g[kSmallAhead / 2][4];
        int64_t target[kSmallAhead / 2][4];
#pragma unroll
        for (int u = 0; u < kSmallAhead / 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t row = base + 8 * u + 4 * half + e, r = row < share.end ? row : share.end - 1;
                x[u][e] = row >= share.end ? 0.0f : f < a.K ? load_as<DT>(a.X, row * a.ldx + f) : f == a.K ? 1.0f : 0.0f;
                z[u][e] = row < share.end && c_there ? k.z[row * k.step + c] : 0.0f;
                target[u][e] = row < share.end ? a.target[r] : a.ignore;
                lse[u][e] = lse_of(r);
                g[u][e] = each ? a.dloss[r] : 1.0f;
            }
#pragma unroll
        for (int u = 0; u < kSmallAhead / 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = target[u][e] != a.ignore && c_there ? small_dz(z[u][e], c, target[u][e], lse[u][e], g[u][e]) : 0.0f;
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[u][e], d, acc, 0, 0, 0);
            }
    }
    join_waves(acc, lds, wave, lane, [&](int e, int, float s) {
        const int64_t i = f0 + 8 * (e >> 2) + 4 * half + (e & 3);
        if (!c_there) return;
        if (k.w_parts > 1) {
            if (i <= a.K) k.w_slices[((int64_t)part * (a.K + 1) + i) * a.N + c] = s;
            return;
        }
        if (i < a.K && a.dW) store_as<DT>(a.dW, i * a.N + c, s * factor);
        if (i == a.K && a.dbias) {
            if (a.bias_dtype == kBf16) store_as<kBf16>(a.dbias, c, s * factor);
            else store_as<kF32>(a.dbias, c, s * factor);
        }
    });
}

// dW and db of few rows (up to MM), fp32: a thread has four classes' dz of all of them in registers and writes kOuterLines lines of
// dW, so that only dW itself is moved (1 x 4096 x 128000 in fp32: 2 GB).
constexpr int kOuterLines = 64, kOuterRows = 16;
template <int MM>
__global__ __launch_bounds__(kThreads) void xent_outer_kernel(XentArgs a, SmallArgs k)
{
    __shared__ float x[MM][kOuterLines];
    const int64_t f0 = (int64_t)blockIdx.y * kOuterLines, c0 = (int64_t)blockIdx.x * (4 * kThreads) + threadIdx.x;
    const float factor = (a.reduction == kNone ? 1.0f : (a.dloss ? *a.dloss : 1.0f)) * a.saved[a.M];
    for (int i = threadIdx.x; i < MM * kOuterLines; i += kThreads) {
        const int m = i / kOuterLines, f = i % kOuterLines;
        x[m][f] = m < a.M && f0 + f < a.K ? load_as<kF32>(a.X, m * a.ldx + f0 + f) : 0.0f;
    }
    float d[MM][4];
#pragma unroll
    for (int m = 0; m < MM; ++m) {
        const bool counted = m < a.M && a.target[m < a.M ? m : 0] != a.ignore;
        const int64_t target = counted ? a.target[m] : -1;
        const float lse = counted ? a.saved[m] : 0.0f, each = counted ? row_factor(a, m) * factor : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = c0 + e * kThreads;
            d[m][e] = counted && c < a.N ? small_dz(k.z[m * k.step + c], c, target, lse, each) : 0.0f;
        }
    }
    __syncthreads();
    if (a.dbias && blockIdx.y == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = c0 + e * kThreads;
            float s = 0.0f;
#pragma unroll
            for (int m = 0; m < MM; ++m) s += d[m][e];
            if (c >= a.N) continue;
            if (a.bias_dtype == kBf16) store_as<kBf16>(a.dbias, c, s);
            else store_as<kF32>(a.dbias, c, s);
        }
    if (!a.dW) return;
    const int lines = a.K - f0 < kOuterLines ? (int)(a.K - f0) : kOuterLines;
    for (int f = 0; f < lines; ++f) {
        float s[4] = {};
#pragma unroll
        for (int m = 0; m < MM; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fmaf(x[m][f], d[m][e], s[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = c0 + e * kThreads;
            if (c < a.N) store_as<kF32>(a.dW, (f0 + f) * a.N + c, s[e]);
        }
    }
}

// dX's parts added up, and dW's and db's behind them
__global__ __launch_bounds__(kThreads) void xent_small_add_kernel(XentArgs a, SmallArgs k, int64_t of_x, int64_t of_w)
{
    const float factor = (a.reduction == kNone ? 1.0f : (a.dloss ? *a.dloss : 1.0f)) * a.saved[a.M];
    int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (at >= of_x + of_w) return;
    const bool x = at < of_x;
    at -= x ? 0 : of_x;
    const float* from = (x ? k.slices : k.w_slices) + at;
    const int64_t size = x ? a.M * a.K : (a.K + 1) * a.N;
    const uint32_t parts = x ? k.x_parts : k.w_parts;
    float v = 0.0f;
#pragma unroll 4
    for (uint32_t i = 0; i < parts; ++i) v += from[i * size];
    v *= factor;
    const bool bias = !x && at >= a.K * a.N;
    void* to = x ? a.dX : bias ? a.dbias : a.dW;
    if (!to) return;
    if (bias) at -= a.K * a.N;
    if ((bias ? a.bias_dtype : a.dtype) == kBf16) store_as<kBf16>(to, at, v);
    else store_as<kF32>(to, at, v);
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// How a product is cut: large tiles of 256 x 256 (one plane) or 256 x 128 (three), one to a compute unit, or small ones of
// 128 x 128 or 128 x 64, two to a compute unit; and the contraction in parts, which another launch adds up.
struct Cut {
    int a, b;
    bool large;
    uint32_t parts;
    double us;
};

// The cut that a simple model of the time likes best, microseconds: rounds of the workgroups that the chip holds (256, 512), each
// as many stages as a part has, at what a stage takes on a full chip, and 5 to begin and end; for parts the sums written, read
// again at 4 TB/s, and a launch, once for all pieces.  (Stages measured, large and small tiles: 8192 x 4096 x 8192 in bfloat16
// 1.85 and 1.05, in fp32 2.8 and 1.4; 0.75 and 0.8 where a compute unit has one of the small.  What the model chooses between,
// forward, both ways: 2048 cubed in bfloat16 51 and 30 us, 8192 x 4096 x 8192 474 and 537; in fp32 137 and 100, 512 x 1024 x 32768 174 and 196,
// 10000 x 512 x 1000 100 and 71.  Small tiles of 128 x 128 in fp32, one to a compute unit and three stages in LDS: 93, 190, 82.)
Cut cut_of(int64_t RA, int64_t RB, int64_t D, int planes, bool may_split, int64_t pieces = 1)
{
    Cut best{};
    const int64_t stages = (D + bf16::stage_of(planes) - 1) / bf16::stage_of(planes);
    for (const bool large : {true, false}) {
        Cut c{large ? 256 : 128, large ? (planes == 1 ? 256 : 128) : planes == 1 ? 128 : 64, large, 1, 0.0};
        const int64_t tiles = ((RA + c.a - 1) / c.a) * ((RB + c.b - 1) / c.b);
        for (int64_t parts = 1; parts <= 64; ++parts) {
            if (parts > 1 && (!may_split || tiles * parts > 1024 || stages < 4 * parts)) break;
            const int64_t groups = tiles * parts, slots = large ? 256 : 512;
            const double stage = large ? (planes == 1 ? 1.85 : 2.8) : groups > 256 ? (planes == 1 ? 1.05 : 1.4) : planes == 1 ? 0.75 : 0.8;
            double t = (double)((groups + slots - 1) / slots) * ((double)((stages + parts - 1) / parts) * stage + 5.0);
            if (parts > 1) t += (6.0 + 4.0 * (double)(2 * parts + 1) * (double)RA * (double)RB / 4.0e6) / (double)pieces;
            if (best.a == 0 || t < best.us) { best = c; best.parts = (uint32_t)parts; best.us = t; }
        }
    }
    return best;
}

// dz of a piece, and logits that a step keeps, stay within what the memory-side cache holds between their writer and their readers
constexpr int64_t kPieceBytes = (int64_t)128 << 20;

// How a call is cut, and where its pieces of the workspace lie.
struct Plan {
    int planes;                         // 3: fp32
    bool pack_x, pack_w;
    bool whole_w;                       // W is packed as a whole, once for both directions
    int64_t piece;                      // classes of a piece
    int64_t x_step, w_step, dz_step;    // of packed rows, of dz
    size_t x, w;                        // bytes of X packed, of W or a piece of it packed
    size_t pairs, picked, rows;         // forward
    Cut dx;
    size_t dz, dx_slices, slices, column;          // backward
    bool keeps;                         // a step of this size keeps the logits,
    size_t z;                           // in front of those; 0: this call does not
};

bool whole_rows(const void* p, int64_t ld, int64_t cols, int dtype)
{
    return dtype == kBf16 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < (int64_t)1 << 21;
}

// (sizes: for any alignment of the operands; step: the forward and the backward pass in one call)
Plan plan_of(const XentArgs& a, bool sizes, bool step)
{
    Plan p{};
    p.planes = a.dtype == kF32 ? 3 : 1;
    p.pack_x = sizes || !whole_rows(a.X, a.ldx, a.K, a.dtype);
    p.pack_w = sizes || !whole_rows(a.W, a.ldw, a.N, a.dtype);
    p.piece = kPieceBytes / (2 * p.planes * a.M) / 256 * 256;
    if (p.piece < 1024) p.piece = 1024;
    if (p.piece > 65536) p.piece = 65536;
    if (p.piece > a.N) p.piece = a.N;
    const int64_t unit = p.planes == 1 ? 8 : 32;
    p.x_step = p.planes * up(a.K, unit);
    p.whole_w = a.K * a.N <= ((int64_t)256 << 20) / (2 * p.planes);
    p.w_step = p.planes * up(p.whole_w ? a.N : p.piece, unit);
    p.dz_step = p.planes * up(p.piece, 256);
    p.x = p.pack_x ? up256(2 * (size_t)a.M * p.x_step) : 0;
    p.w = p.pack_w ? up256(2 * (size_t)a.K * p.w_step) : 0;
    p.pairs = up256(sizeof(float2) * ((a.N + 127) / 128 + (a.N + p.piece - 1) / p.piece) * a.M);
    p.picked = p.rows = up256(sizeof(float) * a.M);
    p.dz = up256(2 * (size_t)a.M * p.dz_step);
    // (dX is cut alike for all pieces: its parts' sums are kept from one to the next)
    p.dx = cut_of(a.M, a.K, p.piece, p.planes, true, (a.N + p.piece - 1) / p.piece);
    p.dx_slices = p.dx.parts > 1 || p.piece < a.N ? up256(sizeof(float) * p.dx.parts * a.M * a.K) : 0;
    // in fp32, where the classes are one piece, a step keeps the logits: 4 bytes each, written and read, against six products.  (A backward
    // call of its own multiplies them in the launch that makes dz: 777 x 320 x 10007 154.5 us, by way of the logits 155.2; 512 x 2048 x
    // 1000 105 and 111, 128 x 512 x 10000 68 and 75.  What a step loses by the bound: 50000 x 512 x 1000 1164 us, 1392 without its 205 MB.)
    const int64_t z = (int64_t)sizeof(float) * a.M * up(a.N, 256);
    p.keeps = p.planes == 3 && p.piece == a.N && z <= kPieceBytes;
    p.z = step && p.keeps ? up256((size_t)z) : 0;
    const int64_t rows = p.keeps ? kRowsOfDz : p.planes == 3 ? 64 : 128;        // (the smaller tiles')
    p.column = up256(sizeof(float) * (size_t)((a.M + rows - 1) / rows) * p.piece);
    size_t most = 0;
    for (const int64_t classes : {p.piece, a.N - (a.N - 1) / p.piece * p.piece}) {          // (the last piece's dW may be cut another way)
        const size_t parts = cut_of(a.K, classes, a.M, p.planes, true).parts, bytes = parts > 1 ? parts * a.K * classes : 0;
        if (bytes > most) most = bytes;
    }
    p.slices = up256(sizeof(float) * most);
    return p;
}

PackArgs pack_of(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, uint16_t* dst, int64_t step)
{
    const int64_t pairs = (dtype == kBf16 ? step : step / 3) / 2;
    return {src, rows, cols, ld, dst, step, (uint32_t)((pairs + kThreads - 1) / kThreads), 0};
}
// its first rows, as many as kPackGroups workgroups have (a launch has fewer than 2^32 threads: of both operands 2^31 at most)
constexpr int64_t kPackGroups = (int64_t)1 << 22;
PackArgs take_rows(PackArgs* a, int64_t size)
{
    PackArgs first = *a;
    if (!a->rows) return first;
    const int64_t most = kPackGroups / a->across * kPackRows;
    if (first.rows > most) first.rows = most;
    first.groups = a->across * (uint32_t)((first.rows + kPackRows - 1) / kPackRows);
    a->rows -= first.rows;
    a->src = static_cast<const char*>(a->src) + first.rows * a->ld * size;
    a->dst += first.rows * a->step;
    return first;
}
// (either may be empty)
hipError_t launch_pack(PackArgs one, PackArgs other, int dtype, hipStream_t stream)
{
    while (one.rows || other.rows) {
        const PackArgs p = take_rows(&one, dtype_size(dtype)), q = take_rows(&other, dtype_size(dtype));
        const dim3 grid(p.groups + q.groups);
        ProfileScope ps(K_XENT_PACK, stream);
        if (dtype == kBf16) hipLaunchKernelGGL(xent_pack_kernel<kBf16>, grid, dim3(kThreads), 0, stream, p, q);
        else hipLaunchKernelGGL(xent_pack_kernel<kF32>, grid, dim3(kThreads), 0, stream, p, q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool GRAD>
hipError_t launch_logits(int tag, const bf16::Args& g, const RowArgs& r, int planes, bool large, hipStream_t stream)
{
    ProfileScope ps(tag, stream);
    const dim3 grid(8 * g.per_xcd);
    if (planes == 1) {
        if (large) hipLaunchKernelGGL((xent_logits_kernel<GRAD, 1, 256, 256, 2, 4>), grid, dim3(512), 0, stream, g, r);
        else hipLaunchKernelGGL((xent_logits_kernel<GRAD, 1, 128, 128, 2, 2>), grid, dim3(256), 0, stream, g, r);
    } else {
        if (large) hipLaunchKernelGGL((xent_logits_kernel<GRAD, 3, 256, 128, 4, 2>), grid, dim3(512), 0, stream, g, r);
        else hipLaunchKernelGGL((xent_logits_kernel<GRAD, 3, 128, 64, 2, 2>), grid, dim3(256), 0, stream, g, r);
    }
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_gradient(int tag, const bf16::Args& g, const OutArgs& o, int planes, bool large, hipStream_t stream)
{
    {
        ProfileScope ps(tag, stream);
        const dim3 grid(8 * g.per_xcd);
        if (planes == 1) {
            if (large) hipLaunchKernelGGL((xent_gradient_kernel<1, MODE, 256, 256, 2, 4>), grid, dim3(512), 0, stream, g, o);
            else hipLaunchKernelGGL((xent_gradient_kernel<1, MODE, 128, 128, 2, 2>), grid, dim3(256), 0, stream, g, o);
        } else {
            if (large) hipLaunchKernelGGL((xent_gradient_kernel<3, MODE, 256, 128, 4, 2>), grid, dim3(512), 0, stream, g, o);
            else hipLaunchKernelGGL((xent_gradient_kernel<3, MODE, 128, 64, 2, 2>), grid, dim3(256), 0, stream, g, o);
        }
    }
    if (o.parts > 1 && o.last_piece) {
        ProfileScope ps(K_XENT_ADD_PARTS, stream);
        const uint32_t down = (uint32_t)(g.RA < 65535 ? g.RA : 65535);
        if (g.RB % 4 == 0)
            hipLaunchKernelGGL(xent_add_parts_kernel<4>, dim3((uint32_t)((g.RB / 4 + kThreads - 1) / kThreads), down), dim3(kThreads), 0, stream,
                               o, g.RA, g.RB);
        else
            hipLaunchKernelGGL(xent_add_parts_kernel<1>, dim3((uint32_t)((g.RB + kThreads - 1) / kThreads), down), dim3(kThreads), 0, stream,
                               o, g.RA, g.RB);
    }
    return hipGetLastError();
}

// X and a piece of W as the products take them; `have`: another pass has just left them in this workspace
struct Operands {
    bf16::Side x, w;
};
hipError_t operands_of(const XentArgs& a, const Plan& p, char* workspace, int64_t first, int64_t classes, bool have, Operands* o,
                       hipStream_t stream)
{
    const int64_t size = dtype_size(a.dtype);
    const char* w = static_cast<const char*>(a.W) + first * size;
    uint16_t *px = reinterpret_cast<uint16_t*>(workspace), *pw = reinterpret_cast<uint16_t*>(workspace + p.x);
    o->x = p.pack_x ? bf16::Side{px, p.x_step} : bf16::Side{static_cast<const uint16_t*>(a.X), a.ldx};
    o->w = p.pack_w ? bf16::Side{pw + (p.whole_w ? p.planes * first : 0), p.w_step} : bf16::Side{reinterpret_cast<const uint16_t*>(w), a.ldw};
    PackArgs x{}, of_w{};
    if (p.pack_x && !have && first == 0) x = pack_of(a.X, a.dtype, a.M, a.K, a.ldx, px, p.x_step);
    if (p.pack_w && p.whole_w && !have && first == 0) of_w = pack_of(a.W, a.dtype, a.K, a.N, a.ldw, pw, p.w_step);
    if (p.pack_w && !p.whole_w && !(have && p.piece == a.N)) of_w = pack_of(w, a.dtype, a.K, classes, a.ldw, pw, p.w_step);
    return launch_pack(x, of_w, a.dtype, stream);
}

int lanes_of(int64_t tiles)
{
    int lanes = 1;
    while (lanes < 64 && 4 * lanes < tiles) lanes *= 2;
    return lanes;
}
// (four rounds of a workgroup at most: less than another launch)
bool rows_alone(const XentArgs& a, int64_t tiles) { return a.M * lanes_of(tiles) <= 4 * kAlone; }

// from the tiles' pairs to the loss
hipError_t launch_rows(const XentArgs& a, const float2* pairs, int64_t tiles, const float* picked, float* rows, hipStream_t stream)
{
    ProfileScope ps(K_XENT_LOSS, stream);
    const int lanes = lanes_of(tiles);
    if (rows_alone(a, tiles)) {
        hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(kAlone), 0, stream, a, pairs, tiles, picked, rows, lanes, 1);
        return hipGetLastError();
    }
    const int64_t per = kThreads / lanes;
    const dim3 grid((uint32_t)((a.M + per - 1) / per));
    hipLaunchKernelGGL(xent_rows_kernel, grid, dim3(kThreads), 0, stream, a, pairs, tiles, picked, rows, lanes, 0);
    hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(1024), 0, stream, a, rows);
    return hipGetLastError();
}

RowArgs rows_of(const XentArgs& a, int64_t first, int64_t classes)
{
    RowArgs r{};
    r.bias = a.bias ? static_cast<const char*>(a.bias) + first * dtype_size(a.bias_dtype) : nullptr;
    r.bias_dtype = a.bias_dtype; r.classes = classes; r.first_class = first; r.target = a.target; r.ignore = a.ignore; r.M = a.M;
    return r;
}

// ---- small problems ----

constexpr int64_t kSmallLogits = (int64_t)8 << 20;          // of 4 bytes

// (of fewer outputs a launch more is not worth it; bfloat16 problems of so many are not small)
bool few_rows(const XentArgs& a) { return a.dtype == kF32 && a.M <= kOuterRows && a.K * a.N >= (int64_t)4 << 20; }

struct SmallPlan {
    int64_t class_tiles, row_tiles, step;
    uint32_t x_parts, w_parts;              // of dX's and dW's contractions
    size_t z, pairs, picked, rows, x_slices, w_slices;
};
// (gradients: they will be asked for, and read the logits)
SmallPlan small_plan(const XentArgs& a, bool gradients)
{
    SmallPlan p{};
    p.class_tiles = (a.N + kSmallTile - 1) / kSmallTile;
    p.row_tiles = (a.M + kSmallTile - 1) / kSmallTile;
    p.step = up(a.N, 4);
    // where tiles are few several workgroups share a contraction: up to two for a compute unit, two rounds each at least
    auto parts = [](int64_t tiles, int64_t length) {
        const int64_t most = length / (2 * kSmallRound), n = 512 / tiles < most ? 512 / tiles : most;
        return (uint32_t)(n < 1 ? 1 : n);
    };
    p.x_parts = parts(p.row_tiles * ((a.K + kSmallTile - 1) / kSmallTile), a.N);
    p.w_parts = parts(p.class_tiles * (a.K / kSmallTile + 1), a.M);
    p.z = gradients ? up256(sizeof(float) * a.M * p.step) : 0;
    p.pairs = up256(sizeof(float2) * p.class_tiles * a.M);
    p.picked = p.rows = up256(sizeof(float) * a.M);
    p.x_slices = p.x_parts > 1 ? up256(sizeof(float) * p.x_parts * a.M * a.K) : 0;
    p.w_slices = p.w_parts > 1 ? up256(sizeof(float) * p.w_parts * (a.K + 1) * a.N) : 0;
    return p;
}

// Whether a problem is small.  bfloat16: the large products' seven launches are what they take (128 x 512 x 1000 44 us, here 34;
// 512 x 512 x 100 49 and 30; 2048 x 512 x 100 51 and 52), unless W is large, whose single elements are read here (1 x 512 x 33000
// 74 and 298).  fp32: by models of a step's time, microseconds.  Here 512 workgroups at a time, 2 to begin and 3 for every
// round of the contraction, dW's 1 and 4, and a third for each round of the longest chain; of few rows dW at 4 TB/s.  There
// the cuts', what the packing and the logits move at 3.5 TB/s, and 14.  (Fitted to 29 problems, of which both choose the faster
// way, here and there: 128 x 512 x 1000 30 and 59, 512 x 512 x 1000 56 and 72, 32 x 2048 x 4000 101 and 113, 512 x 2048 x 1000 148 and
// 119, 128 x 512 x 10000 119 and 84, 8192 x 512 x 100 102 and 84, 8192 x 64 x 100 39 and 65, 1 x 4096 x 128000 1508 and 4702.)
bool small_problem(const XentArgs& a)
{
    if (a.M * a.N > kSmallLogits) return false;
    if (a.dtype == kBf16) return a.K * a.N <= ((int64_t)3 << 19) && a.M * a.N <= ((int64_t)1 << 26) / a.K;
    const SmallPlan p = small_plan(a, true);
    const double kn = (double)a.K * (double)a.N, mk = (double)a.M * (double)a.K, mn = (double)a.M * (double)a.N;
    auto rounds = [](int64_t length, int64_t of, uint32_t parts) {
        const int64_t n = (length + of - 1) / of;
        return (double)((n + parts - 1) / parts);
    };
    const double z = rounds(a.K, kSmallRound, 1), x = rounds(a.N, kSmallRound, p.x_parts), w = rounds(a.M, kSmallRound / 2, p.w_parts);
    const double k_tiles = (double)((a.K + kSmallTile - 1) / kSmallTile), with_ones = (double)(a.K / kSmallTile + 1);
    double here = 14.0 + 0.35 * (z + (x > w ? x : w));
    here += (double)(p.row_tiles * p.class_tiles) / 512.0 * (2.0 + 3.0 * z) + (double)p.row_tiles * k_tiles * p.x_parts / 512.0 * (2.0 + 3.0 * x);
    if (few_rows(a)) here += 4.0 + 4.0 * kn / 4.0e6;
    else here += (double)p.class_tiles * with_ones * p.w_parts / 512.0 * (1.0 + 4.2 * w);
    const double large = 14.0 + cut_of(a.N, a.M, a.K, 3, false).us + cut_of(a.M, a.K, a.N, 3, true).us + cut_of(a.K, a.N, a.M, 3, true).us +
                         (10.0 * (kn + mk) + 14.0 * mn) / 3.5e6;
    return here <= large;
}

// f(type, whole sixteen or eight bytes)
template <class F>
void with_small(const XentArgs& a, bool vec, F f)
{
    using std::integral_constant;
    if (a.dtype == kBf16) {
        if (vec) f(integral_constant<int, kBf16>{}, std::true_type{});
        else f(integral_constant<int, kBf16>{}, std::false_type{});
    } else {
        if (vec) f(integral_constant<int, kF32>{}, std::true_type{});
        else f(integral_constant<int, kF32>{}, std::false_type{});
    }
}
bool fours(const void* p, int64_t ld, int64_t cols, int dtype)
{
    return reinterpret_cast<uintptr_t>(p) % (size_t)(4 * dtype_size(dtype)) == 0 && ld % 4 == 0 && cols % 4 == 0;
}

bool outer_problem(const XentArgs& a) { return (a.dW || a.dbias) && few_rows(a); }
// whether a step's gradients join the rows' pairs for themselves: few of them
bool joins(const XentArgs& a, const SmallPlan& p)
{
    return !outer_problem(a) && rows_alone(a, p.class_tiles) && p.class_tiles * a.M <= kJoined;
}

// forward: the loss; keep: the logits for the gradients, which may follow
hipError_t launch_small_logits(const XentArgs& a, const SmallPlan& p, char* at, bool forward, bool keep, hipStream_t stream)
{
    SmallArgs k{};
    if (keep) k.z = reinterpret_cast<float*>(at);
    k.step = p.step;
    k.w_across = (uint32_t)p.class_tiles;
    if (forward) {
        k.pairs = reinterpret_cast<float2*>(at + p.z);
        k.picked = reinterpret_cast<float*>(at + p.z + p.pairs);
    }
    {
        ProfileScope ps(K_XENT_LOGITS, stream);
        with_small(a, fours(a.X, a.ldx, a.K, a.dtype), [&](auto dt, auto vec) {
            hipLaunchKernelGGL((xent_small_logits_kernel<dt.value, vec.value>), dim3((uint32_t)(p.class_tiles * p.row_tiles)),
                               dim3(64 * kSmallWaves), 0, stream, a, k);
        });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !forward || (keep && joins(a, p))) return e;
    float* rows = a.reduction == kNone ? a.loss : reinterpret_cast<float*>(at + p.z + p.pairs + p.picked);
    return launch_rows(a, k.pairs, p.class_tiles, k.picked, rows, stream);
}

hipError_t launch_small_gradients(const XentArgs& a, const SmallPlan& p, char* at, bool forward, hipStream_t stream)
{
    SmallArgs k{};
    const bool join = forward && joins(a, p);
    k.pairs = reinterpret_cast<float2*>(at + p.z);
    k.picked = reinterpret_cast<float*>(at + p.z + p.pairs);
    k.rows = a.loss;
    k.lanes = lanes_of(p.class_tiles);
    k.z = reinterpret_cast<float*>(at);
    k.step = p.step;
    k.x_across = (uint32_t)((a.K + kSmallTile - 1) / kSmallTile);
    k.x_tiles = a.dX ? (uint32_t)p.row_tiles * k.x_across : 0;
    k.x_parts = p.x_parts;
    k.w_parts = p.w_parts;
    k.w_across = (uint32_t)p.class_tiles;
    k.slices = reinterpret_cast<float*>(at + p.z + p.pairs + p.picked + p.rows);
    k.w_slices = k.slices + p.x_slices / sizeof(float);
    // (the line of ones may begin a tile of its own)
    const uint32_t w_end = (uint32_t)((a.K + (a.dbias ? 1 : 0) + kSmallTile - 1) / kSmallTile);
    k.w_first = a.dW ? 0 : a.dbias ? w_end - 1 : w_end;
    k.w_tiles = (w_end - k.w_first) * k.w_across;
    if (outer_problem(a)) {
        k.w_tiles = 0;
        const dim3 grid((uint32_t)((a.N + 4 * kThreads - 1) / (4 * kThreads)), a.dW ? (uint32_t)((a.K + kOuterLines - 1) / kOuterLines) : 1);
        ProfileScope ps(K_XENT_DW, stream);
        if (a.M <= 2) hipLaunchKernelGGL(xent_outer_kernel<2>, grid, dim3(kThreads), 0, stream, a, k);
        else if (a.M <= 8) hipLaunchKernelGGL(xent_outer_kernel<8>, grid, dim3(kThreads), 0, stream, a, k);
        else hipLaunchKernelGGL(xent_outer_kernel<kOuterRows>, grid, dim3(kThreads), 0, stream, a, k);
    }
    if (k.x_tiles || k.w_tiles) {
        ProfileScope ps(K_XENT_DX, stream);
        with_small(a, fours(a.W, a.ldw, a.N, a.dtype), [&](auto dt, auto vec) {
            const dim3 grid(k.x_tiles * k.x_parts + k.w_tiles * k.w_parts), block(64 * kSmallWaves);
            if (join) hipLaunchKernelGGL((xent_small_gradients_kernel<dt.value, vec.value, true>), grid, block, 0, stream, a, k);
            else hipLaunchKernelGGL((xent_small_gradients_kernel<dt.value, vec.value, false>), grid, block, 0, stream, a, k);
        });
    }
    const int64_t of_x = a.dX && p.x_parts > 1 ? a.M * a.K : 0, of_w = k.w_tiles && p.w_parts > 1 ? (a.K + 1) * a.N : 0;
    if (of_x + of_w) {
        ProfileScope ps(K_XENT_ADD_PARTS, stream);
        hipLaunchKernelGGL(xent_small_add_kernel, dim3((uint32_t)((of_x + of_w + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a, k,
                           of_x, of_w);
    }
    return hipGetLastError();
}

} // namespace

size_t xent_workspace(const XentArgs& a, bool forward, bool backward)
{
    if (small_problem(a)) {
        const SmallPlan p = small_plan(a, backward);
        return p.z + p.pairs + p.picked + p.rows + (backward ? p.x_slices + p.w_slices : 0);
    }
    const Plan p = plan_of(a, true, forward && backward);
    const size_t f = forward ? p.pairs + p.picked + p.rows : 0, b = backward ? p.dz + p.dx_slices + p.slices + p.column : 0;
    return p.x + p.w + p.z + (f > b ? f : b);
}

hipError_t launch_xent_fwd(const XentArgs& a, void* workspace, bool backward, hipStream_t stream)
{
    if (small_problem(a)) return launch_small_logits(a, small_plan(a, backward), static_cast<char*>(workspace), true, backward, stream);
    const Plan p = plan_of(a, false, backward);
    char* at = static_cast<char*>(workspace) + p.x + p.w;
    char* rest = at + p.z;
    float2* pairs = reinterpret_cast<float2*>(rest);
    float* picked = reinterpret_cast<float*>(rest + p.pairs);
    float* rows = a.reduction == kNone ? a.loss : reinterpret_cast<float*>(rest + p.pairs + p.picked);
    hipError_t e;
    int64_t tiles = 0;
    for (int64_t first = 0; first < a.N; first += p.piece) {
        const int64_t classes = a.N - first < p.piece ? a.N - first : p.piece;
        Operands o;
        if ((e = operands_of(a, p, static_cast<char*>(workspace), first, classes, false, &o, stream)) != hipSuccess) return e;
        RowArgs r = rows_of(a, first, classes);
        r.pairs = pairs + tiles * a.M;
        r.picked = picked;
        if (p.z) r.z = reinterpret_cast<float*>(at);
        r.z_step = up(a.N, 256);
        const Cut t = cut_of(classes, a.M, a.K, p.planes, false);
        const bf16::Args g = bf16::plan(o.w, o.x, classes, a.M, a.K, p.planes, t.a, t.b, 1);
        if ((e = launch_logits<false>(K_XENT_LOGITS, g, r, p.planes, t.large, stream)) != hipSuccess) return e;
        tiles += g.n_at;
    }
    return launch_rows(a, pairs, tiles, picked, rows, stream);
}

// forward: the forward pass has just run in the same workspace
hipError_t launch_xent_bwd(const XentArgs& a, void* workspace, bool forward, hipStream_t stream)
{
    hipError_t e;
    if (small_problem(a)) {
        const SmallPlan s = small_plan(a, true);
        if (!forward && (e = launch_small_logits(a, s, static_cast<char*>(workspace), false, true, stream)) != hipSuccess) return e;
        return launch_small_gradients(a, s, static_cast<char*>(workspace), forward, stream);
    }
    const Plan p = plan_of(a, false, forward);
    float* z = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.x + p.w);
    char* at = reinterpret_cast<char*>(z) + p.z;
    uint32_t dx_parts = 1;
    for (int64_t first = 0; first < a.N; first += p.piece) {
        const int64_t classes = a.N - first < p.piece ? a.N - first : p.piece;
        Operands o;
        if ((e = operands_of(a, p, static_cast<char*>(workspace), first, classes, forward, &o, stream)) != hipSuccess)
            return e;
        RowArgs r = rows_of(a, first, classes);
        r.saved = a.saved; r.dloss = a.dloss; r.each = a.reduction == kNone;
        r.dz = reinterpret_cast<uint16_t*>(at);
        r.step = p.dz_step;
        if (a.dbias) r.column = reinterpret_cast<float*>(at + p.dz + p.dx_slices + p.slices);
        Cut t = cut_of(classes, a.M, a.K, p.planes, false);
        bf16::Args g = bf16::plan(o.w, o.x, classes, a.M, a.K, p.planes, t.a, t.b, 1);
        r.eights = p.keeps;
        const uint32_t row_tiles = p.keeps ? (uint32_t)((a.M + kRowsOfDz - 1) / kRowsOfDz) : g.n_bt;
        if (p.z) {
            r.z = z;
            r.z_step = up(a.N, 256);
            ProfileScope ps(K_XENT_DLOGITS, stream);
            // (rows along x: they may be more than 65535 workgroups)
            hipLaunchKernelGGL(xent_dz_kernel, dim3(row_tiles, (uint32_t)((p.dz_step / 3 + 4 * kThreads - 1) / (4 * kThreads))), dim3(kThreads), 0,
                               stream, r);
            e = hipGetLastError();
        } else {
            e = launch_logits<true>(K_XENT_DLOGITS, g, r, p.planes, t.large, stream);
        }
        if (e != hipSuccess) return e;
        const bf16::Side dz{r.dz, r.step};
        OutArgs out{};
        out.dtype = a.dtype; out.share = a.saved + a.M; out.dloss = r.each ? nullptr : a.dloss;
        out.slices = reinterpret_cast<float*>(at + p.dz + p.dx_slices);
        out.first_piece = out.last_piece = 1;
        if (a.dX) {
            OutArgs x = out;
            x.out = a.dX; x.step = a.K;
            x.slices = reinterpret_cast<float*>(at + p.dz);
            x.first_piece = first == 0; x.last_piece = first + classes == a.N;
            g = bf16::plan(dz, o.w, a.M, a.K, classes, p.planes, p.dx.a, p.dx.b, p.dx.parts);
            if (first == 0) dx_parts = g.parts;
            x.parts = dx_parts;
            if ((e = launch_gradient<kAlong>(K_XENT_DX, g, x, p.planes, p.dx.large, stream)) != hipSuccess) return e;
        }
        if (a.dW) {
            OutArgs w = out;
            w.out = static_cast<char*>(a.dW) + first * dtype_size(a.dtype); w.step = a.N;
            t = cut_of(a.K, classes, a.M, p.planes, true);
            g = bf16::plan(o.x, dz, a.K, classes, a.M, p.planes, t.a, t.b, t.parts);
            w.parts = g.parts;
            if ((e = launch_gradient<kDown>(K_XENT_DW, g, w, p.planes, t.large, stream)) != hipSuccess) return e;
        }
        if (a.dbias) {
            OutArgs b = out;
            b.dtype = a.bias_dtype;
            void* to = static_cast<char*>(a.dbias) + first * dtype_size(a.bias_dtype);
            ProfileScope ps(K_XENT_DBIAS, stream);
            hipLaunchKernelGGL(xent_dbias_kernel, dim3((uint32_t)((classes + 15) / 16)), dim3(kThreads), 0, stream, r.column, row_tiles, classes,
                               to, b);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

} // namespace hdqt
