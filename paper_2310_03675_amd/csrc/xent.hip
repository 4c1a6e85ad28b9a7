// Softmax cross entropy of a linear classifier over N classes, in pieces of the classes, without the logits in memory
// (gfx950):
//   z = X W + b,  lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,target(i)  (0 where the target is to be ignored)
//   dz_ij = g_i (exp(z_ij - lse_i) - [j = target(i)]),  dX = dz W^T,  dW = X^T dz,  db = sum_i dz_ij
// Forward, every tile of the product leaves the largest logit of a row and the sum of exponentials relative to it; a
// second launch joins a row's pairs.  Backward, the logits of a piece of the classes are multiplied again and become dz in
// the workspace, from which the three gradients are taken; dX is added up over the pieces in 32 bits.
//
// The matrix pipe bounds it: four products of 2 M K N operations forward and backward, of which three are what the
// gradients need and one is what not keeping the logits costs.
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
// is |t| 2^-24 of the result.
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
    if (om == -INFINITY && ol == 0.0f) return;
    if (m == -INFINITY && l == 0.0f) { m = om; l = ol; return; }
    const float top = om > m ? om : m;
    l = l * expf(m - top) + ol * expf(om - top);
    m = top;
}

// ---- operands as the products take them: rows of whole 16 bytes, in planes where they are fp32 ----

struct PackArgs {
    const void* src;
    int64_t rows, cols, ld;
    uint16_t* dst;
    int64_t step, plane;
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

template <int DT>
__global__ __launch_bounds__(kThreads) void xent_pack_kernel(PackArgs a)
{
    const int64_t c = 2 * ((int64_t)blockIdx.x * kThreads + threadIdx.x);
    if (c >= a.step) return;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const int64_t from = row * a.ld + c;
        const float x = c < a.cols ? load_as<DT>(a.src, from) : 0.0f, y = c + 1 < a.cols ? load_as<DT>(a.src, from + 1) : 0.0f;
        uint32_t* to = reinterpret_cast<uint32_t*>(a.dst + row * a.step + c);
        if (DT == kBf16) {
            *to = __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xFFFF0000u);
        } else {
            uint32_t p[3], q[3];
            split(x, p);
            split(y, q);
#pragma unroll
            for (int k = 0; k < 3; ++k) to[k * (a.plane / 2)] = p[k] | q[k] << 16;
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
    int64_t step, plane;
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

// Lines of A are classes (W, read down), lines of B rows (X): a lane then holds sums of one row of the logits, and the
// maximum and the sum over classes stay inside it but for one exchange between the wave's halves.
template <bool GRAD, bool PLANES, int TA, int TB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB) __attribute__((amdgpu_waves_per_eu(2, 2))) void xent_logits_kernel(bf16::Args g, RowArgs r)
{
    constexpr int NA = TA / WA / 32, NB = TB / WB / 32;
    __shared__ __align__(1024) uint8_t a0[128 * TA], a1[128 * TA], b0[128 * TB], b1[128 * TB];
    __shared__ __align__(16) float bias[TA];
    __shared__ float2 halves[WA][TB];
    const bf16::Place p = bf16::place_of(g);
    if (!p.there) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (int t = threadIdx.x; t < TA; t += 64 * WA * WB) {
        const int64_t c = (int64_t)p.at * TA + t;
        bias[t] = c >= r.classes ? -INFINITY : r.bias ? any_load(r.bias, r.bias_dtype, c) : 0.0f;
    }
    v16f acc[NA][NB] = {};
    bf16::multiply<kDown, kAlong, TA, TB, WA, WB>(g, p, a0, a1, b0, b1, wave, lane, acc);

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
            top = larger_half(top);
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += exp_of<PLANES>(acc[i][j][e] - base);
            sum = sum_halves(sum);
            if (lane < 32) halves[wave / WB][row0 + 32 * j + lane] = make_float2(top, sum);
        } else {
            const bool counted = there && target != r.ignore;
            const float lse = there ? r.saved[row] : 0.0f, base = lse == -INFINITY ? 0.0f : lse;
            const float each = r.each && counted ? (r.dloss ? r.dloss[row] : 1.0f) : 1.0f;
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = exp_of<PLANES>(acc[i][j][e] - base);
            if (any) {
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (at == 32 * i + 8 * (e >> 2) + (e & 3)) acc[i][j][e] -= 1.0f;
            }
            if (there) {
                uint16_t* to = r.dz + row * r.step + (int64_t)p.at * TA + class0 + 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < NA; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = counted ? acc[i][j][4 * q + e] * each : 0.0f;
                        if constexpr (PLANES) {
                            uint32_t s[4][3];
#pragma unroll
                            for (int e = 0; e < 4; ++e) split(v[e], s[e]);
#pragma unroll
                            for (int k = 0; k < 3; ++k)
                                *reinterpret_cast<uint2*>(to + k * r.plane + 32 * i + 8 * q) =
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
    if constexpr (!GRAD) {
        __syncthreads();
        for (int t = threadIdx.x; t < TB; t += 64 * WA * WB) {
            const int64_t row = (int64_t)p.bt * TB + t;
            if (row >= r.M) continue;
            float2 v = halves[0][t];
            for (int w = 1; w < WA; ++w) join(v.x, v.y, halves[w][t].x, halves[w][t].y);
            r.pairs[(int64_t)p.at * r.M + row] = v;
        }
    }
}

// ---- gradients: dX (lines of A rows, of B features) and dW (lines of A features, of B classes) ----

struct OutArgs {
    void* out;
    int64_t step;
    int dtype;
    const float *share, *dloss;         // factors of all, or null
    float* slices;                      // parts of the contraction: [part][RA][RB], added up by another launch
    float* sums;                        // several pieces: [RA][RB], what they have so far
    int first_piece, last_piece;
};

__device__ __forceinline__ float factor_of(const OutArgs& o) { return (o.share ? *o.share : 1.0f) * (o.dloss ? *o.dloss : 1.0f); }

template <int DT>
__device__ __forceinline__ void finish(const OutArgs& o, int64_t i, int64_t j, int64_t RB, float v, float factor)
{
    if (o.sums) {
        float* s = o.sums + i * RB + j;
        if (!o.first_piece) v += *s;
        if (!o.last_piece) { *s = v; return; }
    }
    store_as<DT>(o.out, i * o.step + j, v * factor);
}

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

template <int MODE, int TA, int TB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB) __attribute__((amdgpu_waves_per_eu(2, 2))) void xent_gradient_kernel(bf16::Args g, OutArgs o)
{
    constexpr int NA = TA / WA / 32, NB = TB / WB / 32;
    __shared__ __align__(1024) uint8_t a0[128 * TA], a1[128 * TA], b0[128 * TB], b1[128 * TB];
    const bf16::Place p = bf16::place_of(g);
    if (!p.there) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    v16f acc[NA][NB] = {};
    bf16::multiply<MODE, MODE, TA, TB, WA, WB>(g, p, a0, a1, b0, b1, wave, lane, acc);
    const int64_t i0 = (int64_t)p.at * TA + (wave / WB) * (TA / WA), j0 = (int64_t)p.bt * TB + (wave % WB) * (TB / WB);
    const bool several = g.parts > 1;
    float* part = several ? o.slices + (int64_t)p.part * g.RA * g.RB : o.sums;
    if (!several && o.sums && !o.first_piece)
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, o.sums + i0 * g.RB + j0, g.RB, [](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
            return v + __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, 4 * at, 0, 0));
        });
    if (several || (o.sums && !o.last_piece)) {
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
                             __builtin_amdgcn_raw_buffer_store_b16((short)to_bf16(v * factor), rs, at >= bf16::kOutside / 4 ? bf16::kOutside : 2 * at, 0, 0);
                             return v;
                         });
    else
        each_sum<NA, NB>(acc, g.RA - i0, g.RB - j0, lane, static_cast<float*>(o.out) + i0 * o.step + j0, o.step,
                         [factor](float v, __amdgpu_buffer_rsrc_t rs, uint32_t at) {
                             __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v * factor), rs, 4 * at, 0, 0);
                             return v;
                         });
}

__global__ __launch_bounds__(kThreads) void xent_add_parts_kernel(OutArgs o, int64_t RA, int64_t RB, uint32_t parts)
{
    const float factor = factor_of(o);
    for (int64_t i = blockIdx.y; i < RA; i += gridDim.y) {
        const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
        if (j >= RB) continue;
        float v = 0.0f;
        for (uint32_t k = 0; k < parts; ++k) v += o.slices[((int64_t)k * RA + i) * RB + j];
        if (o.dtype == kBf16) finish<kBf16>(o, i, j, RB, v, factor);
        else finish<kF32>(o, i, j, RB, v, factor);
    }
}

// ---- sums over rows ----

// a row's pairs joined: its log of the sum of exponentials and its loss
__global__ __launch_bounds__(kThreads) void xent_rows_kernel(XentArgs a, const float2* pairs, int64_t tiles, const float* picked,
                                                             float* rows)
{
    const int64_t row = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (row >= a.M) return;
    float m = -INFINITY, l = 0.0f;
    for (int64_t i = 0; i < tiles; ++i) {
        const float2 p = pairs[i * a.M + row];
        join(m, l, p.x, p.y);
    }
    const int64_t t = a.target[row];
    // (no class left: minus infinity; a logit of plus infinity: no probabilities)
    float lse = m == INFINITY ? NAN : l > 0.0f ? m + logf(l) : l != l ? l : m, loss = 0.0f;
    if (t != a.ignore) {
        if (t < 0 || t >= a.N) lse = NAN;                       // (a target that is no class: seen in the loss and the gradients)
        const float z = t < 0 || t >= a.N ? NAN : picked[row];
        loss = z == -INFINITY && lse == lse ? INFINITY : lse - z;
    }
    a.saved[row] = lse;
    rows[row] = loss;
}

// one workgroup: the loss over all rows and a row's share in it
__global__ __launch_bounds__(1024) void xent_total_kernel(XentArgs a, const float* rows)
{
    __shared__ double sums[16];
    __shared__ long long counts[16];
    double s = 0.0;
    long long n = 0;
    for (int64_t i = threadIdx.x; i < a.M; i += 1024) {
        s += (double)rows[i];
        n += a.target[i] != a.ignore;
    }
    s = wave_sum(s);
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = s; counts[threadIdx.x >> 6] = n; }
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 16; ++w) { s += sums[w]; n += counts[w]; }
    const double share = a.reduction == kMean ? 1.0 / (double)(n > 0 ? n : 1) : 1.0;
    a.saved[a.M] = (float)share;
    if (a.reduction != kNone) a.loss[0] = (float)(s * share);
}

// db of a piece's classes: a column's sum, eight threads to two columns
template <bool PLANES>
__global__ __launch_bounds__(kThreads) void xent_dbias_kernel(RowArgs r, void* dbias, OutArgs o)
{
    __shared__ float2 sums[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t col = 2 * ((int64_t)blockIdx.x * 32 + x);
    float2 s = make_float2(0.0f, 0.0f);
    if (col < r.classes)
        for (int64_t i = y; i < r.M; i += 8)
#pragma unroll
            for (int k = PLANES ? 2 : 0; k >= 0; --k) {
                const uint32_t v = *reinterpret_cast<const uint32_t*>(r.dz + k * r.plane + i * r.step + col);
                s.x += from_bf16(v & 0xFFFFu);
                s.y += __uint_as_float(v & 0xFFFF0000u);
            }
    sums[y][x] = s;
    __syncthreads();
    if (y) return;
    for (int w = 1; w < 8; ++w) { s.x += sums[w][x].x; s.y += sums[w][x].y; }
    const float factor = factor_of(o);
    for (int e = 0; e < 2; ++e) {
        if (col + e >= r.classes) continue;
        const float v = (e ? s.y : s.x) * factor;
        if (o.dtype == kBf16) store_as<kBf16>(dbias, col + e, v);
        else store_as<kF32>(dbias, col + e, v);
    }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

constexpr int kBig = 256, kMid = 128;

// How a call is cut, and where its pieces of the workspace lie.
struct Plan {
    bool planes;                        // fp32
    bool pack_x, pack_w;
    int64_t piece;                      // classes of a piece
    int64_t x_step, w_step, dz_step;    // of packed rows, of dz
    size_t x, w, rest;                  // bytes of X packed, of a piece of W packed, of what lies behind them
    size_t pairs, picked, rows;         // forward
    size_t dz, sums, slices;            // backward
};

// products of few tiles: the contraction in parts, so that there are about two workgroups for a compute unit, each part
// at least 512 long
uint32_t parts_of(int64_t RA, int64_t RB, int64_t D, int tile)
{
    const int64_t tiles = ((RA + tile - 1) / tile) * ((RB + tile - 1) / tile), full = tile == kBig ? 256 : 512;
    int64_t parts = full / tiles;
    if (parts > D / 512) parts = D / 512;
    return (uint32_t)(parts < 1 ? 1 : parts > 64 ? 64 : parts);
}

int tile_of(int64_t RA, int64_t RB)
{
    const int64_t tiles = ((RA + kBig - 1) / kBig) * ((RB + kBig - 1) / kBig);
    return tiles >= 192 ? kBig : kMid;
}

bool whole(const void* p, int64_t ld, int64_t cols, int dtype)
{
    return dtype == kBf16 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < (int64_t)1 << 21;
}

// (sizes: for any alignment of the operands)
Plan plan_of(const XentArgs& a, bool sizes)
{
    Plan p{};
    p.planes = a.dtype == kF32;
    const int n = p.planes ? 3 : 1;
    p.pack_x = sizes || !whole(a.X, a.ldx, a.K, a.dtype);
    p.pack_w = sizes || !whole(a.W, a.ldw, a.N, a.dtype);
    // dz of a piece stays within 128 MB, which the memory-side cache holds between its writer and its readers
    p.piece = ((int64_t)128 << 20) / (2 * n * a.M) / kBig * kBig;
    if (p.piece < 1024) p.piece = 1024;
    if (p.piece > 65536) p.piece = 65536;
    if (p.piece > a.N) p.piece = a.N;
    p.x_step = up(a.K, 8);
    p.w_step = up(p.piece, 8);
    p.dz_step = up(p.piece, kBig);
    p.x = p.pack_x ? up256(2 * (size_t)n * a.M * p.x_step) : 0;
    p.w = p.pack_w ? up256(2 * (size_t)n * a.K * p.w_step) : 0;
    p.pairs = up256(sizeof(float2) * ((a.N + kMid - 1) / kMid + (a.N + p.piece - 1) / p.piece) * a.M);
    p.picked = p.rows = up256(sizeof(float) * a.M);
    p.dz = up256(2 * (size_t)n * a.M * p.dz_step);
    p.sums = p.piece < a.N ? up256(sizeof(float) * a.M * a.K) : 0;
    size_t most = 0;
    for (const int64_t classes : {p.piece, a.N - (a.N - 1) / p.piece * p.piece}) {          // (the last piece may be cut another way)
        const uint32_t px = parts_of(a.M, a.K, classes, tile_of(a.M, a.K)), pw = parts_of(a.K, classes, a.M, tile_of(a.K, classes));
        const size_t sx = px > 1 ? (size_t)px * a.M * a.K : 0, sw = pw > 1 ? (size_t)pw * a.K * classes : 0;
        if (sx > most) most = sx;
        if (sw > most) most = sw;
    }
    p.slices = up256(sizeof(float) * most);
    return p;
}

hipError_t launch_pack(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, uint16_t* dst, int64_t step, hipStream_t stream)
{
    const PackArgs a{src, rows, cols, ld, dst, step, rows * step};
    const dim3 grid((uint32_t)((step / 2 + kThreads - 1) / kThreads), (uint32_t)(rows < 65535 ? rows : 65535));
    ProfileScope ps(K_XENT_PACK, stream);
    if (dtype == kBf16) hipLaunchKernelGGL(xent_pack_kernel<kBf16>, grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL(xent_pack_kernel<kF32>, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <bool GRAD>
hipError_t launch_logits(int tag, const bf16::Args& g, const RowArgs& r, int tile, hipStream_t stream)
{
    ProfileScope ps(tag, stream);
    const dim3 grid(8 * g.per_xcd);
    if (tile == kBig) {
        if (g.terms > 1) hipLaunchKernelGGL((xent_logits_kernel<GRAD, true, 256, 256, 2, 4>), grid, dim3(512), 0, stream, g, r);
        else hipLaunchKernelGGL((xent_logits_kernel<GRAD, false, 256, 256, 2, 4>), grid, dim3(512), 0, stream, g, r);
    } else {
        if (g.terms > 1) hipLaunchKernelGGL((xent_logits_kernel<GRAD, true, 128, 128, 2, 2>), grid, dim3(256), 0, stream, g, r);
        else hipLaunchKernelGGL((xent_logits_kernel<GRAD, false, 128, 128, 2, 2>), grid, dim3(256), 0, stream, g, r);
    }
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_gradient(int tag, const bf16::Args& g, const OutArgs& o, int tile, hipStream_t stream)
{
    {
        ProfileScope ps(tag, stream);
        const dim3 grid(8 * g.per_xcd);
        if (tile == kBig) hipLaunchKernelGGL((xent_gradient_kernel<MODE, 256, 256, 2, 4>), grid, dim3(512), 0, stream, g, o);
        else hipLaunchKernelGGL((xent_gradient_kernel<MODE, 128, 128, 2, 2>), grid, dim3(256), 0, stream, g, o);
    }
    if (g.parts > 1) {
        ProfileScope ps(K_XENT_ADD_PARTS, stream);
        hipLaunchKernelGGL(xent_add_parts_kernel, dim3((uint32_t)((g.RB + kThreads - 1) / kThreads), (uint32_t)(g.RA < 65535 ? g.RA : 65535)),
                           dim3(kThreads), 0, stream, o, g.RA, g.RB, g.parts);
    }
    return hipGetLastError();
}

// X and a piece of W as the products take them
struct Operands {
    bf16::Side x, w;
};
hipError_t operands_of(const XentArgs& a, const Plan& p, char* workspace, int64_t first, int64_t classes, bool have_x, bool have_w,
                       Operands* o, hipStream_t stream)
{
    const int64_t size = dtype_size(a.dtype);
    const char* w = static_cast<const char*>(a.W) + first * size;
    uint16_t *px = reinterpret_cast<uint16_t*>(workspace), *pw = reinterpret_cast<uint16_t*>(workspace + p.x);
    o->x = p.pack_x ? bf16::Side{px, p.x_step, a.M * p.x_step} : bf16::Side{static_cast<const uint16_t*>(a.X), a.ldx, 0};
    o->w = p.pack_w ? bf16::Side{pw, p.w_step, a.K * p.w_step} : bf16::Side{reinterpret_cast<const uint16_t*>(w), a.ldw, 0};
    hipError_t e = hipSuccess;
    if (p.pack_x && !have_x) e = launch_pack(a.X, a.dtype, a.M, a.K, a.ldx, px, p.x_step, stream);
    if (p.pack_w && !have_w && e == hipSuccess) e = launch_pack(w, a.dtype, a.K, classes, a.ldw, pw, p.w_step, stream);
    return e;
}

RowArgs rows_of(const XentArgs& a, int64_t first, int64_t classes)
{
    RowArgs r{};
    r.bias = a.bias ? static_cast<const char*>(a.bias) + first * dtype_size(a.bias_dtype) : nullptr;
    r.bias_dtype = a.bias_dtype; r.classes = classes; r.first_class = first; r.target = a.target; r.ignore = a.ignore; r.M = a.M;
    return r;
}

} // namespace

size_t xent_workspace(const XentArgs& a, bool backward)
{
    const Plan p = plan_of(a, true);
    return p.x + p.w + (backward ? p.dz + p.sums + p.slices : p.pairs + p.picked + p.rows);
}

hipError_t launch_xent_fwd(const XentArgs& a, void* workspace, hipStream_t stream)
{
    const Plan p = plan_of(a, false);
    char* at = static_cast<char*>(workspace) + p.x + p.w;
    float2* pairs = reinterpret_cast<float2*>(at);
    float* picked = reinterpret_cast<float*>(at + p.pairs);
    float* rows = a.reduction == kNone ? a.loss : reinterpret_cast<float*>(at + p.pairs + p.picked);
    hipError_t e;
    int64_t tiles = 0;
    for (int64_t first = 0; first < a.N; first += p.piece) {
        const int64_t classes = a.N - first < p.piece ? a.N - first : p.piece;
        Operands o;
        if ((e = operands_of(a, p, static_cast<char*>(workspace), first, classes, first > 0, false, &o, stream)) != hipSuccess) return e;
        RowArgs r = rows_of(a, first, classes);
        r.pairs = pairs + tiles * a.M;
        r.picked = picked;
        const int tile = tile_of(classes, a.M);
        const bf16::Args g = bf16::plan(o.w, o.x, classes, a.M, a.K, p.planes, tile, tile, 1);
        if ((e = launch_logits<false>(K_XENT_LOGITS, g, r, tile, stream)) != hipSuccess) return e;
        tiles += g.n_at;
    }
    ProfileScope ps(K_XENT_LOSS, stream);
    hipLaunchKernelGGL(xent_rows_kernel, dim3((uint32_t)((a.M + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a, pairs, tiles,
                       picked, rows);
    hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(1024), 0, stream, a, rows);
    return hipGetLastError();
}

// forward: the forward pass has just run in the same workspace
hipError_t launch_xent_bwd(const XentArgs& a, void* workspace, bool forward, hipStream_t stream)
{
    const Plan p = plan_of(a, false);
    char* at = static_cast<char*>(workspace) + p.x + p.w;
    hipError_t e;
    for (int64_t first = 0; first < a.N; first += p.piece) {
        const int64_t classes = a.N - first < p.piece ? a.N - first : p.piece;
        Operands o;
        if ((e = operands_of(a, p, static_cast<char*>(workspace), first, classes, forward || first > 0, forward && p.piece == a.N, &o, stream)) != hipSuccess)
            return e;
        RowArgs r = rows_of(a, first, classes);
        r.saved = a.saved; r.dloss = a.dloss; r.each = a.reduction == kNone;
        r.dz = reinterpret_cast<uint16_t*>(at);
        r.step = p.dz_step; r.plane = a.M * p.dz_step;
        int tile = tile_of(classes, a.M);
        bf16::Args g = bf16::plan(o.w, o.x, classes, a.M, a.K, p.planes, tile, tile, 1);
        if ((e = launch_logits<true>(K_XENT_DLOGITS, g, r, tile, stream)) != hipSuccess) return e;
        const bf16::Side dz{r.dz, r.step, r.plane};
        OutArgs out{};
        out.dtype = a.dtype; out.share = a.saved + a.M; out.dloss = r.each ? nullptr : a.dloss;
        out.slices = reinterpret_cast<float*>(at + p.dz + p.sums);
        out.first_piece = out.last_piece = 1;
        if (a.dX) {
            OutArgs x = out;
            x.out = a.dX; x.step = a.K;
            x.sums = p.sums ? reinterpret_cast<float*>(at + p.dz) : nullptr;
            x.first_piece = first == 0; x.last_piece = first + classes == a.N;
            tile = tile_of(a.M, a.K);
            g = bf16::plan(dz, o.w, a.M, a.K, classes, p.planes, tile, tile, parts_of(a.M, a.K, classes, tile));
            if ((e = launch_gradient<kAlong>(K_XENT_DX, g, x, tile, stream)) != hipSuccess) return e;
        }
        if (a.dW) {
            OutArgs w = out;
            w.out = static_cast<char*>(a.dW) + first * dtype_size(a.dtype); w.step = a.N;
            tile = tile_of(a.K, classes);
            g = bf16::plan(o.x, dz, a.K, classes, a.M, p.planes, tile, tile, parts_of(a.K, classes, a.M, tile));
            if ((e = launch_gradient<kDown>(K_XENT_DW, g, w, tile, stream)) != hipSuccess) return e;
        }
        if (a.dbias) {
            OutArgs b = out;
            b.dtype = a.bias_dtype;
            void* to = static_cast<char*>(a.dbias) + first * dtype_size(a.bias_dtype);
            const dim3 grid((uint32_t)((classes + 63) / 64));
            ProfileScope ps(K_XENT_DBIAS, stream);
            if (p.planes) hipLaunchKernelGGL(xent_dbias_kernel<true>, grid, dim3(kThreads), 0, stream, r, to, b);
            else hipLaunchKernelGGL(xent_dbias_kernel<false>, grid, dim3(kThreads), 0, stream, r, to, b);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

} // namespace hdqt
