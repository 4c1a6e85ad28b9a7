// Softmax cross entropy of a linear classifier over N classes, in pieces of the classes, without the logits in memory
// (gfx950):
//   z = X W + b,  lse_i = log sum_j exp z_ij,  loss_i = lse_i - z_i,target(i)  (0 where the target is to be ignored)
//   dz_ij = g_i (exp(z_ij - lse_i) - [j = target(i)]),  dX = dz W^T,  dW = X^T dz,  db = sum_i dz_ij
// Forward, every tile of the product leaves the largest logit of a row and the sum of exponentials relative to it; a
// second launch joins a row's pairs.  Backward, the logits of a piece of the classes are multiplied again and become dz in
// the workspace, from which the three gradients are taken; dX is added up over the pieces in 32 bits.
#include "train.hpp"

#include <type_traits>

namespace hdqt {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64, kStage = 16;

// An operand of a product as it lies in memory: element (line, k) at line * line_step + k * k_step.
struct Operand {
    const void* p;
    int64_t line_step, k_step;
    int dtype;
};

enum Epilogue { kLogits, kDlogits, kOut };

struct ProductArgs {
    Operand A, B;
    int64_t RA, RB, D;                  // lines of A, lines of B, contraction
    // kLogits, kDlogits: lines of A are rows, lines of B classes from first_class on
    const void* bias;
    int bias_dtype;
    const int64_t* target;
    int64_t ignore, first_class;
    float2* pairs;                      // [tiles of classes][M]: largest logit, sum of exponentials
    float* picked;                      // [M]: the target's logit
    const float *saved, *dloss;
    int dloss_each;
    float* dz;                          // [M][RB]
    // kOut
    void* out;                          // [RA][RB], out_step apart
    int64_t out_step;
    int out_dtype;
    float* sums;                        // null, or [RA][RB] in 32 bits, of several pieces
    int first_piece, last_piece;
};

__device__ __forceinline__ float any_load(const void* p, int dtype, int64_t i)
{
    return dtype == kBf16 ? load_as<kBf16>(p, i) : load_as<kF32>(p, i);
}

// exp(z - lse) with z - lse <= 0 up to rounding; nothing where a class is masked by minus infinity
__device__ __forceinline__ float prob(float z, float lse) { return z == -INFINITY ? (lse != lse ? lse : 0.0f) : expf(z - lse); }

// (largest, sum of exponentials relative to it) of two parts together
__device__ __forceinline__ void join(float& m, float& l, float om, float ol)
{
    if (om == -INFINITY && ol == 0.0f) return;
    if (m == -INFINITY && l == 0.0f) { m = om; l = ol; return; }
    const float top = om > m ? om : m;
    l = l * expf(m - top) + ol * expf(om - top);
    m = top;
}

template <int EPI>
__global__ __launch_bounds__(kThreads) void xent_product_kernel(ProductArgs g)
{
    __shared__ float a[kStage][kTile + 4], b[kStage][kTile + 4];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t i0 = (int64_t)blockIdx.x * kTile, j0 = (int64_t)blockIdx.y * kTile;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < g.D; k0 += kStage) {
        for (int e = threadIdx.x; e < kStage * kTile; e += kThreads) {
            // (neighbouring threads take neighbouring elements in memory)
            const int la = g.A.k_step == 1 ? e / kStage : e % kTile, ka = g.A.k_step == 1 ? e % kStage : e / kTile;
            const int lb = g.B.k_step == 1 ? e / kStage : e % kTile, kb = g.B.k_step == 1 ? e % kStage : e / kTile;
            a[ka][la] = i0 + la < g.RA && k0 + ka < g.D ? any_load(g.A.p, g.A.dtype, (i0 + la) * g.A.line_step + (k0 + ka) * g.A.k_step) : 0.0f;
            b[kb][lb] = j0 + lb < g.RB && k0 + kb < g.D ? any_load(g.B.p, g.B.dtype, (j0 + lb) * g.B.line_step + (k0 + kb) * g.B.k_step) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kStage; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[k][ty * 4 + i], b[k][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = i0 + ty * 4 + i;
        const bool there = row < g.RA;
        if constexpr (EPI == kOut) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t col = j0 + tx * 4 + j;
                if (!there || col >= g.RB) continue;
                float v = acc[i][j];
                if (g.sums) {
                    float* s = g.sums + row * g.RB + col;
                    if (!g.first_piece) v += *s;
                    if (!g.last_piece) *s = v;
                }
                if (g.last_piece) {
                    if (g.out_dtype == kBf16) store_as<kBf16>(g.out, row * g.out_step + col, v);
                    else store_as<kF32>(g.out, row * g.out_step + col, v);
                }
            }
        } else {
            const int64_t t = there ? g.target[row] - g.first_class : -1;
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t col = j0 + tx * 4 + j;
                if (!there || col >= g.RB) continue;
                float z = acc[i][j];
                if (g.bias) z += any_load(g.bias, g.bias_dtype, g.first_class + col);
                if constexpr (EPI == kLogits) {
                    if (col == t) g.picked[row] = z;
                    join(m, l, z, z == -INFINITY ? 0.0f : 1.0f);
                }
                acc[i][j] = z;
            }
            if constexpr (EPI == kLogits) {
#pragma unroll
                for (int s = 1; s < 16; s <<= 1) {
                    const float om = __shfl_xor(m, s), ol = __shfl_xor(l, s);
                    join(m, l, om, ol);
                }
                if (there && tx == 0) g.pairs[(int64_t)blockIdx.y * g.RA + row] = make_float2(m, l);
            } else if (there) {
                const bool counted = g.target[row] != g.ignore;
                const float lse = g.saved[row];
                const float scale = counted ? (g.dloss ? g.dloss[g.dloss_each ? row : 0] : 1.0f) * g.saved[g.RA] : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int64_t col = j0 + tx * 4 + j;
                    if (col >= g.RB) continue;
                    g.dz[row * g.RB + col] = counted ? (prob(acc[i][j], lse) - (col == t ? 1.0f : 0.0f)) * scale : 0.0f;
                }
            }
        }
    }
}

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
        loss = z == -INFINITY ? INFINITY : lse - z;
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

// db of a piece's classes: a column's sum, eight threads to a column
__global__ __launch_bounds__(kThreads) void xent_dbias_kernel(const float* dz, int64_t M, int64_t classes, void* dbias, int dtype)
{
    __shared__ float sums[8][32];
    const int64_t col = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int y = threadIdx.x >> 5;
    float s = 0.0f;
    if (col < classes)
        for (int64_t i = y; i < M; i += 8) s += dz[i * classes + col];
    sums[y][threadIdx.x & 31] = s;
    __syncthreads();
    if (y || col >= classes) return;
    for (int w = 1; w < 8; ++w) s += sums[w][threadIdx.x];
    if (dtype == kBf16) store_as<kBf16>(dbias, col, s);
    else store_as<kF32>(dbias, col, s);
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
uint32_t tiles_of(int64_t n) { return (uint32_t)((n + kTile - 1) / kTile); }

// classes of a piece: dz of it stays within 128 MB, which the memory-side cache holds between its writer and its readers
int64_t piece_of(const XentArgs& a)
{
    int64_t n = ((int64_t)128 << 20) / (4 * a.M) / kTile * kTile;
    if (n < 1024) n = 1024;
    return n < a.N ? n : a.N;
}

template <int EPI>
hipError_t launch_product(int tag, const ProductArgs& g, hipStream_t stream)
{
    ProfileScope ps(tag, stream);
    hipLaunchKernelGGL(xent_product_kernel<EPI>, dim3(tiles_of(g.RA), tiles_of(g.RB)), dim3(kThreads), 0, stream, g);
    return hipGetLastError();
}

ProductArgs logits_args(const XentArgs& a, int64_t first, int64_t classes)
{
    const int64_t size = dtype_size(a.dtype);
    ProductArgs g{};
    g.A = {a.X, a.ldx, 1, a.dtype};
    g.B = {static_cast<const char*>(a.W) + first * size, 1, a.ldw, a.dtype};
    g.RA = a.M; g.RB = classes; g.D = a.K;
    g.bias = a.bias; g.bias_dtype = a.bias_dtype; g.target = a.target; g.ignore = a.ignore; g.first_class = first;
    return g;
}

} // namespace

size_t xent_workspace(const XentArgs& a, bool backward)
{
    if (!backward) return up256(sizeof(float2) * tiles_of(a.N) * a.M) + 2 * up256(sizeof(float) * a.M);
    const int64_t piece = piece_of(a);
    return up256(sizeof(float) * a.M * piece) + (piece < a.N ? up256(sizeof(float) * a.M * a.K) : 0);
}

hipError_t launch_xent_fwd(const XentArgs& a, void* workspace, hipStream_t stream)
{
    float2* pairs = static_cast<float2*>(workspace);
    float* picked = reinterpret_cast<float*>(static_cast<char*>(workspace) + up256(sizeof(float2) * tiles_of(a.N) * a.M));
    float* rows = a.reduction == kNone ? a.loss : picked + up256(sizeof(float) * a.M) / 4;
    ProductArgs g = logits_args(a, 0, a.N);
    g.pairs = pairs;
    g.picked = picked;
    hipError_t e = launch_product<kLogits>(K_XENT_LOGITS, g, stream);
    if (e != hipSuccess) return e;
    ProfileScope ps(K_XENT_LOSS, stream);
    hipLaunchKernelGGL(xent_rows_kernel, dim3((uint32_t)((a.M + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a, pairs,
                       tiles_of(a.N), picked, rows);
    hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(1024), 0, stream, a, rows);
    return hipGetLastError();
}

hipError_t launch_xent_bwd(const XentArgs& a, void* workspace, hipStream_t stream)
{
    const int64_t piece = piece_of(a), size = dtype_size(a.dtype);
    float* dz = static_cast<float*>(workspace);
    float* sums = piece < a.N ? reinterpret_cast<float*>(static_cast<char*>(workspace) + up256(sizeof(float) * a.M * piece)) : nullptr;
    for (int64_t first = 0; first < a.N; first += piece) {
        const int64_t classes = a.N - first < piece ? a.N - first : piece;
        ProductArgs g = logits_args(a, first, classes);
        g.saved = a.saved; g.dloss = a.dloss; g.dloss_each = a.reduction == kNone; g.dz = dz;
        hipError_t e = launch_product<kDlogits>(K_XENT_DLOGITS, g, stream);
        if (e != hipSuccess) return e;
        if (a.dX) {
            ProductArgs x{};
            x.A = {dz, classes, 1, kF32};
            x.B = {static_cast<const char*>(a.W) + first * size, a.ldw, 1, a.dtype};
            x.RA = a.M; x.RB = a.K; x.D = classes;
            x.out = a.dX; x.out_step = a.K; x.out_dtype = a.dtype;
            x.sums = sums; x.first_piece = first == 0; x.last_piece = first + classes == a.N;
            if ((e = launch_product<kOut>(K_XENT_DX, x, stream)) != hipSuccess) return e;
        }
        if (a.dW) {
            ProductArgs w{};
            w.A = {a.X, 1, a.ldx, a.dtype};
            w.B = {dz, 1, classes, kF32};
            w.RA = a.K; w.RB = classes; w.D = a.M;
            w.out = static_cast<char*>(a.dW) + first * size; w.out_step = a.N; w.out_dtype = a.dtype;
            w.first_piece = w.last_piece = 1;
            if ((e = launch_product<kOut>(K_XENT_DW, w, stream)) != hipSuccess) return e;
        }
        if (a.dbias) {
            ProfileScope ps(K_XENT_DBIAS, stream);
            hipLaunchKernelGGL(xent_dbias_kernel, dim3((uint32_t)((classes + 31) / 32)), dim3(kThreads), 0, stream, dz, a.M, classes,
                               static_cast<char*>(a.dbias) + first * dtype_size(a.bias_dtype), a.bias_dtype);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

} // namespace hdqt
