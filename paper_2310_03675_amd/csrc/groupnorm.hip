// Group normalisation with an activation behind it, channels innermost (gfx950):
//   mu, var over the P pixels and C/G channels of a group;  xh = (x - mu) / sqrt(var + eps);
//   pre = xh w + b;  y = act(pre)
// and its gradients, with d = dy act'(pre):
//   db = sum d, dw = sum d xh (over images and pixels);  dx = (w d - mean(w d) - xh mean(w d xh)) / sqrt(var + eps).
// Nothing but x (and dy) is read: xh and pre are recomputed.  Memory bounds it.
//
// An image's channels that fit a workgroup's registers (whole groups, all pixels) are read once and stay there: one launch
// forward, one backward and one that adds dw and db up over the images.  Larger ones take three launches either way, sums of
// slices of the pixels, their joining, and the result, and are read twice; the last launch walks from the end to the start,
// where what it begins with is still in the memory-side cache.
//
// 128 x 1024 x 64 in fp32, an image's slab in registers: 20 us forward (67 MB, 3.4 TB/s; the 512 workgroups all at once), 34 backward (101
// MB, 3.0; 70 registers, one workgroup to a compute unit, two rounds), 134 in three launches each way and 60 so, all of it; 8 x 65536 x 320 in bfloat16, which the chip's registers do not hold (336 MB): sums
// 77 and 146 us (4.4 and 4.6 TB/s), results 129 and 193 (5.2, some of it from that cache), 570 in all, where a copy moves 4.8.
// 1 x 49 x 96: 5 us, a launch; 128 x 16 x 512: 18, three launches.
//
// A thread has a vector of neighbouring channels (16 bytes where the channels come in whole ones) and walks down the
// pixels; sums stand in places of their own and are added in order, so that results do not depend on what finishes
// first.  Variances are sums of squares around the mean where the values are at hand; of slices they are sums around a value
// of the thread's own, joined by the rule for two parts' means and squares, in 32 bits inside a slice and in 64 across
// slices: no cancellation against a large mean.
#include "train.hpp"

#include <type_traits>

namespace hdqt {

namespace {

constexpr int kThreads = 256;

// How a launch cuts the tensor: workgroup = (tile of channels, slice of pixels, image).
struct Cut {
    uint32_t tx, ty;                // threads side by side in the channels, and down the pixels
    Divisor by_tx;
    uint32_t vectors;               // of a pixel
    uint32_t slice, slices;         // pixels of a slice
    uint32_t tiles;                 // of channels
};

template <int DT, int V>
__device__ __forceinline__ void load_vec(const void* p, int64_t i, float (&v)[V])
{
    if constexpr (V == 1) {
        v[0] = load_as<DT>(p, i);
    } else {
        const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + i * (16 / V));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < V; ++j)
            v[j] = DT == kF32 ? __uint_as_float(w[j]) : __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
}

template <int DT, int V>
__device__ __forceinline__ void store_vec(void* p, int64_t i, const float (&v)[V])
{
    if constexpr (V == 1) {
        store_as<DT>(p, i, v[0]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = DT == kF32 ? __float_as_uint(v[j % V]) : to_bf16(v[2 * j % V]) | to_bf16(v[(2 * j + 1) % V]) << 16;
        *reinterpret_cast<uint4*>(static_cast<char*>(p) + i * (16 / V)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__device__ __forceinline__ float param(const void* p, int dtype, int c, float otherwise)
{
    return !p ? otherwise : dtype == kBf16 ? load_as<kBf16>(p, c) : load_as<kF32>(p, c);
}

// 1 / (1 + exp(-pre)) by the chip's reciprocal (one unit in the last place): a division's ten instructions would be most of
// what an element of the backward pass costs (8 x 65536 x 320 in bfloat16, the sums: 178 us with it).  The exponential is the chip's
// power of two of the rounded product with log2 e: |pre| 2^-24 of it, in fp32 too, where pre is behind a normalisation and seldom beyond
// 10 (128 x 1024 x 64: outputs off by 1.88e-7 in the 2-norm, by exact functions 1.78e-7).
__device__ __forceinline__ float logistic(float pre) { return __builtin_amdgcn_rcpf(1.0f + __expf(-pre)); }

template <int ACT>
__device__ __forceinline__ float act(float pre)
{
    if (ACT == kRelu) return pre > 0.0f ? pre : (pre != pre ? pre : 0.0f);
    if (ACT == kSilu) return pre * logistic(pre);
    return pre;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float pre)
{
    if (ACT == kRelu) return pre > 0.0f ? 1.0f : 0.0f;
    if (ACT == kSilu) {
        const float s = logistic(pre);
        return s * fmaf(pre, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

// where a thread stands: its first channel, its pixels
struct Spot {
    int c;                          // first channel of its vector, -1: none
    uint32_t ix, iy;
    int64_t p, end, base;           // first pixel, end of the slice, the image's first element
};
template <int V>
__device__ __forceinline__ Spot spot_of(const NormArgs& a, const Cut& k, uint32_t slice, uint32_t image)
{
    Spot s;
    s.iy = divide(threadIdx.x, k.by_tx);
    s.ix = threadIdx.x - s.iy * k.tx;
    const uint32_t vec = blockIdx.x * k.tx + s.ix;
    s.c = s.iy < k.ty && vec < k.vectors ? (int)vec * V : -1;
    const int64_t begin = (int64_t)slice * k.slice;
    s.end = begin + k.slice < a.P ? begin + k.slice : a.P;
    s.p = begin + s.iy;
    s.base = (int64_t)image * a.P * a.C;
    return s;
}

// (count, mean, sum of squares around it) of two parts together
__device__ __forceinline__ void join(float& n, float& mean, float& m2, float on, float omean, float om2)
{
    if (on == 0.0f) return;
    const float sum = n + on, d = omean - mean, share = on / sum;
    mean += d * share;
    m2 += om2 + d * d * n * share;
    n = sum;
}

// 16 bytes of a tensor, or one element in x
template <int DT, int V>
__device__ __forceinline__ uint4 hold(const void* p, int64_t i)
{
    if constexpr (V == 1) return make_uint4(DT == kBf16 ? static_cast<const uint16_t*>(p)[i] : static_cast<const uint32_t*>(p)[i], 0, 0, 0);
    else return *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + i * (16 / V));
}
template <int DT, int V>
__device__ __forceinline__ float held(const uint4& q, int j)
{
    const uint32_t w = DT == kF32 ? (j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w)
                                  : (j / 2 == 0 ? q.x : j / 2 == 1 ? q.y : j / 2 == 2 ? q.z : q.w);
    return DT == kF32 ? __uint_as_float(w) : __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
}

struct Two {
    uint4 x, dy;
};

// take(load(p)) for a thread's pixels, AHEAD of them loaded before the first is taken
template <int AHEAD, class L, class F>
__device__ __forceinline__ void each_vector(const Spot& s, uint32_t step, L load, F take)
{
    int64_t p = s.p;
    for (; p + (AHEAD - 1) * (int64_t)step < s.end; p += AHEAD * (int64_t)step) {
        decltype(load(p)) q[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) q[u] = load(p + u * (int64_t)step);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) take(q[u]);
    }
    for (; p < s.end; p += step) take(load(p));
}

// parts[image][slice][channel]: mean and sum of squares around it
template <int DT, int V>
__global__ __launch_bounds__(kThreads) void norm_fwd_sums_kernel(NormArgs a, Cut k, float2* parts)
{
    __shared__ float2 lds[kThreads * V];
    const Spot s = spot_of<V>(a, k, blockIdx.y, blockIdx.z);
    float first[V], s1[V] = {}, s2[V] = {}, n = 0.0f;
    if (s.c >= 0 && s.p < s.end) {
        load_vec<DT, V>(a.x, s.base + s.p * a.C + s.c, first);
        auto take = [&](const uint4& q) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = held<DT, V>(q, j) - first[j];
                s1[j] += d;
                s2[j] = fmaf(d, d, s2[j]);
            }
            n += 1.0f;
        };
        each_vector<8>(s, k.ty, [&](int64_t p) { return hold<DT, V>(a.x, s.base + p * a.C + s.c); }, take);
    }
    float mean[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float m = n ? s1[j] / n : 0.0f;
        mean[j] = n ? first[j] + m : 0.0f;
        m2[j] = fmaf(-s1[j], m, s2[j]);
        lds[j * kThreads + threadIdx.x] = make_float2(mean[j], m2[j]);
    }
    __syncthreads();
    if (s.iy || s.c < 0) return;
    for (uint32_t y = 1; y < k.ty; ++y) {
        const int64_t p = s.p + y;
        if (p >= s.end) break;
        const float on = (float)((s.end - p + k.ty - 1) / k.ty);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float2 o = lds[j * kThreads + y * k.tx + s.ix];
            float sum = n;
            join(sum, mean[j], m2[j], on, o.x, o.y);
        }
        n += on;
    }
    float2* to = parts + ((int64_t)blockIdx.z * k.slices + blockIdx.y) * a.C + s.c;
#pragma unroll
    for (int j = 0; j < V; ++j) to[j] = make_float2(mean[j], m2[j]);
}

// a workgroup's sum of doubles, in every thread
__device__ __forceinline__ double block_sum(double v, double* lds)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (uint32_t w = 1; w < blockDim.x / kWave; ++w) v += lds[w];
    return v;
}

// one workgroup to a group of an image
__global__ __launch_bounds__(kThreads) void norm_fwd_finish_kernel(NormArgs a, Cut k, Divisor Cg, Divisor G, const float2* parts)
{
    __shared__ double lds[kThreads / kWave];
    const uint32_t image = divide(blockIdx.x, G), g = blockIdx.x - image * G.d, width = Cg.d < kThreads ? Cg.d : kThreads;
    const float2* of = parts + (int64_t)image * k.slices * a.C + g * Cg.d;
    // threads side by side in the channels, down the slices; around the first part's mean, which costs no more bits of 53
    // than twice the distance of the means in deviations
    const uint32_t y = Cg.d < kThreads ? divide(threadIdx.x, Cg) : 0, down = kThreads / width;
    const double about = (double)of[0].x;
    double s1 = 0.0, s2 = 0.0;
    if (y < down)
        for (uint32_t c = threadIdx.x - y * width; c < Cg.d; c += kThreads)
#pragma unroll 4
            for (uint32_t slice = y; slice < k.slices; slice += down) {
                const double n = (double)(slice + 1 < k.slices ? k.slice : (uint32_t)(a.P - (int64_t)slice * k.slice));
                const float2 part = of[(int64_t)slice * a.C + c];
                const double d = (double)part.x - about;
                s1 += n * d;
                s2 += (double)part.y + n * d * d;
            }
    s1 = block_sum(s1, lds);
    s2 = block_sum(s2, lds);
    if (threadIdx.x) return;
    const double count = (double)a.P * Cg.d, mean = s1 / count, var = s2 / count - mean * mean;
    a.saved[2 * blockIdx.x] = (float)(about + mean);
    a.saved[2 * blockIdx.x + 1] = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)a.eps));
}

// the group's mean and reciprocal deviation, and the parameters, of a thread's channels
template <int V>
struct Channel {
    float mean[V], rstd[V], w[V], b[V];
    __device__ __forceinline__ Channel(const NormArgs& a, int64_t image, int c)
    {
        const int Cg = a.C / a.G;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int64_t g = image * a.G + (c + j) / Cg;
            mean[j] = a.saved[2 * g];
            rstd[j] = a.saved[2 * g + 1];
            w[j] = param(a.weight, a.param_dtype, c + j, 1.0f);
            b[j] = param(a.bias, a.param_dtype, c + j, 0.0f);
        }
    }
};

template <int DT, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(NormArgs a, Cut k)
{
    const uint32_t image = (uint32_t)a.B - 1 - blockIdx.z;          // (from the end to the start)
    const Spot s = spot_of<V>(a, k, k.slices - 1 - blockIdx.y, image);
    if (s.c < 0 || s.p >= s.end) return;
    const Channel<V> ch(a, image, s.c);
#pragma unroll 4
    for (int64_t p = s.p; p < s.end; p += k.ty) {
        const int64_t at = s.base + p * a.C + s.c;
        float v[V];
        load_vec<DT, V>(a.x, at, v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = act<ACT>(fmaf((v[j] - ch.mean[j]) * ch.rstd[j], ch.w[j], ch.b[j]));
        store_vec<DT, V>(a.y, at, v);
    }
}

// parts[image][slice][channel]: sums of d and of d xh
template <int DT, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_bwd_sums_kernel(NormArgs a, Cut k, float2* parts)
{
    __shared__ float2 lds[kThreads * V];
    const Spot s = spot_of<V>(a, k, blockIdx.y, blockIdx.z);
    float s1[V] = {}, s2[V] = {};
    if (s.c >= 0 && s.p < s.end) {
        const Channel<V> ch(a, blockIdx.z, s.c);
        auto take = [&](const Two& q) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (held<DT, V>(q.x, j) - ch.mean[j]) * ch.rstd[j];
                const float d = held<DT, V>(q.dy, j) * act_slope<ACT>(fmaf(xh, ch.w[j], ch.b[j]));
                s1[j] += d;
                s2[j] = fmaf(d, xh, s2[j]);
            }
        };
        each_vector<4>(s, k.ty, [&](int64_t p) {
            const int64_t at = s.base + p * a.C + s.c;
            return Two{hold<DT, V>(a.x, at), hold<DT, V>(a.dy, at)};
        }, take);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) lds[j * kThreads + threadIdx.x] = make_float2(s1[j], s2[j]);
    __syncthreads();
    if (s.iy || s.c < 0) return;
    float2* to = parts + ((int64_t)blockIdx.z * k.slices + blockIdx.y) * a.C + s.c;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        for (uint32_t y = 1; y < k.ty; ++y) {
            const float2 o = lds[j * kThreads + y * k.tx + s.ix];
            s1[j] += o.x;
            s2[j] += o.y;
        }
        to[j] = make_float2(s1[j], s2[j]);
    }
}

// A group's two means, one workgroup to a group of an image, and the image's sums of its channels
__global__ __launch_bounds__(kThreads) void norm_bwd_finish_kernel(NormArgs a, Cut k, Divisor Cg, Divisor G, const float2* parts,
                                                                   float2* images, float2* means)
{
    __shared__ double lds[2 * kThreads];
    const uint32_t image = divide(blockIdx.x, G), g = blockIdx.x - image * G.d, width = Cg.d < kThreads ? Cg.d : kThreads;
    const float2* of = parts + (int64_t)image * k.slices * a.C + g * Cg.d;
    const uint32_t y = Cg.d < kThreads ? divide(threadIdx.x, Cg) : 0, down = kThreads / width, x = threadIdx.x - y * width;
    double m1 = 0.0, m2 = 0.0;
    for (uint32_t c = x; c - x < Cg.d; c += kThreads) {          // (as often for every thread)
        double s1 = 0.0, s2 = 0.0;
        if (y < down && c < Cg.d)
#pragma unroll 4
            for (uint32_t slice = y; slice < k.slices; slice += down) {
                const float2 part = of[(int64_t)slice * a.C + c];
                s1 += (double)part.x;
                s2 += (double)part.y;
            }
        lds[threadIdx.x] = s1;
        lds[kThreads + threadIdx.x] = s2;
        __syncthreads();
        if (y == 0 && c < Cg.d) {
            for (uint32_t w = 1; w < down; ++w) {
                s1 += lds[w * width + x];
                s2 += lds[kThreads + w * width + x];
            }
            images[(int64_t)image * a.C + g * Cg.d + c] = make_float2((float)s1, (float)s2);
            const double w = (double)param(a.weight, a.param_dtype, g * Cg.d + c, 1.0f);
            m1 += w * s1;
            m2 += w * s2;
        }
        __syncthreads();
    }
    m1 = block_sum(m1, lds);
    m2 = block_sum(m2, lds);
    const double count = (double)a.P * Cg.d;
    if (threadIdx.x == 0) means[blockIdx.x] = make_float2((float)(m1 / count), (float)(m2 / count));
}

// dw and db: the images' sums of 16 channels, 64 images at a time
constexpr int kParamThreads = 1024;
__global__ __launch_bounds__(kParamThreads) void norm_params_kernel(NormArgs a, const float2* images)
{
    __shared__ double lds[2][kParamThreads / 16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = (int)blockIdx.x * 16 + x;
    double s1 = 0.0, s2 = 0.0;
    if (c < a.C)
#pragma unroll 4
        for (int64_t i = y; i < a.B; i += kParamThreads / 16) {
            const float2 v = images[i * a.C + c];
            s1 += (double)v.x;
            s2 += (double)v.y;
        }
    lds[0][y][x] = s1;
    lds[1][y][x] = s2;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    const int of = threadIdx.x >> 4;
    double v = 0.0;
    for (int i = 0; i < kParamThreads / 16; ++i) v += lds[of][i][x];
    void* to = of ? a.dweight : a.dbias;
    if (!to || c >= a.C) return;
    if (a.param_dtype == kBf16) store_as<kBf16>(to, c, (float)v);
    else store_as<kF32>(to, c, (float)v);
}

template <int DT, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(NormArgs a, Cut k, const float2* means)
{
    const uint32_t image = (uint32_t)a.B - 1 - blockIdx.z;          // (from the end to the start)
    const Spot s = spot_of<V>(a, k, k.slices - 1 - blockIdx.y, image);
    if (s.c < 0 || s.p >= s.end) return;
    const Channel<V> ch(a, image, s.c);
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 m = means[(int64_t)image * a.G + (s.c + j) / (a.C / a.G)];
        m1[j] = m.x;
        m2[j] = m.y;
    }
#pragma unroll 2
    for (int64_t p = s.p; p < s.end; p += k.ty) {
        const int64_t at = s.base + p * a.C + s.c;
        float v[V], d[V];
        load_vec<DT, V>(a.x, at, v);
        load_vec<DT, V>(a.dy, at, d);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float xh = (v[j] - ch.mean[j]) * ch.rstd[j];
            d[j] *= act_slope<ACT>(fmaf(xh, ch.w[j], ch.b[j]));
            v[j] = ch.rstd[j] * (fmaf(ch.w[j], d[j], -m1[j]) - xh * m2[j]);
        }
        store_vec<DT, V>(a.dx, at, v);
    }
}

// ---- images whose channels fit a workgroup's registers ----

// How: workgroup = (slab of channels: whole groups, whole vectors; image), a thread has R vectors of the slab's pixels.
struct Slab {
    uint32_t channels, groups;      // of the slab; its groups
    uint32_t tx, ty;                // vectors of a pixel, threads down the pixels
    Divisor by_tx, by_channels, Cg;
    uint32_t rows;                  // parts that a channel's sum over ty is taken in
    Divisor slabs;                  // of an image
    uint32_t total, per_xcd;        // workgroups
};

// Workgroups go to the eight XCDs in turn: each gets a run of its own, so that slabs side by side, which share lines of memory,
// share an L2.  false: none of this number.
__device__ __forceinline__ bool slab_place(const Slab& k, uint32_t& image, uint32_t& slab)
{
    const uint32_t idx = (blockIdx.x & 7) * k.per_xcd + (blockIdx.x >> 3);
    image = divide(idx, k.slabs);
    slab = idx - image * k.slabs.d;
    return idx < k.total;
}

// Sums over the slab's pixels of S values a channel, v[k][j] of a thread's channel j: to sums[k][part][channel], of k.rows
// parts, which whoever reads them adds up.  `lds` has room for a value of every thread's channels.
template <int S, int V, int T>
__device__ __forceinline__ void channel_sums(const Slab& k, const float (&v)[S][V], uint32_t ix, uint32_t iy, bool there, float* lds,
                                             float (*sums)[T])
{
#pragma unroll
    for (int n = 0; n < S; ++n) {
        __syncthreads();
        if (there)
#pragma unroll
            for (int j = 0; j < V; ++j) lds[iy * k.channels + ix * V + j] = v[n][j];
        __syncthreads();
        const uint32_t part = divide(threadIdx.x, k.by_channels), c = threadIdx.x - part * k.channels;
        if (part < k.rows) {
            float s = 0.0f;
            for (uint32_t y = part; y < k.ty; y += k.rows) s += lds[y * k.channels + c];
            sums[n][part * k.channels + c] = s;
        }
    }
    __syncthreads();
}

// A group's sum of weight(channel) sums[part][channel], by a wave, in every lane
template <class W>
__device__ __forceinline__ float group_sum(const Slab& k, uint32_t g, const float* sums, W weight)
{
    float s = 0.0f;
    for (uint32_t c = threadIdx.x & 63; c < k.Cg.d; c += 64) {
        float t = 0.0f;
        for (uint32_t p = 0; p < k.rows; ++p) t += sums[p * k.channels + g * k.Cg.d + c];
        s += t * weight(g * k.Cg.d + c);
    }
    return wave_sum(s);
}

template <int DT, int V, int ACT, int T, int R>
__global__ __launch_bounds__(T) void norm_fwd_slab_kernel(NormArgs a, Slab k)
{
    __shared__ float lds[T * V];
    __shared__ float sums[1][T];
    __shared__ float2 of_group[T];
    uint32_t image, slab;
    if (!slab_place(k, image, slab)) return;
    const uint32_t iy = divide(threadIdx.x, k.by_tx), ix = threadIdx.x - iy * k.tx, wave = threadIdx.x >> 6;
    const bool there = iy < k.ty;
    const uint32_t c0 = slab * k.channels, c = c0 + ix * V;
    const int64_t base = (int64_t)image * a.P * a.C + c;
    const uint32_t P = there ? (uint32_t)a.P : 0;
    uint4 x[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P) x[r] = hold<DT, V>(a.x, base + (int64_t)(iy + r * k.ty) * a.C);
    float v[1][V] = {};
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P)
#pragma unroll
            for (int j = 0; j < V; ++j) v[0][j] += held<DT, V>(x[r], j);
    channel_sums<1, V, T>(k, v, ix, iy, there, lds, sums);
    const float count = (float)a.P * k.Cg.d;
    for (uint32_t g = wave; g < k.groups; g += T / 64) {
        const float s = group_sum(k, g, sums[0], [](uint32_t) { return 1.0f; });
        if ((threadIdx.x & 63) == 0) of_group[g].x = s / count;
    }
    __syncthreads();
    float mean[V], rstd[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        mean[j] = there ? of_group[divide(ix * V + j, k.Cg)].x : 0.0f;
        v[0][j] = 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = held<DT, V>(x[r], j) - mean[j];
                v[0][j] = fmaf(d, d, v[0][j]);
            }
    channel_sums<1, V, T>(k, v, ix, iy, there, lds, sums);
    for (uint32_t g = wave; g < k.groups; g += T / 64) {
        const float s = group_sum(k, g, sums[0], [](uint32_t) { return 1.0f; });
        if ((threadIdx.x & 63) == 0) {
            of_group[g].y = 1.0f / sqrtf(s / count + a.eps);
            reinterpret_cast<float2*>(a.saved)[(int64_t)image * a.G + slab * k.groups + g] = of_group[g];
        }
    }
    __syncthreads();
    if (!there) return;
    float w[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        rstd[j] = of_group[divide(ix * V + j, k.Cg)].y;
        w[j] = param(a.weight, a.param_dtype, c + j, 1.0f);
        b[j] = param(a.bias, a.param_dtype, c + j, 0.0f);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P) {
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = act<ACT>(fmaf((held<DT, V>(x[r], j) - mean[j]) * rstd[j], w[j], b[j]));
            store_vec<DT, V>(a.y, base + (int64_t)(iy + r * k.ty) * a.C, y);
        }
}

// images[image][channel]: sums of d and of d xh
template <int DT, int V, int ACT, int T, int R>
__global__ __launch_bounds__(T) void norm_bwd_slab_kernel(NormArgs a, Slab k, float2* images)
{
    __shared__ float lds[T * V];
    __shared__ float sums[2][T];
    __shared__ float2 of_group[T];
    uint32_t image, slab;
    if (!slab_place(k, image, slab)) return;
    const uint32_t iy = divide(threadIdx.x, k.by_tx), ix = threadIdx.x - iy * k.tx, wave = threadIdx.x >> 6;
    const bool there = iy < k.ty;
    const uint32_t c0 = slab * k.channels, c = c0 + ix * V;
    const int64_t base = (int64_t)image * a.P * a.C + c;
    const uint32_t P = there ? (uint32_t)a.P : 0;
    uint4 x[R], dy[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P) {
            x[r] = hold<DT, V>(a.x, base + (int64_t)(iy + r * k.ty) * a.C);
            dy[r] = hold<DT, V>(a.dy, base + (int64_t)(iy + r * k.ty) * a.C);
        }
    float mean[V], rstd[V], w[V], b[V], v[2][V] = {};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint32_t cj = there ? c + j : 0;
        const float2 s = reinterpret_cast<const float2*>(a.saved)[(int64_t)image * a.G + divide(cj, k.Cg)];
        mean[j] = s.x;
        rstd[j] = s.y;
        w[j] = param(a.weight, a.param_dtype, cj, 1.0f);
        b[j] = param(a.bias, a.param_dtype, cj, 0.0f);
    }
    // xh and d take x's and dy's place where they are no wider (fp32); of bfloat16 they are computed again
    auto word = [](uint4& q, int j) -> uint32_t& { return j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w; };
    auto both = [&](int r, int j, bool again, float& xh, float& d) {
        if (DT == kF32 && again) {
            xh = __uint_as_float(word(x[r], j));
            d = __uint_as_float(word(dy[r], j));
            return;
        }
        xh = (held<DT, V>(x[r], j) - mean[j]) * rstd[j];
        d = held<DT, V>(dy[r], j) * act_slope<ACT>(fmaf(xh, w[j], b[j]));
        if (DT == kF32) {
            word(x[r], j) = __float_as_uint(xh);
            word(dy[r], j) = __float_as_uint(d);
        }
    };
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float xh, d;
                both(r, j, false, xh, d);
                v[0][j] += d;
                v[1][j] = fmaf(d, xh, v[1][j]);
            }
    channel_sums<2, V, T>(k, v, ix, iy, there, lds, sums);
    if (images)
        for (uint32_t i = threadIdx.x; i < k.channels; i += T) {
            float2 s = make_float2(0.0f, 0.0f);
            for (uint32_t p = 0; p < k.rows; ++p) {
                s.x += sums[0][p * k.channels + i];
                s.y += sums[1][p * k.channels + i];
            }
            images[(int64_t)image * a.C + c0 + i] = s;
        }
    if (!a.dx) return;
    const float count = (float)a.P * k.Cg.d;
    for (uint32_t g = wave; g < k.groups; g += T / 64) {
        auto weight = [&](uint32_t i) { return param(a.weight, a.param_dtype, c0 + i, 1.0f); };
        const float s1 = group_sum(k, g, sums[0], weight), s2 = group_sum(k, g, sums[1], weight);
        if ((threadIdx.x & 63) == 0) of_group[g] = make_float2(s1 / count, s2 / count);
    }
    __syncthreads();
    if (!there) return;
    float2 m[V];
#pragma unroll
    for (int j = 0; j < V; ++j) m[j] = of_group[divide(ix * V + j, k.Cg)];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (iy + r * k.ty < P) {
            float dx[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float xh, d;
                both(r, j, true, xh, d);
                dx[j] = rstd[j] * (fmaf(w[j], d, -m[j].x) - xh * m[j].y);
            }
            store_vec<DT, V>(a.dx, base + (int64_t)(iy + r * k.ty) * a.C, dx);
        }
}

// 16 bytes at a time where every pixel starts at a multiple of them, else an element (both ways, 128 x 1024 x 65 in fp32 109 us, of 64
// channels 56; 8 x 65536 x 321 in bfloat16 1008, of 320 560)
int vector_of(const NormArgs& a)
{
    const int v = a.dtype == kBf16 ? 8 : 4;
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.dy) | reinterpret_cast<uintptr_t>(a.y) |
                         reinterpret_cast<uintptr_t>(a.dx);
    return a.C % v == 0 && at % 16 == 0 ? v : 1;
}

Cut cut_of(const NormArgs& a, int V)
{
    Cut k{};
    k.vectors = (uint32_t)(a.C / V);
    // of the numbers of tiles, the first with the fewest idle threads
    const uint32_t least = (k.vectors + kThreads - 1) / kThreads;
    uint32_t best = 0;
    for (uint32_t n = least; n <= least + 2; ++n) {
        const uint32_t tx = (k.vectors + n - 1) / n, busy = kThreads / tx * k.vectors / n;
        if (n == least || busy > best) { best = busy; k.tiles = n; k.tx = tx; }
    }
    k.ty = kThreads / k.tx;
    k.by_tx = make_divisor(k.tx);
    // a thread has 64 pixels, fewer where that leaves less than eight workgroups to a compute unit
    int64_t down = 64;
    while (down > 4 && (int64_t)k.tiles * ((a.P + k.ty * down - 1) / (k.ty * down)) * a.B < 2048) down /= 2;
    int64_t slice = k.ty * down;
    if ((a.P + slice - 1) / slice > 32768) slice = (a.P + 32767) / 32768;      // (what the y axis of a grid holds)
    k.slice = (uint32_t)(slice < a.P ? slice : a.P);
    k.slices = (uint32_t)((a.P + k.slice - 1) / k.slice);
    return k;
}

constexpr uint32_t kSlabThreads = 1024;

// The slab for an image's channels, and how many threads and vectors each; false where no slab fits.
// Slabs are 64 bytes of a pixel and more (whole sectors), wider where there still are two for every compute unit, and threads as few as
// hold the slab with four vectors each, 1024 with up to sixteen (backward, of x and dy both, eight).  Two of 1024 are on a compute
// unit at once where a thread has 64 registers at most (forward with four vectors, single elements), else one.
struct SlabPlan {
    Slab k;
    uint32_t threads, vectors;
};
bool slab_of(const NormArgs& a, int V, bool backward, SlabPlan* plan)
{
    const uint32_t C = (uint32_t)a.C, Cg = C / (uint32_t)a.G, size = (uint32_t)dtype_size(a.dtype);
    uint32_t unit = Cg;                     // whole groups and whole vectors
    while (unit % V) unit += Cg;
    const uint32_t units = C / unit, most = backward ? 8 : 16;
    auto fits = [&](uint32_t channels) {
        const uint32_t across = channels / V;
        return channels <= kSlabThreads && (uint64_t)a.P * across <= (uint64_t)(kSlabThreads / across * across) * most;
    };
    uint32_t channels = 0;
    for (uint32_t m = 1; m <= units; ++m) {
        if (units % m) continue;
        const uint32_t s = m * unit;
        if (!fits(s)) break;
        if (channels && channels * size >= 64 && (s * size > 256 || (uint64_t)a.B * (C / s) < 512)) break;
        channels = s;
    }
    if (!channels || (channels * size < 32 && channels < C)) return false;
    Slab& k = plan->k;
    k.channels = channels;
    k.groups = channels / Cg;
    k.tx = channels / V;
    plan->threads = 256;
    auto holds = [&](uint32_t threads) { return threads >= channels && (uint64_t)a.P <= (uint64_t)(threads / k.tx) * 4; };
    while (plan->threads < kSlabThreads && !holds(plan->threads)) plan->threads *= 2;
    k.ty = plan->threads / k.tx;
    if (k.ty > a.P) k.ty = (uint32_t)a.P;
    plan->vectors = (uint32_t)((a.P + k.ty - 1) / k.ty);
    k.by_tx = make_divisor(k.tx);
    k.by_channels = make_divisor(channels);
    k.Cg = make_divisor(Cg);
    k.rows = plan->threads / channels;
    k.slabs = make_divisor(C / channels);
    k.total = C / channels * (uint32_t)a.B;
    k.per_xcd = (k.total + 7) / 8;
    // (a launch has fewer than 2^32 threads along an axis; the slices' grid is spread over three)
    return (uint64_t)8 * k.per_xcd * plan->threads < (uint64_t)1 << 32;
}

// f(threads, vectors as types): no more vectors than the threads' number asks for
template <class F>
void with_slab(const SlabPlan& p, F f)
{
    auto is = [&](auto t, auto r) {
        if (p.threads != t.value || p.vectors > r.value) return false;
        f(t, r);
        return true;
    };
    using std::integral_constant;
    is(integral_constant<int, 256>{}, integral_constant<int, 1>{}) || is(integral_constant<int, 256>{}, integral_constant<int, 2>{}) ||
        is(integral_constant<int, 256>{}, integral_constant<int, 4>{}) || is(integral_constant<int, 512>{}, integral_constant<int, 4>{}) ||
        is(integral_constant<int, 1024>{}, integral_constant<int, 4>{}) || is(integral_constant<int, 1024>{}, integral_constant<int, 8>{}) ||
        is(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

size_t images_bytes(const NormArgs& a) { return ((size_t)a.B * a.C * sizeof(float2) + 255) / 256 * 256; }
size_t parts_bytes(const NormArgs& a, const Cut& k) { return ((size_t)a.B * k.slices * a.C * sizeof(float2) + 255) / 256 * 256; }

// f(kernel arguments as types): DT, V, ACT
template <class F>
void with_types(const NormArgs& a, int V, F f)
{
    auto with_act = [&](auto dt, auto v) {
        if (a.act == kRelu) f(dt, v, std::integral_constant<int, kRelu>{});
        else if (a.act == kSilu) f(dt, v, std::integral_constant<int, kSilu>{});
        else f(dt, v, std::integral_constant<int, kNoAct>{});
    };
    using one = std::integral_constant<int, 1>;
    if (a.dtype == kBf16) {
        std::integral_constant<int, kBf16> dt;
        if (V > 1) with_act(dt, std::integral_constant<int, 8>{});
        else with_act(dt, one{});
    } else {
        std::integral_constant<int, kF32> dt;
        if (V > 1) with_act(dt, std::integral_constant<int, 4>{});
        else with_act(dt, one{});
    }
}

} // namespace

size_t norm_workspace(const NormArgs& a, bool backward)
{
    // (whatever the tensors' alignment turns out to be: the larger of both ways; slices' sums only where a way has slices)
    size_t most = 0;
    for (const int V : {1, a.dtype == kBf16 ? (a.C % 8 ? 1 : 8) : (a.C % 4 ? 1 : 4)}) {
        SlabPlan slab;
        if (slab_of(a, V, backward, &slab)) continue;
        const size_t need = (backward ? (size_t)a.B * a.G * sizeof(float2) : 0) + parts_bytes(a, cut_of(a, V));
        if (need > most) most = need;
    }
    most += backward ? images_bytes(a) : 0;
    return most ? most : 256;           // (none is what invalid arguments have)
}

hipError_t launch_norm_fwd(const NormArgs& a, void* workspace, hipStream_t stream)
{
    const int V = vector_of(a);
    SlabPlan slab;
    if (slab_of(a, V, false, &slab)) {
        ProfileScope ps(K_NORM_FWD, stream);
        const dim3 grid(8 * slab.k.per_xcd);
        with_types(a, V, [&](auto dt, auto v, auto act) {
            with_slab(slab, [&](auto t, auto r) {
                hipLaunchKernelGGL((norm_fwd_slab_kernel<dt.value, v.value, act.value, t.value, r.value>), grid, dim3(t.value), 0, stream, a, slab.k);
            });
        });
        return hipGetLastError();
    }
    const Cut k = cut_of(a, V);
    float2* parts = static_cast<float2*>(workspace);
    const dim3 grid(k.tiles, k.slices, (uint32_t)a.B), block(kThreads);
    const Divisor Cg = make_divisor((uint32_t)(a.C / a.G)), G = make_divisor((uint32_t)a.G);
    with_types(a, V, [&](auto dt, auto v, auto act) {
        {
            ProfileScope ps(K_NORM_FWD_SUMS, stream);
            hipLaunchKernelGGL((norm_fwd_sums_kernel<dt.value, v.value>), grid, block, 0, stream, a, k, parts);
        }
        {
            ProfileScope ps(K_NORM_FWD_FINISH, stream);
            hipLaunchKernelGGL(norm_fwd_finish_kernel, dim3((uint32_t)(a.B * a.G)), block, 0, stream, a, k, Cg, G, parts);
        }
        ProfileScope ps(K_NORM_FWD, stream);
        hipLaunchKernelGGL((norm_fwd_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k);
    });
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, void* workspace, hipStream_t stream)
{
    const int V = vector_of(a);
    float2* images = static_cast<float2*>(workspace);
    SlabPlan slab;
    const bool fits = slab_of(a, V, true, &slab), params = a.dweight || a.dbias;
    with_types(a, V, [&](auto dt, auto v, auto act) {
        if (fits) {
            ProfileScope ps(K_NORM_BWD, stream);
            const dim3 grid(8 * slab.k.per_xcd);
            with_slab(slab, [&](auto t, auto r) {
                if constexpr (r.value <= 8)
                    hipLaunchKernelGGL((norm_bwd_slab_kernel<dt.value, v.value, act.value, t.value, r.value>), grid, dim3(t.value), 0, stream,
                                       a, slab.k, params ? images : nullptr);
            });
            return;
        }
        const Cut k = cut_of(a, V);
        float2* means = reinterpret_cast<float2*>(static_cast<char*>(workspace) + images_bytes(a));
        float2* parts = means + a.B * a.G;
        const dim3 grid(k.tiles, k.slices, (uint32_t)a.B), block(kThreads);
        {
            ProfileScope ps(K_NORM_BWD_SUMS, stream);
            hipLaunchKernelGGL((norm_bwd_sums_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k, parts);
        }
        {
            ProfileScope ps(K_NORM_BWD_FINISH, stream);
            const Divisor Cg = make_divisor((uint32_t)(a.C / a.G)), G = make_divisor((uint32_t)a.G);
            hipLaunchKernelGGL(norm_bwd_finish_kernel, dim3((uint32_t)(a.B * a.G)), block, 0, stream, a, k, Cg, G, parts, images, means);
        }
        if (!a.dx) return;
        ProfileScope ps(K_NORM_BWD, stream);
        hipLaunchKernelGGL((norm_bwd_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k, means);
    });
    if (params) {
        ProfileScope ps(K_NORM_PARAMS, stream);
        hipLaunchKernelGGL(norm_params_kernel, dim3((uint32_t)((a.C + 15) / 16)), dim3(kParamThreads), 0, stream, a, images);
    }
    return hipGetLastError();
}

} // namespace hdqt
