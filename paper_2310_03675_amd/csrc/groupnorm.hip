// Group normalisation with an activation behind it, channels innermost (gfx950):
//   mu, var over the P pixels and C/G channels of a group;  xh = (x - mu) / sqrt(var + eps);
//   pre = xh w + b;  y = act(pre)
// and its gradients, with d = dy act'(pre):
//   db = sum d, dw = sum d xh (over images and pixels);  dx = (w d - mean(w d) - xh mean(w d xh)) / sqrt(var + eps).
// Nothing but x (and dy) is read: xh and pre are recomputed.  Memory bounds it.
//
// A thread has a vector of neighbouring channels (16 bytes where the channels come in whole ones) and walks down the
// pixels of a slice; the sums of a slice stand in a place of their own and are added in order, so that results do not depend
// on what finishes first.  Variances are sums of squares around a value of the thread's own, joined by the rule for two parts'
// means and squares, in 32 bits inside a slice and in 64 across slices: no cancellation against a large mean.
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

template <int ACT>
__device__ __forceinline__ float act(float pre)
{
    if (ACT == kRelu) return pre > 0.0f ? pre : (pre != pre ? pre : 0.0f);
    if (ACT == kSilu) return pre / (1.0f + __expf(-pre));
    return pre;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float pre)
{
    if (ACT == kRelu) return pre > 0.0f ? 1.0f : 0.0f;
    if (ACT == kSilu) {
        const float s = 1.0f / (1.0f + __expf(-pre));
        return s * (1.0f + pre * (1.0f - s));
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
__device__ __forceinline__ Spot spot_of(const NormArgs& a, const Cut& k)
{
    Spot s;
    s.iy = divide(threadIdx.x, k.by_tx);
    s.ix = threadIdx.x - s.iy * k.tx;
    const uint32_t vec = blockIdx.x * k.tx + s.ix;
    s.c = s.iy < k.ty && vec < k.vectors ? (int)vec * V : -1;
    const int64_t begin = (int64_t)blockIdx.y * k.slice;
    s.end = begin + k.slice < a.P ? begin + k.slice : a.P;
    s.p = begin + s.iy;
    s.base = (int64_t)blockIdx.z * a.P * a.C;
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

// parts[image][slice][channel]: mean and sum of squares around it
template <int DT, int V>
__global__ __launch_bounds__(kThreads) void norm_fwd_sums_kernel(NormArgs a, Cut k, float2* parts)
{
    __shared__ float2 lds[kThreads * V];
    const Spot s = spot_of<V>(a, k);
    float first[V], s1[V] = {}, s2[V] = {}, n = 0.0f;
    if (s.c >= 0 && s.p < s.end) {
        load_vec<DT, V>(a.x, s.base + s.p * a.C + s.c, first);
#pragma unroll 4
        for (int64_t p = s.p; p < s.end; p += k.ty) {
            float v[V];
            load_vec<DT, V>(a.x, s.base + p * a.C + s.c, v);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = v[j] - first[j];
                s1[j] += d;
                s2[j] = fmaf(d, d, s2[j]);
            }
            n += 1.0f;
        }
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
__global__ __launch_bounds__(kThreads) void norm_fwd_finish_kernel(NormArgs a, Cut k, const float2* parts)
{
    __shared__ double lds[kThreads / kWave];
    const int Cg = a.C / a.G;
    const int64_t image = blockIdx.x / a.G, items = (int64_t)k.slices * Cg;
    const int g = (int)(blockIdx.x - image * a.G);
    const float2* of = parts + image * k.slices * a.C + g * Cg;
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < items; i += kThreads) {
        const int64_t slice = i / Cg;
        const int64_t n = slice + 1 < k.slices ? k.slice : a.P - slice * k.slice;
        s += (double)n * (double)of[slice * a.C + (i - slice * Cg)].x;
    }
    const double count = (double)a.P * Cg, mean = block_sum(s, lds) / count;
    s = 0.0;
    for (int64_t i = threadIdx.x; i < items; i += kThreads) {
        const int64_t slice = i / Cg;
        const int64_t n = slice + 1 < k.slices ? k.slice : a.P - slice * k.slice;
        const float2 part = of[slice * a.C + (i - slice * Cg)];
        const double d = (double)part.x - mean;
        s += (double)part.y + (double)n * d * d;
    }
    const double var = block_sum(s, lds) / count;
    if (threadIdx.x == 0) {
        a.saved[2 * blockIdx.x] = (float)mean;
        a.saved[2 * blockIdx.x + 1] = (float)(1.0 / sqrt(var + (double)a.eps));
    }
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
    const Spot s = spot_of<V>(a, k);
    if (s.c < 0 || s.p >= s.end) return;
    const Channel<V> ch(a, blockIdx.z, s.c);
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
    const Spot s = spot_of<V>(a, k);
    float s1[V] = {}, s2[V] = {};
    if (s.c >= 0 && s.p < s.end) {
        const Channel<V> ch(a, blockIdx.z, s.c);
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
                s1[j] += d[j];
                s2[j] = fmaf(d[j], xh, s2[j]);
            }
        }
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

// Workgroups 0 .. B G - 1: the two means of a group of an image, into means.  Behind them: 64 channels each, dw and db.
__global__ __launch_bounds__(kThreads) void norm_bwd_finish_kernel(NormArgs a, Cut k, const float2* parts, float2* means)
{
    __shared__ double lds[2 * kThreads];
    const int64_t groups = a.B * a.G;
    if (blockIdx.x < groups) {
        const int Cg = a.C / a.G;
        const int64_t image = blockIdx.x / a.G, items = (int64_t)k.slices * Cg;
        const int g = (int)(blockIdx.x - image * a.G);
        const float2* of = parts + image * k.slices * a.C + g * Cg;
        double s1 = 0.0, s2 = 0.0;
        for (int64_t i = threadIdx.x; i < items; i += kThreads) {
            const int64_t slice = i / Cg;
            const int c = (int)(i - slice * Cg);
            const float2 part = of[slice * a.C + c];
            const double w = (double)param(a.weight, a.param_dtype, g * Cg + c, 1.0f);
            s1 += w * (double)part.x;
            s2 += w * (double)part.y;
        }
        const double count = (double)a.P * Cg;
        s1 = block_sum(s1, lds);
        s2 = block_sum(s2, lds);
        if (threadIdx.x == 0) means[blockIdx.x] = make_float2((float)(s1 / count), (float)(s2 / count));
        return;
    }
    const int c = (int)(blockIdx.x - groups) * 64 + (threadIdx.x & 63), q = threadIdx.x >> 6;
    double s1 = 0.0, s2 = 0.0;
    if (c < a.C)
        for (int64_t i = q; i < a.B * k.slices; i += kThreads / 64) {
            const float2 part = parts[i * a.C + c];
            s1 += (double)part.x;
            s2 += (double)part.y;
        }
    lds[threadIdx.x] = s1;
    lds[kThreads + threadIdx.x] = s2;
    __syncthreads();
    if (q || c >= a.C) return;
    for (int w = 1; w < kThreads / 64; ++w) {
        s1 += lds[threadIdx.x + 64 * w];
        s2 += lds[kThreads + threadIdx.x + 64 * w];
    }
    auto put = [&](void* p, double v) {
        if (p && a.param_dtype == kBf16) store_as<kBf16>(p, c, (float)v);
        else if (p) store_as<kF32>(p, c, (float)v);
    };
    put(a.dbias, s1);
    put(a.dweight, s2);
}

template <int DT, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(NormArgs a, Cut k, const float2* means)
{
    const Spot s = spot_of<V>(a, k);
    if (s.c < 0 || s.p >= s.end) return;
    const Channel<V> ch(a, blockIdx.z, s.c);
    float m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 m = means[(int64_t)blockIdx.z * a.G + (s.c + j) / (a.C / a.G)];
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

// 16 bytes at a time where every pixel starts at a multiple of them
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
    // (whatever the tensors' alignment turns out to be: an image's slices are not longer for single elements)
    const Cut one = cut_of(a, 1), wide = cut_of(a, a.dtype == kBf16 ? (a.C % 8 ? 1 : 8) : (a.C % 4 ? 1 : 4));
    const size_t p = parts_bytes(a, one), q = parts_bytes(a, wide);
    return (p > q ? p : q) + (backward ? (size_t)a.B * a.G * sizeof(float2) : 0);
}

hipError_t launch_norm_fwd(const NormArgs& a, void* workspace, hipStream_t stream)
{
    const int V = vector_of(a);
    const Cut k = cut_of(a, V);
    float2* parts = static_cast<float2*>(workspace);
    const dim3 grid(k.tiles, k.slices, (uint32_t)a.B), block(kThreads);
    with_types(a, V, [&](auto dt, auto v, auto act) {
        {
            ProfileScope ps(K_NORM_FWD_SUMS, stream);
            hipLaunchKernelGGL((norm_fwd_sums_kernel<dt.value, v.value>), grid, block, 0, stream, a, k, parts);
        }
        {
            ProfileScope ps(K_NORM_FWD_FINISH, stream);
            hipLaunchKernelGGL(norm_fwd_finish_kernel, dim3((uint32_t)(a.B * a.G)), block, 0, stream, a, k, parts);
        }
        ProfileScope ps(K_NORM_FWD, stream);
        hipLaunchKernelGGL((norm_fwd_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k);
    });
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs& a, void* workspace, hipStream_t stream)
{
    const int V = vector_of(a);
    const Cut k = cut_of(a, V);
    float2 *parts = static_cast<float2*>(workspace), *means = reinterpret_cast<float2*>(static_cast<char*>(workspace) + parts_bytes(a, k));
    const dim3 grid(k.tiles, k.slices, (uint32_t)a.B), block(kThreads);
    with_types(a, V, [&](auto dt, auto v, auto act) {
        {
            ProfileScope ps(K_NORM_BWD_SUMS, stream);
            hipLaunchKernelGGL((norm_bwd_sums_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k, parts);
        }
        {
            ProfileScope ps(K_NORM_BWD_FINISH, stream);
            hipLaunchKernelGGL(norm_bwd_finish_kernel, dim3((uint32_t)(a.B * a.G + (a.C + 63) / 64)), block, 0, stream, a, k, parts, means);
        }
        if (!a.dx) return;
        ProfileScope ps(K_NORM_BWD, stream);
        hipLaunchKernelGGL((norm_bwd_kernel<dt.value, v.value, act.value>), grid, block, 0, stream, a, k, means);
    });
    return hipGetLastError();
}

} // namespace hdqt
