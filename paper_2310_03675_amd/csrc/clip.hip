// The global norm of many tensors and their clipping by it (gfx950):
//   n = sqrt(sum over all elements g^2) or max |g|,   c = min(1, max_norm / (n + eps)),   g <- c g.
// Every element is read twice, once for n and once for the product, and written once: three transfers, and nothing that
// can be had with fewer, since the product needs all of n.  Memory bounds it.  The tensors' addresses travel in the kernel's
// arguments (kClipMost of them to a launch), so that nothing is copied to the device and a call can be captured.  Tensors are
// cut into pieces of 32 KB times a power of two, one workgroup each; every workgroup leaves the sum of its piece in a word of
// its own and one workgroup adds those in order: no atomics, the same result every time.  Squares are summed in 64 bits, which
// memory hides, and in which no square of a finite 32-bit number overflows.
//
// 60 tensors, 400 million elements of both types (1.18 GB): 632 us, the norm 208 (5.7 TB/s), the product 422 (5.6), where a plain
// sum reads 3.9 TB/s and a copy moves 4.8.  ResNet-18's 62 gradients, 45 MB: 26 us in two launches, the second read from the
// memory-side cache.
#include "train.hpp"

namespace hdqt {

namespace {

constexpr int kThreads = kClipThreads, kLoads = kClipLoads;
constexpr int64_t kClipStream = (int64_t)128 << 20;         // bytes of all pieces above which the product goes past the caches

// the tensor that piece `p` of the launch belongs to
__device__ __forceinline__ int tensor_of(const ClipTable& t, uint32_t p)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.t[mid].first <= p) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// |x| as a number that orders like it, NaN above infinity
__device__ __forceinline__ uint32_t order(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

struct Sum {
    double s = 0.0;
    uint32_t m = 0;
    template <bool LARGEST>
    __device__ __forceinline__ void take(float x)
    {
        if (LARGEST) m = order(x) > m ? order(x) : m;
        else s = fma((double)x, (double)x, s);
    }
};

template <bool LARGEST, int DT>
__device__ __forceinline__ void piece_norm(const ClipTensor& t, int64_t begin, int64_t end, bool wide, Sum& sum)
{
    constexpr int V = DT == kBf16 ? 8 : 4;
    if (!wide) {
        for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) sum.take<LARGEST>(load_as<DT>(t.src, i));
        return;
    }
    const int64_t whole = begin + (end - begin) / V * V;
    const uint4* src = reinterpret_cast<const uint4*>(t.src);
    for (int64_t at = begin / V + threadIdx.x; at < whole / V; at += (int64_t)kThreads * kLoads) {
        uint4 v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            v[k] = at + k * kThreads < whole / V ? src[at + k * kThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (DT == kBf16) {
                    sum.take<LARGEST>(from_bf16(w[j] & 0xFFFFu));
                    sum.take<LARGEST>(__uint_as_float(w[j] & 0xFFFF0000u));
                } else {
                    sum.take<LARGEST>(__uint_as_float(w[j]));
                }
            }
        }
    }
    if (whole + threadIdx.x < end) sum.take<LARGEST>(load_as<DT>(t.src, whole + threadIdx.x));      // (fewer than V)
}

// the piece's elements [begin, end) of its tensor, and whether 16 bytes at a time are aligned
struct Piece {
    int64_t begin, end;
    bool wide;
};
__device__ __forceinline__ Piece piece_of(const ClipTable& t, const ClipTensor& x, uint32_t p)
{
    const int64_t len = (int64_t)t.loads * kThreads * (x.dtype == kBf16 ? 8 : 4);
    Piece r;
    r.begin = (int64_t)(p - x.first) * len;
    r.end = x.n - r.begin < len ? x.n : r.begin + len;
    r.wide = ((reinterpret_cast<uintptr_t>(x.src) | reinterpret_cast<uintptr_t>(x.dst)) & 15u) == 0;
    return r;
}

template <bool LARGEST>
__global__ __launch_bounds__(kThreads) void clip_norm_kernel(ClipTable t, double* parts)
{
    __shared__ double sums[kThreads / kWave];
    __shared__ uint32_t tops[kThreads / kWave];
    const ClipTensor x = t.t[tensor_of(t, blockIdx.x)];
    const Piece p = piece_of(t, x, blockIdx.x);
    Sum sum;
    if (x.dtype == kBf16) piece_norm<LARGEST, kBf16>(x, p.begin, p.end, p.wide, sum);
    else piece_norm<LARGEST, kF32>(x, p.begin, p.end, p.wide, sum);
    if (LARGEST) sum.m = wave_max_bits(sum.m);
    else sum.s = wave_sum(sum.s);
    if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = sum.s; tops[threadIdx.x >> 6] = sum.m; }
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < kThreads / kWave; ++w) {
        sum.s += sums[w];
        sum.m = tops[w] > sum.m ? tops[w] : sum.m;
    }
    // (a pattern as a number: exact in 64 bits, and ordered)
    parts[t.first + blockIdx.x] = LARGEST ? (double)sum.m : sum.s;
}

// The pieces' sums added up by a workgroup of T threads, in order; every thread has n and c.
struct Factor {
    float norm, scale;
};
template <bool LARGEST, int T>
__device__ __forceinline__ Factor factor_of(const double* parts, uint32_t pieces, float max_norm, float eps, double* lds)
{
    double s = 0.0;
    auto add = [](double p, double q) { return LARGEST ? (q > p ? q : p) : p + q; };
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < pieces; i += T) s = add(s, parts[i]);
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) s = add(s, __shfl_xor(s, m));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lds[0];
    for (int w = 1; w < T / kWave; ++w) s = add(s, lds[w]);
    Factor f;
    f.norm = LARGEST ? __uint_as_float((uint32_t)s) : (float)sqrt(s);
    const float c = max_norm / (f.norm + eps);
    f.scale = c >= 1.0f ? 1.0f : c;         // (a NaN among the gradients stays one in all of them)
    return f;
}

constexpr int kFinish = 1024;

template <bool LARGEST>
__global__ __launch_bounds__(kFinish) void clip_finish_kernel(const double* parts, uint32_t pieces, float max_norm, float eps,
                                                              float* norm, float* scale)
{
    __shared__ double lds[kFinish / kWave];
    const Factor f = factor_of<LARGEST, kFinish>(parts, pieces, max_norm, eps, lds);
    if (threadIdx.x) return;
    *norm = f.norm;
    *scale = f.scale;
}

// sixteen bytes, and where they are not to stay in the caches
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ uint4 take(const uint4* p)
{
    if constexpr (!STREAM) return *p;
    const v4u q = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p));
    return make_uint4(q.x, q.y, q.z, q.w);
}
template <bool STREAM>
__device__ __forceinline__ void put(uint4* p, uint4 v)
{
    if constexpr (!STREAM) *p = v;
    else __builtin_nontemporal_store(v4u{v.x, v.y, v.z, v.w}, reinterpret_cast<v4u*>(p));
}

template <bool STREAM, int DT>
__device__ __forceinline__ void piece_scale(const ClipTensor& t, int64_t begin, int64_t end, bool wide, float c)
{
    constexpr int V = DT == kBf16 ? 8 : 4;
    if (!wide) {
        for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) store_as<DT>(t.dst, i, c * load_as<DT>(t.src, i));
        return;
    }
    const int64_t whole = begin + (end - begin) / V * V;
    const uint4* src = reinterpret_cast<const uint4*>(t.src);
    uint4* dst = reinterpret_cast<uint4*>(t.dst);
    for (int64_t at = begin / V + threadIdx.x; at < whole / V; at += (int64_t)kThreads * kLoads) {
        uint4 v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (at + k * kThreads < whole / V) v[k] = take<STREAM>(src + at + k * kThreads);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (DT == kBf16)
                    w[j] = to_bf16(c * from_bf16(w[j] & 0xFFFFu)) | to_bf16(c * __uint_as_float(w[j] & 0xFFFF0000u)) << 16;
                else
                    w[j] = __float_as_uint(c * __uint_as_float(w[j]));
            }
            if (at + k * kThreads < whole / V) put<STREAM>(dst + at + k * kThreads, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
    const int64_t i = whole + threadIdx.x;
    if (i < end) store_as<DT>(t.dst, i, c * load_as<DT>(t.src, i));
}

// Of few pieces every workgroup adds up the sums itself, one after a launch of a single workgroup would (ResNet-18's 62
// gradients, 1400 pieces: a launch less); of many it reads what that launch has left.  (From the last piece to the first, which
// the memory-side cache may still hold, is no faster: 453 us either way for 2.4 GB, 18.6 against 17.4 for ResNet-18's.)
// STREAM: past the caches.  With a pass over the results behind it, out of place, of 100 MB 112 us, 104 through the caches; of 150
// MB 152 and 168, 300 MB 304 and 333, 1 GB 1014 and 1055.
template <bool LARGEST, bool OWN, bool STREAM>
__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipTable t, const double* parts, uint32_t pieces, float max_norm, float eps,
                                                              float* norm, const float* scale)
{
    __shared__ double lds[kThreads / kWave];
    const uint32_t piece = blockIdx.x;
    const ClipTensor x = t.t[tensor_of(t, piece)];
    float c;
    if constexpr (OWN) {
        const Factor f = factor_of<LARGEST, kThreads>(parts, pieces, max_norm, eps, lds);
        c = f.scale;
        if (t.first == 0 && blockIdx.x == 0 && threadIdx.x == 0) *norm = f.norm;
    } else {
        c = *scale;
    }
    if (c == 1.0f && x.src == x.dst) return;
    const Piece p = piece_of(t, x, piece);
    if (x.dtype == kBf16) piece_scale<STREAM, kBf16>(x, p.begin, p.end, p.wide, c);
    else piece_scale<STREAM, kF32>(x, p.begin, p.end, p.wide, c);
}

} // namespace

hipError_t launch_clip_norm(const ClipTable& t, bool largest, double* parts, hipStream_t stream)
{
    ProfileScope ps(K_CLIP_NORM, stream);
    if (largest) hipLaunchKernelGGL(clip_norm_kernel<true>, dim3(t.pieces), dim3(kThreads), 0, stream, t, parts);
    else hipLaunchKernelGGL(clip_norm_kernel<false>, dim3(t.pieces), dim3(kThreads), 0, stream, t, parts);
    return hipGetLastError();
}

hipError_t launch_clip_finish(const double* parts, uint32_t pieces, bool largest, float max_norm, float eps, float* norm,
                              float* scale, hipStream_t stream)
{
    ProfileScope ps(K_CLIP_FINISH, stream);
    if (largest) hipLaunchKernelGGL(clip_finish_kernel<true>, dim3(1), dim3(kFinish), 0, stream, parts, pieces, max_norm, eps, norm, scale);
    else hipLaunchKernelGGL(clip_finish_kernel<false>, dim3(1), dim3(kFinish), 0, stream, parts, pieces, max_norm, eps, norm, scale);
    return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipTable& t, const double* parts, uint32_t pieces, bool largest, float max_norm, float eps,
                             float* norm, const float* scale, hipStream_t stream)
{
    ProfileScope ps(K_CLIP_SCALE, stream);
    const dim3 grid(t.pieces), block(kThreads);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, t, parts, pieces, max_norm, eps, norm, scale); };
    const bool large = (int64_t)pieces * t.loads * kThreads * 16 > kClipStream;
    if (!clip_scales_alone(pieces)) launch(large ? clip_scale_kernel<false, false, true> : clip_scale_kernel<false, false, false>);
    else launch(largest ? clip_scale_kernel<true, true, false> : clip_scale_kernel<false, true, false>);
    return hipGetLastError();
}

} // namespace hdqt
