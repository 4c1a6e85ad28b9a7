// Dropout, added to a residual or not (gfx950):  y = residual + (u(e) < p 2^32 ? 0 : x / (1 - p)),  element by element, with the
// mask of dropout.hpp.  The gradient of x is the same call on y's gradient.  Memory bounds it: a thread takes eight elements, one
// block of the generator, so that the next workgroups' loads hide what its 20 wide multiplications cost.  65536 x 1152 in fp32, added to
// a residual and its gradient, 1.5 GB: 264 us, 5.7 TB/s (a large copy: 5.1); 128 x 512: 3.0 us a launch.
#include "dropout.hpp"

namespace hdqt {

namespace {

constexpr int kThreads = 256;

template <int DT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const void* x, const void* residual, void* y, int64_t n, DropArgs d)
{
    const uint64_t key = drop_key(d);
    const int64_t step = (int64_t)gridDim.x * kThreads * 8;
    auto dropped = [&](int64_t e, Eight<DT>& q, const Eight<DT>& r) {
        const uint32_t keep = kept_block(d, key, (uint64_t)e >> 3);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float of = residual ? r.get(j) : 0.0f;
            v[j] = keep >> j & 1 ? (residual ? fmaf(q.get(j), d.rate, of) : q.get(j) * d.rate) : of;
        }
        q.set(v);
    };
    for (int64_t e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8; e < n; e += step) {
        Eight<DT> r{};
        if (n - e >= 8) {
            Eight<DT> q = load_eight<DT>(x, e);
            if (residual) r = load_eight<DT>(residual, e);
            dropped(e, q, r);
            store_eight<DT>(y, e, q);
        } else {
            Eight<DT> q = load_some<DT>(x, e, (int)(n - e));
            if (residual) r = load_some<DT>(residual, e, (int)(n - e));
            dropped(e, q, r);
            store_some<DT>(y, e, 0, (int)(n - e), q);
        }
    }
}

} // namespace

hipError_t launch_dropout(const void* x, const void* residual, void* y, int64_t n, int dtype, const DropArgs& d, hipStream_t stream)
{
    ProfileScope ps(K_DROPOUT, stream);
    const int64_t groups = (n + 8 * kThreads - 1) / (8 * kThreads), most = (int64_t)1 << 22;
    const dim3 grid((uint32_t)(groups < most ? groups : most)), block(kThreads);
    if (dtype == kBf16) hipLaunchKernelGGL(dropout_kernel<kBf16>, grid, block, 0, stream, x, residual, y, n, d);
    else hipLaunchKernelGGL(dropout_kernel<kF32>, grid, block, 0, stream, x, residual, y, n, d);
    return hipGetLastError();
}

} // namespace hdqt
