// C ABI of the operators of a residual block around an adapted layer: argument validation and the sequence of launches of each
// entry point.  See include/hdqt.h for the contract of every function.
#include "../../include/hdqt.h"
#include "train.hpp"

#include <math.h>

namespace {

using hdqt::hip_fail;

constexpr int64_t kMaxElems = (int64_t)1 << 40;
constexpr int64_t kMaxRows = (int64_t)1 << 31;

bool known_dtype(int d) { return d == HDQT_F32 || d == HDQT_BF16; }
bool off(const void* p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size != 0; }
bool short_of(const void* workspace, size_t have, size_t need) { return need > 0 && (!workspace || have < need); }

// what the kernels take of a description; NULL: no dropout
int drop_of(const hdqt_dropout_t* d, hdqt::DropArgs* out)
{
    *out = hdqt::DropArgs{};
    if (!d) return HDQT_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return HDQT_EINVAL_OPTION;
    if (off(d->step, 8)) return HDQT_EALIGN;
    const uint64_t bound = (uint64_t)llrint(d->p * 4294967296.0), all = (uint64_t)1 << 32;
    out->seed = d->seed;
    out->step = d->step;
    out->hi = (uint32_t)(bound >> 16);
    out->lo = (uint32_t)(bound & 0xFFFF);
    out->tensor_id = d->tensor_id;
    out->rate = bound == all ? 0.0f : (float)((double)all / (double)(all - bound));
    out->on = 1;
    return HDQT_OK;
}

int check_layernorm(const hdqt::LayerNormArgs& a)
{
    if (!known_dtype(a.dtype) || !known_dtype(a.param_dtype)) return HDQT_EINVAL_DTYPE;
    if (a.M < 1 || a.M >= kMaxRows || a.C < 1 || a.C > hdqt::kLayerNormColumns) return HDQT_EINVAL_DIM;
    if (!(a.eps >= 0.0f) || !isfinite(a.eps)) return HDQT_EINVAL_OPTION;
    const int64_t size = hdqt::dtype_size(a.dtype), psize = hdqt::dtype_size(a.param_dtype);
    for (const void* p : {a.x, a.residual, (const void*)a.sum, (const void*)a.y, a.s, a.dy, a.dsum, (const void*)a.dx, (const void*)a.dresidual})
        if (off(p, size)) return HDQT_EALIGN;
    for (const void* p : {a.weight, a.bias, (const void*)a.dweight, (const void*)a.dbias})
        if (off(p, psize)) return HDQT_EALIGN;
    return off(a.saved, 8) ? HDQT_EALIGN : HDQT_OK;
}

// (as for the products; a classifier's features)
constexpr int64_t kMaxTokens = (int64_t)65535 * 64, kMaxFeatures = (int64_t)1 << 21;

bool sized(const hdqt::AdapterArgs& a)
{
    return a.M >= 1 && a.M <= kMaxTokens && a.K >= 1 && a.K <= kMaxFeatures && a.N >= 1 && a.N <= kMaxFeatures && a.r >= 1 &&
           a.r <= hdqt::kRankMost && a.n >= 1 && a.n <= hdqt::kAdaptersMost && known_dtype(a.dtype);
}

hdqt::AdapterArgs sizes_of(int64_t M, int64_t K, int64_t N, int r, int n, int dtype)
{
    hdqt::AdapterArgs a{};
    a.M = M; a.K = K; a.N = N; a.r = r; a.n = n; a.dtype = dtype;
    return a;
}

int check_adapters(const hdqt::AdapterArgs& a, size_t saved_bytes)
{
    if (!a.x || !a.A || !a.B || !a.ids || !a.saved) return HDQT_EINVAL_NULL;
    if (!known_dtype(a.dtype)) return HDQT_EINVAL_DTYPE;
    if (!sized(a)) return HDQT_EINVAL_DIM;
    const int64_t size = hdqt::dtype_size(a.dtype);
    for (const void* p : {a.x, a.A, a.B, a.base, (const void*)a.out, a.dy, (const void*)a.dA, (const void*)a.dB})
        if (off(p, size)) return HDQT_EALIGN;
    if (off(a.ids, 8) || off(a.scale, 4) || off(a.saved, 16)) return HDQT_EALIGN;
    return saved_bytes < hdqt::adapters_saved(a) ? HDQT_EWORKSPACE : HDQT_OK;
}

} // namespace

extern "C" {

int hdqt_dropout(const void* x, const void* residual, void* y, int64_t elements, int dtype, const hdqt_dropout_t* dropout, void* stream)
{
    if (!x || !y || !dropout) return HDQT_EINVAL_NULL;
    if (elements < 1 || elements > kMaxElems) return HDQT_EINVAL_DIM;
    if (!known_dtype(dtype)) return HDQT_EINVAL_DTYPE;
    hdqt::DropArgs d;
    const int rc = drop_of(dropout, &d);
    if (rc) return rc;
    const int64_t size = hdqt::dtype_size(dtype);
    if (off(x, size) || off(residual, size) || off(y, size)) return HDQT_EALIGN;
    const hipError_t e = hdqt::launch_dropout(x, residual, y, elements, dtype, d, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

int hdqt_layernorm_fwd(const void* x, const void* residual, const hdqt_dropout_t* dropout, const void* weight, const void* bias, void* sum,
                       void* y, float* saved, int64_t M, int64_t C, float eps, int dtype, int param_dtype, void* stream)
{
    if (!x || !y) return HDQT_EINVAL_NULL;
    hdqt::LayerNormArgs a{};
    a.x = x; a.residual = residual; a.weight = weight; a.bias = bias; a.y = y; a.saved = saved; a.M = M; a.eps = eps;
    a.C = C < 1 || C > hdqt::kLayerNormColumns ? 0 : (int)C;
    a.sum = residual || dropout ? sum : nullptr;
    a.dtype = dtype; a.param_dtype = param_dtype;
    int rc = drop_of(dropout, &a.drop);
    if (!rc) rc = check_layernorm(a);
    if (rc) return rc;
    const hipError_t e = hdqt::launch_layernorm_fwd(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

size_t hdqt_layernorm_bwd_workspace_size(int64_t M, int64_t C, int dtype)
{
    hdqt::LayerNormArgs a{};
    a.M = M; a.dtype = dtype;
    a.C = C < 1 || C > hdqt::kLayerNormColumns ? 0 : (int)C;
    return check_layernorm(a) ? 0 : hdqt::layernorm_workspace(a);
}

int hdqt_layernorm_bwd(const void* dy, const void* dsum, const void* s, const hdqt_dropout_t* dropout, const void* weight,
                       const float* saved, void* dx, void* dresidual, void* dweight, void* dbias, int64_t M, int64_t C, int dtype,
                       int param_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dy || !s || !saved || (!dx && !dresidual && !dweight && !dbias)) return HDQT_EINVAL_NULL;
    hdqt::LayerNormArgs a{};
    a.dy = dy; a.dsum = dsum; a.s = s; a.weight = weight; a.saved = const_cast<float*>(saved); a.dx = dx; a.dresidual = dresidual;
    a.dweight = dweight; a.dbias = dbias; a.M = M; a.dtype = dtype; a.param_dtype = param_dtype;
    a.C = C < 1 || C > hdqt::kLayerNormColumns ? 0 : (int)C;
    int rc = drop_of(dropout, &a.drop);
    if (!rc) rc = check_layernorm(a);
    if (rc) return rc;
    if (dweight || dbias) {
        if (short_of(workspace, workspace_bytes, hdqt::layernorm_workspace(a))) return HDQT_EWORKSPACE;
        if (off(workspace, 16)) return HDQT_EALIGN;
    }
    const hipError_t e = hdqt::launch_layernorm_bwd(a, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

size_t hdqt_adapters_saved_size(int64_t M, int64_t K, int64_t N, int r, int n, int dtype)
{
    const hdqt::AdapterArgs a = sizes_of(M, K, N, r, n, dtype);
    return sized(a) ? hdqt::adapters_saved(a) : 0;
}

size_t hdqt_adapters_bwd_workspace_size(int64_t M, int64_t K, int64_t N, int r, int n, int dtype)
{
    const hdqt::AdapterArgs a = sizes_of(M, K, N, r, n, dtype);
    return sized(a) ? hdqt::adapters_workspace(a) : 0;
}

int hdqt_adapters_fwd(const void* x, const void* A, const void* B, const int64_t* ids, const float* scale, const void* base, void* out,
                      void* saved, size_t saved_bytes, int64_t M, int64_t K, int64_t N, int r, int n, int dtype, void* stream)
{
    if (!out) return HDQT_EINVAL_NULL;
    hdqt::AdapterArgs a = sizes_of(M, K, N, r, n, dtype);
    a.x = x; a.A = A; a.B = B; a.ids = ids; a.scale = scale; a.base = base; a.out = out; a.saved = saved;
    const int rc = check_adapters(a, saved_bytes);
    if (rc) return rc;
    const hipError_t e = hdqt::launch_adapters_fwd(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

int hdqt_adapters_bwd(const void* dy, const void* x, const void* A, const void* B, const int64_t* ids, const float* scale,
                      const void* saved, size_t saved_bytes, const void* base, void* dx, void* dA, void* dB, int64_t M, int64_t K, int64_t N,
                      int r, int n, int dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dy || (!dx && !dA && !dB)) return HDQT_EINVAL_NULL;
    hdqt::AdapterArgs a = sizes_of(M, K, N, r, n, dtype);
    a.dy = dy; a.x = x; a.A = A; a.B = B; a.ids = ids; a.scale = scale; a.base = base; a.out = dx; a.dA = dA; a.dB = dB;
    a.saved = const_cast<void*>(saved);
    const int rc = check_adapters(a, saved_bytes);
    if (rc) return rc;
    if (short_of(workspace, workspace_bytes, hdqt::adapters_workspace(a))) return HDQT_EWORKSPACE;
    if (off(workspace, 16)) return HDQT_EALIGN;
    const hipError_t e = hdqt::launch_adapters_bwd(a, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

} // extern "C"
