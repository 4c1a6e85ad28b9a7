// C ABI of the operators around the integer products: argument validation and the sequence of launches of each entry
// point.  See include/hdqt.h for the contract of every function.
#include "../../include/hdqt.h"
#include "train.hpp"

#include <math.h>

namespace {

using hdqt::hip_fail;

constexpr int64_t kMaxDim = (int64_t)65535 * 64 + 1;        // as for the products
constexpr int64_t kMaxElems = (int64_t)1 << 40;
constexpr int64_t kMaxFeatures = (int64_t)1 << 21;          // of a classifier: 128 rows of three planes within 32 bits of bytes

bool known_dtype(int d) { return d == HDQT_F32 || d == HDQT_BF16; }
bool off(const void* p, int64_t size) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)size != 0; }
bool short_of(const void* workspace, size_t have, size_t need) { return need > 0 && (!workspace || have < need); }

// tensors with elements, and whether every description is one
int check_tensors(const hdqt_tensor_t* tensors, int64_t count, bool clip)
{
    if (count < 0 || count > (int64_t)1 << 24) return HDQT_EINVAL_DIM;
    if (count && !tensors) return HDQT_EINVAL_NULL;
    for (int64_t i = 0; i < count; ++i) {
        const hdqt_tensor_t& t = tensors[i];
        if (t.elements < 0 || t.elements >= kMaxElems) return HDQT_EINVAL_DIM;
        if (!known_dtype(t.dtype)) return HDQT_EINVAL_DTYPE;
        if (t.elements == 0) continue;
        if (!t.src || (clip && !t.dst)) return HDQT_EINVAL_NULL;
        const int64_t size = hdqt::dtype_size(t.dtype);
        if (off(t.src, size) || (clip && off(t.dst, size))) return HDQT_EALIGN;
    }
    return HDQT_OK;
}

struct ClipCall {
    hdqt::ClipPlan plan{};
    bool fits = false;
};

ClipCall plan_of(const hdqt_tensor_t* tensors, int64_t count)
{
    ClipCall c;
    c.fits = hdqt::plan_clip([&](int64_t i) { return tensors[i].elements * hdqt::dtype_size(tensors[i].dtype); }, count, &c.plan);
    return c;
}

size_t clip_bytes(const hdqt::ClipPlan& plan) { return 256 + sizeof(double) * (size_t)plan.pieces; }

// f(table) for every launch that the tensors take
template <class F>
hipError_t each_table(const hdqt_tensor_t* tensors, int64_t count, const hdqt::ClipPlan& plan, bool clip, F f)
{
    hdqt::ClipTable t{};
    t.loads = plan.loads;
    for (int64_t i = 0; i < count; ++i) {
        const hdqt_tensor_t& x = tensors[i];
        if (x.elements) {
            t.t[t.count++] = {x.src, clip ? x.dst : nullptr, x.elements, t.pieces, x.dtype};
            t.pieces += hdqt::clip_pieces(x.elements * hdqt::dtype_size(x.dtype), plan);
        }
        if (t.count && (t.count == hdqt::kClipMost || i + 1 == count)) {
            const hipError_t e = f(t);
            if (e != hipSuccess) return e;
            t.first += t.pieces;
            t.count = 0;
            t.pieces = 0;
        }
    }
    return hipSuccess;
}

int run_clip(const hdqt_tensor_t* tensors, int64_t count, int kind, bool clip, float max_norm, float eps, float* norm,
             void* workspace, size_t workspace_bytes, void* stream)
{
    if (!norm) return HDQT_EINVAL_NULL;
    if (kind != HDQT_NORM_2 && kind != HDQT_NORM_MAX) return HDQT_EINVAL_OPTION;
    if (clip && (!(max_norm >= 0.0f) || !(eps >= 0.0f))) return HDQT_EINVAL_OPTION;
    const int rc = check_tensors(tensors, count, clip);
    if (rc) return rc;
    if (off(norm, 4)) return HDQT_EALIGN;
    const ClipCall call = plan_of(tensors, count);
    if (!call.fits) return HDQT_EINVAL_DIM;
    if (short_of(workspace, workspace_bytes, clip_bytes(call.plan))) return HDQT_EWORKSPACE;
    if (off(workspace, 16)) return HDQT_EALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float* scale = static_cast<float*>(workspace);
    double* parts = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
    hipError_t e = each_table(tensors, count, call.plan, clip,
                              [&](const hdqt::ClipTable& t) { return hdqt::launch_clip_norm(t, kind == HDQT_NORM_MAX, parts, st); });
    const bool largest = kind == HDQT_NORM_MAX;
    const uint32_t pieces = call.plan.pieces;
    if (e == hipSuccess && !(clip && hdqt::clip_scales_alone(pieces)))
        e = hdqt::launch_clip_finish(parts, pieces, largest, max_norm, eps, norm, scale, st);
    if (e == hipSuccess && clip)
        e = each_table(tensors, count, call.plan, clip, [&](const hdqt::ClipTable& t) {
            return hdqt::launch_clip_scale(t, parts, pieces, largest, max_norm, eps, norm, scale, st);
        });
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

int check_norm(const hdqt::NormArgs& a)
{
    if (!known_dtype(a.dtype) || !known_dtype(a.param_dtype)) return HDQT_EINVAL_DTYPE;
    if (a.B < 1 || a.B > 65535 || a.P < 1 || a.P >= (int64_t)1 << 31 || a.C < 1 || a.C > 65536 || a.G < 1 || a.G > a.C || a.C % a.G)
        return HDQT_EINVAL_DIM;
    if (a.B * a.G > (int64_t)1 << 23 || a.P * a.C > kMaxElems / a.B) return HDQT_EINVAL_DIM;
    if (a.act != HDQT_ACT_NONE && a.act != HDQT_ACT_RELU && a.act != HDQT_ACT_SILU) return HDQT_EINVAL_OPTION;
    if (!(a.eps >= 0.0f) || !isfinite(a.eps)) return HDQT_EINVAL_OPTION;
    const int64_t size = hdqt::dtype_size(a.dtype), psize = hdqt::dtype_size(a.param_dtype);
    for (const void* p : {a.x, a.dy, (const void*)a.y, (const void*)a.dx})
        if (p && off(p, size)) return HDQT_EALIGN;
    for (const void* p : {a.weight, a.bias, (const void*)a.dweight, (const void*)a.dbias})
        if (p && off(p, psize)) return HDQT_EALIGN;
    return off(a.saved, 8) ? HDQT_EALIGN : HDQT_OK;
}

int check_xent(const hdqt::XentArgs& a)
{
    if (!a.X || !a.W || !a.target || !a.saved) return HDQT_EINVAL_NULL;
    if (!known_dtype(a.dtype) || !known_dtype(a.bias_dtype)) return HDQT_EINVAL_DTYPE;
    if (a.M < 1 || a.K < 1 || a.N < 1 || a.M >= kMaxDim || a.K > kMaxFeatures || a.N >= kMaxDim) return HDQT_EINVAL_DIM;
    if (a.ldx < a.K || a.ldw < a.N || a.ldx > kMaxElems / a.M || a.ldw > kMaxElems / a.K) return HDQT_EINVAL_DIM;
    if (a.reduction != HDQT_REDUCE_NONE && a.reduction != HDQT_REDUCE_MEAN && a.reduction != HDQT_REDUCE_SUM) return HDQT_EINVAL_OPTION;
    const int64_t size = hdqt::dtype_size(a.dtype), bsize = hdqt::dtype_size(a.bias_dtype);
    for (const void* p : {a.X, a.W, (const void*)a.dX, (const void*)a.dW})
        if (p && off(p, size)) return HDQT_EALIGN;
    for (const void* p : {a.bias, (const void*)a.dbias})
        if (p && off(p, bsize)) return HDQT_EALIGN;
    if (off(a.target, 8) || off(a.saved, 4) || off(a.loss, 4) || off(a.dloss, 4)) return HDQT_EALIGN;
    return HDQT_OK;
}

hdqt::XentArgs sizes_of(int64_t M, int64_t K, int64_t N, int dtype, int reduction)
{
    hdqt::XentArgs a{};
    a.M = M; a.K = K; a.N = N; a.dtype = dtype; a.reduction = reduction;
    a.ldx = K; a.ldw = N;
    return a;
}

bool sized(const hdqt::XentArgs& a)
{
    return a.M >= 1 && a.K >= 1 && a.N >= 1 && a.M < kMaxDim && a.K <= kMaxFeatures && a.N < kMaxDim && known_dtype(a.dtype) &&
           a.K <= kMaxElems / a.M && a.N <= kMaxElems / a.K;
}

} // namespace

extern "C" {

size_t hdqt_clip_grad_norm_workspace_size(const hdqt_tensor_t* tensors, int64_t count)
{
    if (check_tensors(tensors, count, false)) return 0;
    const ClipCall call = plan_of(tensors, count);
    return call.fits ? clip_bytes(call.plan) : 0;
}

int hdqt_grad_norm(const hdqt_tensor_t* tensors, int64_t count, int kind, float* norm, void* workspace, size_t workspace_bytes,
                   void* stream)
{
    return run_clip(tensors, count, kind, false, 0.0f, 0.0f, norm, workspace, workspace_bytes, stream);
}

int hdqt_clip_grad_norm(const hdqt_tensor_t* tensors, int64_t count, float max_norm, float eps, int kind, float* norm,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    return run_clip(tensors, count, kind, true, max_norm, eps, norm, workspace, workspace_bytes, stream);
}

size_t hdqt_groupnorm_workspace_size(int64_t B, int64_t P, int C, int G, int dtype, int backward)
{
    hdqt::NormArgs a{};
    a.B = B; a.P = P; a.C = C; a.G = G; a.dtype = dtype;
    return check_norm(a) ? 0 : hdqt::norm_workspace(a, backward != 0);
}

int hdqt_groupnorm_fwd(const void* x, const void* weight, const void* bias, void* y, float* saved, int64_t B, int64_t P, int C,
                       int G, float eps, int act, int dtype, int param_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !y || !saved) return HDQT_EINVAL_NULL;
    hdqt::NormArgs a{};
    a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.saved = saved; a.B = B; a.P = P; a.C = C; a.G = G; a.eps = eps;
    a.act = act; a.dtype = dtype; a.param_dtype = param_dtype;
    const int rc = check_norm(a);
    if (rc) return rc;
    if (short_of(workspace, workspace_bytes, hdqt::norm_workspace(a, false))) return HDQT_EWORKSPACE;
    if (off(workspace, 16)) return HDQT_EALIGN;
    const hipError_t e = hdqt::launch_norm_fwd(a, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

int hdqt_groupnorm_bwd(const void* dy, const void* x, const void* weight, const void* bias, const float* saved, void* dx,
                       void* dweight, void* dbias, int64_t B, int64_t P, int C, int G, int act, int dtype, int param_dtype,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    if (!dy || !x || !saved || (!dx && !dweight && !dbias)) return HDQT_EINVAL_NULL;
    hdqt::NormArgs a{};
    a.x = x; a.dy = dy; a.weight = weight; a.bias = bias; a.dx = dx; a.dweight = dweight; a.dbias = dbias;
    a.saved = const_cast<float*>(saved); a.B = B; a.P = P; a.C = C; a.G = G; a.act = act; a.dtype = dtype; a.param_dtype = param_dtype;
    const int rc = check_norm(a);
    if (rc) return rc;
    if (short_of(workspace, workspace_bytes, hdqt::norm_workspace(a, true))) return HDQT_EWORKSPACE;
    if (off(workspace, 16)) return HDQT_EALIGN;
    const hipError_t e = hdqt::launch_norm_bwd(a, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

size_t hdqt_xent_saved_size(int64_t M) { return M < 1 || M >= kMaxDim ? 0 : sizeof(float) * (size_t)(M + 1); }

size_t hdqt_xent_fwd_workspace_size(int64_t M, int64_t K, int64_t N, int dtype)
{
    const hdqt::XentArgs a = sizes_of(M, K, N, dtype, HDQT_REDUCE_MEAN);
    return sized(a) ? hdqt::xent_workspace(a, true, false) : 0;
}

size_t hdqt_xent_bwd_workspace_size(int64_t M, int64_t K, int64_t N, int dtype)
{
    const hdqt::XentArgs a = sizes_of(M, K, N, dtype, HDQT_REDUCE_MEAN);
    return sized(a) ? hdqt::xent_workspace(a, false, true) : 0;
}

size_t hdqt_xent_step_workspace_size(int64_t M, int64_t K, int64_t N, int dtype)
{
    const hdqt::XentArgs a = sizes_of(M, K, N, dtype, HDQT_REDUCE_MEAN);
    return sized(a) ? hdqt::xent_workspace(a, true, true) : 0;
}

static int run_xent(hdqt::XentArgs a, bool forward, bool backward, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_xent(a);
    if (rc) return rc;
    if (short_of(workspace, workspace_bytes, hdqt::xent_workspace(a, forward, backward))) return HDQT_EWORKSPACE;
    if (off(workspace, 256)) return HDQT_EALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    if (forward) e = hdqt::launch_xent_fwd(a, workspace, backward, st);
    if (backward && e == hipSuccess) e = hdqt::launch_xent_bwd(a, workspace, forward, st);
    return e == hipSuccess ? HDQT_OK : hip_fail(e);
}

int hdqt_xent_fwd(const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias, const int64_t* target,
                  int64_t ignore_index, int64_t M, int64_t K, int64_t N, int dtype, int bias_dtype, int reduction, float* loss,
                  float* saved, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!loss) return HDQT_EINVAL_NULL;
    const hdqt::XentArgs a{X, W, bias, ldx, ldw, target, ignore_index, M, K, N, dtype, bias_dtype, reduction,
                           saved, loss, nullptr, nullptr, nullptr, nullptr};
    return run_xent(a, true, false, workspace, workspace_bytes, stream);
}

int hdqt_xent_bwd(const float* dloss, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias,
                  const int64_t* target, int64_t ignore_index, int64_t M, int64_t K, int64_t N, int dtype, int bias_dtype,
                  int reduction, const float* saved, void* dX, void* dW, void* dbias, void* workspace, size_t workspace_bytes,
                  void* stream)
{
    if (!dX && !dW && !dbias) return HDQT_EINVAL_NULL;
    const hdqt::XentArgs a{X, W, bias, ldx, ldw, target, ignore_index, M, K, N, dtype, bias_dtype, reduction,
                           const_cast<float*>(saved), nullptr, dloss, dX, dW, dbias};
    return run_xent(a, false, true, workspace, workspace_bytes, stream);
}

int hdqt_xent_step(const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias, const int64_t* target,
                   int64_t ignore_index, int64_t M, int64_t K, int64_t N, int dtype, int bias_dtype, int reduction, float* loss,
                   float* saved, void* dX, void* dW, void* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!loss || (!dX && !dW && !dbias)) return HDQT_EINVAL_NULL;
    const hdqt::XentArgs a{X, W, bias, ldx, ldw, target, ignore_index, M, K, N, dtype, bias_dtype, reduction,
                           saved, loss, nullptr, dX, dW, dbias};
    return run_xent(a, true, true, workspace, workspace_bytes, stream);
}

} // extern "C"
