// Declarations of the operators around the integer products of a training step (api_train.hip and api_block.hip are their C
// ABI): clipping of gradients by their global norm (clip.hip), group normalisation (groupnorm.hip), the classifier's
// loss (xent.hip), dropout (dropout.hip), layer normalisation (layernorm.hip), low-rank adapters (adapters.hip).
#pragma once
#include "common.hpp"

namespace hdqt {

// these operators' kernels, behind the others' (common.hpp is left as it is: the benchmark's counters are tied to it)
enum TrainKernelId {
    K_CLIP_NORM = K_COUNT, K_CLIP_FINISH, K_CLIP_SCALE, K_NORM_FWD_SUMS, K_NORM_FWD_FINISH, K_NORM_FWD, K_NORM_BWD_SUMS,
    K_NORM_BWD_FINISH, K_NORM_BWD, K_XENT_LOGITS, K_XENT_LOSS, K_XENT_DLOGITS, K_XENT_DX, K_XENT_DW, K_XENT_DBIAS,
    K_XENT_PACK, K_XENT_ADD_PARTS, K_NORM_PARAMS, K_DROPOUT, K_LAYERNORM_FWD, K_LAYERNORM_BWD, K_LAYERNORM_PARAMS,
    K_ADAPT_PLAN, K_ADAPT_DOWN, K_ADAPT_UP, K_ADAPT_DOWN_UP, K_ADAPT_WEIGHTS,
    K_ALL_COUNT
};
int hip_fail(hipError_t e);          // notes the error for hdqt_last_hip_error (api.hip); HDQT_EHIP

enum Dtype { kF32 = 0, kBf16 = 1 };
inline int64_t dtype_size(int d) { return d == kBf16 ? 2 : 4; }

// ---- device helpers ----

__device__ __forceinline__ float from_bf16(uint32_t bits) { return __uint_as_float(bits << 16); }

// bf16_bits for any value: a NaN stays one (its fraction is not rounded away or into the sign)
__device__ __forceinline__ uint32_t to_bf16(float x) { return x != x ? (__float_as_uint(x) >> 16) | 0x40u : bf16_bits(x); }

template <int DT>
__device__ __forceinline__ float load_as(const void* p, int64_t i)
{
    return DT == kBf16 ? from_bf16(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
template <int DT>
__device__ __forceinline__ void store_as(void* p, int64_t i, float v)
{
    if (DT == kBf16) static_cast<uint16_t*>(p)[i] = (uint16_t)to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// sums over a wave, the same in every lane
template <class T>
__device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// ---- clip.hip ----

struct ClipTensor {
    const void* src;
    void* dst;              // null: only the norm is asked for
    int64_t n;
    uint32_t first;         // its first piece
    int32_t dtype;
};
constexpr int kClipMost = 120;          // tensors of a launch: its arguments are at most 4 KB
struct ClipTable {
    ClipTensor t[kClipMost];
    int count;
    uint32_t first, pieces;             // of the launch among all, its number
    int loads;                          // 16-byte loads of a thread per piece: kClipLoads times a power of two
};
// How tensors are cut: pieces of all of them, and of what length.
struct ClipPlan {
    uint32_t pieces;
    int loads;
};
constexpr int kClipThreads = 256;
constexpr int kClipLoads = 8;                   // 16-byte loads of a thread in flight: a piece has that many times a power of two
constexpr uint32_t kClipPieces = 8192;          // beyond, pieces are longer: one workgroup adds up what they leave
inline uint32_t clip_pieces(int64_t bytes, const ClipPlan& plan)
{
    const int64_t piece = (int64_t)plan.loads * kClipThreads * 16;
    return (uint32_t)((bytes + piece - 1) / piece);
}
// bytes(i) of `count` tensors; false: too many pieces
template <class F>
bool plan_clip(F bytes, int64_t count, ClipPlan* plan)
{
    for (plan->loads = kClipLoads; plan->loads <= 1 << 20; plan->loads *= 2) {
        const int64_t piece = (int64_t)plan->loads * kClipThreads * 16;
        int64_t pieces = 0, least = 0;
        for (int64_t i = 0; i < count; ++i) {
            pieces += (bytes(i) + piece - 1) / piece;
            least += bytes(i) > 0;
        }
        plan->pieces = (uint32_t)pieces;
        if (pieces <= kClipPieces || pieces <= 2 * least) return pieces < ((int64_t)1 << 24);
    }
    return false;
}
hipError_t launch_clip_norm(const ClipTable& t, bool largest, double* parts, hipStream_t stream);
hipError_t launch_clip_finish(const double* parts, uint32_t pieces, bool largest, float max_norm, float eps, float* norm,
                              float* scale, hipStream_t stream);
// whether the product's workgroups add the pieces' sums up themselves; else launch_clip_finish goes before
inline bool clip_scales_alone(uint32_t pieces) { return pieces > 0 && pieces <= 2048; }
hipError_t launch_clip_scale(const ClipTable& t, const double* parts, uint32_t pieces, bool largest, float max_norm, float eps,
                             float* norm, const float* scale, hipStream_t stream);

// ---- groupnorm.hip ----

enum Activation { kNoAct = 0, kRelu = 1, kSilu = 2 };

struct NormArgs {
    const void *x, *dy;                 // [B, P, C], channels innermost
    void *y, *dx;
    const void *weight, *bias;          // [C] or null (ones, zeros)
    void *dweight, *dbias;              // or null
    float* saved;                       // [B, G] pairs: mean, 1 / standard deviation
    int64_t B, P;
    int C, G;
    float eps;
    int act, dtype, param_dtype;
};
size_t norm_workspace(const NormArgs& a, bool backward);
hipError_t launch_norm_fwd(const NormArgs& a, void* workspace, hipStream_t stream);
hipError_t launch_norm_bwd(const NormArgs& a, void* workspace, hipStream_t stream);

// ---- xent.hip ----

enum Reduction { kNone = 0, kMean = 1, kSum = 2 };

struct XentArgs {
    const void *X, *W, *bias;           // [M, K] rows ldx apart, [K, N] rows ldw apart, [N] or null
    int64_t ldx, ldw;
    const int64_t* target;              // [M]
    int64_t ignore;
    int64_t M, K, N;
    int dtype, bias_dtype, reduction;
    float* saved;                       // [M] log of the sum of exponentials, then the share of a row in the loss
    float* loss;                        // [M] or one
    const float* dloss;                 // its gradient, as many; null: ones
    void *dX, *dW, *dbias;              // [M, K], [K, N], [N]; any may be null
};
size_t xent_workspace(const XentArgs& a, bool forward, bool backward);        // both: a step
// backward: the backward pass will run in the same workspace
hipError_t launch_xent_fwd(const XentArgs& a, void* workspace, bool backward, hipStream_t stream);
// forward: the forward pass has just run in the same workspace
hipError_t launch_xent_bwd(const XentArgs& a, void* workspace, bool forward, hipStream_t stream);

// ---- dropout.hip ----

struct DropArgs {
    uint64_t seed;
    const int64_t* step;                // device: added to the seed; or null
    uint32_t hi, lo;                    // round(p 2^32): what is above its 16 lowest bits (2^16: nothing is kept), and those
    uint32_t tensor_id;
    float rate;                         // what is kept is multiplied by: 1 / (1 - p)
    int on;                             // 0: there is no dropout
};
hipError_t launch_dropout(const void* x, const void* residual, void* y, int64_t n, int dtype, const DropArgs& d, hipStream_t stream);

// ---- layernorm.hip ----

constexpr int64_t kLayerNormColumns = 32768;        // what 1024 threads hold in registers, forward and backward
struct LayerNormArgs {
    const void *x, *residual;           // [M, C]; residual may be null
    void *sum, *y;                      // sum may be null
    const void *s, *dy, *dsum;          // backward: what was normalised; dsum may be null
    void *dx, *dresidual;               // either may be null
    const void *weight, *bias;          // [C] or null (ones, zeros)
    void *dweight, *dbias;              // or null
    float* saved;                       // [M] pairs: mean, 1 / standard deviation; forward may be null
    DropArgs drop;
    int64_t M;
    int C;
    float eps;
    int dtype, param_dtype;
};
size_t layernorm_workspace(const LayerNormArgs& a);         // of the backward pass
hipError_t launch_layernorm_fwd(const LayerNormArgs& a, hipStream_t stream);
hipError_t launch_layernorm_bwd(const LayerNormArgs& a, void* workspace, hipStream_t stream);

// ---- adapters.hip ----

constexpr int kAdaptersMost = 1024, kRankMost = 128;
struct AdapterArgs {
    const void *x, *A, *B;              // [M, K], [n, K, r], [n, r, N]
    const int64_t* ids;                 // [M]
    const float* scale;                 // [n] or null
    const void* base;                   // [M, N] (backward: of dx, [M, K]) or null
    void* out;                          // [M, N]; backward: dx [M, K] or null
    const void* dy;                     // [M, N]
    void *dA, *dB;                      // as A and B, or null
    void* saved;
    int64_t M, K, N;
    int r, n, dtype;
};
size_t adapters_saved(const AdapterArgs& a);
size_t adapters_workspace(const AdapterArgs& a);            // of the backward pass
hipError_t launch_adapters_fwd(const AdapterArgs& a, hipStream_t stream);
hipError_t launch_adapters_bwd(const AdapterArgs& a, void* workspace, hipStream_t stream);

} // namespace hdqt
