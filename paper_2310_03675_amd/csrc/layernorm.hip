// Layer normalisation of rows, with the residual sum and the dropout in front of it (gfx950):
//   s = x, or residual + dropout(x), rounded to the tensors' type;  mu, var over a row's C values;
//   xh = (s - mu) / sqrt(var + eps);  y = xh w + b
// and its gradients, d = w dy:
//   ds = (d - mean(d) - xh mean(d xh)) / sqrt(var + eps) + dsum;  dresidual = ds, dx = dropout(ds);  dw = sum dy xh, db = sum dy
// (over rows; dsum: the gradient that reaches s past the normalisation).  Memory bounds it.
//
// A row stays in registers: R vectors of eight to each of a power of two of threads, 64 at most where that holds it, so that
// its sums stay inside a wave, else several waves' through LDS.  Variances are sums of squares around the mean.  Backward, a
// workgroup keeps the parameters' gradients of the columns that its threads have over all its rows, and leaves one part of them,
// which a second launch adds up in 64 bits: no atomics, results do not depend on what finishes first.
//
// Measured, with a residual forward and a gradient of s backward (a large copy: 5.1 TB/s): 8192 x 4096 in bfloat16 44 us (6.1 TB/s) and 65 us
// (4.1), in fp32 102 us (5.3) and 116 us (4.6); 20011 x 1031 in bfloat16 43 and 52 us (3.8 and 3.2 TB/s: its vectors are one more than
// places, and rows start and end anywhere; 1024 columns 30 and 39); 131072 x 64 in fp32 22 and 28 us; 128 x 512 in fp32 3.6 and 3.5 us, a launch each.
#include "dropout.hpp"
#include "lane_ops.hpp"

#include <type_traits>

namespace hdqt {

namespace {

// How rows lie on threads.
struct Rows {
    uint32_t width;                 // threads to a row
    uint32_t R;                     // vectors to a thread
    uint32_t at_once;               // rows of a workgroup
    uint32_t groups;                // workgroups
};

// sum over the `width` (a power of two up to 64) neighbouring lanes of a lane, the same in each
__device__ __forceinline__ float lanes_sum(float v, uint32_t width)
{
    auto half = [&](uint32_t m) { return width > m; };
    if (half(1)) v += lanes::lane_xor<1>(v);
    if (half(2)) v += lanes::lane_xor<2>(v);
    if (half(4)) v += lanes::lane_xor<4>(v);
    if (half(8)) v += lanes::lane_xor<8>(v);
#ifdef __HIP_DEVICE_COMPILE__
    if (half(16)) {
        const lanes::v2u r = __builtin_amdgcn_permlane16_swap(lanes::as_u(v), lanes::as_u(v), false, false);
        v = lanes::as_f(r[0]) + lanes::as_f(r[1]);
    }
    if (half(32)) {
        const lanes::v2u r = __builtin_amdgcn_permlane32_swap(lanes::as_u(v), lanes::as_u(v), false, false);
        v = lanes::as_f(r[0]) + lanes::as_f(r[1]);
    }
#endif
    return v;
}

// Sums of N values over a row's threads, in each of them.  Every thread of the workgroup comes here.  lds: N values a wave; two
// calls in turn have one each.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], uint32_t width, float* lds)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], width < 64 ? width : 64);
    if (width <= 64) return;
    const uint32_t wave = threadIdx.x >> 6, waves = width >> 6, first = wave & ~(waves - 1);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[N * wave + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float s = 0.0f;
        for (uint32_t w = 0; w < waves; ++w) s += lds[N * (first + w) + i];
        v[i] = s;
    }
}

// How rows end: whole vectors; with one that begins eight before the row's end, and what it has of the one before is left out; a row
// is less than a vector.
enum End { kWhole, kOverlap, kShort };

// A thread's vector of a row: columns c + lo to c + hi of it.  Only the thread's last may be a row's last, or behind it.
template <int END>
struct Span {
    int c, lo, hi;
    bool there, ends;
    __device__ __forceinline__ Span(uint32_t vector, int C, bool row, bool last)
    {
        const int first = 8 * (int)vector;
        ends = last && END != kWhole;
        there = row && (!last || first < C);
        c = END != kOverlap || !last || first + 8 <= C ? first : C - 8;
        lo = END == kOverlap ? first - c : 0;
        hi = END == kShort ? C : 8;
    }
    __device__ __forceinline__ bool has(int j) const { return !ends || (END == kOverlap ? j >= lo : j < hi); }
    template <int DT>
    __device__ __forceinline__ Eight<DT> load(const void* p, int64_t base) const
    {
        if constexpr (END == kShort) return load_some<DT>(p, base + c, hi);
        else return load_eight<DT>(p, base + c);
    }
    template <int DT>
    __device__ __forceinline__ void store(void* p, int64_t base, const Eight<DT>& q) const
    {
        if (END != kShort && (!ends || lo == 0)) store_eight<DT>(p, base + c, q);
        else store_some<DT>(p, base + c, lo, hi, q);
    }
    // of the parameters, or `otherwise`
    __device__ __forceinline__ void params(const void* p, int dtype, float otherwise, float (&v)[8]) const
    {
        if (!p) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = otherwise;
        } else if (dtype == kBf16) {
            const Eight<kBf16> q = load<kBf16>(p, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = q.get(j);
        } else {
            const Eight<kF32> q = load<kF32>(p, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = q.get(j);
        }
    }
};

template <int DT, int R, int END, int T>
__global__ __launch_bounds__(T) void layernorm_fwd_kernel(LayerNormArgs a, Rows k)
{
    __shared__ float lds[2][T / 64];
    const uint32_t group = threadIdx.x / k.width, t = threadIdx.x & (k.width - 1);
    const bool drops = a.drop.on, changed = drops || a.residual;
    const uint64_t key = drops ? drop_key(a.drop) : 0;
    const float count = (float)a.C;
    // (as often for every thread: they meet)
    for (int64_t first = (int64_t)blockIdx.x * k.at_once; first < a.M; first += (int64_t)k.groups * k.at_once) {
        const int64_t row = first + group, base = row * a.C;
        const bool there = row < a.M;
        Eight<DT> q[R], res[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            q[r] = res[r] = Eight<DT>{};
            if (at.there) q[r] = at.template load<DT>(a.x, base);
            if (at.there && a.residual) res[r] = at.template load<DT>(a.residual, base);
        }
        float sum[1] = {0.0f}, squares[1] = {0.0f};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            if (!at.there) continue;
            if (changed) {
                const uint32_t keep = drops ? kept_eight(a.drop, key, base + at.c) : 0;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = q[r].get(j), of = res[r].get(j);
                    if (drops) v[j] = keep >> j & 1 ? (a.residual ? fmaf(x, a.drop.rate, of) : x * a.drop.rate) : of;
                    else v[j] = of + x;
                }
                q[r].set(v);
                if (a.sum) at.store(a.sum, base, q[r]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += at.has(j) ? q[r].get(j) : 0.0f;
        }
        row_sums(sum, k.width, lds[0]);
        const float mean = sum[0] / count;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            q[r].renew();
            if (!at.there) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = at.has(j) ? q[r].get(j) - mean : 0.0f;
                squares[0] = fmaf(d, d, squares[0]);
            }
        }
        row_sums(squares, k.width, lds[1]);
        const float rstd = 1.0f / sqrtf(squares[0] / count + a.eps);
        if (a.saved && there && t == 0) reinterpret_cast<float2*>(a.saved)[row] = make_float2(mean, rstd);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            q[r].renew();
            if (!at.there) continue;
            float w[8], b[8], v[8];
            at.params(a.weight, a.param_dtype, 1.0f, w);
            at.params(a.bias, a.param_dtype, 0.0f, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf((q[r].get(j) - mean) * rstd, w[j], b[j]);
            q[r].set(v);
            at.store(a.y, base, q[r]);
        }
    }
}

// Of few rows: both parameters' gradients of 32 columns, over all rows, by one workgroup, beside those that the rows have.
constexpr int64_t kFewRows = 1024;
template <int DT, int T>
__device__ __forceinline__ void columns_alone(const LayerNormArgs& a, uint32_t block)
{
    __shared__ double lds[2][T / 32][33];
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5, slices = T / 32;
    const int c = (int)(32 * block + x);
    float dw = 0.0f, db = 0.0f;
    if (c < a.C)
#pragma unroll 8
        for (int64_t row = y; row < a.M; row += slices) {
            const float2 stats = reinterpret_cast<const float2*>(a.saved)[row];
            const float g = load_as<DT>(a.dy, row * a.C + c);
            dw = fmaf(g, (load_as<DT>(a.s, row * a.C + c) - stats.x) * stats.y, dw);
            db += g;
        }
    lds[0][y][x] = (double)dw;
    lds[1][y][x] = (double)db;
    __syncthreads();
    void* to = y == 0 ? a.dweight : a.dbias;
    if (y > 1 || c >= a.C || !to) return;
    double s = 0.0;
    for (uint32_t i = 0; i < slices; ++i) s += lds[y][i][x];
    if (a.param_dtype == kBf16) store_as<kBf16>(to, c, (float)s);
    else store_as<kF32>(to, c, (float)s);
}

// parts[workgroup][2][C]: sums over its rows of dy xh and of dy; null: they are not wanted.  ALONE: the workgroups behind k.groups have
// the parameters' gradients.
template <int DT, int R, int END, int T, bool ALONE>
__global__ __launch_bounds__(T) void layernorm_bwd_kernel(LayerNormArgs a, Rows k, float* parts)
{
    // rows that take more registers than there are beside the gradients' sums are read again for the result (500 x 30000 in fp32: 135 us,
    // held 174; 8192 x 4096 in fp32: held 116 us, read again 130)
    constexpr bool kHold = R * T < 4096;
    __shared__ float lds[2][2 * (T / 64)];
    extern __shared__ float columns[];          // [2][C], where a workgroup has several rows at once
    if (ALONE) {
        if (blockIdx.x >= k.groups) {
            columns_alone<DT, T>(a, blockIdx.x - k.groups);
            return;
        }
        if (!a.dx && !a.dresidual) return;
    }
    const uint32_t group = threadIdx.x / k.width, t = threadIdx.x & (k.width - 1);
    const bool drops = a.drop.on && a.dx;
    const uint64_t key = drops ? drop_key(a.drop) : 0;
    const float count = (float)a.C;
    float dw[R][8] = {}, db[R][8] = {};
    uint32_t turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * k.at_once; first < a.M; first += (int64_t)k.groups * k.at_once) {
        const int64_t row = first + group, base = row * a.C;
        const bool there = row < a.M;
        Eight<DT> s[R], dy[R], more[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            s[r] = dy[r] = more[r] = Eight<DT>{};
            if (at.there) s[r] = at.template load<DT>(a.s, base);
            if (at.there) dy[r] = at.template load<DT>(a.dy, base);
            if (kHold && at.there && a.dsum) more[r] = at.template load<DT>(a.dsum, base);
        }
        const float2 stats = there ? reinterpret_cast<const float2*>(a.saved)[row] : make_float2(0.0f, 0.0f);
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            if (!at.there) continue;
            float w[8];
            at.params(a.weight, a.param_dtype, 1.0f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xh = (s[r].get(j) - stats.x) * stats.y, g = dy[r].get(j), d = g * w[j];
                if (!at.has(j)) continue;
                dw[r][j] = fmaf(g, xh, dw[r][j]);
                db[r][j] += g;
                sums[0] += d;
                sums[1] = fmaf(d, xh, sums[1]);
            }
        }
        if (!a.dx && !a.dresidual) continue;            // (all of the workgroup: it does not meet)
        row_sums(sums, k.width, lds[turn]);
        turn ^= 1;
        const float m1 = sums[0] / count, m2 = sums[1] / count;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const Span<END> at(t + r * k.width, a.C, there, r + 1 == R);
            s[r].renew();
            dy[r].renew();
            if (!at.there) continue;
            if (!kHold) {
                s[r] = at.template load<DT>(a.s, base);
                dy[r] = at.template load<DT>(a.dy, base);
                if (a.dsum) more[r] = at.template load<DT>(a.dsum, base);
            }
            float w[8], v[8];
            at.params(a.weight, a.param_dtype, 1.0f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xh = (s[r].get(j) - stats.x) * stats.y, d = dy[r].get(j) * w[j], g = d - m1 - xh * m2;
                v[j] = fmaf(stats.y, g, more[r].get(j));
            }
            Eight<DT> q;
            if (a.dresidual || !drops) {
                q.set(v);
                if (a.dresidual) at.store(a.dresidual, base, q);
                if (a.dx && !drops) at.store(a.dx, base, q);
            }
            if (drops) {
                const uint32_t keep = kept_eight(a.drop, key, base + at.c);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = keep >> j & 1 ? v[j] * a.drop.rate : 0.0f;
                q.set(v);
                at.store(a.dx, base, q);
            }
        }
    }
    if (ALONE || !parts) return;
    // the rows that a wave has side by side, then one wave's, or one row's several waves, after the other
    for (uint32_t m = k.width; m < 64; m <<= 1)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[r][j] += __shfl_xor(dw[r][j], (int)m);
                db[r][j] += __shfl_xor(db[r][j], (int)m);
            }
    const uint32_t wide = k.width < 64 ? 64 : k.width, turns = blockDim.x / wide, mine = threadIdx.x / wide;
    float* const to = parts + (int64_t)blockIdx.x * 2 * a.C;
    for (uint32_t g = 0; g < turns; ++g) {
        if (mine == g && threadIdx.x - mine * wide < k.width) {
            float* const into = g + 1 == turns ? to : columns;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const Span<END> at(t + r * k.width, a.C, true, r + 1 == R);
                if (!at.there) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int c = at.c + j;
                    if (!at.has(j)) continue;
                    if (g) {
                        dw[r][j] += columns[c];
                        db[r][j] += columns[a.C + c];
                    }
                    into[c] = dw[r][j];
                    into[a.C + c] = db[r][j];
                }
            }
        }
        if (g + 1 < turns) __syncthreads();
    }
}

// dw and db: the parts' sums of 32 columns (backward, 16, 32 and 64 of them: 8192 x 4096 in bfloat16 68.5, 65 and 66 us, 131072 x 64 27.8, 28.3
// and 29.9)
constexpr int kParamThreads = 512;
__global__ __launch_bounds__(kParamThreads) void layernorm_params_kernel(LayerNormArgs a, const float* parts, uint32_t groups)
{
    __shared__ double lds[kParamThreads / 32][33];
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x, of = blockIdx.y;
    double s = 0.0;
    if (c < (uint32_t)a.C)
#pragma unroll 8
        for (uint32_t g = y; g < groups; g += kParamThreads / 32) s += (double)parts[((int64_t)g * 2 + of) * a.C + c];
    lds[y][x] = s;
    __syncthreads();
    void* to = of ? a.dbias : a.dweight;
    if (y || c >= (uint32_t)a.C || !to) return;
    for (int i = 1; i < kParamThreads / 32; ++i) s += lds[i][x];
    if (a.param_dtype == kBf16) store_as<kBf16>(to, c, (float)s);
    else store_as<kF32>(to, c, (float)s);
}

uint32_t power_from(uint32_t n)
{
    uint32_t p = 1;
    while (p < n) p *= 2;
    return p;
}

// As many threads to a row as it has vectors, half of them and again while that leaves enough waves for the chip and `most` vectors
// hold the row.  (In bfloat16, at most one vector, two and three.  Forward: 20011 x 1031 60, 44 and 43 us, 8192 x 4096 47, 44 and 44;
// in fp32 the latter 96, 102 and 102.  Backward, where the gradients' sums take registers too: 20011 x 1031 56, 52 and 72 us,
// 8192 x 4096 67, 65 and 65.)
Rows rows_of(const LayerNormArgs& a, uint32_t most, uint32_t threads, int64_t waves)
{
    Rows k{};
    const uint32_t vectors = (uint32_t)((a.C + 7) / 8);
    k.width = power_from(vectors) < 1024 ? power_from(vectors) : 1024;
    auto need = [&](uint32_t width) { return (vectors + width - 1) / width; };
    while (k.width > 64 && need(k.width / 2) <= most && a.M * (k.width / 2) >= waves * 64) k.width /= 2;
    k.R = need(k.width);
    if (threads < k.width) threads = k.width;
    k.at_once = threads / k.width;
    return k;
}

// (with 512 threads forward 8192 x 4096 in bfloat16 takes 45 us for 44, with 256 backward 77 for 65)
constexpr uint32_t kFwdThreads = 256, kBwdThreads = 512, kFwdMost = 3, kBwdMost = 2;

Rows fwd_rows(const LayerNormArgs& a)
{
    Rows k = rows_of(a, kFwdMost, kFwdThreads, 4096);
    const int64_t groups = (a.M + k.at_once - 1) / k.at_once;
    k.groups = (uint32_t)(groups < (1 << 20) ? groups : 1 << 20);
    return k;
}
// Two workgroups to a compute unit, what registers leave room for, each with one part of the parameters' gradients; one, and half as many
// parts, where they have 1024 threads, or come round to fewer than four turns each.  (One, two and three, bfloat16: 20011 x 1031 70, 52 and
// 64 us, 8192 x 4096 70, 65 and 74; 2000 x 1031, few turns, one and two: 15.6 and 18.7, 2048 x 4096 27 and 31; of 1024 threads 2048 x 16384
// 83 and 110.  Few rows leave no parts: 300 x 4096 6.1 and 5.1.)
bool few_rows(const LayerNormArgs& a, const Rows& k) { return a.M <= kFewRows && k.R <= kBwdMost; }
Rows bwd_rows(const LayerNormArgs& a)
{
    Rows k = rows_of(a, kBwdMost, kBwdThreads, 2048);
    const int64_t groups = (a.M + k.at_once - 1) / k.at_once, most = 256 * (k.width == 1024 || (groups < 2048 && !few_rows(a, k)) ? 1 : 2);
    k.groups = (uint32_t)(groups < most ? groups : most);
    return k;
}

// f(type, R, how rows end, how many threads a workgroup has at most): of more than MOST vectors only 1024
template <int MOST, class F>
void with_rows(const LayerNormArgs& a, const Rows& k, F f)
{
    using std::integral_constant;
    auto of = [&](auto dt) {
        auto ended = [&](auto r, auto e) {
            if constexpr (e.value != kShort)
                if (r.value > MOST || k.width * k.at_once > 512) return f(dt, r, e, integral_constant<int, 1024>{});
            if constexpr (r.value <= MOST) f(dt, r, e, integral_constant<int, 512>{});
        };
        auto held = [&](auto r) {
            if (a.C % 8 == 0) ended(r, integral_constant<int, kWhole>{});
            else if (a.C > 8) ended(r, integral_constant<int, kOverlap>{});
            else if constexpr (r.value == 1) ended(r, integral_constant<int, kShort>{});
        };
        if (k.R == 1) held(integral_constant<int, 1>{});
        else if (k.R == 2) held(integral_constant<int, 2>{});
        else if (k.R == 3) held(integral_constant<int, 3>{});
        else held(integral_constant<int, 4>{});
    };
    if (a.dtype == kBf16) of(integral_constant<int, kBf16>{});
    else of(integral_constant<int, kF32>{});
}

} // namespace

size_t layernorm_workspace(const LayerNormArgs& a) { return (size_t)bwd_rows(a).groups * 2 * a.C * sizeof(float); }

hipError_t launch_layernorm_fwd(const LayerNormArgs& a, hipStream_t stream)
{
    const Rows k = fwd_rows(a);
    ProfileScope ps(K_LAYERNORM_FWD, stream);
    with_rows<kFwdMost>(a, k, [&](auto dt, auto r, auto end, auto t) {
        hipLaunchKernelGGL((layernorm_fwd_kernel<dt.value, r.value, end.value, t.value>), dim3(k.groups), dim3(k.width * k.at_once), 0, stream,
                           a, k);
    });
    return hipGetLastError();
}

hipError_t launch_layernorm_bwd(const LayerNormArgs& a, void* workspace, hipStream_t stream)
{
    const Rows k = bwd_rows(a);
    // (in the same launch only where no row's gradients are written over what the columns' sums read)
    const bool over = a.dx && (a.dx == a.dy || a.dx == a.s), over_too = a.dresidual && (a.dresidual == a.dy || a.dresidual == a.s);
    const bool params = a.dweight || a.dbias, alone = params && few_rows(a, k) && !over && !over_too;
    float* parts = params && !alone ? static_cast<float*>(workspace) : nullptr;
    {
        ProfileScope ps(K_LAYERNORM_BWD, stream);
        // (several rows of 256 threads at most, two vectors to each: 32 KB)
        const size_t lds = k.at_once > 1 && parts ? 2 * (size_t)a.C * sizeof(float) : 0;
        const dim3 grid(k.groups + (alone ? (uint32_t)((a.C + 31) / 32) : 0));
        with_rows<kBwdMost>(a, k, [&](auto dt, auto r, auto end, auto t) {
            if (alone) {
                if constexpr (r.value <= kBwdMost)
                    hipLaunchKernelGGL((layernorm_bwd_kernel<dt.value, r.value, end.value, t.value, true>), grid, dim3(t.value), 0, stream, a, k, parts);
            } else {
                hipLaunchKernelGGL((layernorm_bwd_kernel<dt.value, r.value, end.value, t.value, false>), grid, dim3(t.value), lds, stream, a, k, parts);
            }
        });
    }
    if (parts) {
        ProfileScope ps(K_LAYERNORM_PARAMS, stream);
        hipLaunchKernelGGL(layernorm_params_kernel, dim3((uint32_t)((a.C + 31) / 32), 2), dim3(kParamThreads), 0, stream, a, parts, k.groups);
    }
    return hipGetLastError();
}

} // namespace hdqt
