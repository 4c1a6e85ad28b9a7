// Low-rank adapters beside a shared projection, rows of one call with adapters of their own (gfx950):
//   h_i = x_i A_a,   out_i = base_i + scale_a h_i B_a,   a = ids[i], A [K, r], B [r, N] of each adapter
// and the gradients, g = dy B^T of a row's adapter times scale_a:
//   dx_i = base_i + g_i A_a^T,   dA_a = sum x_i^T g_i,   dB_a = sum scale_a h_i^T dy_i   (over the rows that have a)
// Four products with an axis of r, at most 128: memory bounds them, reading x, dy and the adapters and writing what is as large.
//
// Rows are grouped by adapter, in their order, first: tiles of 32 rows of one adapter, which a launch of one workgroup writes down
// (the plan); up to 64 rows need none, a wave sees them all by a ballot.  Then "down": a tile's h, or g, the contraction over K or N
// split over a workgroup's eight waves and, where tiles are few, over workgroups, whose parts whoever reads h adds up; "up": a
// tile's part of out or dx; "weights": an adapter's gradients, 128 columns (64 in fp32) to a workgroup.
//
// All three take their operands from memory straight into the matrix instructions' registers, 16 bytes a lane and load: the order
// of a contraction is free as long as both operands have the same, and so is which of the product's columns a lane's are.  Where
// memory runs along the contraction, a load is a fragment; where it runs across it, a lane loads as many lines of the contraction as
// a fragment has, and turns them in registers: lane i then has the columns i kLane to i kLane + kLane - 1, in as many
// products.  Nothing goes through LDS but the sums of waves.
//
// bfloat16: h, g and their sums are held in 32 bits.  Where they are multiplied again each is taken as two bfloat16 values, the first
// cut off and the second rounded: off by 2^-16 of itself at most.  fp32: products in 32 bits.
#include "train.hpp"

#include <type_traits>

namespace hdqt {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int kSubs = 2, kTile = 16 * kSubs;        // rows of a tile, in blocks of the matrix instruction
constexpr int kDownWaves = 8, kUpWaves = 4, kWeightWaves = 4;
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kMostGroups = kAdaptersMost + 2;

enum Mode { kAlong, kDown };        // memory runs along the contraction, or across it

// 16 bytes of a line: eight bfloat16 values or four of 32 bits
struct Piece {
    uint32_t w[4];
};
template <int DT>
constexpr int lane_of() { return DT == kF32 ? 4 : 8; }

// (n: how many of them there are; the others are zero)
template <int DT>
__device__ __forceinline__ Piece load_piece(const void* p, int64_t at, int n)
{
    constexpr int L = lane_of<DT>();
    Piece q{};
    const char* from = static_cast<const char*>(p) + at * (16 / L);
    if (n >= L) {
        __builtin_memcpy(q.w, from, 16);
    } else {
#pragma unroll
        for (int j = 0; j < L - 1; ++j)
            if (j < n) {
                if (DT == kF32) q.w[j & 3] = static_cast<const uint32_t*>(p)[at + j];
                else q.w[j / 2] |= (uint32_t)static_cast<const uint16_t*>(p)[at + j] << 16 * (j & 1);
            }
    }
    return q;
}
template <int DT>
__device__ __forceinline__ void store_piece(void* p, int64_t at, int n, const Piece& q)
{
    constexpr int L = lane_of<DT>();
    if (n >= L) {
        __builtin_memcpy(static_cast<char*>(p) + at * (16 / L), q.w, 16);
        return;
    }
#pragma unroll
    for (int j = 0; j < L - 1; ++j)
        if (j < n) {
            if (DT == kF32) static_cast<uint32_t*>(p)[at + j] = q.w[j & 3];
            else static_cast<uint16_t*>(p)[at + j] = (uint16_t)(q.w[j / 2] >> 16 * (j & 1));
        }
}
template <int DT>
__device__ __forceinline__ float value(const Piece& q, int j)
{
    if (DT == kF32) return __uint_as_float(q.w[j & 3]);
    return __uint_as_float(j & 1 ? q.w[j / 2] & 0xFFFF0000u : q.w[j / 2] << 16);
}
template <int DT>
__device__ __forceinline__ Piece piece_of(const float (&v)[lane_of<DT>()])
{
    Piece q;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == kF32) q.w[j] = __float_as_uint(v[j]);
        else q.w[j] = to_bf16(v[2 * j]) | to_bf16(v[2 * j + 1]) << 16;
    }
    return q;
}

// N neighbouring elements of a line, in the first places of a piece
template <int DT, int N>
__device__ __forceinline__ Piece load_few(const void* p, int64_t at, int n)
{
    if constexpr (N == lane_of<DT>()) return load_piece<DT>(p, at, n);
    Piece q{};
    const char* from = static_cast<const char*>(p) + at * (DT == kF32 ? 4 : 2);
    if (n >= N) {
        __builtin_memcpy(q.w, from, N * (DT == kF32 ? 4 : 2));
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < n) {
                if (DT == kF32) q.w[j & 3] = static_cast<const uint32_t*>(p)[at + j];
                else q.w[j / 2] |= (uint32_t)static_cast<const uint16_t*>(p)[at + j] << 16 * (j & 1);
            }
    }
    return q;
}

// Fragment t of lines that run across the contraction: element t of each
template <int DT>
__device__ __forceinline__ Piece turned(const Piece (&in)[lane_of<DT>()], int t)
{
    Piece out;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        if constexpr (DT == kF32) out.w[d] = in[d].w[t & 3];
        else out.w[d] = __builtin_amdgcn_perm(in[2 * d + 1].w[t / 2], in[2 * d].w[t / 2], t & 1 ? 0x07060302u : 0x05040100u);
    }
    return out;
}

// d(i, j) += sum over the fragments' contraction of a(i) b(j): lane l has line l % 16 of either and of the contraction the
// elements from kLane (l / 16) on; of d column l % 16, rows 4 (l / 16) to 4 (l / 16) + 3
template <int DT>
__device__ __forceinline__ v4f multiply(const Piece& a, const Piece& b, v4f d)
{
#ifdef __HIP_DEVICE_COMPILE__
    if constexpr (DT == kF32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) d = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[k]), __uint_as_float(b.w[k]), d, 0, 0, 0);
    } else {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), d, 0, 0, 0);
    }
#endif
    return d;
}

// 32-bit values as the matrix instructions take them: themselves, or two planes of bfloat16
template <int DT>
constexpr int planes_of() { return DT == kF32 ? 1 : 2; }
template <int DT>
__device__ __forceinline__ void split(const float (&v)[lane_of<DT>()], Piece (&to)[planes_of<DT>()])
{
    if constexpr (DT == kF32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[0].w[j] = __float_as_uint(v[j]);
    } else {
        uint32_t first[8], second[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            first[j] = __float_as_uint(v[j]) >> 16;
            const float cut = from_bf16(first[j]);
            second[j] = v[j] == cut ? 0u : to_bf16(v[j] - cut);         // (equal: an infinity has no rest)
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            to[0].w[j] = first[2 * j] | first[2 * j + 1] << 16;
            to[1].w[j] = second[2 * j] | second[2 * j + 1] << 16;
        }
    }
}

// ---- which rows have which adapter ----

// groups: an adapter's rows for each of n; n: rows without one; n + 1: rows whose number is none
__device__ __forceinline__ uint32_t group_of(int64_t id, int n) { return id < 0 ? (uint32_t)n : id < n ? (uint32_t)id : (uint32_t)n + 1; }

// The plan in memory: start[groups + 1] (a group's first place in the order), tiles, order[M] (rows), tile[..] (group, first place)
struct Plan {
    const uint32_t *start, *tiles, *order;
    const uint2* tile;
};
__host__ __device__ inline size_t plan_words(int64_t M, int n) { return (size_t)(n + 3 + 1 + M); }
__host__ __device__ inline int64_t most_tiles(int64_t M, int n) { return M / kTile + (n + 2 < M ? n + 2 : M); }
__host__ __device__ inline Plan plan_at(const void* p, int64_t M, int n)
{
    const uint32_t* w = static_cast<const uint32_t*>(p);
    return {w, w + n + 3, w + n + 4, reinterpret_cast<const uint2*>(w + (plan_words(M, n) + 1) / 2 * 2)};
}

constexpr int64_t kDirect = 64;         // as many rows a wave sees at once

// lanes with the same value of `bits` bits
__device__ __forceinline__ uint64_t same_lanes(uint32_t v, int bits, uint64_t among)
{
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(v >> b & 1);
        among &= v >> b & 1 ? set : ~set;
    }
    return among;
}

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const int64_t* ids, int64_t M, int n, int bits, uint32_t* plan)
{
    __shared__ uint32_t counts[kPlanWaves][kMostGroups];
    __shared__ uint32_t starts[kMostGroups + 1], tiles[kMostGroups + 1], waves[2][kPlanWaves];
    const Plan p = plan_at(plan, M, n);
    uint32_t *start = const_cast<uint32_t*>(p.start), *order = const_cast<uint32_t*>(p.order);
    const uint32_t groups = (uint32_t)n + 2;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t rows = (M + 64 * kPlanWaves - 1) / (64 * kPlanWaves) * 64, first = wave * rows, end = first + rows < M ? first + rows : M;
    for (uint32_t i = threadIdx.x; i < kPlanWaves * kMostGroups; i += kPlanThreads) (&counts[0][0])[i] = 0;
    __syncthreads();
#pragma unroll 4
    for (int64_t i = first + lane; i < end; i += 64) atomicAdd(&counts[wave][group_of(ids[i], n)], 1u);
    __syncthreads();
    // a thread's two groups: their rows and tiles, and the sums of those of the groups before
    uint32_t have[2] = {0, 0}, cut[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g < groups)
            for (int w = 0; w < kPlanWaves; ++w) {
                const uint32_t c = counts[w][g];
                counts[w][g] = have[u];             // (of the group's rows, those of the waves before)
                have[u] += c;
            }
        cut[u] = (have[u] + kTile - 1) / kTile;
    }
    uint32_t before[2] = {have[0] + have[1], cut[0] + cut[1]};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t own = before[u];
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t up = __shfl_up(before[u], m);
            if (lane >= m) before[u] += up;
        }
        if (lane == 63) waves[u][wave] = before[u];
        before[u] -= own;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
        for (int w = 0; w < wave; ++w) before[u] += waves[u][w];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g <= groups) {
            starts[g] = before[0];
            tiles[g] = before[1];
            start[g] = before[0];
        }
        before[0] += have[u];
        before[1] += cut[u];
    }
    __syncthreads();
    const uint32_t total = tiles[groups];
    if (threadIdx.x == 0) *const_cast<uint32_t*>(p.tiles) = total;
    for (uint32_t i = threadIdx.x; i < total; i += kPlanThreads) {
        uint32_t lo = 0, hi = groups;               // the last group whose first tile is not behind this one
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (tiles[mid] <= i) lo = mid;
            else hi = mid;
        }
        const_cast<uint2*>(p.tile)[i] = make_uint2(lo, starts[lo] + kTile * (i - tiles[lo]));
    }
    for (int64_t i = first; i < end; i += 64) {
        const bool there = i + lane < end;
        const uint32_t g = there ? group_of(ids[i + lane], n) : 0;
        const uint64_t same = same_lanes(g, bits, __ballot(there));
        const int leader = __ffsll((unsigned long long)same) - 1;
        uint32_t at = 0;
        if (there && lane == leader) at = atomicAdd(&counts[wave][g], (uint32_t)__popcll(same));
        at = __shfl(at, leader & 63);
        if (there) order[starts[g] + at + (uint32_t)__popcll(same & ((1ull << lane) - 1))] = (uint32_t)(i + lane);
    }
}

// Rows of one group, for a wave: `count` of them, place p's row by row(p).
struct Group {
    uint32_t group, count;
    const uint32_t* order;          // the plan's, from the group's or the tile's first place on, or null:
    uint32_t listed;                // of up to 64 rows, lane p has place p's
    __device__ __forceinline__ uint32_t row(uint32_t place) const
    {
        return order ? order[place] : __shfl(listed, (int)place);
    }
};

// of up to 64 rows, those of a group
__device__ __forceinline__ Group listed_group(uint32_t group, uint32_t of_lane, bool there)
{
    const int lane = threadIdx.x & 63;
    const uint64_t same = __ballot(there && of_lane == group);
    const uint64_t lower = (1ull << lane) - 1;
    // (the others go behind them, each to a place of its own)
    const int count = __popcll(same), to = same >> lane & 1 ? __popcll(same & lower) : count + __popcll(~same & lower);
    return {group, (uint32_t)count, nullptr, (uint32_t)__builtin_amdgcn_ds_permute(4 * to, lane)};
}

struct RowArgs {
    const int64_t* ids;
    const void* plan;
    int64_t M;
    int n;
};

// The rows of workgroup `tile`: none where there is no such tile, or where an earlier row of the few has them.
__device__ __forceinline__ Group tile_rows(const RowArgs& a, uint32_t tile)
{
    if (a.M <= kDirect) {
        const int lane = threadIdx.x & 63;
        const bool there = lane < a.M;
        const uint32_t g = there ? group_of(a.ids[lane], a.n) : 0;
        const uint32_t mine = __shfl(g, (int)tile);
        Group of = listed_group(mine, g, there);
        const uint64_t same = __ballot(there && g == mine);
        if ((uint32_t)__ffsll((unsigned long long)same) - 1 != tile) of.count = 0;
        return of;
    }
    const Plan p = plan_at(a.plan, a.M, a.n);
    if (tile >= *p.tiles) return {0, 0, p.order, 0};
    const uint2 t = p.tile[tile];
    const uint32_t left = p.start[t.x + 1] - t.y;
    return {t.x, left < kTile ? left : kTile, p.order + t.y, 0};
}
__device__ __forceinline__ Group adapter_rows(const RowArgs& a, uint32_t adapter)
{
    if (a.M <= kDirect) {
        const int lane = threadIdx.x & 63;
        const bool there = lane < a.M;
        return listed_group(adapter, there ? group_of(a.ids[lane], a.n) : 0, there);
    }
    const Plan p = plan_at(a.plan, a.M, a.n);
    return {adapter, p.start[adapter + 1] - p.start[adapter], p.order + p.start[adapter], 0};
}

// ---- down ----

struct DownArgs {
    RowArgs rows;
    const void *x, *W;              // [M, D]; of an adapter [D, r] (kDown) or [r, D] (kAlong)
    float* h;                       // [parts][M][16 RT]
    int64_t D;
    int r;
    uint32_t parts, chunks;         // of the contraction: parts, and how many times 4 kLane a part has
};

template <int DT, int RT, int MODE>
__global__ __launch_bounds__(64 * kDownWaves) void down_kernel(DownArgs a)
{
    constexpr int L = lane_of<DT>(), kChunk = 4 * L, RL = RT < L ? RT : L, RQ = RT / RL;
    // tile t + RL q of the ranks: a lane's is 16 RL q + RL (l % 16) + t
    __shared__ v4f sums[kDownWaves / 2][kSubs][RT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const Group rows = tile_rows(a.rows, blockIdx.x);
    if (!rows.count || rows.group >= (uint32_t)a.rows.n) return;
    const char* W = static_cast<const char*>(a.W) + (int64_t)rows.group * a.D * a.r * (16 / L);
    const int64_t first = (int64_t)blockIdx.y * a.chunks, all = (a.D + kChunk - 1) / kChunk;
    const int64_t last = first + a.chunks < all ? first + a.chunks : all;
    for (uint32_t place = 0; place < rows.count; place += kTile) {
        int64_t line[kSubs];
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
            const uint32_t p = place + 16 * s + j;          // (rows behind the last: any that there is)
            line[s] = (int64_t)rows.row(p < rows.count ? p : place) * a.D;
        }
        v4f acc[kSubs][RT] = {};
        auto chunk = [&](int64_t c, auto whole) {
            const int64_t k = c * kChunk + L * g;
            const int n = whole.value || k + L <= a.D ? L : k < a.D ? (int)(a.D - k) : 0;
            Piece x[kSubs], w[RT];
#pragma unroll
            for (int s = 0; s < kSubs; ++s) x[s] = load_piece<DT>(a.x, line[s] + k, whole.value ? L : n);
#pragma unroll
            for (int q = 0; q < RQ; ++q) {
                const int c0 = 16 * RL * q + RL * j;
                if constexpr (MODE == kDown) {
                    Piece lines[L];
#pragma unroll
                    for (int e = 0; e < L; ++e) {
                        lines[e] = Piece{};
                        if (whole.value || e < n) lines[e] = load_few<DT, RL>(W, (k + e) * a.r + c0, a.r - c0);
                    }
#pragma unroll
                    for (int t = 0; t < RL; ++t) w[RL * q + t] = turned<DT>(lines, t);
                } else {
#pragma unroll
                    for (int t = 0; t < RL; ++t) {
                        w[RL * q + t] = Piece{};
                        if (c0 + t < a.r) w[RL * q + t] = load_piece<DT>(W, (c0 + t) * a.D + k, whole.value ? L : n);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[s][t] = multiply<DT>(x[s], w[t], acc[s][t]);
        };
        const int64_t full = a.D / kChunk < last ? a.D / kChunk : last;
        int64_t c = first + wave;
#pragma unroll 4
        for (; c < full; c += kDownWaves) chunk(c, std::true_type{});
        if (c < last) chunk(c, std::false_type{});
#pragma unroll
        for (int half = kDownWaves / 2; half; half /= 2) {
            __syncthreads();
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int s = 0; s < kSubs; ++s)
#pragma unroll
                    for (int t = 0; t < RT; ++t) sums[wave - half][s][t][lane] = acc[s][t];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int s = 0; s < kSubs; ++s)
#pragma unroll
                    for (int t = 0; t < RT; ++t) acc[s][t] += sums[wave][s][t][lane];
        }
        if (wave == 0)
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t p = place + 16 * s + 4 * g + i;
                    const uint32_t row = rows.row(p < rows.count ? p : place);
                    if (p >= rows.count) continue;
                    float* to = a.h + ((int64_t)blockIdx.y * a.rows.M + row) * (16 * RT);
#pragma unroll
                    for (int q = 0; q < RQ; ++q)
#pragma unroll
                        for (int t = 0; t < RL; ++t) {
                            const int c0 = 16 * RL * q + RL * j + t;
                            to[c0] = c0 < a.r ? acc[s][RL * q + t][i] : 0.0f;       // (0 x infinity behind the last rank)
                        }
                }
    }
}

// ---- up ----

struct UpArgs {
    RowArgs rows;
    const float* h;                 // [parts][M][16 RT]
    const float* scale;             // [n] or null
    const void* W;                  // of an adapter [r, N] (kDown) or [N, r] (kAlong)
    const void* base;               // [M, N] or null
    void* out;                      // [M, N]
    int64_t N;
    int r;
    uint32_t parts;
};

// a row's values from `rank` on, all parts together, times `scale`
template <int N>
__device__ __forceinline__ void load_h(const float* h, int64_t part, uint32_t parts, float scale, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = 0.0f;
    for (uint32_t s = 0; s < parts; ++s)
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const float4 q = *reinterpret_cast<const float4*>(h + s * part + j);
            v[j] += q.x;
            v[j + 1] += q.y;
            v[j + 2] += q.z;
            v[j + 3] += q.w;
        }
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] *= scale;
}

template <int DT, int RT, int MODE>
__global__ __launch_bounds__(64 * kUpWaves) void up_kernel(UpArgs a)
{
    constexpr int L = lane_of<DT>(), kChunk = 4 * L, kColumns = 16 * L;
    // bfloat16, one tile of ranks: both planes are one chunk, the second beside the same lines of W again
    constexpr bool kFolded = DT == kBf16 && RT == 1;
    constexpr int P = kFolded ? 1 : planes_of<DT>(), C = 16 * RT < kChunk ? 1 : 16 * RT / kChunk, kRanks = 16 * RT;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const Group rows = tile_rows(a.rows, blockIdx.x);
    if (!rows.count) return;
    const bool none = rows.group == (uint32_t)a.rows.n, wrong = rows.group > (uint32_t)a.rows.n;
    if (none && a.base == a.out) return;
    const char* W = static_cast<const char*>(a.W) + (none || wrong ? 0 : (int64_t)rows.group * a.N * a.r * (16 / L));
    const float scale = a.scale && !none && !wrong ? a.scale[rows.group] : 1.0f;
    const int at = L * (kFolded ? g & 1 : g);              // a lane's first rank of a chunk
    for (uint32_t place = 0; place < rows.count; place += kTile) {
        Piece h[kSubs][C][P];
        int64_t line[kSubs][4];
        bool there[kSubs][4];
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
            const uint32_t p = place + 16 * s + j;
            const uint32_t row = rows.row(p < rows.count ? p : place);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[L] = {};
                if (!none && !wrong) load_h<L>(a.h + (int64_t)row * kRanks + kChunk * c + at, a.rows.M * kRanks, a.parts, scale, v);
                Piece two[planes_of<DT>()];
                split<DT>(v, two);
                if constexpr (kFolded) h[s][c][0] = g < 2 ? two[0] : two[1];
                else
#pragma unroll
                    for (int k = 0; k < P; ++k) h[s][c][k] = two[k];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t q = place + 16 * s + 4 * g + i;
                there[s][i] = q < rows.count;
                line[s][i] = (int64_t)rows.row(there[s][i] ? q : place) * a.N;
            }
        }
        for (int64_t c0 = ((int64_t)blockIdx.y * kUpWaves + wave) * kColumns; c0 < a.N; c0 += (int64_t)gridDim.y * kUpWaves * kColumns) {
            const int64_t col = c0 + L * j;
            const int n = col + L <= a.N ? L : col < a.N ? (int)(a.N - col) : 0;
            Piece base[kSubs][4];
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    base[s][i] = Piece{};
                    if (a.base && there[s][i]) base[s][i] = load_piece<DT>(a.base, line[s][i] + col, n);
                }
            v4f acc[kSubs][L] = {};
            if (!none && !wrong)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int rank = kChunk * c + at;
                    Piece w[L];
                    if constexpr (MODE == kDown) {
                        Piece lines[L];
#pragma unroll
                        for (int e = 0; e < L; ++e) {
                            lines[e] = Piece{};
                            if (rank + e < a.r) lines[e] = load_piece<DT>(W, (rank + e) * a.N + col, n);
                        }
#pragma unroll
                        for (int t = 0; t < L; ++t) w[t] = turned<DT>(lines, t);
                    } else {
#pragma unroll
                        for (int t = 0; t < L; ++t) {
                            w[t] = Piece{};
                            if (t < n) w[t] = load_piece<DT>(W, (col + t) * a.r + rank, a.r - rank);
                        }
                    }
#pragma unroll
                    for (int k = P - 1; k >= 0; --k)
#pragma unroll
                        for (int s = 0; s < kSubs; ++s)
#pragma unroll
                            for (int t = 0; t < L; ++t) acc[s][t] = multiply<DT>(h[s][c][k], w[t], acc[s][t]);
                }
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[L];
#pragma unroll
                    for (int t = 0; t < L; ++t) v[t] = wrong ? __builtin_nanf("") : value<DT>(base[s][i], t) + acc[s][t][i];
                    if (there[s][i]) store_piece<DT>(a.out, line[s][i] + col, n, piece_of<DT>(v));
                }
        }
    }
}

// ---- weights ----

// an adapter's gradient: W[j][c] = sum over its rows of scale h[row][j] v[row][c]
struct WeightArgs {
    RowArgs rows;
    const float* h[2];              // dA: g; dB: h.  [parts][M][16 RT]
    const void* v[2];               // dA: x; dB: dy
    void* out[2];                   // [n][K][r]; [n][r][N]; either may be null
    float* sums;                    // where a gradient is added up over parts of the rows, [split][n][r][K + N], else null
    const float* scale;
    int64_t N[2];
    int r;
    uint32_t parts[2], blocks[2], split;        // blocks of columns
};

template <int DT, int RT>
__global__ __launch_bounds__(64 * kWeightWaves) void weights_kernel(WeightArgs a)
{
    constexpr int L = lane_of<DT>(), kChunk = 4 * L, kColumns = 16 * L, RW = RT < 2 ? RT : 2, P = planes_of<DT>();
    __shared__ v4f sums[kWeightWaves / 2][RW][L][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int of = blockIdx.x >= a.blocks[0];
    if (!a.out[of]) return;
    const int64_t N = a.N[of], c0 = (int64_t)(blockIdx.x - (of ? a.blocks[0] : 0)) * kColumns, col = c0 + L * j;
    const uint32_t adapter = blockIdx.y, rank0 = blockIdx.z / a.split * (16 * RW), part = blockIdx.z % a.split;
    const Group rows = adapter_rows(a.rows, adapter);
    const float* h = a.h[of] + rank0 + j;
    const int n = col + L <= N ? L : col < N ? (int)(N - col) : 0;
    v4f acc[RW][L] = {};
    // (as often for every lane of a wave: the rows of a few are handed from lane to lane)
    const uint32_t step = kChunk * kWeightWaves * a.split;
    for (uint32_t first = kChunk * (part * kWeightWaves + wave); first < rows.count; first += step) {
        Piece lines[L];
        float u[RW][L];
#pragma unroll
        for (int e = 0; e < L; ++e) {
            const uint32_t p = first + L * g + e;
            const bool there = p < rows.count;
            const int64_t row = rows.row(there ? p : first);
            lines[e] = Piece{};
            if (there) lines[e] = load_piece<DT>(a.v[of], row * N + col, n);
#pragma unroll
            for (int t = 0; t < RW; ++t) {
                u[t][e] = 0.0f;
                if (there)
                    for (uint32_t s = 0; s < a.parts[of]; ++s) u[t][e] += h[(s * a.rows.M + row) * (16 * RT) + 16 * t];
            }
        }
        Piece up[RW][P];
#pragma unroll
        for (int t = 0; t < RW; ++t) split<DT>(u[t], up[t]);
#pragma unroll
        for (int c = 0; c < L; ++c) {
            const Piece w = turned<DT>(lines, c);
#pragma unroll
            for (int t = 0; t < RW; ++t)
#pragma unroll
                for (int k = P - 1; k >= 0; --k) acc[t][c] = multiply<DT>(up[t][k], w, acc[t][c]);
        }
    }
#pragma unroll
    for (int half = kWeightWaves / 2; half; half /= 2) {
        __syncthreads();
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int t = 0; t < RW; ++t)
#pragma unroll
                for (int c = 0; c < L; ++c) sums[wave - half][t][c][lane] = acc[t][c];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int t = 0; t < RW; ++t)
#pragma unroll
                for (int c = 0; c < L; ++c) acc[t][c] += sums[wave][t][c][lane];
    }
    if (wave) return;
    const float scale = a.scale ? a.scale[adapter] : 1.0f;
    // a lane has ranks rank0 + 16 t + 4 g to + 3 of columns col to col + kLane - 1
#pragma unroll
    for (int t = 0; t < RW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int rank = (int)rank0 + 16 * t + 4 * g + i;
            if (rank >= a.r) continue;
            float v[L];
#pragma unroll
            for (int c = 0; c < L; ++c) v[c] = acc[t][c][i] * scale;
            if (a.sums) {
                float* to = a.sums + ((int64_t)(part * gridDim.y + adapter) * a.r) * (a.N[0] + a.N[1]) + (of ? (int64_t)a.r * a.N[0] : 0) + rank * N + col;
                for (int c = 0; c < n; ++c) to[c] = v[c];
            } else if (of) {
                store_piece<DT>(a.out[1], ((int64_t)adapter * a.r + rank) * N + col, n, piece_of<DT>(v));
            } else {
                for (int c = 0; c < n; ++c) store_as<DT>(a.out[0], ((int64_t)adapter * N + col + c) * a.r + rank, v[c]);
            }
        }
}

// the gradients where their rows are in parts
template <int DT>
__global__ __launch_bounds__(256) void add_parts_kernel(WeightArgs a, uint32_t n)
{
    const int64_t one = (int64_t)a.r * (a.N[0] + a.N[1]), all = one * n;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    float s = 0.0f;
    for (uint32_t part = 0; part < a.split; ++part) s += a.sums[part * all + i];
    const int64_t adapter = i / one, in = i - adapter * one, dA = (int64_t)a.r * a.N[0];
    if (in < dA) {
        const int64_t rank = in / a.N[0], c = in - rank * a.N[0];
        if (a.out[0]) store_as<DT>(a.out[0], (adapter * a.N[0] + c) * a.r + rank, s);
    } else if (a.out[1]) {
        store_as<DT>(a.out[1], adapter * a.r * a.N[1] + in - dA, s);
    }
}

int tiles_of_rank(int r) { return r <= 16 ? 1 : r <= 32 ? 2 : r <= 64 ? 4 : 8; }

// (what a grid has: tiles that may be)
uint32_t grid_tiles(const AdapterArgs& a) { return (uint32_t)(a.M <= kDirect ? a.M : most_tiles(a.M, a.n)); }

// Parts of a contraction over D: as many as make 512 workgroups, none of fewer than eight waves' chunks.
struct Parts {
    uint32_t parts, chunks;
};
Parts parts_of(const AdapterArgs& a, int64_t D)
{
    const int64_t chunk = a.dtype == kBf16 ? 32 : 16, chunks = (D + chunk - 1) / chunk;
    const int64_t tiles = a.M <= kDirect ? (a.M < a.n ? a.M : a.n) : a.M / kTile + (a.n < a.M / kTile ? a.n : a.M / kTile);
    int64_t parts = 512 / (tiles > 0 ? tiles : 1);
    if (parts > 8) parts = 8;
    while (parts > 1 && chunks < parts * kDownWaves) --parts;
    if (parts < 1) parts = 1;
    const int64_t each = (chunks + parts - 1) / parts;
    return {(uint32_t)((chunks + each - 1) / each), (uint32_t)each};
}

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t plan_bytes(const AdapterArgs& a)
{
    return a.M <= kDirect ? 0 : rounded((plan_words(a.M, a.n) + 1) / 2 * 8 + sizeof(uint2) * (size_t)most_tiles(a.M, a.n));
}
size_t h_bytes(const AdapterArgs& a, int64_t D)
{
    return rounded((size_t)parts_of(a, D).parts * (size_t)a.M * 16 * tiles_of_rank(a.r) * sizeof(float));
}

// Parts of the rows that the adapters' gradients are added up over: where columns and adapters are few workgroups, as many as make 1024
// of them, none of fewer than 128 rows to an adapter.
uint32_t split_of(const AdapterArgs& a)
{
    const int64_t columns = a.dtype == kBf16 ? 128 : 64, RT = tiles_of_rank(a.r);
    const int64_t groups = ((a.K + columns - 1) / columns + (a.N + columns - 1) / columns) * a.n * (RT < 2 ? 1 : RT / 2);
    int64_t split = 1024 / groups;
    const int64_t most = a.M / (128 * (int64_t)a.n);
    if (split > most) split = most;
    return (uint32_t)(split < 1 ? 1 : split > 16 ? 16 : split);
}
size_t sums_bytes(const AdapterArgs& a)
{
    const uint32_t split = split_of(a);
    return split > 1 ? rounded((size_t)split * a.n * a.r * (size_t)(a.K + a.N) * sizeof(float)) : 0;
}

// f(type, tiles of ranks)
template <class F>
void with_types(const AdapterArgs& a, F f)
{
    using std::integral_constant;
    auto ranks = [&](auto dt) {
        switch (tiles_of_rank(a.r)) {
        case 1: f(dt, integral_constant<int, 1>{}); break;
        case 2: f(dt, integral_constant<int, 2>{}); break;
        case 4: f(dt, integral_constant<int, 4>{}); break;
        default: f(dt, integral_constant<int, 8>{}); break;
        }
    };
    if (a.dtype == kBf16) ranks(integral_constant<int, kBf16>{});
    else ranks(integral_constant<int, kF32>{});
}

template <int MODE>
void launch_down(const AdapterArgs& a, const void* x, const void* W, float* h, int64_t D, const RowArgs& rows, hipStream_t stream)
{
    ProfileScope ps(K_ADAPT_DOWN, stream);
    const Parts p = parts_of(a, D);
    const DownArgs d{rows, x, W, h, D, a.r, p.parts, p.chunks};
    with_types(a, [&](auto dt, auto rt) {
        hipLaunchKernelGGL((down_kernel<dt.value, rt.value, MODE>), dim3(grid_tiles(a), p.parts), dim3(64 * kDownWaves), 0, stream, d);
    });
}
template <int MODE>
void launch_up(const AdapterArgs& a, const float* h, const void* W, const void* base, void* out, int64_t N, int64_t D, const RowArgs& rows,
               hipStream_t stream)
{
    ProfileScope ps(K_ADAPT_UP, stream);
    const UpArgs u{rows, h, a.scale, W, base, out, N, a.r, parts_of(a, D).parts};
    const int64_t columns = (a.dtype == kBf16 ? 128 : 64) * kUpWaves;
    int64_t across = (N + columns - 1) / columns;
    if (across > 32768) across = 32768;
    with_types(a, [&](auto dt, auto rt) {
        hipLaunchKernelGGL((up_kernel<dt.value, rt.value, MODE>), dim3(grid_tiles(a), (uint32_t)across), dim3(64 * kUpWaves), 0, stream, u);
    });
}

} // namespace

size_t adapters_saved(const AdapterArgs& a) { return plan_bytes(a) + h_bytes(a, a.K); }
size_t adapters_workspace(const AdapterArgs& a) { return h_bytes(a, a.N) + sums_bytes(a); }

hipError_t launch_adapters_fwd(const AdapterArgs& a, hipStream_t stream)
{
    float* h = reinterpret_cast<float*>(static_cast<char*>(a.saved) + plan_bytes(a));
    const RowArgs rows{a.ids, a.saved, a.M, a.n};
    if (a.M > kDirect) {
        ProfileScope ps(K_ADAPT_PLAN, stream);
        int bits = 1;
        while ((1 << bits) < a.n + 2) ++bits;
        hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a.ids, a.M, a.n, bits, static_cast<uint32_t*>(a.saved));
    }
    launch_down<kDown>(a, a.x, a.A, h, a.K, rows, stream);
    launch_up<kDown>(a, h, a.B, a.base, a.out, a.N, a.K, rows, stream);
    return hipGetLastError();
}

hipError_t launch_adapters_bwd(const AdapterArgs& a, void* workspace, hipStream_t stream)
{
    float* h = reinterpret_cast<float*>(static_cast<char*>(a.saved) + plan_bytes(a));
    float* g = static_cast<float*>(workspace);
    const RowArgs rows{a.ids, a.saved, a.M, a.n};
    if (a.out || a.dA) launch_down<kAlong>(a, a.dy, a.B, g, a.N, rows, stream);
    if (a.out) launch_up<kAlong>(a, g, a.A, a.base, a.out, a.K, a.N, rows, stream);
    if (a.dA || a.dB) {
        ProfileScope ps(K_ADAPT_WEIGHTS, stream);
        const int64_t columns = a.dtype == kBf16 ? 128 : 64, RT = tiles_of_rank(a.r);
        WeightArgs w{};
        w.rows = rows;
        w.h[0] = g; w.h[1] = h;
        w.v[0] = a.x; w.v[1] = a.dy;
        w.out[0] = a.dA; w.out[1] = a.dB;
        w.scale = a.scale;
        w.N[0] = a.K; w.N[1] = a.N;
        w.r = a.r;
        w.parts[0] = parts_of(a, a.N).parts; w.parts[1] = parts_of(a, a.K).parts;
        w.blocks[0] = (uint32_t)((a.K + columns - 1) / columns); w.blocks[1] = (uint32_t)((a.N + columns - 1) / columns);
        w.split = split_of(a);
        if (w.split > 1) w.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + h_bytes(a, a.N));
        with_types(a, [&](auto dt, auto rt) {
            hipLaunchKernelGGL((weights_kernel<dt.value, rt.value>), dim3(w.blocks[0] + w.blocks[1], (uint32_t)a.n, (uint32_t)(RT < 2 ? 1 : RT / 2) * w.split),
                               dim3(64 * kWeightWaves), 0, stream, w);
            if (w.split > 1) {
                const int64_t all = (int64_t)a.n * a.r * (a.K + a.N);
                hipLaunchKernelGGL((add_parts_kernel<dt.value>), dim3((uint32_t)((all + 255) / 256)), dim3(256), 0, stream, w, (uint32_t)a.n);
            }
        });
    }
    return hipGetLastError();
}

} // namespace hdqt
