// Low-rank adapters beside a shared projection, rows of one call with adapters of their own (gfx950):
//   h_i = x_i A_a,   out_i = base_i + scale_a h_i B_a,   a = ids[i], A [K, r], B [r, N] of each adapter
// and the gradients, g = dy B^T of a row's adapter times scale_a:
//   dx_i = base_i + g_i A_a^T,   dA_a = sum x_i^T g_i,   dB_a = sum scale_a h_i^T dy_i   (over the rows that have a)
// Four products with an axis of r, at most 128: memory bounds them, reading x, dy and the adapters and writing what is as large.
//
// Rows are grouped by adapter, in their order, first: tiles of 32 rows of one adapter, which a launch of one workgroup writes down,
// or three of more than 8192 rows (the plan); few rows need none, every wave sees them all by ballots.  Then "down": a tile's h, or g, the contraction over K or N
// split over a workgroup's eight waves and, where tiles are few, over workgroups, whose parts whoever reads h adds up; "up": a
// tile's part of out or dx; "weights": an adapter's gradients, 128 columns (64 in fp32) to a workgroup.  A small tile goes down and up
// in one launch.
//
// Operands come in loads of 16 bytes a lane: the order of a contraction is free as long as both operands have the same, and so is
// which of the product's columns a lane's are.  Where memory runs across the contraction, a lane loads as many lines of it as a
// fragment has, and turns them in registers: lane i then has the columns i kLane to i kLane + kLane - 1, in as many products.  Where it
// runs along the contraction a load is a fragment, but sixteen lines apart from lane to lane: what is long so, x and dy, is loaded
// line by line and takes the way through LDS.  h, which all of a workgroup's columns take, lies there as fragments.
//
// Measured in a step of 8192 x 4096 x 16384, rank 64, 32 adapters, bfloat16 (a large copy: 5.1 TB/s): plan 12 us; forward down 42 (x
// and A read: 2.0 TB/s), up 136 (base read, out written: 4.0 TB/s); backward down 131 (dy and B: 2.6 TB/s; every tile of 32 rows
// reads its adapter's B again, twice its rows' bytes, from L2), up 40 (dx and A), weights 124 (x, dy and the gradients: 3.3 TB/s).
//
// bfloat16: h and g are sums in 32 bits.  Where they are multiplied again each is taken as two bfloat16 values, the first cut off and the
// second rounded: off by 2^-16 of itself at most; so they are left in memory, in as many bytes, but where parts are still to be added up,
// which are in fp32.  fp32: products in 32 bits.
#include "dropout.hpp"

#include <type_traits>

namespace hdqt {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

constexpr int kSubs = 2, kTile = 16 * kSubs;        // rows of a tile, in blocks of the matrix instruction
constexpr int kDownWaves = 8, kUpWaves = 4, kWeightWaves = 4, kMostParts = 4;
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kMostGroups = kAdaptersMost + 2;

enum Mode { kAlong, kDown };        // memory runs along the contraction, or across it

// What the lanes of a wave have done in LDS that is the wave's own is before what they do there next.  (A wave's LDS operations are carried
// out in order: it is the compiler that is kept from moving them across each other.)
__device__ __forceinline__ void wave_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 bytes of a line: eight bfloat16 values or four of 32 bits
struct __attribute__((aligned(16))) Piece {
    uint32_t w[4];
};
template <int DT>
constexpr int lane_of() { return DT == kF32 ? 4 : 8; }

// N neighbouring elements of a line, in the first places of a piece.  WHOLE: all are there.  Else the first `n` of them are, and the
// others zero: element by element, at addresses that are inside (`at` is), so that no branch comes between one load and the next.
template <int DT, int N, bool WHOLE>
__device__ __forceinline__ Piece load_few(const void* p, int64_t at, int n)
{
    Piece q{};
    if constexpr (WHOLE) {
        __builtin_memcpy(q.w, static_cast<const char*>(p) + at * (DT == kF32 ? 4 : 2), N * (DT == kF32 ? 4 : 2));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int64_t i = at + (j < n ? j : 0);
            if (DT == kF32) {
                const uint32_t v = static_cast<const uint32_t*>(p)[i];
                q.w[j & 3] = j < n ? v : 0u;
            } else {
                const uint32_t v = static_cast<const uint16_t*>(p)[i];
                q.w[j / 2] |= (j < n ? v : 0u) << 16 * (j & 1);
            }
        }
    }
    return q;
}
template <int DT, bool WHOLE>
__device__ __forceinline__ Piece load_piece(const void* p, int64_t at, int n)
{
    return load_few<DT, lane_of<DT>(), WHOLE>(p, at, n);
}
__device__ __forceinline__ Piece only_if(bool there, const Piece& q) { return there ? q : Piece{}; }
// zeros for the first n elements (chosen, not masked: masks are registers, and 170 of them instead of 166 are a wave of three to a SIMD
// less for the way up of one tile of ranks in bfloat16: 8192 x 4096 x 4096 of rank 12, dx alone, 39.7 us for 35.1)
template <int DT>
__device__ __forceinline__ Piece without(Piece q, int n)
{
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        if (DT == kF32) q.w[d] = d < n ? 0u : q.w[d];
        else q.w[d] = 2 * d + 1 < n ? 0u : 2 * d < n ? q.w[d] & 0xFFFF0000u : q.w[d];
    }
    return q;
}

// elements lo to hi - 1
template <int DT>
__device__ __forceinline__ void store_piece(void* p, int64_t at, int lo, int hi, const Piece& q)
{
    constexpr int L = lane_of<DT>();
    if (lo <= 0 && hi >= L) {
        __builtin_memcpy(static_cast<char*>(p) + at * (16 / L), q.w, 16);
        return;
    }
#pragma unroll
    for (int j = 0; j < L; ++j)
        if (j >= lo && j < hi) {
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
        else q.w[j] = two_bf16(v[2 * j], v[2 * j + 1]);
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

// planes of a value of 32 bits as the matrix instructions take it: itself, or two of bfloat16
template <int DT>
constexpr int planes_of() { return DT == kF32 ? 1 : 2; }

// A value as two planes of bfloat16 side by side, the first, cut off, in the upper half, the second, rounded, in the lower: off by 2^-16
// of itself at most.  (Equal: an infinity has no rest.)  So is h held by bfloat16 calls where it is no sum of parts.
__device__ __forceinline__ uint32_t paired(float v)
{
    const float cut = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
    return (__float_as_uint(v) & 0xFFFF0000u) | (two_bf16(v == cut ? 0.0f : v - cut, 0.0f) & 0xFFFFu);
}
// the planes of such values, or those themselves
template <int DT>
__device__ __forceinline__ void unpaired(const uint32_t (&v)[lane_of<DT>()], Piece (&to)[planes_of<DT>()])
{
    if constexpr (DT == kF32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[0].w[j] = v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            to[0].w[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x07060302u);
            to[1].w[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x05040100u);
        }
    }
}

// ---- which rows have which adapter ----

// groups: an adapter's rows for each of n; n: rows without one; n + 1: rows whose number is none
__device__ __forceinline__ uint32_t group_of(int64_t id, int n) { return id < 0 ? (uint32_t)n : id < n ? (uint32_t)id : (uint32_t)n + 1; }

// The plan in memory, of more rows than a wave sees at once: start[groups + 1] (a group's first place in the order), tiles, order[M] (rows), tile[..] (group, first place)
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

constexpr int64_t kDirect = 256;        // as many rows a wave sees at once (without a plan)

// lanes with the same value of `bits` bits
__device__ __forceinline__ uint64_t same_lanes(uint32_t v, int bits, uint64_t among)
{
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(v >> b & 1);
        among &= v >> b & 1 ? set : ~set;
    }
    return among;
}

// A workgroup looks through 8192 rows, eight times 64 to a wave, all loaded before the first is taken.
constexpr int kAhead = 8;
constexpr int64_t kChunkRows = 64 * kPlanWaves * kAhead;
__host__ __device__ inline int64_t chunks_of(int64_t M) { return (M + kChunkRows - 1) / kChunkRows; }

struct Chunk {
    int64_t first, end;                     // a wave's rows
    uint32_t group[kAhead], before[kAhead]; // of a lane's: the group, and its rows in the wave before it
};
// Leaves in counts[wave] how many rows of every group the wave has.  (No barrier behind it.)
__device__ __forceinline__ void look_through(const int64_t* ids, int64_t from, int64_t M, int n, int bits, uint32_t (*counts)[kMostGroups], Chunk& c)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t left = M - from < kChunkRows ? M - from : kChunkRows, rows = (left + 64 * kPlanWaves - 1) / (64 * kPlanWaves) * 64;
    c.first = from + wave * rows;
    c.end = c.first + rows < from + left ? c.first + rows : from + left;
    int64_t id[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int64_t at = c.first + 64 * u + lane;
        id[u] = at < c.end ? ids[at] : 0;
    }
    for (uint32_t i = lane; i < (uint32_t)n + 2; i += 64) counts[wave][i] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        if (c.first + 64 * u >= c.end) break;
        const bool there = c.first + 64 * u + lane < c.end;
        c.group[u] = group_of(id[u], n);
        // the group's rows of the wave so far, and those of this 64 before a lane's, which are counted
        const uint64_t same = same_lanes(c.group[u], bits, __ballot(there));
        const int leader = __ffsll((unsigned long long)same) - 1;
        uint32_t at = 0;
        if (there && lane == leader) at = atomicAdd(&counts[wave][c.group[u]], (uint32_t)__popcll(same));
        c.before[u] = __shfl(at, leader & 63) + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        wave_in_order();                        // (the next 64 rows' leader of the group may be another lane)
    }
}
// Writes the rows to their places, counts[wave][group] being where the wave's rows of the group begin.
__device__ __forceinline__ void put_in_order(const Chunk& c, const uint32_t (*counts)[kMostGroups], uint32_t* order)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int64_t row = c.first + 64 * u + lane;
        if (row < c.end) order[counts[wave][c.group[u]] + c.before[u]] = (uint32_t)row;
    }
}

struct PlanLds {
    uint32_t starts[kMostGroups + 1], tiles[kMostGroups + 1], waves[2][kPlanWaves];
};
// From how many rows a thread's two groups have: where groups begin, and the tiles
__device__ __forceinline__ void lay_out(const uint32_t (&have)[2], const Plan& p, uint32_t groups, PlanLds& lds)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint32_t cut[2], before[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) cut[u] = (have[u] + kTile - 1) / kTile;
    before[0] = have[0] + have[1];
    before[1] = cut[0] + cut[1];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t own = before[u];
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t up = __shfl_up(before[u], m);
            if (lane >= m) before[u] += up;
        }
        if (lane == 63) lds.waves[u][wave] = before[u];
        before[u] -= own;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
        for (int w = 0; w < wave; ++w) before[u] += lds.waves[u][w];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g <= groups) {
            lds.starts[g] = before[0];
            lds.tiles[g] = before[1];
            const_cast<uint32_t*>(p.start)[g] = before[0];
        }
        before[0] += have[u];
        before[1] += cut[u];
    }
    __syncthreads();
    const uint32_t total = lds.tiles[groups];
    if (threadIdx.x == 0) *const_cast<uint32_t*>(p.tiles) = total;
    for (uint32_t i = threadIdx.x; i < total; i += kPlanThreads) {
        uint32_t lo = 0, hi = groups;               // the last group whose first tile is not behind this one
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (lds.tiles[mid] <= i) lo = mid;
            else hi = mid;
        }
        const_cast<uint2*>(p.tile)[i] = make_uint2(lo, lds.starts[lo] + kTile * (i - lds.tiles[lo]));
    }
}

// Up to 8192 rows, by one workgroup.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(const int64_t* ids, int64_t M, int n, int bits, uint32_t* plan)
{
    __shared__ uint32_t counts[kPlanWaves][kMostGroups];
    __shared__ PlanLds lds;
    const Plan p = plan_at(plan, M, n);
    const uint32_t groups = (uint32_t)n + 2;
    Chunk c;
    look_through(ids, 0, M, n, bits, counts, c);
    __syncthreads();
    uint32_t have[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g < groups)
            for (int w = 0; w < kPlanWaves; ++w) have[u] += counts[w][g];
    }
    lay_out(have, p, groups, lds);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g < groups) {
            uint32_t at = lds.starts[g];
            for (int w = 0; w < kPlanWaves; ++w) {
                const uint32_t own = counts[w][g];
                counts[w][g] = at;
                at += own;
            }
        }
    }
    __syncthreads();
    put_in_order(c, counts, const_cast<uint32_t*>(p.order));
}

// Of more rows: how many of every group each 8192 have; where those begin; the order.  (Three launches: 16384 rows 19 us, 65536 of ten adapters
// 21, a million 41; one workgroup for all of them 23, 76 and 1095.)
__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(const int64_t* ids, int64_t M, int n, int bits, uint32_t* chunks)
{
    __shared__ uint32_t counts[kPlanWaves][kMostGroups];
    const uint32_t groups = (uint32_t)n + 2;
    Chunk c;
    look_through(ids, blockIdx.x * kChunkRows, M, n, bits, counts, c);
    __syncthreads();
    for (uint32_t g = threadIdx.x; g < groups; g += kPlanThreads) {
        uint32_t s = 0;
        for (int w = 0; w < kPlanWaves; ++w) s += counts[w][g];
        chunks[(int64_t)blockIdx.x * groups + g] = s;
    }
}
__global__ __launch_bounds__(kPlanThreads) void plan_starts_kernel(int64_t M, int n, uint32_t* plan, uint32_t* chunks, uint32_t of_them)
{
    __shared__ PlanLds lds;
    const uint32_t groups = (uint32_t)n + 2;
    uint32_t have[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t g = 2 * threadIdx.x + u;
        if (g < groups)
#pragma unroll 8
            for (uint32_t i = 0; i < of_them; ++i) have[u] += chunks[(int64_t)i * groups + g];
    }
    lay_out(have, plan_at(plan, M, n), groups, lds);
    for (uint32_t g = threadIdx.x; g < groups; g += kPlanThreads) {
        uint32_t at = lds.starts[g];
        for (uint32_t i = 0; i < of_them; i += 8) {
            uint32_t own[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) own[k] = i + k < of_them ? chunks[(int64_t)(i + k) * groups + g] : 0;
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
                if (i + k < of_them) chunks[(int64_t)(i + k) * groups + g] = at;
                at += own[k];
            }
        }
    }
}
__global__ __launch_bounds__(kPlanThreads) void plan_order_kernel(const int64_t* ids, int64_t M, int n, int bits, uint32_t* plan, const uint32_t* chunks)
{
    __shared__ uint32_t counts[kPlanWaves][kMostGroups];
    const uint32_t groups = (uint32_t)n + 2;
    Chunk c;
    look_through(ids, blockIdx.x * kChunkRows, M, n, bits, counts, c);
    __syncthreads();
    for (uint32_t g = threadIdx.x; g < groups; g += kPlanThreads) {
        uint32_t at = chunks[(int64_t)blockIdx.x * groups + g];
        for (int w = 0; w < kPlanWaves; ++w) {
            const uint32_t own = counts[w][g];
            counts[w][g] = at;
            at += own;
        }
    }
    __syncthreads();
    put_in_order(c, counts, const_cast<uint32_t*>(plan_at(plan, M, n).order));
}

constexpr int kWords = (int)(kDirect / 64);

// Rows of one group, for a wave: `count` of them from place `first` of the group on.
struct Group {
    uint32_t group, count, first;
    const uint32_t* order;          // the plan's, from the group's first place on, or null: of few rows,
    uint32_t listed[kWords];        // 64 at a time, lane p has the p-th of the group, of which
    uint32_t start[kWords];         // so many are before these 64
    uint32_t words;                 // how many 64 there are
    // lane l's: the row at place first + `from` + l, the last one's behind it
    __device__ __forceinline__ uint32_t rows(uint32_t from) const
    {
        const uint32_t at = from + (threadIdx.x & 63), place = first + (at < count ? at : count - 1);
        if (order) return order[place];
        uint32_t row = __shfl(listed[0], (int)place);
#pragma unroll
        for (int w = 1; w < kWords; ++w) {
            if (w >= (int)words) break;
            const uint32_t other = __shfl(listed[w], (int)(place - start[w]));
            row = place >= start[w] ? other : row;
        }
        return row;
    }
};

struct RowArgs {
    const int64_t* ids;
    const void* plan;               // null: none, there are few rows
    int64_t M;
    int n;
};

// A launch of `inner` x `outer` workgroups.  They go to the eight XCDs in turn: each gets a run of its own, inner after inner, so
// that tiles of one adapter, which read the same part of its matrix, share an L2.
// More of them than a launch counts threads for are spread over the grid's other axis, so many `outer` each.
struct Grid {
    Divisor inner;
    uint32_t total, per_xcd, outer, slice;
    uint32_t slices() const { return (outer + slice - 1) / slice; }
};
Grid grid_of(uint32_t inner, uint32_t outer)
{
    const uint32_t most = (1u << 22) / inner, slice = outer < most ? outer : most > 0 ? most : 1, total = inner * slice;
    return {make_divisor(inner), total, (total + 7) / 8, outer, slice};
}
__device__ __forceinline__ bool place_of(const Grid& k, uint32_t& inner, uint32_t& outer)
{
    const uint32_t idx = (blockIdx.x & 7) * k.per_xcd + (blockIdx.x >> 3);
    outer = divide(idx, k.inner);
    inner = idx - outer * k.inner.d;
    outer += blockIdx.y * k.slice;
    return idx < k.total && outer < k.outer;
}

// of few rows, a lane's groups of every 64
__device__ __forceinline__ void groups_of(const RowArgs& a, uint32_t (&g)[kWords])
{
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const int64_t row = 64 * w + (threadIdx.x & 63);
        g[w] = row < a.M ? group_of(a.ids[row], a.n) : ~0u;
    }
}
__device__ __forceinline__ Group listed_rows(const RowArgs& a, const uint32_t (&g)[kWords], uint32_t group)
{
    const int lane = threadIdx.x & 63;
    const uint64_t lower = (1ull << lane) - 1;
    Group of{};
    of.group = group;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        of.start[w] = of.count;
        if (w && 64 * w >= a.M) continue;
        const uint64_t same = __ballot(g[w] == group);
        // (the others go behind them, each to a place of its own)
        const int count = __popcll(same), to = same >> lane & 1 ? __popcll(same & lower) : count + __popcll(~same & lower);
        of.listed[w] = 64 * w + (uint32_t)__builtin_amdgcn_ds_permute(4 * to, lane);
        of.count += (uint32_t)count;
    }
    of.words = (uint32_t)(a.M + 63) / 64;
    return of;
}

// The rows of workgroup `tile`, 32 at most: none where there is no such tile.  Of few rows, every 32nd of a group stands for a tile.
__device__ __forceinline__ Group tile_rows(const RowArgs& a, uint32_t tile)
{
    if (!a.plan) {
        uint32_t g[kWords], before = 0;         // rows of the group before the tile's
        groups_of(a, g);
        const uint32_t mine = group_of(a.ids[tile], a.n);
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const uint64_t same = __ballot(g[w] == mine), until = (1ull << (tile & 63)) - 1;
            before += (uint32_t)w < tile >> 6 ? __popcll(same) : (uint32_t)w == tile >> 6 ? __popcll(same & until) : 0;
        }
        if (before % kTile) return Group{};
        Group of = listed_rows(a, g, mine);
        of.first = before;
        of.count = of.count - before < kTile ? of.count - before : kTile;
        return of;
    }
    const Plan p = plan_at(a.plan, a.M, a.n);
    Group of{};
    of.order = p.order;
    if (tile >= *p.tiles) return of;
    const uint2 t = p.tile[tile];
    const uint32_t left = p.start[t.x + 1] - t.y;
    of.group = t.x;
    of.count = left < kTile ? left : kTile;
    of.first = t.y;
    return of;
}
__device__ __forceinline__ Group adapter_rows(const RowArgs& a, uint32_t adapter)
{
    if (!a.plan) {
        uint32_t g[kWords];
        groups_of(a, g);
        return listed_rows(a, g, adapter);
    }
    const Plan p = plan_at(a.plan, a.M, a.n);
    Group of{};
    of.group = adapter;
    of.order = p.order;
    of.first = p.start[adapter];
    of.count = p.start[adapter + 1] - of.first;
    return of;
}

// ---- down ----

struct DownArgs {
    RowArgs rows;
    Grid grid;                      // tiles, parts
    const void *x, *W;              // [M, D]; of an adapter [D, r] (kDown) or [r, D] (kAlong)
    float* h;                       // [parts][M][16 RT]
    int64_t D;
    int r;
    uint32_t steps, parts;          // of the contraction: how many times 8 kLane a part has, parts
};

// The sums of a workgroup's waves, in the first one's
template <int RT>
__device__ __forceinline__ void join_waves(v4f (&acc)[kSubs][RT], v4f* lds, int wave, int lane)
{
#pragma unroll
    for (int half = kDownWaves / 2; half; half /= 2) {
        __syncthreads();
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int t = 0; t < RT; ++t) lds[(((wave - half) * kSubs + s) * RT + t) * 64 + lane] = acc[s][t];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[s][t] += lds[((wave * kSubs + s) * RT + t) * 64 + lane];
    }
}

// A wave's step: 128 bytes of every row, two chunks.  x (and W, where it runs along the contraction) is loaded as memory lies, eight
// lanes to a row, into registers, while the step before is multiplied, and handed to the lanes that multiply it through LDS that is
// the wave's own: asked for as the fragments lie, sixteen rows side by side, every lane's 16 bytes are an access of the cache of their
// own, four times as many (a tile of 8192 x 16384 in bfloat16 against rank 64: 284 us).  A row's pieces are turned by the row's
// number, so that eight lanes' reads lie in different banks.
// SHORT: the contraction is shorter than a step; element by element.  Else the last step, where it is no whole one, begins a step
// before the end, and what it has of the one before is taken for zeros.
template <int DT, int RT, int MODE, bool SHORT>
struct Down {
    static constexpr int L = lane_of<DT>(), kChunk = 4 * L, kStep = 2 * kChunk, RL = RT < L ? RT : L, RQ = RT / RL;
    static constexpr int kRows = kTile + (MODE == kAlong ? 16 * RT : 0), kLoads = kRows / 8;    // of a step, that go through LDS
    static constexpr int kBytes = SHORT ? 0 : 128 * kRows * kDownWaves, kSums = kDownWaves / 2 * kSubs * RT * 64 * (int)sizeof(v4f);
    static constexpr int kLds = kBytes > kSums ? kBytes : kSums;
    static __device__ __forceinline__ void tile(const DownArgs& a, const Group& rows, uint32_t part, char* lds);
};
template <int DT, int RT, int MODE, bool SHORT>
__global__ __launch_bounds__(64 * kDownWaves, 2) void down_kernel(DownArgs a)
{
    typedef Down<DT, RT, MODE, SHORT> D;
    __shared__ __attribute__((aligned(16))) char lds[D::kLds];
    uint32_t tile, part;
    if (!place_of(a.grid, tile, part)) return;
    const Group rows = tile_rows(a.rows, tile);
    if (rows.count && rows.group < (uint32_t)a.rows.n) D::tile(a, rows, part, lds);
}
template <int DT, int RT, int MODE, bool SHORT>
__device__ __forceinline__ void Down<DT, RT, MODE, SHORT>::tile(const DownArgs& a, const Group& rows, uint32_t part, char* lds)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const char* W = static_cast<const char*>(a.W) + (int64_t)rows.group * a.D * a.r * (16 / L);
    // tile t + RL q of the ranks: a lane's is rank[q] + t.  (16 RL q + RL (l % 16); the last lanes' begin RL before the last rank's end,
    // and have ranks of the lanes before again: r is above RL, where that is more than one)
    int rank[RQ];
#pragma unroll
    for (int q = 0; q < RQ; ++q) {
        const int c = 16 * RL * q + RL * j;
        rank[q] = c + RL <= a.r ? c : a.r - RL;
    }
    const int64_t first = (int64_t)part * a.steps, all = (a.D + kStep - 1) / kStep;
    const int64_t last = first + a.steps < all ? first + a.steps : all;
    const uint32_t row = rows.rows(0);
    v4f acc[kSubs][RT] = {};
    // the chunk's products: x's fragments, and W's lines across the contraction or fragments along it
    auto products = [&](const Piece (&x)[kSubs], const Piece (&w)[RQ][MODE == kDown ? L : RL]) {
#pragma unroll
        for (int q = 0; q < RQ; ++q)
#pragma unroll
            for (int t = 0; t < RL; ++t) {
                Piece b;
                if constexpr (MODE == kDown) b = turned<DT>(w[q], t);
                else b = w[q][t];
#pragma unroll
                for (int s = 0; s < kSubs; ++s) acc[s][RL * q + t] = multiply<DT>(x[s], b, acc[s][RL * q + t]);
            }
    };
    if constexpr (SHORT) {
        for (int64_t k0 = (first + wave) * kStep; k0 < a.D && first + wave < last; k0 += kChunk) {
            const int64_t k = k0 + L * g;
            const int n = (int)(a.D - k);
            const int64_t in = n <= 0 ? 0 : k;
            Piece x[kSubs], w[RQ][MODE == kDown ? L : RL];
#pragma unroll
            for (int s = 0; s < kSubs; ++s) x[s] = load_piece<DT, false>(a.x, (int64_t)__shfl(row, 16 * s + j) * a.D + in, n);
#pragma unroll
            for (int q = 0; q < RQ; ++q)
#pragma unroll
                for (int e = 0; e < (MODE == kDown ? L : RL); ++e) {
                    if constexpr (MODE == kDown) w[q][e] = only_if(e < n, load_few<DT, RL, true>(W, (e < n ? k + e : 0) * a.r + rank[q], RL));
                    else w[q][e] = load_piece<DT, false>(W, (int64_t)(rank[q] + e) * a.D + in, n);
                }
            products(x, w);
        }
    } else {
        char* const mine = lds + 128 * kRows * wave;
        // a lane's pieces: piece l % 8 of rows l / 8, 8 + l / 8, ..: the tile's rows, then the ranks in the fragments' order
        const char* from[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = 8 * i + lane / 8;
            if (8 * i < kTile) {
                from[i] = static_cast<const char*>(a.x) + (int64_t)__shfl(row, at) * a.D * (16 / L);
            } else {
                const int f = at - kTile, c = 16 * RL * (f / (16 * RL)) + RL * (f % 16);        // fragment f / 16 - RL q, line f % 16
                from[i] = W + (int64_t)((c + RL <= a.r ? c : a.r - RL) + f / 16 % RL) * a.D * (16 / L);
            }
            from[i] += 16 * (lane % 8);
        }
        Piece next[kLoads], lines[2][MODE == kDown ? RQ : 1][MODE == kDown ? L : 1];
        auto load = [&](int64_t step) {
            const int64_t k = (step + 1) * kStep <= a.D ? step * kStep : a.D - kStep;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) __builtin_memcpy(next[i].w, from[i] + k * (16 / L), 16);
            if constexpr (MODE == kDown)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int q = 0; q < RQ; ++q)
#pragma unroll
                        for (int e = 0; e < L; ++e) lines[c][q][e] = load_few<DT, RL, true>(W, (k + kChunk * c + L * g + e) * a.r + rank[q], RL);
        };
        int64_t step = first + wave;
        if (step < last) load(step);
        for (; step < last; step += kDownWaves) {
            const int skip = (step + 1) * kStep <= a.D ? 0 : (int)((step + 1) * kStep - a.D);
            if (skip) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) next[i] = without<DT>(next[i], skip - L * (lane % 8));
                if constexpr (MODE == kDown)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int q = 0; q < RQ; ++q)
#pragma unroll
                            for (int e = 0; e < L; ++e) lines[c][q][e] = only_if(kChunk * c + L * g + e >= skip, lines[c][q][e]);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                *reinterpret_cast<Piece*>(mine + 1024 * i + 128 * (lane / 8) + 16 * ((lane ^ lane / 8) % 8)) = next[i];
            Piece w[2][RQ][MODE == kDown ? L : RL];
            if constexpr (MODE == kDown)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int q = 0; q < RQ; ++q)
#pragma unroll
                        for (int e = 0; e < L; ++e) w[c][q][e] = lines[c][q][e];
            if (step + kDownWaves < last) load(step + kDownWaves);
            wave_in_order();                            // the pieces are there for the lanes that take them
            auto fragment = [&](int f, int c) {         // 16 rows from 16 f on
                return *reinterpret_cast<const Piece*>(mine + 2048 * f + 128 * j + 16 * ((4 * c + g) ^ (j & 7)));
            };
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                Piece x[kSubs];
#pragma unroll
                for (int s = 0; s < kSubs; ++s) x[s] = fragment(s, c);
                if constexpr (MODE == kAlong)
#pragma unroll
                    for (int q = 0; q < RQ; ++q)
#pragma unroll
                        for (int t = 0; t < RL; ++t) w[c][q][t] = fragment(kSubs + RL * q + t, c);
                products(x, w[c]);
            }
            wave_in_order();                            // and are taken before the next step's are put over them
        }
    }
    join_waves<RT>(acc, reinterpret_cast<v4f*>(lds), wave, lane);
    if (wave == 0)
#pragma unroll
        for (int s = 0; s < kSubs; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t of = __shfl(row, 16 * s + 4 * g + i);
                if (16 * s + 4 * g + i >= rows.count) continue;
                float* to = a.h + ((int64_t)part * a.rows.M + of) * (16 * RT);
#pragma unroll
                for (int q = 0; q < RQ; ++q)
#pragma unroll
                    for (int t = 0; t < RL; ++t) {
                        const int c = 16 * RL * q + RL * j + t;
                        const float v = acc[s][RL * q + t][i];
                        to[rank[q] + t] = DT == kBf16 && a.parts == 1 ? __uint_as_float(paired(v)) : v;
                        if (c >= a.r) to[c] = 0.0f;     // (behind the last rank)
                    }
            }
}

// ---- up ----

struct UpArgs {
    RowArgs rows;
    Grid grid;                      // workgroups over the columns, tiles
    const float* h;                 // [parts][M][16 RT]
    const float* scale;             // [n] or null
    const void* W;                  // of an adapter [r, N] (kDown) or [N, r] (kAlong)
    const void* base;               // [M, N] or null
    void* out;                      // [M, N]
    int64_t N;
    int r;
    uint32_t parts;
};

// Planes of a row's values from any of them on, all parts together (four are asked for at once), the first `skip` taken for zeros: P of
// them, or, of two in one (P = 1), a lane's own.  (Chosen word by word: a choice between the two in memory would put them into LDS, at an
// address that a load from the host's queue decides, 10 us of a small call.)
template <int DT, int P>
__device__ __forceinline__ void load_h(const float* h, int64_t part, uint32_t parts, int skip, bool second, Piece (&to)[P])
{
    constexpr int N = lane_of<DT>(), V = N / 4;
    v4f q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) __builtin_memcpy(&q[j], h + 4 * j, 16);
    if (parts > 1) {
        v4f more[kMostParts - 1][V];
#pragma unroll
        for (int u = 1; u < kMostParts; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) __builtin_memcpy(&more[u - 1][j], h + (u < (int)parts ? u : 0) * part + 4 * j, 16);
#pragma unroll
        for (int u = 1; u < kMostParts; ++u)
#pragma unroll
            for (int j = 0; j < V; ++j) q[j] += u < (int)parts ? more[u - 1][j] : v4f{};
        if constexpr (DT == kBf16)
#pragma unroll
            for (int j = 0; j < N; ++j) q[j / 4][j % 4] = __uint_as_float(paired(q[j / 4][j % 4]));
    }
    uint32_t v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = j < skip ? 0u : __float_as_uint(q[j / 4][j % 4]);
    if constexpr (DT == kBf16 && P == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[0].w[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], second ? 0x05040100u : 0x07060302u);
    } else {
        unpaired<DT>(v, to);
    }
}

// How columns end.  kShort: there are fewer than a wave has, or (kAlong) fewer ranks than a load, and W and base are loaded element by
// element.  Else the last columns, and the last ranks of a line along them, begin so far before the end that loads are whole; what
// others have already is not written, and zero in h and in W.  kEven: columns, and ranks along a line, are whole loads, so that a lane writes
// all of its own or none and has no ranks of others'.
enum End { kEven, kOdd, kShort };
template <int DT, int RT, int MODE, int END, int WAVES>
struct Up {
    static constexpr bool SHORT = END == kShort;
    static constexpr int L = lane_of<DT>(), kChunk = 4 * L, kColumns = 16 * L;
    // bfloat16, one tile of ranks: both planes are one chunk, the second beside the same lines of W again
    static constexpr bool kFolded = DT == kBf16 && RT == 1;
    static constexpr int P = kFolded ? 1 : planes_of<DT>(), C = 16 * RT < kChunk ? 1 : 16 * RT / kChunk, kRanks = 16 * RT;
    struct Lds {
        Piece h[kSubs * C][P][64];
    };
    // every `across`-th group of WAVES blocks of columns, from `over` on
    static __device__ __forceinline__ void tile(const UpArgs& a, const Group& rows, uint32_t over, uint32_t across, Lds& lds);
};
template <int DT, int RT, int MODE, int END>
__global__ __launch_bounds__(64 * kUpWaves, 2) void up_kernel(UpArgs a)
{
    typedef Up<DT, RT, MODE, END, kUpWaves> U;
    __shared__ typename U::Lds lds;
    uint32_t tile, over;
    if (!place_of(a.grid, over, tile)) return;
    const Group rows = tile_rows(a.rows, tile);
    if (rows.count) U::tile(a, rows, over, a.grid.inner.d, lds);
}
// Both ways by one workgroup to a tile, h by way of memory.
template <int DT, int RT, int MODE, int END>
__global__ __launch_bounds__(64 * kDownWaves, 2) void down_up_kernel(DownArgs d, UpArgs u)
{
    typedef Down<DT, RT, MODE, false> D;
    typedef Up<DT, RT, MODE, END, kDownWaves> U;
    __shared__ __attribute__((aligned(16))) char lds[D::kLds > (int)sizeof(typename U::Lds) ? D::kLds : (int)sizeof(typename U::Lds)];
    uint32_t tile, none;
    if (!place_of(d.grid, tile, none)) return;
    const Group rows = tile_rows(d.rows, tile);
    if (!rows.count) return;
    if (rows.group < (uint32_t)d.rows.n) D::tile(d, rows, 0, lds);
    __syncthreads();
    U::tile(u, rows, 0, 1, *reinterpret_cast<typename U::Lds*>(lds));
}
template <int DT, int RT, int MODE, int END, int WAVES>
__device__ __forceinline__ void Up<DT, RT, MODE, END, WAVES>::tile(const UpArgs& a, const Group& rows, uint32_t over, uint32_t across, Lds& lds)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const bool none = rows.group == (uint32_t)a.rows.n, wrong = rows.group > (uint32_t)a.rows.n;
    if (none && a.base == a.out) return;
    const char* W = static_cast<const char*>(a.W) + (none || wrong ? 0 : (int64_t)rows.group * a.N * a.r * (16 / L));
    // (rows without an adapter: minus one times zero, which leaves any base as it is)
    const float scale = wrong ? __builtin_nanf("") : none ? -1.0f : a.scale ? a.scale[rows.group] : 1.0f;
    // a lane's ranks of a chunk: from first(c) on, those before own(c) another lane's
    auto own = [&](int c) { return kChunk * c + L * (kFolded ? g & 1 : g); };
    auto first = [&](int c) { return MODE == kDown || SHORT || own(c) + L <= a.r ? own(c) : a.r - L; };
    const uint32_t all = rows.rows(0);
    uint32_t row[kSubs][4];
#pragma unroll
    for (int s = 0; s < kSubs; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) row[s][i] = __shfl(all, 16 * s + 4 * g + i);
    // a lane's columns from c0 on: from col, those from lo to hi its own
    int64_t col;
    int lo, hi;
    Piece base[kSubs][4] = {}, w[L];
    auto lines = [&](int c) {
#pragma unroll
        for (int e = 0; e < L; ++e) {
            if constexpr (MODE == kDown) {             // line own(c) + e
                const int rank = own(c) + e < a.r ? own(c) + e : 0;
                w[e] = load_piece<DT, !SHORT>(W, rank * a.N + col, hi);
            } else {                                   // column col + e
                const int rank = first(c) < a.r ? first(c) : 0;
                w[e] = load_piece<DT, !SHORT>(W, (col + (SHORT && e >= hi ? 0 : e)) * a.r + rank, a.r - first(c));
            }
        }
    };
    auto fetch = [&](int64_t c0) {
        const int64_t from = SHORT || c0 + kColumns <= a.N ? c0 : a.N - kColumns;
        lo = (int)(c0 - from) - L * j;
        hi = SHORT ? (int)(a.N - c0) - L * j : L;
        col = SHORT && hi <= 0 ? c0 : from + L * j;
        if (a.base)
#pragma unroll
            for (int s = 0; s < kSubs; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) base[s][i] = load_piece<DT, !SHORT>(a.base, row[s][i] * a.N + col, hi);
        if (!none && !wrong) lines(0);
    };
    // the first columns are on their way while the tile's h is split, for all waves
    int64_t c0 = ((int64_t)over * WAVES + wave) * kColumns;
    const int64_t step = (int64_t)across * WAVES * kColumns;
    if (c0 < a.N) fetch(c0);
    for (int f = wave; f < kSubs * C; f += WAVES) {
        const int s = f / C, c = f % C;
        const uint32_t of = __shfl(all, 16 * s + j);
        Piece planes[P];
        if (none || wrong) continue;
        load_h<DT, P>(a.h + (int64_t)of * kRanks + first(c), a.rows.M * kRanks, a.parts, own(c) - first(c), g >= 2, planes);
#pragma unroll
        for (int k = 0; k < P; ++k) lds.h[f][k][lane] = planes[k];
    }
    __syncthreads();
    for (; c0 < a.N; c0 += step) {
        v4f acc[kSubs][L] = {};
        if (!none && !wrong)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (c) lines(c);
                if (a.r != kRanks) {                   // (h is zero there, but W may be infinite)
#pragma unroll
                    for (int e = 0; e < L; ++e) {
                        if constexpr (MODE == kAlong && END == kOdd) w[e] = without<DT>(w[e], own(c) - first(c));
                        else w[e] = only_if(own(c) + (MODE == kDown ? e : 0) < a.r, w[e]);
                    }
                }
#pragma unroll
                for (int t = 0; t < L; ++t) {
                    const Piece b = MODE == kDown ? turned<DT>(w, t) : w[t];
#pragma unroll
                    for (int k = P - 1; k >= 0; --k)
#pragma unroll
                        for (int s = 0; s < kSubs; ++s) acc[s][t] = multiply<DT>(lds.h[s * C + c][k][lane], b, acc[s][t]);
                }
            }
#pragma unroll
        for (int s = 0; s < kSubs; ++s) {
            if (16 * s >= rows.count) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[L];
#pragma unroll
                for (int t = 0; t < L; ++t) {
                    v[t] = fmaf(scale, acc[s][t][i], value<DT>(base[s][i], t));
                }
                if (16 * s + 4 * g + i >= rows.count || hi <= 0 || lo >= L) continue;
                if constexpr (END == kEven) store_piece<DT>(a.out, row[s][i] * a.N + col, 0, L, piece_of<DT>(v));
                else store_piece<DT>(a.out, row[s][i] * a.N + col, lo, hi, piece_of<DT>(v));
            }
        }
        if (c0 + step < a.N) fetch(c0 + step);
    }
}

// ---- weights ----

// an adapter's gradient: W[j][c] = sum over its rows of scale h[row][j] v[row][c]
struct WeightArgs {
    RowArgs rows;
    Grid grid;                      // blocks of columns of both, and adapters times parts of the rows
    const float* h[2];              // dA: g; dB: h.  [parts][M][16 RT]
    const void* v[2];               // dA: x; dB: dy
    void* out[2];                   // [n][K][r]; [n][r][N]; either may be null
    float* sums;                    // where a gradient is added up over parts of the rows, [split][n K r + n r N], else null
    const float* scale;
    int64_t N[2];
    int r;
    uint32_t parts[2], blocks, split;           // blocks: of dA's columns
    Divisor by_split;
    // elements of a part's sums, and of those dA's
    __device__ __forceinline__ int64_t of_a_part() const { return (int64_t)rows.n * r * (N[0] + N[1]); }
    __device__ __forceinline__ int64_t of_dA() const { return (int64_t)rows.n * r * N[0]; }
};

// A workgroup has 128 columns (64 in fp32) and all ranks of one gradient: a wave four tiles of ranks at most, and of the rows what the
// waves with the same ranks share.  Tile t of a wave: line m is rank rank0 + RL m + t, so that a load of h has a lane's ranks of all
// its tiles.
template <int DT, int RT>
__global__ __launch_bounds__(64 * kWeightWaves, 2) void weights_kernel(WeightArgs a)
{
    constexpr int L = lane_of<DT>(), kChunk = 4 * L, kColumns = 16 * L, P = planes_of<DT>(), RL = RT < 2 ? RT : DT == kBf16 || RT < 4 ? 2 : 4;
    constexpr int kShares = kWeightWaves / (RT / RL);
    __shared__ v4f sums[kWeightWaves / 2][RL][L][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    uint32_t block, which;
    if (!place_of(a.grid, block, which)) return;
    const int of = block >= a.blocks;
    if (!a.out[of]) return;
    const int64_t N = a.N[of], c0 = (int64_t)(block - (of ? a.blocks : 0)) * kColumns, col = c0 + L * j;
    const uint32_t adapter = divide(which, a.by_split), part = which - adapter * a.split;
    const int half = wave / kShares, rank0 = 16 * RL * half, share = wave % kShares;
    const Group rows = adapter_rows(a.rows, adapter);
    const float* h = a.h[of] + rank0 + RL * j;
    const int n = col + L <= N ? L : col < N ? (int)(N - col) : 0;
    v4f acc[RL][L] = {};
    auto sum = [&](auto whole) {
        constexpr bool WHOLE = whole.value;
        // (as often for every lane of a wave: the rows of a few are handed from lane to lane)
        const uint32_t step = kChunk * kShares * a.split;
        uint32_t first = kChunk * (part * kShares + share), next = 0;
        if (first < rows.count) next = rows.rows(first);
        for (; first < rows.count; first += step) {
            const uint32_t now = next;
            Piece lines[L];
            float u[L][RL];
#pragma unroll
            for (int e = 0; e < L; ++e) {
                const uint32_t row = __shfl(now, L * g + e);               // (behind the last: one that there is, taken for zeros)
                lines[e] = load_piece<DT, WHOLE>(a.v[of], row * N + (WHOLE || n > 0 ? col : 0), n);
                __builtin_memcpy(u[e], h + row * (uint32_t)(16 * RT), 4 * RL);
            }
            const uint32_t ahead = first + step;
            if (ahead < rows.count) next = rows.rows(ahead);
            if (a.parts[of] > 1)
#pragma unroll
                for (int e = 0; e < L; ++e) {
                    const uint32_t row = __shfl(now, L * g + e);
                    for (uint32_t s = 1; s < a.parts[of]; ++s)
#pragma unroll
                        for (int t = 0; t < RL; ++t) u[e][t] += h[(s * a.rows.M + row) * (16 * RT) + t];
#pragma unroll
                    for (int t = 0; t < RL; ++t)
                        if (DT == kBf16) u[e][t] = __uint_as_float(paired(u[e][t]));
                }
            if (first + kChunk > rows.count)
#pragma unroll
                for (int e = 0; e < L; ++e) {
                    const bool has = first + L * g + e < rows.count;
                    lines[e] = only_if(has, lines[e]);
#pragma unroll
                    for (int t = 0; t < RL; ++t) u[e][t] = has ? u[e][t] : 0.0f;
                }
            Piece up[RL][P];
#pragma unroll
            for (int t = 0; t < RL; ++t) {
                uint32_t v[L];
#pragma unroll
                for (int e = 0; e < L; ++e) v[e] = __float_as_uint(u[e][t]);
                unpaired<DT>(v, up[t]);
            }
#pragma unroll
            for (int c = 0; c < L; ++c) {
                const Piece w = turned<DT>(lines, c);
#pragma unroll
                for (int k = P - 1; k >= 0; --k)
#pragma unroll
                    for (int t = 0; t < RL; ++t) acc[t][c] = multiply<DT>(up[t][k], w, acc[t][c]);
            }
        }
    };
    if (c0 + kColumns <= N) sum(std::true_type{});
    else sum(std::false_type{});
    // the waves with the same ranks together, as far as there were rows for them
    const uint32_t begun = part * kShares * kChunk;
#pragma unroll
    for (int m = kShares / 2; m; m /= 2) {
        if (rows.count <= begun + m * kChunk) continue;
        __syncthreads();
        if (share >= m && share < 2 * m)
#pragma unroll
            for (int t = 0; t < RL; ++t)
#pragma unroll
                for (int c = 0; c < L; ++c) sums[half * (kShares / 2) + share - m][t][c][lane] = acc[t][c];
        __syncthreads();
        if (share < m)
#pragma unroll
            for (int t = 0; t < RL; ++t)
#pragma unroll
                for (int c = 0; c < L; ++c) acc[t][c] += sums[half * (kShares / 2) + share][t][c][lane];
    }
    if (share || n <= 0) return;
    const float scale = a.scale && rows.count > begun ? a.scale[adapter] : 1.0f;     // (of no rows, or none in this part: zeros, whatever the scale)
    float* parts = a.sums ? a.sums + (int64_t)part * a.of_a_part() + (of ? a.of_dA() : 0) : nullptr;
    // a lane has ranks rank0 + RL (4 g + i) + t of columns col + c: of a rank's run in dB kLane elements, of a column's in dA RL of each i
    if (of) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < RL; ++t) {
                const int rank = rank0 + RL * (4 * g + i) + t;
                if (rank >= a.r) continue;
                const int64_t to = ((int64_t)adapter * a.r + rank) * N + col;
                float v[L];
#pragma unroll
                for (int c = 0; c < L; ++c) v[c] = scale * acc[t][c][i];
                if (parts) {
#pragma unroll
                    for (int c = 0; c < L; ++c)
                        if (c < n) parts[to + c] = v[c];
                } else {
                    store_piece<DT>(a.out[1], to, 0, n, piece_of<DT>(v));
                }
            }
        return;
    }
    const int rank = rank0 + 4 * RL * g, left = a.r - rank;
#pragma unroll
    for (int c = 0; c < L; ++c) {
        if (c >= n || left <= 0) continue;
        const int64_t to = ((int64_t)adapter * N + col + c) * a.r + rank;
        float v[4 * RL];
#pragma unroll
        for (int m = 0; m < 4 * RL; ++m) v[m] = scale * acc[m % RL][c][m / RL];
        if (left >= 4 * RL && !parts && DT == kBf16) {
            uint32_t two[2 * RL];
#pragma unroll
            for (int m = 0; m < 2 * RL; ++m) two[m] = two_bf16(v[2 * m], v[2 * m + 1]);
            __builtin_memcpy(static_cast<uint16_t*>(a.out[0]) + to, two, 8 * RL);
        } else if (left >= 4 * RL) {
            __builtin_memcpy((parts ? parts : static_cast<float*>(a.out[0])) + to, v, 16 * RL);
        } else {
#pragma unroll
            for (int m = 0; m < 4 * RL; ++m)
                if (m < left) {
                    if (parts) parts[to + m] = v[m];
                    else store_as<DT>(a.out[0], to + m, v[m]);
                }
        }
    }
}

// the gradients where their rows are in parts
template <int DT>
__global__ __launch_bounds__(256) void add_parts_kernel(WeightArgs a)
{
    const int64_t all = a.of_a_part(), dA = a.of_dA(), i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int of = i >= dA;
    if (i >= all || !a.out[of]) return;
    float s = 0.0f;
    for (uint32_t part = 0; part < a.split; ++part) s += a.sums[part * all + i];
    store_as<DT>(a.out[of], of ? i - dA : i, s);
}

int tiles_of_rank(int r) { return r <= 16 ? 1 : r <= 32 ? 2 : r <= 64 ? 4 : 8; }

// Where what a tile's workgroup reads and writes by itself, the adapter and its rows either way, takes less time than a launch, and
// tiles do not fill the chip by themselves.  A forward call, two launches and one: 64 x 512 x 512 of rank 16 in bfloat16 (96 KB)
// 9.4 and 6.9 us, 256 x 512 x 512 of rank 16 10.9 and 8.5, 1000 x 512 x 512 of rank 16 in fp32 (192 KB) 14.9 and 14.5, 1 x 4096 x 4096 of rank 16 (272 KB) 9.8 and 15.5,
// 8192 x 512 x 512 of rank 8 25.6 and 26.2.
bool small_tile(const AdapterArgs& a)
{
    const int64_t rows = a.M < kTile ? a.M : kTile;
    return a.M <= 4096 && (a.K + a.N) * (a.r + rows) * dtype_size(a.dtype) <= 192 << 10;
}

// Rows without a plan: every workgroup, of a tile for every row, of which all but the first of 32 have none, looks through all of them.
// With a launch for the plan, a forward call: 32 x 4096 x 4096 of 64 adapters in bfloat16 14.0 us for 9.9, 100 x 4096 x 4096 of 64 20.5 for
// 16.1, 200 x 1024 x 1024 of 10, a small tile, 14.0 for 9.8; the other way round 256 x 4096 x 4096 of 4 15.7 for 18.3, and 20.9 for 28.2
// backward.
bool direct(const AdapterArgs& a) { return a.M <= 128 || (a.M <= kDirect && small_tile(a)); }
// (what a grid has: tiles that may be)
uint32_t grid_tiles(const AdapterArgs& a) { return (uint32_t)(direct(a) ? a.M : most_tiles(a.M, a.n)); }

// Parts of a contraction over D: as many as make 128 workgroups, none of fewer than a step for each of the eight waves; one of a small
// tile.  (Whoever reads h reads all parts.  In bfloat16, rank 16, as many as make 64, 128 and 256, and one: 32 x 4096 x 4096 of 64 adapters
// forward 11.5, 9.9, 10.0 and 14.1 us; 100 rows 18.8, 16.1, 17.6 and 18.8; 1000 rows of 10 adapters 23.8, 19.7, 18.8 and 23.7, and
// backward 21.4, 23.9, 25.8 and 21.4.)
struct Parts {
    uint32_t parts, steps;
};
Parts parts_of(const AdapterArgs& a, int64_t D)
{
    const int64_t step = a.dtype == kBf16 ? 64 : 32, steps = (D + step - 1) / step;
    const int64_t tiles = direct(a) ? (a.M < a.n ? a.M : a.n) : a.M / kTile + (a.n < a.M / kTile ? a.n : a.M / kTile);
    int64_t parts = small_tile(a) ? 1 : 128 / (tiles > 0 ? tiles : 1);
    if (parts > kMostParts) parts = kMostParts;
    while (parts > 1 && steps < parts * kDownWaves) --parts;
    if (parts < 1) parts = 1;
    const int64_t each = (steps + parts - 1) / parts;
    return {(uint32_t)((steps + each - 1) / each), (uint32_t)each};
}

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }
// the plan, and behind it, of more than one workgroup's rows, their counts
size_t counts_at(const AdapterArgs& a) { return (plan_words(a.M, a.n) + 1) / 2 * 8 + sizeof(uint2) * (size_t)most_tiles(a.M, a.n); }
size_t plan_bytes(const AdapterArgs& a)
{
    if (direct(a)) return 0;
    return rounded(counts_at(a) + (a.M > kChunkRows ? sizeof(uint32_t) * (size_t)chunks_of(a.M) * (a.n + 2) : 0));
}
size_t h_bytes(const AdapterArgs& a, int64_t D)
{
    return rounded((size_t)parts_of(a, D).parts * (size_t)a.M * 16 * tiles_of_rank(a.r) * sizeof(float));
}

// Parts of the rows that the adapters' gradients are added up over: where columns and adapters are few workgroups, as many as make 256
// of them, none of fewer than 128 rows to an adapter.  (Backward, 8192 x 4096 x 4096 of rank 16 in bfloat16, one part, 256 workgroups and
// 1024: of one adapter 102, 66 and 68 us, of four 64, 64 and 66; 8192 x 1024 x 1024 of rank 8 and four in fp32 51, 44 and 43.)
uint32_t split_of(const AdapterArgs& a)
{
    const int64_t columns = a.dtype == kBf16 ? 128 : 64;
    const int64_t groups = ((a.K + columns - 1) / columns + (a.N + columns - 1) / columns) * a.n;
    int64_t split = 256 / groups;
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

// Whether a tile goes both ways in one launch, which needs whole loads.
bool one_launch(const AdapterArgs& a, int64_t D, int64_t N, bool along)
{
    const int L = a.dtype == kBf16 ? 8 : 4;
    return small_tile(a) && D >= 8 * L && N >= 16 * L && a.r <= 64 && !(along && a.r < L);
}

template <int MODE>
void launch_pass(const AdapterArgs& a, const void* x, const void* W1, float* h, const void* W2, const void* base, void* out, int64_t D, int64_t N,
                 const RowArgs& rows, hipStream_t stream)
{
    const Parts p = parts_of(a, D);
    const uint32_t tiles = grid_tiles(a);
    const DownArgs d{rows, grid_of(tiles, p.parts), x, W1, h, D, a.r, p.steps, p.parts};
    // (a workgroup has a tile's columns in so many parts: as few as make 2048 workgroups.  With 512 and 8192, 8192 x 4096 x 16384 of rank 64
    // in bfloat16 forward 245 and 214 us for 207)
    const int64_t columns = (a.dtype == kBf16 ? 128 : 64) * kUpWaves, most = (N + columns - 1) / columns, want = 2048 / tiles + 1;
    const uint32_t across = (uint32_t)(most < want ? most : want);
    const UpArgs u{rows, grid_of(across, tiles), h, a.scale, W2, base, out, N, a.r, p.parts};
    const dim3 down(8 * d.grid.per_xcd, d.grid.slices()), up(8 * u.grid.per_xcd, u.grid.slices());
    with_types(a, [&](auto dt, auto rt) {
        constexpr int DT = dt.value, RT = rt.value, L = lane_of<DT>();
        const bool odd = N % L || (MODE == kAlong && a.r % L);
        if constexpr (RT <= 4)
            if (out && one_launch(a, D, N, MODE == kAlong)) {
                ProfileScope ps(K_ADAPT_DOWN_UP, stream);
                if (odd) hipLaunchKernelGGL((down_up_kernel<DT, RT, MODE, kOdd>), down, dim3(64 * kDownWaves), 0, stream, d, u);
                else hipLaunchKernelGGL((down_up_kernel<DT, RT, MODE, kEven>), down, dim3(64 * kDownWaves), 0, stream, d, u);
                return;
            }
        {
            ProfileScope ps(K_ADAPT_DOWN, stream);
            if (D < 8 * L) hipLaunchKernelGGL((down_kernel<DT, RT, MODE, true>), down, dim3(64 * kDownWaves), 0, stream, d);
            else hipLaunchKernelGGL((down_kernel<DT, RT, MODE, false>), down, dim3(64 * kDownWaves), 0, stream, d);
        }
        if (!out) return;
        ProfileScope ps(K_ADAPT_UP, stream);
        if (N < 16 * L || (MODE == kAlong && a.r < L)) hipLaunchKernelGGL((up_kernel<DT, RT, MODE, kShort>), up, dim3(64 * kUpWaves), 0, stream, u);
        else if (odd) hipLaunchKernelGGL((up_kernel<DT, RT, MODE, kOdd>), up, dim3(64 * kUpWaves), 0, stream, u);
        else hipLaunchKernelGGL((up_kernel<DT, RT, MODE, kEven>), up, dim3(64 * kUpWaves), 0, stream, u);
    });
}

} // namespace

size_t adapters_saved(const AdapterArgs& a) { return plan_bytes(a) + h_bytes(a, a.K); }
size_t adapters_workspace(const AdapterArgs& a) { return h_bytes(a, a.N) + sums_bytes(a); }

hipError_t launch_adapters_fwd(const AdapterArgs& a, hipStream_t stream)
{
    float* h = reinterpret_cast<float*>(static_cast<char*>(a.saved) + plan_bytes(a));
    const RowArgs rows{a.ids, direct(a) ? nullptr : a.saved, a.M, a.n};
    if (rows.plan) {
        ProfileScope ps(K_ADAPT_PLAN, stream);
        int bits = 1;
        while ((1 << bits) < a.n + 2) ++bits;
        uint32_t *plan = static_cast<uint32_t*>(a.saved), *counts = reinterpret_cast<uint32_t*>(static_cast<char*>(a.saved) + counts_at(a));
        const uint32_t chunks = (uint32_t)chunks_of(a.M);
        if (chunks == 1) {
            hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a.ids, a.M, a.n, bits, plan);
        } else {
            hipLaunchKernelGGL(plan_count_kernel, dim3(chunks), dim3(kPlanThreads), 0, stream, a.ids, a.M, a.n, bits, counts);
            hipLaunchKernelGGL(plan_starts_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a.M, a.n, plan, counts, chunks);
            hipLaunchKernelGGL(plan_order_kernel, dim3(chunks), dim3(kPlanThreads), 0, stream, a.ids, a.M, a.n, bits, plan, counts);
        }
    }
    launch_pass<kDown>(a, a.x, a.A, h, a.B, a.base, a.out, a.K, a.N, rows, stream);
    return hipGetLastError();
}

hipError_t launch_adapters_bwd(const AdapterArgs& a, void* workspace, hipStream_t stream)
{
    float* h = reinterpret_cast<float*>(static_cast<char*>(a.saved) + plan_bytes(a));
    float* g = static_cast<float*>(workspace);
    const RowArgs rows{a.ids, direct(a) ? nullptr : a.saved, a.M, a.n};
    if (a.out || a.dA) launch_pass<kAlong>(a, a.dy, a.B, g, a.A, a.base, a.out, a.N, a.K, rows, stream);
    if (a.dA || a.dB) {
        ProfileScope ps(K_ADAPT_WEIGHTS, stream);
        const int64_t columns = a.dtype == kBf16 ? 128 : 64;
        WeightArgs w{};
        w.rows = rows;
        w.h[0] = g; w.h[1] = h;
        w.v[0] = a.x; w.v[1] = a.dy;
        w.out[0] = a.dA; w.out[1] = a.dB;
        w.scale = a.scale;
        w.N[0] = a.K; w.N[1] = a.N;
        w.r = a.r;
        w.parts[0] = parts_of(a, a.N).parts; w.parts[1] = parts_of(a, a.K).parts;
        w.split = split_of(a);
        w.by_split = make_divisor(w.split);
        w.blocks = (uint32_t)((a.K + columns - 1) / columns);
        w.grid = grid_of(w.blocks + (uint32_t)((a.N + columns - 1) / columns), (uint32_t)a.n * w.split);
        if (w.split > 1) w.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + h_bytes(a, a.N));
        with_types(a, [&](auto dt, auto rt) {
            hipLaunchKernelGGL((weights_kernel<dt.value, rt.value>), dim3(8 * w.grid.per_xcd, w.grid.slices()), dim3(64 * kWeightWaves), 0, stream, w);
            if (w.split > 1) {
                const int64_t all = (int64_t)a.n * a.r * (a.K + a.N);
                hipLaunchKernelGGL((add_parts_kernel<dt.value>), dim3((uint32_t)((all + 255) / 256)), dim3(256), 0, stream, w);
            }
        });
    }
    return hipGetLastError();
}

} // namespace hdqt
