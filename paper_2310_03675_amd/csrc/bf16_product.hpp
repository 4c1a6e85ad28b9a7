// A product of bfloat16 matrices on the matrix cores, sums in 32 bits: out(i, j) = sum_k A(i, k) B(j, k), for what an
// epilogue makes of a workgroup's part of it (gfx950).
//
// An operand lies in memory with its contraction along the rows (kAlong) or down them (kDown); both ways come to LDS by loads
// that write there directly, 16 bytes a lane, and neither needs a copy in another order: fragments of kDown are read by
// the transposing LDS reads of this chip.  fp32 operands are three bfloat16 matrices (planes) that add up to them, 8
// bits each, and the product the six products of planes that are not below 2^-24 of the whole, smallest first.
#pragma once
#include "train.hpp"

#include <type_traits>

namespace hdqt {
namespace bf16 {

enum Mode { kAlong, kDown };

// An operand in memory, bfloat16: rows `step` elements apart, 16-byte aligned with step a multiple of 8, and so is what a row
// holds (zeros behind the end, where there is padding).  kAlong: a row is a line of the product; kDown: a line is a column.
struct Side {
    const uint16_t* p;
    int64_t step, plane;            // elements from a row, from a plane, to the next
};

struct Args {
    Side A, B;
    int64_t RA, RB, D;              // lines of A, of B; contraction
    int terms;                      // 1, or 6 products of planes
    uint32_t n_at, n_bt, tiles, per_xcd;
    Divisor group, out_tiles;
    uint32_t stages, part_stages, parts;        // of 64 along the contraction
};

constexpr uint32_t kOutside = 0x80000000u;
constexpr int kStage = 64;          // of the contraction

typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

// planes of the six products, smallest first
__device__ __forceinline__ int plane_a(int term) { return (0x201100 >> (4 * (5 - term))) & 3; }
__device__ __forceinline__ int plane_b(int term) { return (0x021010 >> (4 * (5 - term))) & 3; }

inline Args plan(const Side& A, const Side& B, int64_t RA, int64_t RB, int64_t D, bool planes, int ta, int tb, uint32_t parts)
{
    Args g{};
    g.A = A; g.B = B; g.RA = RA; g.RB = RB; g.D = D; g.terms = planes ? 6 : 1;
    g.n_at = (uint32_t)((RA + ta - 1) / ta); g.n_bt = (uint32_t)((RB + tb - 1) / tb);
    g.stages = (uint32_t)((D + kStage - 1) / kStage);
    g.part_stages = (g.stages + parts - 1) / parts;
    g.parts = (g.stages + g.part_stages - 1) / g.part_stages;
    g.tiles = g.n_at * g.n_bt * g.parts;
    g.per_xcd = (g.tiles + 7) / 8;
    g.group = make_divisor(8 * g.n_bt);
    g.out_tiles = make_divisor(g.n_at * g.n_bt);
    return g;
}

// Workgroups go to the eight XCDs in turn: each gets a run of tiles of its own, in groups of eight tiles of A, tile of B by
// tile of B, whose panels its L2 holds.
struct Place {
    uint32_t part, at, bt, first, n;            // stages of the part
    bool there;
};
__device__ __forceinline__ Place place_of(const Args& g)
{
    Place p;
    const uint32_t idx = (blockIdx.x & 7) * g.per_xcd + (blockIdx.x >> 3);
    p.there = idx < g.tiles;
    p.part = divide(idx, g.out_tiles);
    const uint32_t it = idx - p.part * g.out_tiles.d;
    const uint32_t grp = divide(it, g.group), in = it - grp * g.group.d;
    const uint32_t tall = g.n_at - 8 * grp < 8 ? g.n_at - 8 * grp : 8;
    p.bt = in / tall;
    p.at = 8 * grp + in - p.bt * tall;
    p.first = p.part * g.part_stages;
    p.n = g.stages - p.first < g.part_stages ? g.stages - p.first : g.part_stages;
    return p;
}

// One operand of a workgroup: T lines of it, brought by WAVES waves.
//
// In LDS a stage is T rows of 64 codes (kAlong) or 64 rows of T (kDown), and a row's 16-byte pieces are turned by the row's
// number, so that what a fragment's reads touch together lies in different banks.
template <int MODE, int T, int WAVES>
struct Panel {
    static constexpr int kRowBytes = MODE == kAlong ? 2 * kStage : 2 * T;
    static constexpr int kPieces = kRowBytes / 16;
    static constexpr int kBytes = 2 * kStage * T;
    static constexpr int kLoads = kBytes / (1024 * WAVES);          // of a wave, 1 KB each
    static_assert(kLoads >= 1 && kPieces >= 8 && 1024 % kRowBytes == 0, "a load is whole rows");
    static constexpr int kRowsOfLoad = 1024 / kRowBytes;

    static __device__ __forceinline__ int turn(int row)
    {
        if (MODE == kAlong) return (row >> 1) & 7;
        return kPieces >= 16 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
    }

    uint32_t off[kLoads];           // of a lane's piece, from the stage's first byte
    int64_t lines_left, d;
    const uint16_t* base;
    int64_t step, plane;
    int col[kLoads > 1 ? 2 : 1];    // kAlong: first code of a lane's piece in even and odd loads

    __device__ __forceinline__ Panel(const Side& s, int64_t lines, int64_t line0, int64_t D, int wave, int lane)
    {
        step = s.step; plane = s.plane; d = D;
        lines_left = lines - line0;
        base = s.p + (MODE == kAlong ? line0 * s.step : line0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int row = (wave * kLoads + j) * kRowsOfLoad + lane / kPieces;
            const int piece = (lane % kPieces) ^ turn(row);
            off[j] = (uint32_t)row * (uint32_t)step * 2 + 16 * piece;
            if (MODE == kAlong) col[j & (kLoads > 1)] = 8 * piece;          // (turns repeat every 16 rows: two loads)
            else if (8 * piece >= lines_left) off[j] = kOutside;
        }
    }

    // stage `s` of plane `pl` to LDS
    template <class L>
    __device__ __forceinline__ void bring(L* lds, uint32_t s, int pl, int wave) const
    {
        const int64_t at = (int64_t)s * kStage;
        const uint16_t* from = base + pl * plane + (MODE == kAlong ? at : at * step);
        // elements from here to the operand's end
        const int64_t rows = MODE == kAlong ? lines_left : d - at, width = MODE == kAlong ? d - at : lines_left;
        const int64_t bytes = 2 * ((rows - 1) * step + (width + 7) / 8 * 8);
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint16_t*>(from), 0, bytes <= 0 ? 0 : bytes < (int64_t)kOutside ? (int)bytes : (int)(kOutside - 1), 0x00020000);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            uint32_t o = off[j];
            if (MODE == kAlong) o = at + col[j & (kLoads > 1)] < d ? o : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + j) * 1024), 16, o, 0, 0, 0);
        }
    }
};

// Fragments of a wave's lines: N blocks of 32, sixteen of the contraction at a time (lane: line lane % 32, the eight codes
// from 8 (lane / 32) on).
template <int MODE, int T, int N>
struct Fragments {
    uint32_t at[MODE == kAlong ? 4 : N];
    __device__ __forceinline__ Fragments(int line0, int lane)
    {
        if constexpr (MODE == kAlong) {
            const int row = line0 + (lane & 31);
#pragma unroll
            for (int q = 0; q < 4; ++q) at[q] = row * 128 + 16 * ((2 * q + (lane >> 5)) ^ ((row >> 1) & 7));
        } else {
            // sixteen lanes read four rows of 16 codes; lane i gets column i
            const int k = 8 * (lane >> 5) + ((lane >> 2) & 3);
            const int turn = Panel<MODE, T, 1>::turn(k);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int column = line0 + 32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                at[i] = k * 2 * T + 16 * ((column >> 3) ^ turn) + 2 * (column & 7);
            }
        }
    }
    template <class L>
    __device__ __forceinline__ v8b read(const L* lds, int i, int q) const
    {
        if constexpr (MODE == kAlong) {
            return *reinterpret_cast<const v8b*>(lds + at[q] + 4096 * i);
        } else {
            typedef __attribute__((address_space(3))) v4s* local;
            const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((local)(lds + at[i] + 32 * T * q));
            const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((local)(lds + at[i] + 32 * T * q + 8 * T));
            return __builtin_bit_cast(v8b, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// The part's sums: acc[i][j], block i of the wave's lines of A and j of B.  The two stages in LDS are objects of their own, so
// that the compiler knows which loads a read must wait for.  A wave waits for its own part of a stage, and for its own
// reads of the buffer that is brought next, in front of the barrier.
template <int MA, int MB, int TA, int TB, int WA, int WB, class LA, class LB>
__device__ __forceinline__ void multiply(const Args& g, const Place& p, LA* a0, LA* a1, LB* b0, LB* b1, int wave, int lane,
                                         v16f (&acc)[TA / WA / 32][TB / WB / 32])
{
    constexpr int NA = TA / WA / 32, NB = TB / WB / 32;
    const Panel<MA, TA, WA * WB> pa(g.A, g.RA, (int64_t)p.at * TA, g.D, wave, lane);
    const Panel<MB, TB, WA * WB> pb(g.B, g.RB, (int64_t)p.bt * TB, g.D, wave, lane);
    const Fragments<MA, TA, NA> fa((wave / WB) * (TA / WA), lane);
    const Fragments<MB, TB, NB> fb((wave % WB) * (TB / WB), lane);
    uint32_t s = 0;                 // what is brought next
    int term = 0;
    auto bring = [&](LA* a, LB* b) {
        const bool one = g.terms == 1;
        pa.bring(a, p.first + s, one ? 0 : plane_a(term), wave);
        pb.bring(b, p.first + s, one ? 0 : plane_b(term), wave);
        if (++s == p.n) { s = 0; ++term; }
    };
    auto arrived = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);         // vmcnt(0) lgkmcnt(0), as the compiler's own bookkeeping takes it
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto products = [&](const LA* a, const LB* b) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            __builtin_amdgcn_sched_barrier(0);
            v8b x[NA], y[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) y[j] = fb.read(b, j, q);
#pragma unroll
            for (int i = 0; i < NA; ++i) x[i] = fa.read(a, i, q);
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
        }
    };
    const uint32_t total = p.n * (uint32_t)g.terms;
    bring(a0, b0);
    for (uint32_t done = 0; done < total; done += 2) {
        arrived();
        if (done + 1 < total) bring(a1, b1);
        products(a0, b0);
        if (done + 1 < total) {
            arrived();
            if (done + 2 < total) bring(a0, b0);
            products(a1, b1);
        }
    }
    // (what follows may write where the last stage lies)
    arrived();
}

} // namespace bf16
} // namespace hdqt
