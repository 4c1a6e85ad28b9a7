// A product of bfloat16 matrices on the matrix cores, sums in 32 bits: out(i, j) = sum_k A(i, k) B(j, k), for what an
// epilogue makes of a workgroup's part of it (gfx950).
//
// An operand lies in memory with its contraction along the rows (kAlong) or down them (kDown); both ways come to LDS by loads
// that write there directly, 16 bytes a lane, and neither needs a copy in another order: fragments of kDown are read by
// the transposing LDS reads of this chip.  fp32 operands (P = 3) are three bfloat16 matrices, planes, that add up to them, 8
// bits each, and the product is the six products of planes that are not below 2^-24 of the whole, smallest first; a stage
// holds all planes, so that six products share the loads and the LDS reads of six planes.
//
// What bounds it: 8192 x 4096 x 16384 in tiles of 256 x 256, eight waves, the matrix pipe is busy 57 to 64 % of the time at
// the 1.7 to 1.85 GHz that the chip holds under it, LDS 22 %, without conflicts; a stage of 64 takes 1.85 us, of which the
// products are 1.1.  A step of the classifier's loss over 128000 classes takes 28.2 ms, with one set of fragments 29.8; with the matrix
// instructions at a higher wave priority, or without the fences around the reads, 28.7 and 29.6; with four waves of 128 x 128,
// one to a SIMD, 31.8.
#pragma once
#include "train.hpp"

#include <type_traits>

namespace hdqt {
namespace bf16 {

enum Mode { kAlong, kDown };

// An operand in memory, bfloat16: rows `step` elements apart, 16-byte aligned with step a multiple of 8.
// One plane: what a row holds is a multiple of 8 (zeros behind the end, where there is padding).
// Three: 32 codes of a plane stand together, [row][column / 32][plane][column % 32], and a row is a multiple of 32 columns.
// kAlong: a row is a line of the product; kDown: a line is a column.
struct Side {
    const uint16_t* p;
    int64_t step;
};

struct Args {
    Side A, B;
    int64_t RA, RB, D;              // lines of A, of B; contraction
    uint32_t n_at, n_bt, tiles, per_xcd;
    Divisor group, out_tiles;
    uint32_t stages, part_stages, parts;        // of stage_of(P) along the contraction
};

constexpr uint32_t kOutside = 0x80000000u;
constexpr int stage_of(int planes) { return planes == 1 ? 64 : 32; }

typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));

inline Args plan(const Side& A, const Side& B, int64_t RA, int64_t RB, int64_t D, int planes, int ta, int tb, uint32_t parts)
{
    Args g{};
    g.A = A; g.B = B; g.RA = RA; g.RB = RB; g.D = D;
    g.n_at = (uint32_t)((RA + ta - 1) / ta); g.n_bt = (uint32_t)((RB + tb - 1) / tb);
    g.stages = (uint32_t)((D + stage_of(planes) - 1) / stage_of(planes));
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

// (there: else nothing is in range.  A mask: a choice makes the compiler branch around the arithmetic, inside the loop)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const uint16_t* from, int64_t elements, bool there)
{
    int64_t bytes = 2 * elements;
    bytes = bytes < 0 ? 0 : bytes;
    bytes = bytes < (int64_t)kOutside ? bytes : (int64_t)kOutside - 1;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(from), 0, (int)bytes & -(int)there, 0x00020000);
}

// One operand of a workgroup, T lines of it, brought by WAVES waves: a stage to LDS.
//
// One plane: T rows of 64 codes (kAlong) or 64 rows of T (kDown), and a row's 16-byte pieces are turned by the row's
// number, so that what a fragment's reads touch together lies in different banks.
template <int P, int MODE, int T, int WAVES>
struct Panel {
    static constexpr int kStage = 64, kRowBytes = MODE == kAlong ? 2 * kStage : 2 * T, kPieces = kRowBytes / 16;
    static constexpr int kBytes = 2 * kStage * T;
    static constexpr int kLoads = kBytes / (1024 * WAVES);          // of a wave, 1 KB each
    static_assert(P == 1 && kLoads > 1 && (MODE == kAlong || kPieces >= 16) && 1024 % kRowBytes == 0, "a load is whole rows");

    static __device__ __forceinline__ int turn(int row)
    {
        return MODE == kAlong ? (row >> 1) & 7 : 4 * (row & 3);
    }

    uint32_t off[kLoads];           // of a lane's piece, from the stage's first byte
    int64_t lines_left, d, step;
    const uint16_t* base;
    int col[2];                     // kAlong: first code of a lane's piece in even and odd loads

    __device__ __forceinline__ Panel(const Side& s, int64_t lines, int64_t line0, int64_t D, int wave, int lane)
    {
        step = s.step; d = D;
        lines_left = lines - line0;
        base = s.p + (MODE == kAlong ? line0 * s.step : line0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int row = (wave * kLoads + j) * (1024 / kRowBytes) + lane / kPieces;
            const int piece = (lane % kPieces) ^ turn(row);
            off[j] = (uint32_t)row * (uint32_t)step * 2 + 16 * piece;
            if (MODE == kAlong) col[j & 1] = 8 * piece;          // (turns repeat every 16 rows: two loads)
            else if (8 * piece >= lines_left) off[j] = kOutside;
        }
    }

    __device__ __forceinline__ void bring(uint8_t* lds, uint32_t s, bool there, int wave) const
    {
        const int64_t at = (int64_t)s * kStage;
        const int64_t rows = MODE == kAlong ? lines_left : d - at, width = MODE == kAlong ? d - at : lines_left;
        const __amdgpu_buffer_rsrc_t rs = range_of(base + (MODE == kAlong ? at : at * step), (rows - 1) * step + (width + 7) / 8 * 8, there);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            uint32_t o = off[j];
            if (MODE == kAlong) o = at + col[j & 1] < d ? o : kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + j) * 1024), 16, o, 0, 0, 0);
        }
    }
};

// Three planes, 32 of the contraction: T rows of 192 bytes (kAlong; neighbours of two pieces change places every four rows) or
// 32 rows of 6 T (kDown; blocks of 32 columns are turned by the row's number).
template <int MODE, int T, int WAVES>
struct Panel<3, MODE, T, WAVES> {
    static constexpr int kStage = 32, kPieces = MODE == kAlong ? 12 : 12 * T / 32, kBytes = 192 * T;
    static constexpr int kLoads = kBytes / (1024 * WAVES);
    static_assert(kLoads >= 1 && kLoads * 1024 * WAVES == kBytes && T % 64 == 0, "whole loads, blocks of columns to turn");
    static constexpr int kTurns = T >= 128 ? 3 : 1;          // (of two blocks only pairs of rows are kept apart)

    uint32_t off[kLoads];
    int64_t rows_left, step;        // kDown: rows of the whole contraction
    const uint16_t* base;
    int64_t width;                  // of a row from the base on

    __device__ __forceinline__ Panel(const Side& s, int64_t lines, int64_t line0, int64_t D, int wave, int lane)
    {
        step = s.step;
        rows_left = MODE == kAlong ? lines - line0 : D;
        base = s.p + (MODE == kAlong ? line0 * s.step : 3 * line0);
        width = MODE == kAlong ? step : step - 3 * line0;
        const int64_t room = 3 * ((lines - line0 + 31) / 32 * 32);      // (kDown: the columns that there are)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int g = (wave * kLoads + j) * 64 + lane, row = g / kPieces, at = g % kPieces;
            const int piece = MODE == kAlong ? at ^ ((row >> 2) & 1) : ((at / 12) ^ (row & kTurns)) * 12 + at % 12;
            off[j] = (uint32_t)row * (uint32_t)step * 2 + 16 * piece;
            if (MODE == kDown && 8 * piece >= room) off[j] = kOutside;
        }
    }

    __device__ __forceinline__ void bring(uint8_t* lds, uint32_t s, bool there, int wave) const
    {
        const int64_t at = (int64_t)s * kStage;
        const int64_t elements = MODE == kAlong ? (rows_left - 1) * step + width - 3 * at : (rows_left - at - 1) * step + width;
        const __amdgpu_buffer_rsrc_t rs = range_of(base + (MODE == kAlong ? 3 * at : at * step), elements, there);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(lds + (wave * kLoads + j) * 1024), 16, off[j], 0, 0, 0);
    }
};

__device__ __forceinline__ v8b read_turned(const uint8_t* lds, int row_bytes)
{
    typedef __attribute__((address_space(3))) v4s* local;
    const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((local)lds), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((local)(lds + 4 * row_bytes));
    return __builtin_bit_cast(v8b, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Fragments of a wave's lines: N blocks of 32, sixteen of the contraction at a time (lane: line lane % 32, the eight codes
// from 8 (lane / 32) on).  kDown: sixteen lanes read four rows of 16 codes, and lane i gets column i.
template <int P, int MODE, int T, int N>
struct Fragments {
    uint32_t at[MODE == kAlong ? 4 : N];
    __device__ __forceinline__ Fragments(int line0, int lane)
    {
        if constexpr (MODE == kAlong) {
            const int row = line0 + (lane & 31);
#pragma unroll
            for (int q = 0; q < 4; ++q) at[q] = row * 128 + 16 * ((2 * q + (lane >> 5)) ^ ((row >> 1) & 7));
        } else {
            const int k = 8 * (lane >> 5) + ((lane >> 2) & 3);
            const int turn = Panel<P, MODE, T, 1>::turn(k);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int column = line0 + 32 * i + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
                at[i] = k * 2 * T + 16 * ((column >> 3) ^ turn) + 2 * (column & 7);
            }
        }
    }
    __device__ __forceinline__ v8b read(const uint8_t* lds, int i, int q, int) const
    {
        if constexpr (MODE == kAlong) return *reinterpret_cast<const v8b*>(lds + at[q] + 4096 * i);
        else return read_turned(lds + at[i] + 32 * T * q, 2 * T);
    }
};

template <int MODE, int T, int N>
struct Fragments<3, MODE, T, N> {
    uint32_t at[MODE == kAlong ? 1 : N];
    __device__ __forceinline__ Fragments(int line0, int lane)
    {
        if constexpr (MODE == kAlong) {
            const int row = line0 + (lane & 31);
            at[0] = row * 192 + 16 * ((lane >> 5) ^ ((row >> 2) & 1));
        } else {
            const int m = (lane >> 2) & 3, k = 8 * (lane >> 5) + m;
#pragma unroll
            for (int i = 0; i < N; ++i)
                at[i] = k * 6 * T + 192 * (((line0 >> 5) + i) ^ (m & (T >= 128 ? 3 : 1))) + 2 * (16 * ((lane >> 4) & 1) + 4 * (lane & 3));
        }
    }
    __device__ __forceinline__ v8b read(const uint8_t* lds, int i, int q, int plane) const
    {
        if constexpr (MODE == kAlong) return *reinterpret_cast<const v8b*>(lds + at[0] + 6144 * i + 32 * q + 64 * plane);
        else return read_turned(lds + at[i] + 96 * T * q + 64 * plane, 6 * T);
    }
};

// A wave's loads have arrived, and all it reads from LDS; then every wave's.  (The wait is one that the compiler's own
// bookkeeping takes in.)
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

struct Stages {
    uint8_t *a[2], *b[2];
};

// The part's sums: acc[i][j], block i of the wave's lines of A and j of B.  Two stages in LDS, objects of their own, so that the
// compiler knows which loads a read must wait for.  A wave waits for its own part of a stage, and for its own reads of the
// buffer that is brought next, in front of the barrier.
template <int P, int MA, int MB, int TA, int TB, int WA, int WB, int NA, int NB>
__device__ __forceinline__ void multiply(const Args& g, const Place& p, const Stages& lds, int wave, int lane,
                                         v16f (&acc)[NA][NB])
{
#ifdef __HIP_DEVICE_COMPILE__       // (the host's pass has no use for the body, nor all of its builtins)
    static_assert(NA == TA / WA / 32 && NB == TB / WB / 32, "a wave's blocks");
    typedef Panel<P, MA, TA, WA * WB> PanelA;
    typedef Panel<P, MB, TB, WA * WB> PanelB;
    const PanelA pa(g.A, g.RA, (int64_t)p.at * TA, g.D, wave, lane);
    const PanelB pb(g.B, g.RB, (int64_t)p.bt * TB, g.D, wave, lane);
    const Fragments<P, MA, TA, NA> fa((wave / WB) * (TA / WA), lane);
    const Fragments<P, MB, TB, NB> fb((wave % WB) * (TB / WB), lane);
    auto bring = [&](uint32_t s, uint8_t* a, uint8_t* b) {
        pa.bring(a, p.first + s, s < p.n, wave);
        pb.bring(b, p.first + s, s < p.n, wave);
    };
    // fragments of sixteen of the contraction, two sets: one is read while the other is multiplied
    struct Set {
        v8b x[NA][P], y[NB][P];
    } set[2];
    auto read = [&](Set& f, int u, int q) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = P - 1; k >= 0; --k) {
#pragma unroll
            for (int j = 0; j < NB; ++j) f.y[j][k] = fb.read(lds.b[u], j, q, k);
#pragma unroll
            for (int i = 0; i < NA; ++i) f.x[i][k] = fa.read(lds.a[u], i, q, k);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](const Set& f) {
        auto term = [&](int ka, int kb) {
#pragma unroll
            for (int i = 0; i < NA; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.x[i][ka], f.y[j][kb], acc[i][j], 0, 0, 0);
        };
        if constexpr (P == 3) {
            term(2, 0);
            term(0, 2);
            term(1, 1);
            term(1, 0);
            term(0, 1);
        }
        term(0, 0);
    };
    constexpr int kSteps = stage_of(P) / 16;
    static_assert(kSteps % 2 == 0, "the sets take turns");
    // (stages behind the last are zeros: whole rounds of two, and the same waits everywhere)
    bring(0, lds.a[0], lds.b[0]);
    wait_and_meet();
    bring(1, lds.a[1], lds.b[1]);
    read(set[0], 0, 0);
    for (uint32_t s = 0; s < p.n; s += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int q = 0; q + 1 < kSteps; ++q) {
                read(set[(q + 1) & 1], u, q + 1);
                products(set[q & 1]);
            }
            // the stage has been read: what is brought next goes into its place, while the last sixteen are multiplied
            wait_and_meet();
            bring(s + u + 2, lds.a[u], lds.b[u]);
            read(set[0], 1 - u, 0);
            products(set[1]);
        }
    }
    wait_and_meet();                // (what follows may write where a stage lies)
#endif
}

} // namespace bf16
} // namespace hdqt
