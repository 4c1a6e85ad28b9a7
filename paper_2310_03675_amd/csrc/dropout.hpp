// Dropout's mask from the counter-based generator of the stochastic rounding, for the kernels that apply it, and the vectors of
// eight elements, one block of the generator's fields, that they walk in.
//
// Element e of a tensor has a draw u(e) of 32 bits.  Its upper half is field e mod 8 (16 bits, lowest first) of the block
// Philox4x32-10(counter = (e / 8, tensor id, 1), key = seed), its lower half the same field under the counter's last word 2; the
// stochastic rounding's last word is 0.  e is dropped where u(e) < round(p 2^32).  The upper half alone decides but where it
// equals the bound's, once in 65536 elements, so that eight elements cost one block and a branch that few waves take, and the
// probability is exact to 2^-33 all the same.  A block is 20 multiplications of 32 x 32 bits at a quarter of the other
// instructions' rate: with 32 bits of each block to an element the generator would bound a bfloat16 tensor, not memory.
#pragma once
#include "train.hpp"

namespace hdqt {

// Two values as bfloat16, rounded to nearest even, in one instruction of this chip (a NaN stays one).
__device__ __forceinline__ uint32_t two_bf16(float a, float b)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2b));
}

// Eight neighbouring elements, wherever they start.
template <int DT>
struct Eight {
    static constexpr int kWords = DT == kF32 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float get(int j) const
    {
        if (DT == kF32) return __uint_as_float(w[j % kWords]);
        return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int j = 0; j < kWords; ++j) w[j] = DT == kF32 ? __float_as_uint(v[j]) : two_bf16(v[2 * j % 8], v[(2 * j + 1) % 8]);
    }
    // The compiler takes the values for new ones: what it made of them before is not kept in registers, twice as wide, but made again.
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int j = 0; j < kWords; ++j) asm("" : "+v"(w[j]));
    }
};

// (16 bytes at a time at any alignment of an element)
template <int DT>
__device__ __forceinline__ Eight<DT> load_eight(const void* p, int64_t at)
{
    Eight<DT> q;
    const char* from = static_cast<const char*>(p) + at * (DT == kF32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < Eight<DT>::kWords; i += 4) __builtin_memcpy(q.w + i, from + 4 * i, 16);
    return q;
}
template <int DT>
__device__ __forceinline__ void store_eight(void* p, int64_t at, const Eight<DT>& q)
{
    char* to = static_cast<char*>(p) + at * (DT == kF32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < Eight<DT>::kWords; i += 4) __builtin_memcpy(to + 4 * i, q.w + i, 16);
}
// the first n of them; the others are zero, and nothing else is read
template <int DT>
__device__ __forceinline__ Eight<DT> load_some(const void* p, int64_t at, int n)
{
    Eight<DT> q{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) {
            if (DT == kF32) q.w[j % Eight<DT>::kWords] = static_cast<const uint32_t*>(p)[at + j];
            else q.w[j / 2] |= (uint32_t)static_cast<const uint16_t*>(p)[at + j] << 16 * (j & 1);
        }
    return q;
}
// those from `lo` on and before `hi`, one by one: a row's end (one, two and four at a time were no faster, at 20011 x 1031 in fp32
// backward 94 us for 77)
template <int DT>
__device__ __forceinline__ void store_some(void* p, int64_t at, int lo, int hi, const Eight<DT>& q)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j >= lo && j < hi) {
            if (DT == kF32) static_cast<uint32_t*>(p)[at + j] = q.w[j % Eight<DT>::kWords];
            else static_cast<uint16_t*>(p)[at + j] = (uint16_t)(q.w[j / 2] >> 16 * (j & 1));
        }
}

// the generator's key: the seed, and what a counter on the device has come to
__device__ __forceinline__ uint64_t drop_key(const DropArgs& d) { return d.step ? d.seed + (uint64_t)*d.step : d.seed; }

// Bit j: whether element 8 block + j is kept.
__device__ __forceinline__ uint32_t kept_block(const DropArgs& d, uint64_t key, uint64_t block)
{
    uint32_t r[4], keep = 0, open = 0;
    philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), d.tensor_id, 1u, (uint32_t)key, (uint32_t)(key >> 32), r);
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        const uint32_t u = sr_halfword(r, j);
        keep |= (uint32_t)(u > d.hi) << j;
        open |= (uint32_t)(u == d.hi) << j;
    }
    if (open) {
        philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), d.tensor_id, 2u, (uint32_t)key, (uint32_t)(key >> 32), r);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) keep |= open & (uint32_t)(sr_halfword(r, j) >= d.lo) << j;
    }
    return keep;
}

// Bit j: whether element e + j is kept.
__device__ __forceinline__ uint32_t kept_eight(const DropArgs& d, uint64_t key, int64_t e)
{
    const uint64_t block = (uint64_t)e >> 3;
    const int shift = (int)(e & 7);
    uint32_t keep = kept_block(d, key, block) >> shift;
    if (shift) keep |= kept_block(d, key, block + 1) << (8 - shift);
    return keep;
}

} // namespace hdqt
