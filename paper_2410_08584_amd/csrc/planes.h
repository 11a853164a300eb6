// fp32 numbers as planes of bf16 for the matrix cores, shared by the fp32 forms of attention.
#pragma once
#include "common.h"

namespace zipvl {

// Eight fp32 values as three bf16 planes, x = hi + mid + lo (8 significant bits and a sign each, rounded to nearest, so
// that a plane holds at most 2^-9 of the one before): exactly from 2^-109 on; below, the last plane ends at bf16's smallest number and
// the sum is off by up to 2^-134.  An infinity, a NaN or a value that rounds to one leaves a NaN in mid or lo.
struct Planes { uintx4 hi, mid, lo; };
// The smallest magnitude other than 0 of some fp32 values, as 2 |x| - 1 of the bits: 0 is the largest of all.
struct Least {
    uint32_t key = ~0u;
    __device__ __forceinline__ void add(uint32_t x) { key = min(key, 2 * x - 1); }
    __device__ __forceinline__ bool below(float x) const { return key < 2 * __float_as_uint(x) - 1; }        // x > 0
};
// Planes are off by 2^-134 where a number is small: nothing in a logit as long as what the number is multiplied by is below this.  Tiles that meet larger numbers are taken again, in fp32
// products.
constexpr float kPlaneHigh = 0x1p100f;
// x - the low (high) half of a packed pair, in one instruction
// (the factors through a register: as a constant 0xBF800000 is taken for the float -1)
__device__ __forceinline__ float less_half(float x, uint32_t pair, uint32_t factors) {
    asm("" : "+s"(factors));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, factors), x, false);
}
__device__ __forceinline__ float less_low(float x, uint32_t pair) { return less_half(x, pair, 0x0000BF80u); }
__device__ __forceinline__ float less_high(float x, uint32_t pair) { return less_half(x, pair, 0xBF800000u); }
__device__ __forceinline__ Planes split8(const uintx4& a, const uintx4& b) {
    Planes s;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float x0 = __uint_as_float(e < 2 ? a[2 * e] : b[2 * e - 4]), x1 = __uint_as_float(e < 2 ? a[2 * e + 1] : b[2 * e - 3]);
        const uint32_t hi = pack_bf16x2(x0, x1);
        const float r0 = less_low(x0, hi), r1 = less_high(x1, hi);
        const uint32_t mid = pack_bf16x2(r0, r1);
        s.hi[e] = hi;
        s.mid[e] = mid;
        s.lo[e] = pack_bf16x2(less_low(r0, mid), less_high(r1, mid));
    }
    return s;
}
// acc + a b in six products, the small ones first; what is left out (mid lo, lo mid, lo lo) is below 2^-26 of |a| |b|.
__device__ __forceinline__ floatx16 mma_planes(const Planes& a, const Planes& b, floatx16 acc) {
    acc = mma_frag<__bf16>(a.lo, b.hi, acc);
    acc = mma_frag<__bf16>(a.hi, b.lo, acc);
    acc = mma_frag<__bf16>(a.mid, b.mid, acc);
    acc = mma_frag<__bf16>(a.mid, b.hi, acc);
    acc = mma_frag<__bf16>(a.hi, b.mid, acc);
    return mma_frag<__bf16>(a.hi, b.hi, acc);
}

}  // namespace zipvl
