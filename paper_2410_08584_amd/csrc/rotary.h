// Rotary positions: angles as fractions of a turn, rotation of a thread's eight pairs of channels.
#pragma once
#include "common.h"

namespace zipvl {

// zipvl_rope on the device, by value in the kernel arguments.
struct Turns {
    uint64_t turn[ZIPVL_MAX_PAIRS];          // of pair i, a position: freq / (2 pi) without whole turns, in 2^-64 of one
    uint8_t axis[ZIPVL_MAX_PAIRS];           // row of pos
    int axes, pairs, neighbours;
    uint32_t backwards;                      // the sign bit of the sines: 0x80000000 turns the other way
};

// sin and cos of pos * freq.  Whole turns must go before anything is rounded: position 60000 of a frequency of 1 is 9549 turns,
// and a product in fp32 leaves 2^-10 of a turn.  In whole numbers they go by themselves: the low 64 bits of pos * turn are the
// fraction (a negative position included).  A turn is off by up to 3 2^-64, 2.2e-9 radians at 2^31, and the 32 bits that are kept cost 1.5e-9: 3.7e-9 radians at any
// position.  An eighth of a turn to both sides of a quarter is left for the Taylor series (to x^9 / 9! and x^10 / 10!: 2e-9 at pi/4); rounding that and its
// factor to fp32 is most of the error, and sine and cosine are within 3.5 2^-24; v_sin_f32 is not.
__device__ __forceinline__ void turn_of(uint32_t pos, uint64_t turn, uint32_t backwards, float& sn, float& cs) {
    const uint32_t lo = (uint32_t)turn, hi = (uint32_t)(turn >> 32);
    uint32_t f = __umulhi(pos, lo) + pos * hi - ((int32_t)pos < 0 ? lo : 0u);        // in 2^-32 of a turn
    const uint32_t quarter = (f + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(f - (quarter << 30)) * 1.4629180792671596e-09f;  // 2 pi / 2^32
    const float y = x * x;
    const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-06f, -1.9841270e-04f), 8.3333333e-03f), -1.6666667e-01f), x);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-07f, 2.4801587e-05f), -1.3888889e-03f), 4.1666667e-02f), -0.5f), 1.f);
    const uint32_t a = __float_as_uint(quarter & 1 ? c : s), b = __float_as_uint(quarter & 1 ? s : c);
    sn = __uint_as_float(a ^ ((quarter & 2) << 30) ^ backwards);
    cs = __uint_as_float(b ^ (((quarter + 1) & 2) << 30));
}

// A token's positions, and what a thread's eight pairs take of a turn a position: all of it is asked for at once, the axes' positions before it is known
// which of them a pair goes by.
struct Angles {
    uint32_t pos[ZIPVL_MAX_AXES];
    uint64_t turn[8], axis;                                  // a byte a pair
    float sn[8], cs[8];
    __device__ __forceinline__ void ask(const Turns& t, int first, const int32_t* at, int64_t stride) {
#pragma unroll
        for (int a = 0; a < ZIPVL_MAX_AXES; ++a) {
            pos[a] = pos[0];
            if (a < t.axes) pos[a] = (uint32_t)at[a * stride];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) turn[e] = t.turn[first + e];
        axis = *reinterpret_cast<const uint64_t*>(t.axis + first);
    }
    __device__ __forceinline__ void take(const Turns& t) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t a = (uint32_t)(axis >> (8 * e)) & 3;
            uint32_t at = pos[0];
            if (t.axes > 1) {
                at = a == 1 ? pos[1] : at;
                at = a == 2 ? pos[2] : at;
                at = a == 3 ? pos[3] : at;
            }
            turn_of(at, turn[e], t.backwards, sn[e], cs[e]);
        }
    }
};

// Sixteen channels of a row, the share of one of its D / 16 threads: two runs of eight.  Thread c < pairs / 8 has pairs 8 c .. 8 c + 7,
// which are the runs at 8 c and pairs + 8 c (halves) or 16 c and 16 c + 8 (neighbours); the other threads have the channels that no
// pair has.
struct Runs {
    int a, b, first;                         // channels; first pair, -1: none
    __device__ __forceinline__ Runs(int c, int pairs, int neighbours) {
        const int mine = c - pairs / 8;
        if (mine >= 0) { a = 2 * pairs + 16 * mine; b = a + 8; first = -1; }
        else if (neighbours) { a = 16 * c; b = a + 8; first = 8 * c; }
        else { a = 8 * c; b = pairs + a; first = a; }
    }
};

template <typename T> struct Run { uintx4 v[sizeof(T) / 2]; };                       // eight channels
template <typename T>
__device__ __forceinline__ Run<T> load_run(const T* p) {
    Run<T> r;
#pragma unroll
    for (int x = 0; x < (int)sizeof(T) / 2; ++x) r.v[x] = load16(reinterpret_cast<const char*>(p) + 16 * x);
    return r;
}
template <typename T>
__device__ __forceinline__ void store_run(T* p, const Run<T>& r) {
#pragma unroll
    for (int x = 0; x < (int)sizeof(T) / 2; ++x) store16(reinterpret_cast<char*>(p) + 16 * x, r.v[x]);
}
__device__ __forceinline__ void to_floats(const Run<__bf16>& r, float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(r.v[0][e] << 16);
        f[2 * e + 1] = __uint_as_float(r.v[0][e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void to_floats(const Run<float>& r, float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(r.v[e >> 2][e & 3]);
}
__device__ __forceinline__ Run<__bf16> to_run(const float (&f)[8], __bf16) {         // rounded once, to nearest
    Run<__bf16> r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[0][e] = pack_bf16x2(f[2 * e], f[2 * e + 1]);
    return r;
}
__device__ __forceinline__ Run<float> to_run(const float (&f)[8], float) {
    Run<float> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e >> 2][e & 3] = __float_as_uint(f[e]);
    return r;
}

// (x, y) -> (x cos - y sin, x sin + y cos) of the eight pairs in two runs
template <typename T>
__device__ __forceinline__ void turn_runs(Run<T>& ra, Run<T>& rb, const Angles& at, int neighbours) {
    float a[8], b[8], x[8], y[8];
    to_floats(ra, a);
    to_floats(rb, b);
    if (neighbours) {
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = a[2 * e]; y[e] = a[2 * e + 1]; x[e + 4] = b[2 * e]; y[e + 4] = b[2 * e + 1]; }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] = a[e]; y[e] = b[e]; }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float s = x[e], t = y[e];
        x[e] = fmaf(s, at.cs[e], -t * at.sn[e]);
        y[e] = fmaf(s, at.sn[e], t * at.cs[e]);
    }
    if (neighbours) {
#pragma unroll
        for (int e = 0; e < 4; ++e) { a[2 * e] = x[e]; a[2 * e + 1] = y[e]; b[2 * e] = x[e + 4]; b[2 * e + 1] = y[e + 4]; }
        ra = to_run(a, T());
        rb = to_run(b, T());
    } else {
        ra = to_run(x, T());
        rb = to_run(y, T());
    }
}

}  // namespace zipvl
