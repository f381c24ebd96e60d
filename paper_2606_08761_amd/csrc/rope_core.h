// Rotary positions: what the kernels that turn rows share.
//
// Pair j < rot / 2 of a token at position p turns by p freq[j] whole turns:
//   (a, b) -> mag (a cos - b sin, b cos + a sin);
// the pair is (j, j + rot / 2) in the half layout and (2 j, 2 j + 1) in the
// interleaved one, and the values from rot on stay.  A position of any sign and size
// has its angle: the turns are a binary64 product, and only what is left past whole
// turns (exact) goes into the sine.  (In binary32 the angle of position 10^6 would be off
// by 2^-5 of a radian.)
//
// Roundings: cos and sin times mag (binary64) to binary32; each product and their sum to
// binary32, which is what elementary operations in that type give, bit for bit; then to
// binary16.  No fma, which drops one of the products' roundings: a value in ten thousand
// would be another, and a 4-bit code on the way into a cache is decided by such values.  The
// result is 2^-11 of itself and 2^-22 of |a| + |b| off at most.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4_internal.h"
#include "quant_core.h"

namespace apex4 {
namespace rope {
namespace {   // internal linkage in every translation unit that includes it

using quant::h2f;
using quant::u32x4;

// How a head's values go to lanes.  Both but kSingles: D / 16 lanes a head, each
// with two pieces of 8 values.
enum Form : int {
    kHalves = 0,      // half layout, rot % 16 == 0, D % 16 == 0: a lane's two pieces are pairs of each other
    kNeighbours = 1,  // interleaved, rot % 8 == 0, D % 16 == 0: pairs lie inside a piece
    kSingles = 2,     // any other even rot: value by value
};
__host__ __device__ inline int form_of(const Rotary& r, int D) {
    if (D % 16 != 0) return kSingles;
    if (r.interleaved) return r.rot % 8 == 0 ? kNeighbours : kSingles;
    return r.rot % 16 == 0 ? kHalves : kSingles;
}

// (cos, sin) of pair j at position p, times mag.
typedef float Turn __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Turn turn_of(const Rotary& r, int p, int j) {
    const double t = static_cast<double>(p) * r.freq[j];
    double s, c;
    sincospi(2.0 * (t - rint(t)), &s, &c);
    return Turn{static_cast<float>(c * r.mag), static_cast<float>(s * r.mag)};
}

// The compiler may join a product and the sum, or the sum and its rounding to binary16,
// into one instruction that rounds once; the empty statement keeps them apart.
__device__ __forceinline__ float apart(float x) {
    asm("" : "+v"(x));
    return x;
}
__device__ __forceinline__ float first_of(float a, float b, Turn t) { return apart(apart(a * t.x) - apart(b * t.y)); }
__device__ __forceinline__ float second_of(float a, float b, Turn t) { return apart(apart(b * t.x) + apart(a * t.y)); }

// The pieces (of 8 values) of lane l of a head.
template <int FORM>
__device__ __forceinline__ int2 pieces_of(const Rotary& r, int l) {
    if (FORM == kHalves && l < r.rot / 16) return make_int2(l, l + r.rot / 16);
    return make_int2(2 * l, 2 * l + 1);
}

__device__ __forceinline__ float low(uint32_t w) { return h2f(w & 0xFFFFu); }
__device__ __forceinline__ float high(uint32_t w) { return h2f(w >> 16); }
__device__ __forceinline__ uint32_t both(float a, float b) {
    return __half_as_ushort(__float2half_rn(a)) | static_cast<uint32_t>(__half_as_ushort(__float2half_rn(b))) << 16;
}

// Turns lane l's two pieces; turns: the token's rot / 2 (cos, sin).
template <int FORM>
__device__ __forceinline__ void turn_pieces(const Rotary& r, int l, const Turn* turns, u32x4& x, u32x4& y) {
    if constexpr (FORM == kHalves) {
        if (l >= r.rot / 16) return;
        const Turn* t = turns + 8 * l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a0 = low(x[i]), a1 = high(x[i]), b0 = low(y[i]), b1 = high(y[i]);
            const Turn t0 = t[2 * i], t1 = t[2 * i + 1];
            x[i] = both(first_of(a0, b0, t0), first_of(a1, b1, t1));
            y[i] = both(second_of(a0, b0, t0), second_of(a1, b1, t1));
        }
    } else {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (8 * (2 * l + n) >= r.rot) break;
            u32x4& z = n ? y : x;
            const Turn* t = turns + 4 * (2 * l + n);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = both(first_of(low(z[i]), high(z[i]), t[i]), second_of(low(z[i]), high(z[i]), t[i]));
        }
    }
}

// Value e of a head's row (kSingles).
__device__ __forceinline__ uint32_t turned_value(const Rotary& r, const uint16_t* row, int e, const Turn* turns) {
    if (e >= r.rot) return row[e];
    const int half = r.rot / 2;
    const bool second = r.interleaved ? e & 1 : e >= half;
    const int j = r.interleaved ? e >> 1 : second ? e - half : e;
    const float a = h2f(row[r.interleaved ? e & ~1 : j]), b = h2f(row[r.interleaved ? e | 1 : j + half]);
    return __half_as_ushort(__float2half_rn(second ? second_of(a, b, turns[j]) : first_of(a, b, turns[j])));
}
__device__ __forceinline__ u32x4 turned_piece(const Rotary& r, const uint16_t* row, int piece, const Turn* turns) {
    u32x4 z;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        z[i] = turned_value(r, row, 8 * piece + 2 * i, turns) | turned_value(r, row, 8 * piece + 2 * i + 1, turns) << 16;
    return z;
}

}  // namespace
}  // namespace rope
}  // namespace apex4
