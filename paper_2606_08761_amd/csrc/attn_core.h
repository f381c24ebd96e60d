// What the attention kernels over the paged cache share: the tiles of positions
// a range of rows sees, and the arithmetic of the 4-bit codes.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4_internal.h"
#include "kv_cache.h"

namespace apex4 {
namespace attn {
namespace {   // internal linkage in every translation unit that includes it

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
// A running maximum that no finite score is below, and that leaves 2^(s - m)
// zero, not NaN, where every score so far is masked (s = -inf).
constexpr float kNoMax = -1e30f;
// The weights of prefill, whose sums run over a whole length, are scaled by 2^kHeadroom
// when the running maximum is raised, and it is raised again where one passes it by kSlack
// more (in units of log2), just inside binary16's range: after the first tiles a rescale is
// rare (a slack of 8 takes 5 % more time under a window over codes).  Binary16 holds
// the weights to 2^-31 of the largest one, so that a long tail of small weights, rounded
// the same way each, keeps its share (without the headroom 40000 of 2^-25 vanished:
// 1.2e-3 of the result).
constexpr float kHeadroom = 6.f;
constexpr float kSlack = 9.875f;
// Decoding, at most 512 positions a wave: weights below 2^8.
constexpr float kMostWeight = 256.f;
constexpr float kMostSum = 0x1p60f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two weights rounded to binary16 (nearest even), the operand of the second product:
// 2^-11 of a weight at most, which in a sum of many stays about as large as the
// output's own rounding (2.3e-4 to 2.8e-4 of the result against 64 bits, where 32-bit
// weights have 2.0e-4 to 2.1e-4).
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    f16x2 r;
    r[0] = static_cast<_Float16>(a);
    r[1] = static_cast<_Float16>(b);
    return __builtin_bit_cast(uint32_t, r);
}

// Workgroups of a launch: HIP takes less than 2^32 threads along a grid's first
// dimension, so more than 2^22 workgroups (of up to 512 threads) take two.  What is past the
// last one has to return.
inline dim3 grid_of(int64_t blocks) {
    constexpr int64_t kRow = 1 << 22;
    return blocks <= kRow ? dim3(static_cast<unsigned>(blocks))
                          : dim3(static_cast<unsigned>(kRow), static_cast<unsigned>((blocks + kRow - 1) / kRow));
}
__device__ __forceinline__ uint32_t workgroup_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

// New tokens of sequence b of the packed ones: those of rows q_start[b] .. that are
// among the T, none where the start is not.  (So that no row number overflows.)
__device__ __forceinline__ int new_tokens(const AttnArgs& a, int b) {
    const int64_t first = a.q_start[b], n = a.q_start[b + 1] - first, left = a.T - first;
    return static_cast<int>(first < 0 || n < 0 || left < 0 ? 0 : n < left ? n : left);
}

// Tiles of W positions that rows at positions p_lo .. p_hi see (causal, a
// window of `window` positions up to the row's own unless it is 0, and the
// first `sinks`): the tiles of the first positions, then from the window's
// start on, as one list of `count` tiles.
template <int W>
struct Tiles {
    int lo;        // first position the window of the lowest row reaches
    int sinks;     // first positions visible besides
    int n_sink;    // tiles of the list before the window's
    int first;     // tile of the window's start
    int count;
    __device__ __forceinline__ Tiles(int p_lo, int p_hi, int window, int sinks_all) {
        lo = window ? p_lo - window + 1 : 0;
        lo = lo > 0 ? lo : 0;
        sinks = sinks_all < lo ? sinks_all : lo;
        first = lo / W;
        n_sink = (sinks + W - 1) / W;
        n_sink = n_sink < first ? n_sink : first;
        count = p_hi < 0 ? 0 : n_sink + p_hi / W + 1 - first;
    }
    // position of the first token of tile i of the list
    __device__ __forceinline__ int start(int i) const { return (i < n_sink ? i : first + i - n_sink) * W; }
};

// 4-bit codes as binary16 without a conversion.  A two's complement nibble with
// its top bit flipped is code + 8; in bits 0-3 of a half under the exponent of
// 1024 it stands for 1032 + code, in bits 4-7 for 1152 + 16 code, or, under the
// exponent of 64, for 72 + code.  One masked exclusive or sets the exponent and
// flips the bit.  The mask is kept in a vector register: an instruction takes one
// scalar constant.
__device__ __forceinline__ uint32_t masked_xor(uint32_t x, uint32_t mask, uint32_t flip) {
    asm("" : "+v"(mask));
    return (x & mask) ^ flip;
}

// 8 codes, exact: the halves of r[i] are codes i and i + 4.
__device__ __forceinline__ void codes_f16(uint32_t x, uint32_t r[4]) {
    const uint32_t y = x >> 8;
    const uint32_t a[4] = {masked_xor(x, 0x000F000Fu, 0x64086408u), masked_xor(x, 0x00F000F0u, 0x64806480u),
                           masked_xor(y, 0x000F000Fu, 0x64086408u), masked_xor(y, 0x00F000F0u, 0x64806480u)};
    const f16x2 one = {static_cast<_Float16>(1032.f), static_cast<_Float16>(1032.f)};
    const f16x2 six = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
    const f16x2 off = {static_cast<_Float16>(-72.f), static_cast<_Float16>(-72.f)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f16x2 h = __builtin_bit_cast(f16x2, a[i]);
        r[i] = __builtin_bit_cast(uint32_t, (i & 1) ? __builtin_elementwise_fma(h, six, off) : h - one);
    }
}

// code + 72, in the same order and without the subtraction, for a product that
// starts at -72 times the other side's sum (its 32-bit sums lose log2(72) bits
// to the offset: fine for 128 products, not for a sum over all positions).
__device__ __forceinline__ u32x4 codes_bias72(uint32_t x) {
    return u32x4{masked_xor(x << 4, 0x00F000F0u, 0x54805480u), masked_xor(x, 0x00F000F0u, 0x54805480u),
                 masked_xor(x >> 4, 0x00F000F0u, 0x54805480u), masked_xor(x >> 8, 0x00F000F0u, 0x54805480u)};
}

__device__ __forceinline__ float half_of(uint32_t w, int high) {
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    return static_cast<float>(high ? h[1] : h[0]);
}

// y times a half of w (one instruction takes the binary16 operand as it is).
__device__ __forceinline__ float times_half(float y, uint32_t w, int high) { return fmaf(half_of(w, high), y, 0.f); }

// l + both halves of w.
__device__ __forceinline__ float add_pair(uint32_t w, float l) {
    const f16x2 one = {static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)};
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), one, l, false);
}

// 8 binary16 values in the order codes_f16 leaves codes in.
__device__ __forceinline__ u32x4 code_order(u32x4 w) {
    u32x4 r;
    r[0] = __builtin_amdgcn_perm(w[2], w[0], 0x05040100u);
    r[1] = __builtin_amdgcn_perm(w[2], w[0], 0x07060302u);
    r[2] = __builtin_amdgcn_perm(w[3], w[1], 0x05040100u);
    r[3] = __builtin_amdgcn_perm(w[3], w[1], 0x07060302u);
    return r;
}

// The low, or high, halves of two words side by side.
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

}  // namespace
}  // namespace attn
}  // namespace apex4
