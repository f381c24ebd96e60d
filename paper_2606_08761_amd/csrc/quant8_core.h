// 8-bit codes of a token: the arithmetic that the quantizer and the linear that
// quantizes on its way share, so that both give the same bits (described at the top of
// quant_act8.hip).
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "quant_core.h"

namespace apex4 {
namespace quant8 {
namespace {   // internal linkage in every translation unit that includes it

using quant::h2f;
using quant::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

struct Scale {
    float s, inv;  // inv is zero where no code can be other than zero
};

__device__ __forceinline__ Scale scale_of(uint32_t amax_bits) {
    Scale c;
    c.s = h2f(amax_bits) / 127.0f;
    const bool some = c.s > 0.f && amax_bits < 0x7C00u;
    c.inv = some ? __builtin_amdgcn_rcpf(c.s) : 0.f;
    return c;
}

__device__ __forceinline__ int code_of(float x, const Scale& c) {
    float q = rintf(x * c.inv);
    const float d = fmaf(-q, c.s, x), half = 0.5f * c.s;
    const bool odd = static_cast<int>(q) & 1;
    if (fabsf(d) > half || (fabsf(d) == half && odd)) q += d > 0.f ? 1.f : -1.f;
    return static_cast<int>(__builtin_amdgcn_fmed3f(q, -127.f, 127.f));
}

// Nearly always no quotient of the wave's is next to a border, and rint(x inv) is the code:
// RARE looks once for all eight (4096 rows of 8192: 21.9 -> 18.4 us).
template <bool RARE>
__device__ __forceinline__ u32x2 codes8(u32x4 v, const Scale& c) {
    u32x2 out = {0u, 0u};
    if (c.inv == 0.f) return out;
    auto all = [&](auto code) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = v[2 * i + (j >> 1)];
                b[j] = static_cast<uint32_t>(code(h2f(j & 1 ? w >> 16 : w & 0xFFFFu)));
            }
            out[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u),
                                           0x05040100u);
        }
    };
    if constexpr (RARE) {
        float most = 0.f;
        all([&](float x) {
            const float q = rintf(x * c.inv);  // +-127 at most
            most = fmaxf(most, fabsf(fmaf(-q, c.s, x)));
            return static_cast<int>(q);
        });
        if (!__any(most >= 0.5f * c.s)) return out;
    }
    all([&](float x) { return code_of(x, c); });
    return out;
}

// An output from its exact sum: binary32 products, rounded once more to binary16.  The
// empty statement keeps the compiler from one instruction that rounds both at once in
// some kernels and not in others: every kernel gives the same bits.
__device__ __forceinline__ uint32_t result(int sum, float s_token, float s_channel) {
    float y = static_cast<float>(sum) * s_token * s_channel;
    asm("" : "+v"(y));
    return __half_as_ushort(__float2half_rn(y));
}

}  // namespace
}  // namespace quant8
}  // namespace apex4
