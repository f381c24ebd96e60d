// New tokens' keys and values into a paged cache, and back out of it.
//
// One lane moves 8 values (16 bytes of binary16) of one (token, head); blockIdx.y
// picks keys or values.  Into an int4 cache the D / 8 lanes of a head's row
// quantize it on the way (SymQuant with G = D, the codes and scales of
// quant_core.h bit for bit), so the values are read once and a quarter of them
// written.  Bound by the bytes moved, by the launch for a decode step's few
// tokens.  The sequence of a token is a search in q_start, log2(B) loads that
// the caches serve.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "apex4_internal.h"
#include "kv_cache.h"
#include "quant_core.h"

namespace apex4 {
namespace {

using namespace quant;

// Where (token i of the new ones, head h) lies: byte offset of its row in a
// plane, and of its scale.  False where it has no place: before the sequence's
// start, past its table, or on no page.
template <int D, bool I4>
__device__ __forceinline__ bool place(const KvView& c, const int32_t* q_start, int64_t T, int i, int h, int64_t* row,
                                      int64_t* scale) {
    const int b = sequence_of(q_start, c.B, i);
    const int64_t end = q_start ? q_start[b + 1] : i + 1;
    const int64_t pos = c.kv_len[b] - end + i;
    if (pos < 0 || i >= end) return false;
    const int id = page_of(c, b, pos);
    if (id < 0) return false;
    const int page = 1 << c.page_shift, at = static_cast<int>(pos) & (page - 1);
    const int64_t base = id * c.page_bytes;
    const int64_t r = static_cast<int64_t>(h) * page + at;
    *row = base + r * (I4 ? D / 2 : 2 * D);
    *scale = base + static_cast<int64_t>(c.kv_heads) * page * (D / 2) + 2 * r;
    return true;
}

template <int D, bool I4>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView c, const uint16_t* __restrict__ k, int64_t k_stride,
                                                        const uint16_t* __restrict__ v, int64_t v_stride,
                                                        const int32_t* __restrict__ q_start, int64_t T) {
    constexpr int L = D / 8;
    const int64_t slot = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int lane = static_cast<int>(slot & (L - 1));
    const int64_t r = slot / L;
    if (r >= T * c.kv_heads) return;  // whole rows of lanes leave together
    const int i = static_cast<int>(static_cast<uint32_t>(r) / static_cast<uint32_t>(c.kv_heads));
    const int h = static_cast<int>(r) - i * c.kv_heads;
    const uint16_t* src = (blockIdx.y ? v + i * v_stride : k + i * k_stride) + h * D + lane * 8;
    uint8_t* plane = const_cast<uint8_t*>(blockIdx.y ? c.v : c.k);
    const u32x4 t = *reinterpret_cast<const u32x4*>(src);
    int64_t row, scale;
    const bool ok = place<D, I4>(c, q_start, T, i, h, &row, &scale);
    if constexpr (I4) {
        const uint4 x = make_uint4(t[0], t[1], t[2], t[3]);
        uint16_t bits;
        const float s = scale_of(group_max<L>(absmax8_bits(x)), &bits);
        const uint32_t codes = pack8(x, s, inv_of(s));
        if (ok) {
            *reinterpret_cast<uint32_t*>(plane + row + lane * 4) = codes;
            if (lane == 0) *reinterpret_cast<uint16_t*>(plane + scale) = bits;
        }
    } else {
        if (ok) *reinterpret_cast<u32x4*>(plane + row + lane * 16) = t;
    }
}

// Tokens without a place come back as zeros.
template <int D, bool I4>
__global__ __launch_bounds__(256) void kv_gather_kernel(KvView c, uint16_t* __restrict__ k, uint16_t* __restrict__ v,
                                                        const int32_t* __restrict__ q_start, int64_t T) {
    constexpr int L = D / 8;
    const int64_t slot = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int lane = static_cast<int>(slot & (L - 1));
    const int64_t r = slot / L;
    if (r >= T * c.kv_heads) return;
    const int i = static_cast<int>(static_cast<uint32_t>(r) / static_cast<uint32_t>(c.kv_heads));
    const int h = static_cast<int>(r) - i * c.kv_heads;
    const uint8_t* plane = blockIdx.y ? c.v : c.k;
    u32x4 t = {0u, 0u, 0u, 0u};
    int64_t row, scale;
    if (place<D, I4>(c, q_start, T, i, h, &row, &scale)) {
        if constexpr (I4) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(plane + row + lane * 4);
            const float s = h2f(*reinterpret_cast<const uint16_t*>(plane + scale));
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // one rounding: the product has 15 bits at most
                const float lo = static_cast<float>(static_cast<int32_t>(w << (28 - 8 * j)) >> 28) * s;
                const float hi = static_cast<float>(static_cast<int32_t>(w << (24 - 8 * j)) >> 28) * s;
                t[j] = __half_as_ushort(__float2half_rn(lo)) | static_cast<uint32_t>(__half_as_ushort(__float2half_rn(hi))) << 16;
            }
        } else {
            t = *reinterpret_cast<const u32x4*>(plane + row + lane * 16);
        }
    }
    *reinterpret_cast<u32x4*>((blockIdx.y ? v : k) + r * D + lane * 8) = t;
}

dim3 grid_of(const KvView& c, int64_t T) {
    return dim3(static_cast<unsigned>((T * c.kv_heads * (c.D / 8) + 255) / 256), 2);
}

}  // namespace

hipError_t launch_kv_append(const KvView& c, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                            const int32_t* q_start, int64_t T, hipStream_t stream) {
    const dim3 g = grid_of(c, T);
    auto run = [&](auto kernel) { kernel<<<g, 256, 0, stream>>>(c, k, k_stride, v, v_stride, q_start, T); };
    if (c.D == 128) c.i4 ? run(kv_append_kernel<128, true>) : run(kv_append_kernel<128, false>);
    else c.i4 ? run(kv_append_kernel<64, true>) : run(kv_append_kernel<64, false>);
    return hipGetLastError();
}

hipError_t launch_kv_gather(const KvView& c, uint16_t* k, uint16_t* v, const int32_t* q_start, int64_t T,
                            hipStream_t stream) {
    const dim3 g = grid_of(c, T);
    auto run = [&](auto kernel) { kernel<<<g, 256, 0, stream>>>(c, k, v, q_start, T); };
    if (c.D == 128) c.i4 ? run(kv_gather_kernel<128, true>) : run(kv_gather_kernel<128, false>);
    else c.i4 ? run(kv_gather_kernel<64, true>) : run(kv_gather_kernel<64, false>);
    return hipGetLastError();
}

}  // namespace apex4
