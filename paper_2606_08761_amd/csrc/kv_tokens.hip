// New tokens' keys and values into a paged cache, and back out of it.
//
// One lane moves 8 values (16 bytes of binary16) of one (token, head) at a time,
// four in flight; blockIdx.y picks keys or values.  Into an int4 cache the D / 8 lanes
// of a head's row quantize it on the way (SymQuant with G = D, the codes and
// scales of quant_core.h bit for bit), so the values are read once and a quarter of
// them written.  A workgroup looks its tokens' places up first, a thread each (the
// sequence is a search in q_start): that chain of loads, not the bytes, bounds a
// workgroup of few tokens, and long prompts take 8 tokens a workgroup.
//
// Measured, 8 heads of 128: 16 tokens 2.8 us either way (a launch and that chain);
// ragged prompts, 8958 tokens, into an int4 cache 14.4 us (37 MB read, 10 written: 3.2
// TB/s, with the vector units 0.42 busy: neither is full, the chain comes before the
// bytes), back 12.8 us (3.8 TB/s); binary16 there and back 30.4 us (4.8 TB/s).
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "apex4_internal.h"
#include "kv_cache.h"
#include "quant_core.h"

namespace apex4 {
namespace {

using namespace quant;

constexpr int kMost = 8;    // tokens of a workgroup
constexpr int kThreads = 256;

// Where a token lies in a plane: its page, and its place in it; page -1 where it
// has none: before the sequence's start, past its table, or on no page.
struct Place {
    int page, at;
};
__device__ __forceinline__ Place place_of(const KvView& c, const int32_t* q_start, int64_t T, int64_t i) {
    Place p = {-1, 0};
    if (i >= T) return p;
    const int b = sequence_of(q_start, c.B, static_cast<int>(i));
    const int64_t end = q_start ? q_start[b + 1] : i + 1;
    const int64_t pos = c.kv_len[b] - end + i;
    if (pos < 0 || i >= end) return p;
    p.page = page_of(c, b, pos);
    p.at = static_cast<int>(pos) & ((1 << c.page_shift) - 1);
    return p;
}

// Runs move(slot's token, head, lane of the row, place) over the workgroup's
// tokens, U at a time: first load() of all, then use().
template <int D, class Load, class Use>
__device__ __forceinline__ void over_slots(const KvView& c, const Place* places, int tokens, Load load, Use use) {
    constexpr int L = D / 8, U = 4;
    const int slots = tokens * c.kv_heads * L;  // whole rows of lanes: L divides the threads
    for (int s0 = threadIdx.x; s0 < slots; s0 += kThreads * U) {
        u32x4 v[U];
        int tok[U], head[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * kThreads;
            if (s < slots) {
                tok[u] = (s / L) / c.kv_heads;
                head[u] = s / L - tok[u] * c.kv_heads;
                v[u] = load(tok[u], head[u], s % L, places[tok[u]]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s0 + u * kThreads < slots) use(v[u], tok[u], head[u], (s0 + u * kThreads) % L, places[tok[u]]);
    }
}

// Byte offsets in a plane of a token's row, and of its scale.
template <int D, bool I4>
__device__ __forceinline__ int64_t row_at(const KvView& c, const Place& p, int head) {
    return p.page * c.page_bytes + ((static_cast<int64_t>(head) << c.page_shift) + p.at) * (I4 ? D / 2 : 2 * D);
}
template <int D>
__device__ __forceinline__ int64_t scale_at(const KvView& c, const Place& p, int head) {
    return p.page * c.page_bytes + (static_cast<int64_t>(c.kv_heads) << c.page_shift) * (D / 2) +
           2 * ((static_cast<int64_t>(head) << c.page_shift) + p.at);
}

template <int D, bool I4>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvView c, const uint16_t* __restrict__ k, int64_t k_stride,
                                                             const uint16_t* __restrict__ v, int64_t v_stride,
                                                             const int32_t* __restrict__ q_start, int64_t T, int per) {
    __shared__ Place places[kMost];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * per;
    const int tokens = static_cast<int>(T - i0 < per ? T - i0 : per);
    const uint16_t* src = blockIdx.y ? v : k;
    const int64_t stride = blockIdx.y ? v_stride : k_stride;
    uint8_t* plane = const_cast<uint8_t*>(blockIdx.y ? c.v : c.k);
    if (static_cast<int>(threadIdx.x) < per) places[threadIdx.x] = place_of(c, q_start, T, i0 + threadIdx.x);
    __syncthreads();
    over_slots<D>(
        c, places, tokens,
        [&](int t, int h, int lane, const Place&) {
            return *reinterpret_cast<const u32x4*>(src + (i0 + t) * stride + h * D + lane * 8);
        },
        [&](u32x4 x, int, int h, int lane, const Place& p) {
            if constexpr (I4) {
                const uint4 y = make_uint4(x[0], x[1], x[2], x[3]);
                uint16_t bits;
                const float s = scale_of(group_max<D / 8>(absmax8_bits(y)), &bits);
                const uint32_t codes = pack8(y, s, inv_of(s));
                if (p.page >= 0) {
                    *reinterpret_cast<uint32_t*>(plane + row_at<D, true>(c, p, h) + lane * 4) = codes;
                    if (lane == 0) *reinterpret_cast<uint16_t*>(plane + scale_at<D>(c, p, h)) = bits;
                }
            } else {
                if (p.page >= 0) *reinterpret_cast<u32x4*>(plane + row_at<D, false>(c, p, h) + lane * 16) = x;
            }
        });
}

// Tokens without a place come back as zeros.
template <int D, bool I4>
__global__ __launch_bounds__(kThreads) void kv_gather_kernel(KvView c, uint16_t* __restrict__ k, uint16_t* __restrict__ v,
                                                             const int32_t* __restrict__ q_start, int64_t T, int per) {
    __shared__ Place places[kMost];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * per;
    const int tokens = static_cast<int>(T - i0 < per ? T - i0 : per);
    const uint8_t* plane = blockIdx.y ? c.v : c.k;
    uint16_t* out = blockIdx.y ? v : k;
    if (static_cast<int>(threadIdx.x) < per) places[threadIdx.x] = place_of(c, q_start, T, i0 + threadIdx.x);
    __syncthreads();
    over_slots<D>(
        c, places, tokens,
        [&](int, int h, int lane, const Place& p) {
            u32x4 x = {0u, 0u, 0u, 0u};
            if (p.page >= 0) {
                if constexpr (I4) {
                    x[0] = *reinterpret_cast<const uint32_t*>(plane + row_at<D, true>(c, p, h) + lane * 4);
                    x[1] = *reinterpret_cast<const uint16_t*>(plane + scale_at<D>(c, p, h));
                } else {
                    x = *reinterpret_cast<const u32x4*>(plane + row_at<D, false>(c, p, h) + lane * 16);
                }
            }
            return x;
        },
        [&](u32x4 x, int t, int h, int lane, const Place&) {
            if constexpr (I4) {
                const uint32_t w = x[0];
                const float s = h2f(x[1]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {  // one rounding: the product has 15 bits at most
                    const float lo = static_cast<float>(static_cast<int32_t>(w << (28 - 8 * j)) >> 28) * s;
                    const float hi = static_cast<float>(static_cast<int32_t>(w << (24 - 8 * j)) >> 28) * s;
                    x[j] = __half_as_ushort(__float2half_rn(lo)) | static_cast<uint32_t>(__half_as_ushort(__float2half_rn(hi))) << 16;
                }
            }
            *reinterpret_cast<u32x4*>(out + ((i0 + t) * c.kv_heads + h) * D + lane * 8) = x;
        });
}

// Tokens of a workgroup: one while that leaves the compute units with few
// workgroups each, then up to kMost.
int tokens_per_group(int64_t T) {
    const int64_t n = T / (4 * device_cu_count());
    return static_cast<int>(n < 1 ? 1 : n < kMost ? n : kMost);
}
dim3 grid_of(int64_t T, int per) { return dim3(static_cast<unsigned>((T + per - 1) / per), 2); }

}  // namespace

hipError_t launch_kv_append(const KvView& c, const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                            const int32_t* q_start, int64_t T, hipStream_t stream) {
    const int per = tokens_per_group(T);
    auto run = [&](auto kernel) { kernel<<<grid_of(T, per), kThreads, 0, stream>>>(c, k, k_stride, v, v_stride, q_start, T, per); };
    if (c.D == 128) c.i4 ? run(kv_append_kernel<128, true>) : run(kv_append_kernel<128, false>);
    else c.i4 ? run(kv_append_kernel<64, true>) : run(kv_append_kernel<64, false>);
    return hipGetLastError();
}

hipError_t launch_kv_gather(const KvView& c, uint16_t* k, uint16_t* v, const int32_t* q_start, int64_t T,
                            hipStream_t stream) {
    const int per = tokens_per_group(T);
    auto run = [&](auto kernel) { kernel<<<grid_of(T, per), kThreads, 0, stream>>>(c, k, v, q_start, T, per); };
    if (c.D == 128) c.i4 ? run(kv_gather_kernel<128, true>) : run(kv_gather_kernel<128, false>);
    else c.i4 ? run(kv_gather_kernel<64, true>) : run(kv_gather_kernel<64, false>);
    return hipGetLastError();
}

}  // namespace apex4
