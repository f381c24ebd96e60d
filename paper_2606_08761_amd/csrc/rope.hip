// Rotary positions of rows: queries, or queries and keys of one projection, in
// place or into another buffer.
//
// A workgroup takes up to 8 tokens: its threads work out the (cos, sin) of all the
// pairs once, into LDS, and then go through the tokens' heads, a lane with 16 values
// (two loads of 16 bytes) at a time and four of those in flight, so that the sines
// are shared by all heads of a token.  A lane holds both values of each of its
// pairs before it writes either, which is what lets a row be turned in place.
// Bound by memory (4 bytes a value moved, 3 operations): 8192 tokens of 72 heads of 128 take 63
// us (302 MB, 4.8 TB/s), 4001 of 40 heads of 64, interleaved, 9.3 (41 MB, 4.4 TB/s), 16
// tokens of 72 heads 3.8, the launch and one chain of loads.  Value by value (kSingles: 2
// bytes a load, two divisions a pair) 8192 tokens of 72 heads of 128 take 199 us with 120 of them turned
// and 259 with 24, of 72 with all turned 78.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "apex4_internal.h"
#include "rope_core.h"

namespace apex4 {
namespace {

using namespace rope;

constexpr int kThreads = 256, kMost = 8, kMostPairs = 256;  // tokens of a workgroup, pairs of a head

// LANES: lanes of a head (D / 16) where it is known, or 0.
template <int FORM, int LANES>
__global__ __launch_bounds__(kThreads) void rope_kernel(const uint16_t* x, int64_t x_stride, const int32_t* __restrict__ positions,
                                                        int64_t T, int heads, int D, Rotary r, uint16_t* out, int64_t out_stride,
                                                        int per) {
    __shared__ Turn turns[kMost * kMostPairs];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * per;
    const int tokens = static_cast<int>(T - i0 < per ? T - i0 : per);
    const int pairs = r.rot / 2;
    for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) turns[i] = turn_of(r, positions[i0 + i / pairs], i % pairs);
    __syncthreads();
    if constexpr (FORM == kSingles) {
        const int units = pairs + D - r.rot;  // pairs, and the values that stay
        const int n = tokens * heads * units;
        for (int s = threadIdx.x; s < n; s += kThreads) {
            const int row = s / units, u = s - row * units, t = row / heads;
            const uint16_t* from = x + (i0 + t) * x_stride + (row - t * heads) * D;
            uint16_t* to = out + (i0 + t) * out_stride + (row - t * heads) * D;
            if (u >= pairs) {
                to[r.rot + u - pairs] = from[r.rot + u - pairs];
                continue;
            }
            const int ea = r.interleaved ? 2 * u : u, eb = r.interleaved ? 2 * u + 1 : u + pairs;
            const float a = h2f(from[ea]), b = h2f(from[eb]);
            const Turn c = turns[t * pairs + u];
            to[ea] = __half_as_ushort(__float2half_rn(first_of(a, b, c)));
            to[eb] = __half_as_ushort(__float2half_rn(second_of(a, b, c)));
        }
    } else {
        constexpr int U = 4;
        const int lanes = LANES ? LANES : D / 16;
        const int step = kThreads / lanes;  // rows of a round; threads past whole rows stay idle
        const int l = threadIdx.x % lanes, first = threadIdx.x / lanes;
        if (first >= step) return;
        const int2 at = pieces_of<FORM>(r, l);
        const int rows = tokens * heads;
        for (int row0 = first; row0 < rows; row0 += U * step) {
            u32x4 a[U], b[U];
            int tok[U], head[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int row = row0 + u * step;
                tok[u] = row / heads;
                head[u] = row - tok[u] * heads;
                if (row < rows) {
                    const uint16_t* from = x + (i0 + tok[u]) * x_stride + head[u] * D;
                    a[u] = *reinterpret_cast<const u32x4*>(from + 8 * at.x);
                    b[u] = *reinterpret_cast<const u32x4*>(from + 8 * at.y);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (row0 + u * step < rows) {
                    turn_pieces<FORM>(r, l, turns + tok[u] * pairs, a[u], b[u]);
                    uint16_t* to = out + (i0 + tok[u]) * out_stride + head[u] * D;
                    *reinterpret_cast<u32x4*>(to + 8 * at.x) = a[u];
                    *reinterpret_cast<u32x4*>(to + 8 * at.y) = b[u];
                }
            }
        }
    }
}

}  // namespace

hipError_t launch_rope(const uint16_t* x, int64_t x_stride, const int32_t* positions, int64_t T, int heads, int D, const Rotary& r,
                       uint16_t* out, int64_t out_stride, hipStream_t stream) {
    // tokens of a workgroup: one while that leaves the compute units with few workgroups each
    const int64_t n = T / (4 * device_cu_count());
    const int per = static_cast<int>(n < 1 ? 1 : n < kMost ? n : kMost);
    const dim3 grid(static_cast<unsigned>((T + per - 1) / per));
    auto run = [&](auto kernel) { kernel<<<grid, kThreads, 0, stream>>>(x, x_stride, positions, T, heads, D, r, out, out_stride, per); };
    switch (form_of(r, D)) {
        case kHalves: D == 128 ? run(rope_kernel<kHalves, 8>) : D == 64 ? run(rope_kernel<kHalves, 4>) : run(rope_kernel<kHalves, 0>); break;
        case kNeighbours:
            D == 128 ? run(rope_kernel<kNeighbours, 8>) : D == 64 ? run(rope_kernel<kNeighbours, 4>) : run(rope_kernel<kNeighbours, 0>);
            break;
        default: run(rope_kernel<kSingles, 0>);
    }
    return hipGetLastError();
}

}  // namespace apex4
