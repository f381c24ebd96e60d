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
//
// With rotary positions on the way (kv_append_rope_kernel) a lane moves the 16 values
// of one (token, head) that hold both of every pair, and blockIdx.y 0 turns the queries
// into a buffer of their own: one launch for what stands between a layer's projection
// and its attention.
// 64 query and 8 key heads of 128: 16 tokens 4.3 us; five prompts of up to 4001 tokens
// into an int4 cache 75 us (8958 tokens, 340 MB at 4.5 TB/s; the queries, nine tenths of it,
// first: 80 us with them last), into a binary16 one 77 (367 MB, 4.7 TB/s; 81 with
// neighbouring pairs).  Value by value (kSingles: a pair is worked out for each of its two values)
// the latter takes 247 us with 120 of 128 turned and 284 with 24.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <type_traits>

#include "apex4_internal.h"
#include "kv_cache.h"
#include "quant_core.h"
#include "rope_core.h"

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

// The place of new token i, its position, and whether it is a sequence's.
struct Spot {
    Place place;
    int pos;
    bool live;
};
__device__ __forceinline__ Spot spot_of(const KvView& c, const int32_t* q_start, int64_t T, int64_t i) {
    Spot s = {{-1, 0}, 0, false};
    if (i >= T) return s;
    const int b = sequence_of(q_start, c.B, static_cast<int>(i));
    const int64_t end = q_start ? q_start[b + 1] : i + 1;
    if (i >= end) return s;
    const int64_t pos = c.kv_len[b] - end + i;
    s.pos = static_cast<int>(pos);
    s.live = true;
    if (pos < 0) return s;
    s.place.page = page_of(c, b, pos);
    s.place.at = static_cast<int>(pos) & ((1 << c.page_shift) - 1);
    return s;
}

// blockIdx.y: 0 queries (into rows of their own; the longest first), 1 keys, 2 values (not
// turned); without queries 1 and 2 are 0 and 1.  A
// key is turned and rounded to binary16 before it is stored or quantized: what the
// two calls, one after the other, would give, bit for bit.
template <int D, bool I4, int FORM>
__global__ __launch_bounds__(kThreads) void kv_append_rope_kernel(KvView c, RopeRows a, const int32_t* __restrict__ q_start,
                                                                  int64_t T, Rotary r, int per) {
    constexpr int L = D / 16, U = 4;
    __shared__ Spot spots[kMost];
    __shared__ rope::Turn turns[kMost * D / 2];
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * per;
    const int tokens = static_cast<int>(T - i0 < per ? T - i0 : per);
    const int what = static_cast<int>(blockIdx.y) + (a.heads ? 0 : 1);
    const bool turned = what != 2, cached = what != 0;
    const int heads = cached ? c.kv_heads : a.heads, pairs = r.rot / 2;
    const uint16_t* src = what == 0 ? a.q : what == 1 ? a.k : a.v;
    const int64_t stride = what == 0 ? a.q_stride : what == 1 ? a.k_stride : a.v_stride;
    uint8_t* plane = const_cast<uint8_t*>(what == 2 ? c.v : c.k);
    if (static_cast<int>(threadIdx.x) < tokens) spots[threadIdx.x] = spot_of(c, q_start, T, i0 + threadIdx.x);
    __syncthreads();
    if (turned) {
        for (int i = threadIdx.x; i < tokens * pairs; i += kThreads) {
            const int t = i / pairs;
            turns[i] = rope::turn_of(r, a.positions ? a.positions[i0 + t] : spots[t].pos, i - t * pairs);
        }
        __syncthreads();
    }
    const int l = threadIdx.x % L, rows = tokens * heads;
    const int2 at = FORM == rope::kSingles ? make_int2(2 * l, 2 * l + 1) : rope::pieces_of<FORM>(r, l);
    for (int row0 = threadIdx.x / L; row0 < rows; row0 += U * (kThreads / L)) {  // whole rows of lanes
        u32x4 x[U], y[U];
        int tok[U], head[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * (kThreads / L);
            tok[u] = row / heads;
            head[u] = row - tok[u] * heads;
            if (row < rows) {
                const uint16_t* from = src + (i0 + tok[u]) * stride + head[u] * D;
                if (FORM == rope::kSingles && turned) {
                    x[u] = rope::turned_piece(r, from, at.x, turns + tok[u] * pairs);
                    y[u] = rope::turned_piece(r, from, at.y, turns + tok[u] * pairs);
                } else {
                    x[u] = *reinterpret_cast<const u32x4*>(from + 8 * at.x);
                    y[u] = *reinterpret_cast<const u32x4*>(from + 8 * at.y);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row0 + u * (kThreads / L) >= rows) break;
            if constexpr (FORM != rope::kSingles)
                if (turned) rope::turn_pieces<FORM>(r, l, turns + tok[u] * pairs, x[u], y[u]);
            const Spot& s = spots[tok[u]];
            if (!cached) {
                uint16_t* to = a.q_out + ((i0 + tok[u]) * heads + head[u]) * D;
                if (s.live) {
                    *reinterpret_cast<u32x4*>(to + 8 * at.x) = x[u];
                    *reinterpret_cast<u32x4*>(to + 8 * at.y) = y[u];
                }
            } else if constexpr (I4) {
                const uint4 p = make_uint4(x[u][0], x[u][1], x[u][2], x[u][3]), q = make_uint4(y[u][0], y[u][1], y[u][2], y[u][3]);
                const uint32_t mp = absmax8_bits(p), mq = absmax8_bits(q);
                uint16_t bits;
                const float sc = scale_of(group_max<L>(mp > mq ? mp : mq), &bits);
                const uint32_t cp = pack8(p, sc, inv_of(sc)), cq = pack8(q, sc, inv_of(sc));
                if (s.place.page >= 0) {
                    uint8_t* to = plane + row_at<D, true>(c, s.place, head[u]);
                    *reinterpret_cast<uint32_t*>(to + 4 * at.x) = cp;
                    *reinterpret_cast<uint32_t*>(to + 4 * at.y) = cq;
                    if (l == 0) *reinterpret_cast<uint16_t*>(plane + scale_at<D>(c, s.place, head[u])) = bits;
                }
            } else if (s.place.page >= 0) {
                uint8_t* to = plane + row_at<D, false>(c, s.place, head[u]);
                *reinterpret_cast<u32x4*>(to + 16 * at.x) = x[u];
                *reinterpret_cast<u32x4*>(to + 16 * at.y) = y[u];
            }
        }
    }
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

hipError_t launch_kv_append_rope(const KvView& c, const RopeRows& a, const int32_t* q_start, int64_t T, const Rotary& r,
                                 hipStream_t stream) {
    const int per = tokens_per_group(T);
    dim3 grid = grid_of(T, per);
    grid.y = a.heads ? 3 : 2;
    auto run = [&](auto kernel) { kernel<<<grid, kThreads, 0, stream>>>(c, a, q_start, T, r, per); };
    auto form = [&](auto d, auto i4) {
        constexpr int D = decltype(d)::value;
        constexpr bool I4 = decltype(i4)::value;
        switch (rope::form_of(r, D)) {
            case rope::kHalves: run(kv_append_rope_kernel<D, I4, rope::kHalves>); break;
            case rope::kNeighbours: run(kv_append_rope_kernel<D, I4, rope::kNeighbours>); break;
            default: run(kv_append_rope_kernel<D, I4, rope::kSingles>);
        }
    };
    using std::integral_constant;
    using std::bool_constant;
    if (c.D == 128) c.i4 ? form(integral_constant<int, 128>(), bool_constant<true>()) : form(integral_constant<int, 128>(), bool_constant<false>());
    else c.i4 ? form(integral_constant<int, 64>(), bool_constant<true>()) : form(integral_constant<int, 64>(), bool_constant<false>());
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
