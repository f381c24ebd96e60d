// Attention of one new token a sequence over the paged cache, its length split
// over workgroups and joined.
//
//   o = sum_t e^(s_t - m) v_t / sum_t e^(s_t - m),  s_t = scale q . k_t, m = max s_t
//
// over the positions t the token sees (all cached ones, or a window and the
// first few).  Every cached byte is read once, for all the query heads that
// share a key head, and nothing is computed that the reading does not hide:
// the kernel is bound by HBM.
//
// A wave takes tiles of 32 positions.  Its matrix products are laid out so that
// no value moves between lanes and none through LDS:
//   S^T = K Q^T  with 16 x 16 x 32 products: the rows of two products are the
//         positions 8 (m / 4) + 4 u + m % 4 (m < 16, u < 2), so that lane group
//         g = lane / 16 ends up with the scores of positions 8 g .. 8 g + 7 of
//         query head lane % 16, the layout the second product wants its right
//         operand in;
//   O^T = V^T P^T: a lane reads D / 16 consecutive values d of the 8 positions
//         of its group and transposes them in registers (half a v_perm a value);
//         product i takes the rows d = D / 16 (lane % 16) + i.  The order of the
//         rows and of the positions inside a product is free.
// The scores' maximum is kept per head, raised only when a score passes it by
// 2^8: the weights are at most 2^8 and in most tiles nothing is rescaled.
// 4-bit codes enter the products as small integers in binary16 (exact); a
// position's two scales multiply its score and its weight in 32 bits, the
// latter over a power of two near the largest scale so far, so that small scales
// do not push the weights out of binary16's range.
//
// Four waves share a range of positions and add their sums through LDS; with
// more than one range a sequence, a second kernel joins the ranges' sums in
// order (the same bits every time).
#include "attn_core.h"

namespace apex4 {
namespace {

using namespace attn;

constexpr int kTile = 32;      // positions a wave takes at a time
constexpr int kWaves = 4;
constexpr int kMaxTiles = 128; // tiles of a range: 4096 positions, 256 pages at most
constexpr int kHeads = 16;     // query heads a workgroup takes

template <int D, bool I4>
__global__ __launch_bounds__(64 * kWaves) void attn_decode_kernel(KvView c, AttnArgs a, int S, int range,
                                                                  int head_tiles, float* __restrict__ part,
                                                                  float* __restrict__ ml) {
    constexpr int DV = D / 16;  // values d of a lane in the second product
    constexpr int KS = D / 32;  // products along d in the first
    constexpr int P = D + 4;    // floats a row of the sums takes in LDS (rows 16 bytes apart in the banks)
    __shared__ int32_t pages[2 * kMaxTiles];
    __shared__ float sum_ml[2][kWaves][kHeads];
    __shared__ __align__(16) float sums[kWaves][kHeads][P];

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
    uint32_t id = blockIdx.x;
    const int split = static_cast<int>(id % S);
    id /= S;
    const int ht = static_cast<int>(id % head_tiles);
    id /= head_tiles;
    const int h = static_cast<int>(id % c.kv_heads);
    const int b = static_cast<int>(id / c.kv_heads);
    const int group = a.heads / c.kv_heads;
    const int heads = min(kHeads, group - ht * kHeads);  // of this workgroup
    const int64_t row0 = static_cast<int64_t>(b) * a.heads + h * group + ht * kHeads;

    const int len = cached_tokens(c, b);
    const Tiles<kTile> tiles(len - 1, len - 1, a.window, a.sinks);
    const int t0 = split * range, t1 = min(t0 + range, tiles.count);
    if (t0 >= t1) {
        if (S > 1) {
            if (tid < heads) {
                float* o = ml + ((row0 + tid) * S + split) * 2;
                o[0] = kNoMax;
                o[1] = 0.f;
            }
        } else {
            for (int i = tid; i < heads * (D / 8); i += 64 * kWaves)
                reinterpret_cast<u32x4*>(a.out + row0 * D)[i] = u32x4{0u, 0u, 0u, 0u};
        }
        return;
    }

    // the range's pages: an entry for every tile, or for each half of one
    const int halves = c.page_shift == 4 ? 2 : 1;
    for (int i = tid; i < (t1 - t0) * halves; i += 64 * kWaves) {
        const int at = tiles.start(t0 + i / halves) + (i % halves) * 16;
        const int p = page_of(c, b, at);
        pages[i] = p < 0 ? 0 : p;  // positions past the last page are masked, and read page 0
    }

    // q as the right operand of the first product: head r16, d = 32 s + 8 g4 ..
    // (codes: a lane holds 8 KS consecutive d of its position)
    u32x4 qf[KS];
    {
        const uint16_t* q = a.q + b * a.q_stride + static_cast<int64_t>(h * group + ht * kHeads + r16) * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (r16 < heads) {
                qf[s] = *reinterpret_cast<const u32x4*>(q + (I4 ? 8 * KS * g4 + 8 * s : 32 * s + 8 * g4));
                if constexpr (I4) qf[s] = code_order(qf[s]);
            }
        }
    }
    __syncthreads();

    const int page_mask = (1 << c.page_shift) - 1;
    const int64_t head_at = static_cast<int64_t>(h) << c.page_shift;  // row of the head in a page
    const int64_t scale_at = (static_cast<int64_t>(c.kv_heads) << c.page_shift) * (D / 2);
    const int k_off = 8 * (r16 >> 2), v_off = 8 * g4;  // runs of 8 positions lie in one page
    const int k_half = halves == 2 ? k_off >> 4 : 0, v_half = halves == 2 ? v_off >> 4 : 0;

    u32x4 kf[2][I4 ? 1 : KS];
    u32x4 vf[I4 ? 2 : 8];   // a lane's values of 8 positions: DV binary16, or DV codes
    u32x4 ks, vs;           // scales of the lane's 8 positions

    auto load_k = [&](int t) {
        const int at = (tiles.start(t) + k_off) & page_mask;
        const int64_t page = pages[(t - t0) * halves + k_half] * c.page_bytes;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t row = head_at + at + 4 * u + (r16 & 3);
            if constexpr (I4) {
                const uint8_t* p = c.k + page + row * (D / 2) + 4 * KS * g4;
                if constexpr (KS == 4) kf[u][0] = *reinterpret_cast<const u32x4*>(p);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                    kf[u][0][0] = w[0];
                    kf[u][0][1] = w[1];
                }
            } else {
                const uint8_t* p = c.k + page + row * (2 * D) + 16 * g4;
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[u][s] = *reinterpret_cast<const u32x4*>(p + 64 * s);
            }
        }
        if constexpr (I4) {  // scales in the layout of the scores
            const int av = (tiles.start(t) + v_off) & page_mask;
            const int64_t pv = pages[(t - t0) * halves + v_half] * c.page_bytes;
            ks = *reinterpret_cast<const u32x4*>(c.k + pv + scale_at + 2 * (head_at + av));
        }
    };
    auto load_v = [&](int t) {
        const int at = (tiles.start(t) + v_off) & page_mask;
        const int64_t page = pages[(t - t0) * halves + v_half] * c.page_bytes;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t row = head_at + at + j;
            if constexpr (I4) {
                const uint8_t* p = c.v + page + row * (D / 2) + (DV / 2) * r16;
                if constexpr (DV == 8) vf[j >> 2][j & 3] = *reinterpret_cast<const uint32_t*>(p);
                else vf[j >> 2][j & 3] = *reinterpret_cast<const uint16_t*>(p);
            } else {
                const uint8_t* p = c.v + page + row * (2 * D) + 2 * DV * r16;
                if constexpr (DV == 8) vf[j] = *reinterpret_cast<const u32x4*>(p);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                    vf[j][0] = w[0];
                    vf[j][1] = w[1];
                }
            }
        }
        if constexpr (I4) vs = *reinterpret_cast<const u32x4*>(c.v + page + scale_at + 2 * (head_at + at));
    };

    f32x4 o[DV];
#pragma unroll
    for (int i = 0; i < DV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNoMax, l = 0.f, ref = 0.f, ref_inv = 0.f;
    const float to_log2 = a.scale * kLog2e;

    int t = t0 + wave;
    if (t < t1) {
        load_k(t);
        load_v(t);
    }
    for (; t < t1; t += kWaves) {
        const int at = tiles.start(t);
        // scores, 8 positions of one head a lane
        f32x4 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 kk;
                if constexpr (I4) {
                    uint32_t w[4];
                    codes_f16(kf[u][0][s], w);
                    kk = u32x4{w[0], w[1], w[2], w[3]};
                } else {
                    kk = kf[u][s];
                }
                sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kk), __builtin_bit_cast(f16x8, qf[s]),
                                                               sc[u], 0, 0, 0);
            }
        }
        float x[8], w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = sc[j >> 2][j & 3] * to_log2;
            if constexpr (I4) {
                x[j] *= __half2float(__ushort_as_half(static_cast<uint16_t>(ks[j >> 1] >> (16 * (j & 1)))));
                w[j] = __half2float(__ushort_as_half(static_cast<uint16_t>(vs[j >> 1] >> (16 * (j & 1)))));
            }
        }
        const bool more = t + kWaves < t1;
        if (more) load_k(t + kWaves);
        // positions past the end, or between the first ones and the window: their
        // scores do not count, and their values, whatever they are, are zero
        const bool masked = at + kTile > len || (at < tiles.lo && at + kTile > tiles.sinks);
        if (masked) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int p = at + v_off + j;
                const bool seen = p < len && (p >= tiles.lo || p < tiles.sinks);
                x[j] = seen ? x[j] : -INFINITY;
                if constexpr (I4) {
                    w[j] = seen ? w[j] : 0.f;
                } else {
#pragma unroll
                    for (int i = 0; i < DV / 2; ++i) vf[j][i] = seen ? vf[j][i] : 0u;
                }
            }
        }
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        bool raise = top > m + kSlack;
        float wide = 0.f;
        if constexpr (I4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) wide = fmaxf(wide, w[j]);
            raise = raise || wide > 16.f * ref;
        }
        if (__any(raise)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            top = fmaxf(top, m);
            float f = exp2_fast(m - top);
            l *= f;
            m = top;
            if constexpr (I4) {
                wide = fmaxf(wide, __shfl_xor(wide, 16, 64));
                wide = fmaxf(wide, __shfl_xor(wide, 32, 64));
                // the power of two at or below the largest scale
                const float r = fmaxf(ref, __uint_as_float(__float_as_uint(wide) & 0x7F800000u));
                f *= ref == r ? 1.f : ref / r;
                ref = r;
                ref_inv = r > 0.f ? 1.f / r : 0.f;
            }
#pragma unroll
            for (int i = 0; i < DV; ++i) o[i] *= f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = exp2_fast(x[j] - m);
            l += x[j];
            if constexpr (I4) x[j] *= w[j] * ref_inv;
        }
        u32x4 pw;
#pragma unroll
        for (int j = 0; j < 4; ++j) pw[j] = pack_f16(x[2 * j], x[2 * j + 1]);
        // values: 8 positions x DV to DV operands of 8 positions
#pragma unroll
        for (int i = 0; i < DV / 2; ++i) {
            u32x4 even, odd;
            if constexpr (!I4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    even[j] = low_halves(vf[2 * j][i], vf[2 * j + 1][i]);
                    odd[j] = high_halves(vf[2 * j][i], vf[2 * j + 1][i]);
                }
                o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, even), __builtin_bit_cast(f16x8, pw),
                                                                  o[2 * i], 0, 0, 0);
                o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, odd),
                                                                      __builtin_bit_cast(f16x8, pw), o[2 * i + 1], 0, 0, 0);
            }
        }
        if constexpr (I4) {
#pragma unroll
            for (int i = 0; i < DV / 4; ++i) {  // codes 4 i .. 4 i + 3 of the lane's
                uint32_t cf[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t va = vf[j >> 1][2 * (j & 1)], vb = vf[j >> 1][2 * (j & 1) + 1];
                    codes_f16(i ? high_halves(va, vb) : low_halves(va, vb), cf[j]);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const u32x4 av = {cf[0][n], cf[1][n], cf[2][n], cf[3][n]};
                    o[4 * i + n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                        __builtin_bit_cast(f16x8, av), __builtin_bit_cast(f16x8, pw), o[4 * i + n], 0, 0, 0);
                }
            }
        }
        if (more) load_v(t + kWaves);
    }

    // the four waves' sums
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g4 == 0) {
        sum_ml[0][wave][r16] = m;
        sum_ml[1][wave][r16] = l;
    }
    __syncthreads();
    float top = sum_ml[0][0][r16];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, sum_ml[0][i][r16]);
    {
        float f = exp2_fast(m - top);
        if constexpr (I4) f *= ref;
        // lane's rows: d = DV (4 g4 + r) + i
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < DV; i += 4)
                *reinterpret_cast<f32x4*>(&sums[wave][r16][DV * (4 * g4 + r) + i]) =
                    f32x4{o[i][r] * f, o[i + 1][r] * f, o[i + 2][r] * f, o[i + 3][r] * f};
    }
    __syncthreads();
    constexpr int PT = kHeads * D / (64 * kWaves);  // values a thread adds
    const int hd = tid / (D / PT), d0 = (tid % (D / PT)) * PT;
    if (hd >= heads) return;
    float y[PT];
#pragma unroll
    for (int i = 0; i < PT; ++i) y[i] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < PT; i += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(&sums[w][hd][d0 + i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[i + j] += v[j];
        }
    float mt = sum_ml[0][0][hd];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mt = fmaxf(mt, sum_ml[0][w][hd]);
    float lt = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) lt += sum_ml[1][w][hd] * exp2_fast(sum_ml[0][w][hd] - mt);
    if (S == 1) {
        const float inv = lt != 0.f ? 1.f / lt : 0.f;
        uint32_t q[PT / 2];
#pragma unroll
        for (int i = 0; i < PT / 2; ++i) q[i] = pack_f16(y[2 * i] * inv, y[2 * i + 1] * inv);
        uint16_t* out = a.out + (row0 + hd) * D + d0;
        if constexpr (PT == 8) *reinterpret_cast<u32x4*>(out) = u32x4{q[0], q[1], q[2], q[3]};
        else *reinterpret_cast<u32x2*>(out) = u32x2{q[0], q[1]};
    } else {
        const int64_t at = (row0 + hd) * S + split;
        if (d0 == 0) {
            ml[at * 2] = mt;
            ml[at * 2 + 1] = lt;
        }
#pragma unroll
        for (int i = 0; i < PT; i += 4)
            *reinterpret_cast<f32x4*>(part + at * D + d0 + i) = f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]};
    }
}

// out[row] = sum_s part[row][s] 2^(m_s - M) / sum_s l_s 2^(m_s - M).  A workgroup
// takes a row: its threads are D / 4 columns times slices of the parts, added in
// a fixed order.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(const float* __restrict__ part, const float* __restrict__ ml, int S,
                                                        uint16_t* __restrict__ out) {
    constexpr int C = D / 4, N = 256 / C;  // columns, slices
    __shared__ float top_of[4];
    __shared__ float sum_of[N];
    __shared__ __align__(16) f32x4 sums[N][C];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const float* mlr = ml + row * S * 2;
    float top = kNoMax;
    for (int s = tid; s < S; s += 256) top = fmaxf(top, mlr[2 * s]);
#pragma unroll
    for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i, 64));
    if ((tid & 63) == 0) top_of[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
    const int col = tid % C, slice = tid / C;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s = slice; s < S; s += N) {
        const float ls = mlr[2 * s + 1];
        if (ls == 0.f) continue;  // a part without positions wrote no sums
        const float f = exp2_fast(mlr[2 * s] - top);
        l += ls * f;
        const f32x4 v = *reinterpret_cast<const f32x4*>(part + (row * S + s) * D + 4 * col);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = fmaf(v[j], f, y[j]);
    }
    sums[slice][col] = y;
    if (col == 0) sum_of[slice] = l;
    __syncthreads();
    if (slice) return;
#pragma unroll
    for (int s = 1; s < N; ++s) {
        const f32x4 v = sums[s][col];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += v[j];
        l += sum_of[s];
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<u32x2*>(out + row * D + 4 * col) = u32x2{pack_f16(y[0] * inv, y[1] * inv), pack_f16(y[2] * inv, y[3] * inv)};
}

struct Plan {
    int head_tiles;
    int range;   // tiles of a range
    int S;       // ranges a sequence
};

// The longest sequence's tiles cut into ranges so that the workgroups number
// about four a compute unit, of one to 32 tiles a wave.
Plan plan_decode(const KvView& c, const AttnArgs& a) {
    Plan p;
    p.head_tiles = (a.heads / c.kv_heads + kHeads - 1) / kHeads;
    const int64_t most = std::min<int64_t>(c.max_len, static_cast<int64_t>(c.width) << c.page_shift);
    const int64_t full = (most + kTile - 1) / kTile;
    int64_t tiles = full;
    if (a.window) {  // the window's tiles (one more where it starts inside one), and the first ones
        const int64_t w = (static_cast<int64_t>(a.window) + kTile - 2) / kTile + 1 + (static_cast<int64_t>(a.sinks) + kTile - 1) / kTile;
        tiles = std::min(full, w);
    }
    tiles = std::max<int64_t>(tiles, 1);
    const int64_t units = static_cast<int64_t>(c.B) * c.kv_heads * p.head_tiles;
    const int64_t want = (4 * device_cu_count() + units - 1) / units;
    int64_t range = (tiles + want - 1) / want;
    range = std::min<int64_t>(std::max<int64_t>(range, kWaves), kMaxTiles);
    p.range = static_cast<int>((range + kWaves - 1) / kWaves * kWaves);
    p.S = static_cast<int>((tiles + p.range - 1) / p.range);
    return p;
}

int64_t blocks_of(const KvView& c, const Plan& p) {
    return static_cast<int64_t>(c.B) * c.kv_heads * p.head_tiles * p.S;
}

}  // namespace

int64_t attn_decode_workspace(const KvView& c, const AttnArgs& a) {
    const Plan p = plan_decode(c, a);
    if (blocks_of(c, p) > 0x7FFFFFFFll) return -1;
    return p.S == 1 ? 0 : a.T * a.heads * p.S * static_cast<int64_t>(c.D + 2) * 4;
}

hipError_t launch_attn_join(const float* part, const float* ml, int64_t rows, int S, int D, uint16_t* out,
                            hipStream_t stream) {
    auto run = [&](auto kernel) { kernel<<<static_cast<unsigned>(rows), 256, 0, stream>>>(part, ml, S, out); };
    D == 128 ? run(attn_join_kernel<128>) : run(attn_join_kernel<64>);
    return hipGetLastError();
}

hipError_t launch_attn_decode(const KvView& c, const AttnArgs& a, hipStream_t stream) {
    const Plan p = plan_decode(c, a);
    float* part = static_cast<float*>(a.workspace);
    float* ml = part + a.T * a.heads * p.S * c.D;
    auto run = [&](auto kernel) {
        kernel<<<static_cast<unsigned>(blocks_of(c, p)), 64 * kWaves, 0, stream>>>(c, a, p.S, p.range, p.head_tiles, part, ml);
    };
    if (c.D == 128) c.i4 ? run(attn_decode_kernel<128, true>) : run(attn_decode_kernel<128, false>);
    else c.i4 ? run(attn_decode_kernel<64, true>) : run(attn_decode_kernel<64, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.S == 1) return e;
    return launch_attn_join(part, ml, a.T * a.heads, p.S, c.D, a.out, stream);
}

}  // namespace apex4
