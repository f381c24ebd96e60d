// Attention of one new token a sequence, or a few, over the paged cache, its length
// split over workgroups and joined.
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
// The scores' maximum is kept per head, raised only when a weight passes 2^8:
// in most tiles nothing is rescaled.
// 4-bit codes enter the products as small integers in binary16 (exact); a
// position's two scales multiply its score and its weight in 32 bits.  The
// maximum is then that of the score plus log2 of the value's scale, so that
// weights times scales, whatever the scales are, stay in binary16's range.
//
// Four waves (eight where the workgroups are few) share a range of positions and
// add their sums through LDS; with more than one range a sequence, a second kernel
// joins the ranges' sums in order (the same bits every time).
//
// Measured, 8 key heads of 128 and 64 query heads unless said otherwise; a kernel
// that only reads reaches 5.1 TB/s over 0.5 GB and 5.7 over 2:
//   one sequence of 131071, 537 MB           96 us, 5.6 TB/s, the join 4.8
//   27 ragged sequences up to 8192, 502 MB  104 us, 4.8 TB/s, the join 4.8
//   32 of them up to 16384, int4, 342 MB     75 us, 4.6 TB/s, the join 6.4
//   16 under a window of 2048, 40 heads and key heads, 631 MB
//                                           112 us, 5.6 TB/s, the join 4.6
//   one sequence of 517 (one range)         9.4 us: 17 tiles of eight waves are
//                                           three waits on memory and the merge
// A launch of this size has about 10 us besides its bytes (first loads, last merge).
// The codes' kernel issues 18 vector instructions a product, 45 % of what the SIMDs
// issue in that time: there the bound is their latency between two tiles in flight.
#include "attn_core.h"

namespace apex4 {
namespace {

using namespace attn;

constexpr int kTile = 32;      // positions a wave takes at a time
constexpr int kMaxTiles = 64;  // tiles of a range at most
constexpr int kOneRange = 40;  // tiles that are not cut: 5 rounds of eight waves
constexpr int kRows = 16;      // rows (new token, query head) a workgroup takes

template <int D, bool I4, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kWaves == 4 ? 3 : 2) void attn_decode_kernel(KvView c, AttnArgs a, int S, int range,
                                                                  int row_tiles, float* __restrict__ part,
                                                                  float* __restrict__ ml) {
    constexpr int DV = D / 16;  // values d of a lane in the second product
    constexpr int KS = D / 32;  // products along d in the first
    constexpr int P = D + 4;    // floats a row of the sums takes in LDS (rows 16 bytes apart in the banks)
    __shared__ int32_t pages[2 * kMaxTiles];
    __shared__ float sum_ml[2][kWaves][kRows];
    __shared__ __align__(16) float sums[kWaves][kRows][P];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
    // Workgroups go to the 8 XCDs in turn.  Every group of 8 is rotated by its
    // number, so that no XCD gets the same heads or ranges of every sequence, which
    // differ in length; the later ranges, missing from short sequences, come last.
    uint32_t id = workgroup_number();
    if ((id | 7) < gridDim.x * gridDim.y) id = (id & ~7u) | ((id + (id >> 3)) & 7u);
    const int h = static_cast<int>(id % c.kv_heads);
    id /= c.kv_heads;
    const int rt = static_cast<int>(id % row_tiles);
    id /= row_tiles;
    const int b = static_cast<int>(id % c.B);
    const int split = static_cast<int>(id / c.B);
    if (split >= S) return;
    const uint32_t group = a.group;
    // the sequence's rows of this key head: its new tokens times the heads that share it
    const int q0 = a.q_start ? a.q_start[b] : b;
    const int n = a.q_start ? new_tokens(a, b) : 1;
    const int taken = min(n, static_cast<int>(a.max_q));  // past max_q tokens nothing is computed
    const uint32_t all_rows = taken * group, row0 = rt * kRows;  // T heads and max_q heads are below 2^28
    if (row0 >= all_rows) return;
    const int rows = min(static_cast<int>(all_rows - row0), kRows);  // of this workgroup
    struct Row {
        int tok, head;
        bool valid;
        int64_t at;  // its number among all tokens' heads
    };
    auto row_of = [&](int r) {
        Row x;
        x.tok = (row0 + r) / group;
        x.head = h * group + (row0 + r) - x.tok * group;
        x.at = (static_cast<int64_t>(q0) + x.tok) * a.heads + x.head;
        x.valid = r < rows && q0 >= 0 && q0 + x.tok < a.T;
        return x;
    };

    // The range's pages: an entry for every tile, or for each half of one, one a
    // thread.  Without a window their places in the table do not wait for the length.
    static_assert(2 * kMaxTiles <= 64 * kWaves);
    const int halves = c.page_shift == 4 ? 2 : 1;
    const int t0 = split * range;
    int page = 0;
    if (a.window == 0) page = page_of(c, b, (t0 + tid / halves) * kTile + (tid % halves) * 16);
    // q as the right operand of the first product: head r16, d = 32 s + 8 g4 ..
    // (codes: a lane holds 8 KS consecutive d of its position)
    u32x4 qf[KS];
    int tok;
    {
        const Row x = row_of(r16);
        tok = x.tok;
        const uint16_t* q = a.q + (q0 + x.tok) * a.q_stride + x.head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (x.valid) qf[s] = *reinterpret_cast<const u32x4*>(q + (I4 ? 8 * KS * g4 + 8 * s : 32 * s + 8 * g4));
            if constexpr (I4) qf[s] = code_order(qf[s]);
        }
    }
    const int before = cached_tokens(c, b) - n, len = before + taken;  // positions that some row sees end at len
    const int pos = before + tok;  // of the lane's row (negative: it sees nothing)
    const Tiles<kTile> tiles(before, len - 1, a.window, a.sinks);
    const int t1 = min(t0 + range, tiles.count);
    if (t0 >= t1) {
        if (S > 1) {
            const Row x = row_of(tid);
            if (x.valid) {
                float* o = ml + (x.at * S + split) * 2;
                o[0] = kNoMax;
                o[1] = 0.f;
            }
        } else {
            for (int i = tid; i < rows * (D / 8); i += 64 * kWaves) {
                const Row x = row_of(i / (D / 8));
                if (x.valid) reinterpret_cast<u32x4*>(a.out + x.at * D)[i % (D / 8)] = u32x4{0u, 0u, 0u, 0u};
            }
        }
        return;
    }

    if (a.window != 0 && tid < (t1 - t0) * halves)
        page = page_of(c, b, tiles.start(t0 + tid / halves) + (tid % halves) * 16);
    if (tid < 2 * kMaxTiles) pages[tid] = page < 0 ? 0 : page;  // positions past the last page are masked, and read page 0
    __syncthreads();

    const int page_mask = (1 << c.page_shift) - 1;
    const int64_t head_at = static_cast<int64_t>(h) << c.page_shift;  // row of the head in a page
    const int64_t scale_at = (static_cast<int64_t>(c.kv_heads) << c.page_shift) * (D / 2);
    const int k_off = 8 * (r16 >> 2), v_off = 8 * g4;  // runs of 8 positions lie in one page
    const int k_half = halves == 2 ? k_off >> 4 : 0, v_half = halves == 2 ? v_off >> 4 : 0;

    // one tile in registers: a lane's keys of 4 + 4 positions, its values of 8 (DV
    // binary16, or DV codes), and the scales of the 8
    struct Loaded {
        u32x4 k[2][I4 ? 1 : KS];
        u32x4 v[I4 ? 2 : 8];
        u32x4 ks, vs;
    };
    auto load_k = [&](int t, Loaded& x) {
        const int at = (tiles.start(t) + k_off) & page_mask;
        const int64_t page = pages[(t - t0) * halves + k_half] * c.page_bytes;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t row = head_at + at + 4 * u + (r16 & 3);
            if constexpr (I4) {
                const uint8_t* p = c.k + page + row * (D / 2) + 4 * KS * g4;
                if constexpr (KS == 4) x.k[u][0] = *reinterpret_cast<const u32x4*>(p);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                    x.k[u][0][0] = w[0];
                    x.k[u][0][1] = w[1];
                }
            } else {
                const uint8_t* p = c.k + page + row * (2 * D) + 16 * g4;
#pragma unroll
                for (int s = 0; s < KS; ++s) x.k[u][s] = *reinterpret_cast<const u32x4*>(p + 64 * s);
            }
        }
    };
    auto load_v = [&](int t, Loaded& x) {
        const int at = (tiles.start(t) + v_off) & page_mask;
        const int64_t page = pages[(t - t0) * halves + v_half] * c.page_bytes;
        const int64_t row = head_at + at;
        const uint8_t* p = c.v + page + row * (I4 ? D / 2 : 2 * D) + (I4 ? DV / 2 : 2 * DV) * r16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint8_t* pj = p + j * (I4 ? D / 2 : 2 * D);
            if constexpr (I4) {
                if constexpr (DV == 8) x.v[j >> 2][j & 3] = *reinterpret_cast<const uint32_t*>(pj);
                else x.v[j >> 2][j & 3] = *reinterpret_cast<const uint16_t*>(pj);
            } else {
                if constexpr (DV == 8) x.v[j] = *reinterpret_cast<const u32x4*>(pj);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(pj);
                    x.v[j][0] = w[0];
                    x.v[j][1] = w[1];
                }
            }
        }
        if constexpr (I4) {  // both in the layout of the scores
            x.ks = *reinterpret_cast<const u32x4*>(c.k + page + scale_at + 2 * row);
            x.vs = *reinterpret_cast<const u32x4*>(c.v + page + scale_at + 2 * row);
        }
    };

    f32x4 o[DV];
#pragma unroll
    for (int i = 0; i < DV; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNoMax, l = 0.f;
    const float to_log2 = a.scale * kLog2e;
    // the first product of codes + 72 (codes_bias72) starts at -72 sum q
    float minus = 0.f;
    if constexpr (I4) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) minus += half_of(qf[s][i], 0) + half_of(qf[s][i], 1);
        minus += __shfl_xor(minus, 16, 64);
        minus += __shfl_xor(minus, 32, 64);
        minus *= -72.f;
    }

    // first position that the windows of all rows hold
    const int edge = a.window ? len - a.window : 0;

    // One tile.  more(): issues the loads that may go out once the keys, and
    // more_v() once the values, are used.
    auto step = [&](int t, Loaded& x, auto more_k, auto more_v) {
        const int at = tiles.start(t);
        f32x4 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sc[u] = f32x4{minus, minus, minus, minus};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 kk;
                if constexpr (I4) kk = codes_bias72(x.k[u][0][s]);
                else kk = x.k[u][s];
                sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kk), __builtin_bit_cast(f16x8, qf[s]),
                                                               sc[u], 0, 0, 0);
            }
        }
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = sc[j >> 2][j & 3];
            if constexpr (I4) {
                y[j] = times_half(y[j], x.ks[j >> 1], j & 1);
            }
        }
        more_k();
        // positions that a row does not see: their scores do not count, and the values
        // of those that no row sees, whatever they are, are zero
        const bool masked = at + kTile > before + 1 || (at < edge && at + kTile > tiles.sinks);
        if (masked) {
            const int from = a.window ? pos - a.window + 1 : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int p = at + v_off + j;
                const bool seen = p <= pos && (p >= from || p < a.sinks), some = p < len && (p >= tiles.lo || p < tiles.sinks);
                y[j] = seen ? y[j] : -INFINITY;
                if constexpr (I4) {
                    x.vs[j >> 1] &= some ? 0xFFFFFFFFu : (j & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                } else {
#pragma unroll
                    for (int i = 0; i < DV / 2; ++i) x.v[j][i] = some ? x.v[j][i] : 0u;
                }
            }
        }
        // weights under the maximum so far (of a score, or of a score plus log2 of
        // its value's scale); where one is past the slack the maximum is raised first
        float e[8], w[8], top = 0.f, sum_top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = exp2_fast(fmaf(y[j], to_log2, -m));
            w[j] = I4 ? times_half(e[j], x.vs[j >> 1], j & 1) : e[j];
            top = fmaxf(top, w[j]);
            if constexpr (I4) sum_top = fmaxf(sum_top, e[j]);  // a scale of zero leaves the sum alone to grow
        }
        // (only of the rows that need it: what a row gives does not depend on the others)
        if (const uint64_t over = __ballot(top > kMostWeight || (I4 && sum_top > kMostSum))) {
            top = kNoMax;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float z = y[j] * to_log2;
                if constexpr (I4) z += __builtin_amdgcn_logf(fmaxf(half_of(x.vs[j >> 1], j & 1), 0x1p-24f));
                top = fmaxf(top, z);
            }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            top = (over >> r16 & 0x0001000100010001ull) ? fmaxf(top, m) : m;
            const float f = exp2_fast(m - top);
            l *= f;
            m = top;
#pragma unroll
            for (int i = 0; i < DV; ++i) o[i] *= f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = exp2_fast(fmaf(y[j], to_log2, -m));
                w[j] = I4 ? times_half(e[j], x.vs[j >> 1], j & 1) : e[j];
            }
        }
        // A binary16 cache: the weights as a sum of two binary16.  The products are not
        // what bounds the kernel (the times did not change), and so the rounding of the
        // weights (2^-11 of one) is gone from the result, which is then as far from 64
        // bits as its own rounding; with one binary16 1.4 times that.  Codes: one, 1.1
        // times that; their kernel has no time to spare (94 us would be 103).
        u32x4 pw, rest;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            pw[j] = pack_f16(w[2 * j], w[2 * j + 1]);
            if constexpr (!I4) rest[j] = pack_f16(w[2 * j] - half_of(pw[j], 0), w[2 * j + 1] - half_of(pw[j], 1));
            l += e[2 * j] + e[2 * j + 1];
        }
        auto add = [&](int i, const u32x4& v) {
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, pw), o[i], 0, 0, 0);
            if constexpr (!I4)
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, rest), o[i], 0, 0, 0);
        };
        // values: 8 positions x DV to DV operands of 8 positions
        if constexpr (I4) {
#pragma unroll
            for (int i = 0; i < DV / 4; ++i) {  // codes 4 i .. 4 i + 3 of the lane's
                uint32_t cf[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t va = x.v[j >> 1][2 * (j & 1)], vb = x.v[j >> 1][2 * (j & 1) + 1];
                    codes_f16(i ? high_halves(va, vb) : low_halves(va, vb), cf[j]);
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) add(4 * i + n, u32x4{cf[0][n], cf[1][n], cf[2][n], cf[3][n]});
            }
        } else {
#pragma unroll
            for (int i = 0; i < DV / 2; ++i) {
                u32x4 even, odd;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    even[j] = low_halves(x.v[2 * j][i], x.v[2 * j + 1][i]);
                    odd[j] = high_halves(x.v[2 * j][i], x.v[2 * j + 1][i]);
                }
                add(2 * i, even);
                add(2 * i + 1, odd);
            }
        }
        more_v();
    };

    int t = t0 + wave;
    if constexpr (I4) {  // a tile is 4 KB: two in flight
        Loaded x, y;
        auto none = [] {};
        if (t < t1) {
            load_k(t, x);
            load_v(t, x);
        }
        while (t < t1) {
            if (t + kWaves < t1) {
                load_k(t + kWaves, y);
                load_v(t + kWaves, y);
            }
            step(t, x, none, none);
            t += kWaves;
            if (t >= t1) break;
            if (t + kWaves < t1) {
                load_k(t + kWaves, x);
                load_v(t + kWaves, x);
            }
            step(t, y, none, none);
            t += kWaves;
        }
    } else {
        Loaded x;
        if (t < t1) {
            load_k(t, x);
            load_v(t, x);
        }
        for (; t < t1; t += kWaves) {
            const bool more = t + kWaves < t1;
            step(
                t, x, [&] { if (more) load_k(t + kWaves, x); }, [&] { if (more) load_v(t + kWaves, x); });
        }
    }

    // the waves' sums
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
        const float f = exp2_fast(m - top);
        // lane's rows: d = DV (4 g4 + r) + i
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < DV; i += 4)
                *reinterpret_cast<f32x4*>(&sums[wave][r16][DV * (4 * g4 + r) + i]) =
                    f32x4{o[i][r] * f, o[i + 1][r] * f, o[i + 2][r] * f, o[i + 3][r] * f};
    }
    __syncthreads();
    constexpr int PT = kRows * D / (64 * kWaves) > 4 ? kRows * D / (64 * kWaves) : 4;  // values a thread adds
    const int hd = tid / (D / PT), d0 = (tid % (D / PT)) * PT;
    const Row out_row = row_of(hd);
    if (!out_row.valid) return;
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
        uint16_t* out = a.out + out_row.at * D + d0;
        if constexpr (PT == 8) *reinterpret_cast<u32x4*>(out) = u32x4{q[0], q[1], q[2], q[3]};
        else *reinterpret_cast<u32x2*>(out) = u32x2{q[0], q[1]};
    } else {
        const int64_t at = out_row.at * S + split;
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
// takes C columns of four values of a row: its threads are the columns times
// slices of the parts, added in a fixed order.  With many parts a row's columns
// go to several workgroups (64 rows of 256 parts: 13.9 -> 5 us).
template <int D, int C>
__global__ __launch_bounds__(256) void attn_join_kernel(const float* __restrict__ part, const float* __restrict__ ml,
                                                        int64_t rows, int S, uint16_t* __restrict__ out) {
    constexpr int N = 256 / C, kFactors = 1024;
    __shared__ float top_of[4];
    __shared__ int last_of[4];
    __shared__ float factor[kFactors];
    __shared__ float sum_of[4];
    __shared__ __align__(16) f32x4 sums[N][C];
    const uint32_t id = workgroup_number();
    const int64_t row = id / (D / 4 / C);
    if (row >= rows) return;
    const int tid = threadIdx.x, wave = tid >> 6;
    const int col = static_cast<int>(id % (D / 4 / C)) * C + tid % C, slice = tid / C;
    const float* mlr = ml + row * S * 2;
    const float* p = part + row * S * D + 4 * col;
    float top = kNoMax;
    int last = 0;  // parts after the last one with a sum have none, and wrote none
    for (int s = tid; s < S; s += 256) {
        if (mlr[2 * s + 1] != 0.f) {
            top = fmaxf(top, mlr[2 * s]);
            last = s + 1;
        }
    }
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
        top = fmaxf(top, __shfl_xor(top, i, 64));
        last = max(last, __shfl_xor(last, i, 64));
    }
    if ((tid & 63) == 0) {
        top_of[wave] = top;
        last_of[wave] = last;
    }
    __syncthreads();
    top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
    last = max(max(last_of[0], last_of[1]), max(last_of[2], last_of[3]));
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s0 = 0; s0 < last; s0 += kFactors) {
        const int n = min(kFactors, last - s0);
        __syncthreads();  // the factors before are used
        for (int s = tid; s < n; s += 256) {
            const float f = exp2_fast(mlr[2 * (s0 + s)] - top);
            factor[s] = f;
            l = fmaf(mlr[2 * (s0 + s) + 1], f, l);
        }
        __syncthreads();
#pragma unroll 4
        for (int s = slice; s < n; s += N) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(p + static_cast<int64_t>(s0 + s) * D);
            const float f = factor[s];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = fmaf(v[j], f, y[j]);
        }
    }
#pragma unroll
    for (int i = 1; i < 64; i *= 2) l += __shfl_xor(l, i, 64);
    if ((tid & 63) == 0) sum_of[wave] = l;
    sums[slice][tid % C] = y;
    __syncthreads();
    if (slice) return;
#pragma unroll
    for (int s = 1; s < N; ++s) {
        const f32x4 v = sums[s][tid % C];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] += v[j];
    }
    l = (sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]);
    const float inv = l != 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<u32x2*>(out + row * D + 4 * col) = u32x2{pack_f16(y[0] * inv, y[1] * inv), pack_f16(y[2] * inv, y[3] * inv)};
}

// The same for many rows of few parts: D / 4 lanes take a row, so that a workgroup has
// several and the rows are done in few rounds.  (12800 rows of 4 parts: the whole
// call 46 -> 35 us; 256 rows of 12 parts: 17 -> 22, the kernel above waits less.)
constexpr int kFewParts = 16;
template <int D>
__global__ __launch_bounds__(256) void attn_join_few_kernel(const float* __restrict__ part, const float* __restrict__ ml,
                                                            int64_t rows, int S, uint16_t* __restrict__ out) {
    constexpr int C = D / 4;
    const int64_t row = static_cast<int64_t>(workgroup_number()) * (256 / C) + threadIdx.x / C;
    const int col = threadIdx.x % C;
    if (row >= rows) return;
    const float* mlr = ml + row * S * 2;
    const float* p = part + row * S * D + 4 * col;
    float top = kNoMax;
    for (int s = 0; s < S; ++s)
        if (mlr[2 * s + 1] != 0.f) top = fmaxf(top, mlr[2 * s]);
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll 4
    for (int s = 0; s < S; ++s) {
        const float ls = mlr[2 * s + 1], f = exp2_fast(mlr[2 * s] - top);
        const f32x4 v = *reinterpret_cast<const f32x4*>(p + static_cast<int64_t>(s) * D);
        if (ls != 0.f) {  // a part without a sum may have been left unwritten
            l = fmaf(ls, f, l);
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = fmaf(v[j], f, y[j]);
        }
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    *reinterpret_cast<u32x2*>(out + row * D + 4 * col) = u32x2{pack_f16(y[0] * inv, y[1] * inv), pack_f16(y[2] * inv, y[3] * inv)};
}

struct Plan {
    int waves;
    int row_tiles;
    int range;   // tiles of a range
    int S;       // ranges a sequence
};

// A range for every sequence where that is quick: the second launch costs 4 us
// (and as much again on the host), a round of the waves, one tile each, 1.1 us
// (int4: 0.7).  Otherwise the longest sequence's tiles are cut so that the workgroups
// number about four a compute unit, of up to 8 tiles a wave (int4: 16).  Eight
// waves where the workgroups of whole sequences leave compute units idle.
Plan plan_decode(const KvView& c, const AttnArgs& a) {
    Plan p;
    p.row_tiles = static_cast<int>((a.max_q * (a.heads / c.kv_heads) + kRows - 1) / kRows);
    const int64_t most = std::min<int64_t>(c.max_len, static_cast<int64_t>(c.width) << c.page_shift);
    const int64_t full = (most + kTile - 1) / kTile;
    int64_t tiles = full;
    if (a.window) {  // the rows' windows (one more where they start inside a tile), and the first positions
        const int64_t w = (static_cast<int64_t>(a.window) + a.max_q + kTile - 3) / kTile + 1 + (static_cast<int64_t>(a.sinks) + kTile - 1) / kTile;
        tiles = std::min(full, w);
    }
    tiles = std::max<int64_t>(tiles, 1);
    const int64_t units = static_cast<int64_t>(c.B) * c.kv_heads * p.row_tiles, cu = device_cu_count();
    const bool few = units <= cu;
    p.waves = few && tiles <= kOneRange ? 8 : 4;
    int64_t range = (tiles + kOneRange - 1) / kOneRange * kOneRange;
    if (tiles > kOneRange) {
        const int64_t want = (4 * cu + units - 1) / units;
        range = std::min<int64_t>(std::max<int64_t>((tiles + want - 1) / want, p.waves), c.i4 ? kMaxTiles : kMaxTiles / 2);
    }
    p.range = static_cast<int>((range + p.waves - 1) / p.waves * p.waves);
    p.S = static_cast<int>((tiles + p.range - 1) / p.range);
    return p;
}

int64_t blocks_of(const KvView& c, const Plan& p) {
    return static_cast<int64_t>(c.B) * c.kv_heads * p.row_tiles * p.S;
}

}  // namespace

int64_t attn_decode_workspace(const KvView& c, const AttnArgs& a) {
    const Plan p = plan_decode(c, a);
    if (blocks_of(c, p) > 0x7FFFFFFFll) return -1;
    return p.S == 1 ? 0 : a.T * a.heads * p.S * static_cast<int64_t>(c.D + 2) * 4;
}

hipError_t launch_attn_join(const float* part, const float* ml, int64_t rows, int S, int D, uint16_t* out,
                            hipStream_t stream) {
    if (S <= kFewParts && rows >= 8 * device_cu_count()) {
        const int64_t n = 1024 / D;  // rows of a workgroup
        const dim3 grid = grid_of((rows + n - 1) / n);
        if (D == 128) attn_join_few_kernel<128><<<grid, 256, 0, stream>>>(part, ml, rows, S, out);
        else attn_join_few_kernel<64><<<grid, 256, 0, stream>>>(part, ml, rows, S, out);
        return hipGetLastError();
    }
    // 32 parts or more, and rows too few to fill the compute units twice
    const bool wide = S >= 32 && rows < 2 * device_cu_count();
    auto run = [&](auto kernel, int per_row) {
        kernel<<<grid_of(rows * per_row), 256, 0, stream>>>(part, ml, rows, S, out);
    };
    if (D == 128) wide ? run(attn_join_kernel<128, 8>, 4) : run(attn_join_kernel<128, 32>, 1);
    else wide ? run(attn_join_kernel<64, 8>, 2) : run(attn_join_kernel<64, 16>, 1);
    return hipGetLastError();
}

hipError_t launch_attn_decode(const KvView& c, const AttnArgs& a, hipStream_t stream) {
    const Plan p = plan_decode(c, a);
    float* part = static_cast<float*>(a.workspace);
    float* ml = part + a.T * a.heads * p.S * c.D;
    auto run = [&](auto kernel) {
        kernel<<<grid_of(blocks_of(c, p)), 64 * p.waves, 0, stream>>>(c, a, p.S, p.range, p.row_tiles, part, ml);
    };
    auto pick = [&](auto few, auto many) { p.waves == 8 ? run(few) : run(many); };
    if (c.D == 128) {
        if (c.i4) pick(attn_decode_kernel<128, true, 8>, attn_decode_kernel<128, true, 4>);
        else pick(attn_decode_kernel<128, false, 8>, attn_decode_kernel<128, false, 4>);
    } else {
        if (c.i4) pick(attn_decode_kernel<64, true, 8>, attn_decode_kernel<64, true, 4>);
        else pick(attn_decode_kernel<64, false, 8>, attn_decode_kernel<64, false, 4>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.S == 1) return e;
    return launch_attn_join(part, ml, a.T * a.heads, p.S, c.D, a.out, stream);
}

}  // namespace apex4
