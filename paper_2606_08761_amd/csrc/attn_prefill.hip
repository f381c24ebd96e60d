// Attention of packed new tokens over the paged cache (prompts, chunks of them,
// a few tokens at a time): causal, with or without a sliding window and first
// positions that stay visible.
//
// One pass over the positions with the running maximum and sum of the softmax.
// A workgroup takes 128 rows of one key head (a row is a new token and one of
// the query heads that share the key head, so that few tokens still fill it)
// and the tiles of 64 positions that any of them sees; a wave takes 32 rows,
// with q and the output sums in registers.  Bound by the matrix cores and, next
// to them, by the exponentials.
//   S^T = K Q^T   32 x 32 x 16 products: a lane holds 16 positions of one row
//                 in each of the tile's two halves, so the softmax needs no
//                 other lane but lane ^ 32, and that only when the maximum is
//                 raised (kSlack) and at the end;
//   O^T = V^T P^T the scores' layout, rounded to binary16, is the right operand
//                 as it stands: position 16 s + 8 (j / 4) + 4 h + j % 4 is
//                 element j of lane half h in step s.
// Keys and values go through registers into LDS in the order the products read
// them, 16 bytes a lane without bank conflicts: keys as [d / 8][position],
// values transposed on the way (8 positions x 4 values d by v_perm) as
// [step, half][d][8 positions].  The next tile's loads are in flight during a
// tile's products; the buffers alternate, one barrier a tile.
// 4-bit codes become small integers in binary16 (exact) on their way into LDS;
// a position's scales multiply its scores and weights in 32 bits.
// With few rows and a long cache the tiles of a workgroup are cut into S parts,
// joined by the kernel that joins those of attn_decode.hip.
#include "attn_core.h"

namespace apex4 {
namespace {

using namespace attn;

constexpr int kW = 64;            // positions of a tile
constexpr int kWaves = 4;
constexpr int kRows = 32 * kWaves;  // rows of a workgroup
constexpr int kThreads = 64 * kWaves;

template <int D, bool I4>
struct Smem {
    static constexpr int kChunk = kW * 16 + 16;  // bytes of 8 values d of every position; the padding spreads the writes
    uint8_t k[2][D / 8 * kChunk];
    uint8_t v[2][8 * D * 16];
    float ks[2][I4 ? kW : 4];  // scales, the softmax's factor in the keys'
    float vs[2][I4 ? kW : 4];
};

template <int D, bool I4>
__global__ __launch_bounds__(kThreads, 2) void attn_prefill_kernel(KvView c, AttnArgs a, int S, int row_tiles,
                                                                   float* __restrict__ part, float* __restrict__ ml) {
    constexpr int KS = D / 16;                        // products along d in the first
    constexpr int DT = D / 32;                        // tiles of d in the second
    constexpr int KL = I4 ? D / 32 : D / 8;           // lanes a position's 16-byte pieces take
    constexpr int KN = kW * KL / kThreads > 0 ? kW * KL / kThreads : 1;  // pieces a thread loads
    constexpr int KR = kThreads / KL < kW ? kThreads / KL : kW;          // positions the threads cover at a time
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem<D, I4>& sm = *reinterpret_cast<Smem<D, I4>*>(smem_raw);

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, r32 = lane & 31, half = lane >> 5;
    uint32_t id = blockIdx.x;
    const int h = static_cast<int>(id % c.kv_heads);  // workgroups of one key head on one XCD's L2 where the heads allow it
    id /= c.kv_heads;
    const int split = static_cast<int>(id % S);
    id /= S;
    const int b = static_cast<int>(id % c.B);
    const int mt = row_tiles - 1 - static_cast<int>(id / c.B);  // the last rows see the most: first
    const int group = a.heads / c.kv_heads;

    const int q0 = a.q_start[b];
    const int n = a.q_start[b + 1] - q0;
    const int64_t rows = static_cast<int64_t>(n) * group;
    const int64_t R0 = static_cast<int64_t>(mt) * kRows;
    if (R0 >= rows) return;
    const int len = cached_tokens(c, b);
    const int before = len - n;  // position of the sequence's first new token (negative: it has no place)
    const int p_lo = before + static_cast<int>(R0 / group);
    const int p_hi = before + static_cast<int>(((R0 + kRows < rows ? R0 + kRows : rows) - 1) / group);
    const Tiles<kW> tiles(p_lo, p_hi, a.window, a.sinks);
    const int t0 = static_cast<int>(static_cast<int64_t>(tiles.count) * split / S);
    const int t1 = static_cast<int>(static_cast<int64_t>(tiles.count) * (split + 1) / S);

    // the lane's row
    const int64_t R = R0 + wave * 32 + r32;
    const int tok = static_cast<int>(R / group), hq = h * group + static_cast<int>(R % group);
    const bool valid = R < rows && q0 >= 0 && q0 + tok < a.T;
    const int pos = before + tok;
    const int64_t row = (static_cast<int64_t>(q0) + tok) * a.heads + hq;

    u32x4 qf[KS];  // right operand: d = 16 s + 8 half ..
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        qf[s] = u32x4{0u, 0u, 0u, 0u};
        if (valid) qf[s] = *reinterpret_cast<const u32x4*>(a.q + (q0 + tok) * a.q_stride + hq * D + 16 * s + 8 * half);
        if constexpr (I4) qf[s] = code_order(qf[s]);
    }

    const float to_log2 = a.scale * kLog2e;
    const int page_mask = (1 << c.page_shift) - 1;
    const int64_t head_at = static_cast<int64_t>(h) << c.page_shift;
    const int64_t scale_at = (static_cast<int64_t>(c.kv_heads) << c.page_shift) * (D / 2);

    u32x4 kr[KN];
    uint32_t vr[8][I4 ? 1 : 2];
    float ksr = 0.f, vsr = 0.f;
    const int kl = tid % KL, kt = tid / KL;               // piece and first position of a thread's keys
    constexpr int VL = D / 4;                             // threads a position's values take, 4 each
    const int vd = tid % VL, vg = tid / VL;               // values 4 vd .. of positions 16 s + 4 vh .. + 3, and 8 further on
    const int vs_step = vg >> 1, vh = vg & 1;
    const bool v_thread = vg < 8;
    const bool k_thread = kt < kW;

    // the pages of what a thread loads of a tile (16 positions lie in one page)
    int k_page[KN], v_page, s_page;
    auto load_pages = [&](int t) {
        const int at = tiles.start(t);
        auto page = [&](int x) {
            const int p = page_of(c, b, at + x);
            return p < 0 ? 0 : p;  // positions past the last page are masked, and read page 0
        };
#pragma unroll
        for (int i = 0; i < KN; ++i) k_page[i] = page((kt + i * KR) & (kW - 1));
        v_page = page((16 * vs_step) & (kW - 1));
        if constexpr (I4) s_page = page(tid & (kW - 1));
    };

    auto load_tile = [&](int t) {
        const int at = tiles.start(t);
        if (k_thread) {
#pragma unroll
            for (int i = 0; i < KN; ++i) {
                const int x = kt + i * KR;
                const int64_t r = head_at + ((at + x) & page_mask);
                kr[i] = *reinterpret_cast<const u32x4*>(c.k + k_page[i] * c.page_bytes + r * (I4 ? D / 2 : 2 * D) + 16 * kl);
            }
        }
        if (v_thread) {
            const int64_t r = head_at + ((at + 16 * vs_step + 4 * vh) & page_mask);
            const uint8_t* p = c.v + v_page * c.page_bytes + r * (I4 ? D / 2 : 2 * D) + (I4 ? 2 : 8) * vd;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint8_t* pj = p + ((j & 3) + 8 * (j >> 2)) * (I4 ? D / 2 : 2 * D);
                if constexpr (I4) vr[j][0] = *reinterpret_cast<const uint16_t*>(pj);
                else {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(pj);
                    vr[j][0] = w[0];
                    vr[j][1] = w[1];
                }
            }
        }
        if constexpr (I4) {
            if (tid < kW) {
                const int64_t o = s_page * c.page_bytes + scale_at + 2 * (head_at + ((at + tid) & page_mask));
                ksr = __half2float(*reinterpret_cast<const __half*>(c.k + o));
                vsr = __half2float(*reinterpret_cast<const __half*>(c.v + o));
            }
        }
    };
    // positions that no row of the workgroup sees hold anything: their values,
    // times a weight of zero, must not count
    auto seen_by_some = [&](int t) { return t <= p_hi && (t >= tiles.lo || t < tiles.sinks); };
    auto store_tile = [&](int t, int buf) {
        const int at = tiles.start(t);
        const bool edge = at + kW > p_hi + 1 || (at < tiles.lo && at + kW > tiles.sinks);
        if (k_thread) {
#pragma unroll
            for (int i = 0; i < KN; ++i) {
                const int x = kt + i * KR;
                if constexpr (I4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[4];
                        codes_f16(kr[i][j], w);
                        *reinterpret_cast<u32x4*>(&sm.k[buf][(4 * kl + j) * Smem<D, I4>::kChunk + x * 16]) = u32x4{w[0], w[1], w[2], w[3]};
                    }
                } else {
                    *reinterpret_cast<u32x4*>(&sm.k[buf][kl * Smem<D, I4>::kChunk + x * 16]) = kr[i];
                }
            }
        }
        if (v_thread) {
            if (!I4 && edge) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool seen = seen_by_some(at + 16 * vs_step + 4 * vh + (j & 3) + 8 * (j >> 2));
                    vr[j][0] = seen ? vr[j][0] : 0u;
                    if constexpr (!I4) vr[j][1] = seen ? vr[j][1] : 0u;
                }
            }
            u32x4 item[4];  // one of 8 positions for each of the 4 values
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (I4) {
                    uint32_t w[4];
                    codes_f16(low_halves(vr[2 * j][0], vr[2 * j + 1][0]), w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) item[i][j] = w[i];
                } else {
                    item[0][j] = low_halves(vr[2 * j][0], vr[2 * j + 1][0]);
                    item[1][j] = high_halves(vr[2 * j][0], vr[2 * j + 1][0]);
                    item[2][j] = low_halves(vr[2 * j][1], vr[2 * j + 1][1]);
                    item[3][j] = high_halves(vr[2 * j][1], vr[2 * j + 1][1]);
                }
            }
            // value d = 4 vd + i in slot i D/4 + vd: neighbours write side by side
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<u32x4*>(&sm.v[buf][((2 * vs_step + vh) * D + i * VL + vd) * 16]) = item[i];
        }
        if constexpr (I4) {
            if (tid < kW) {
                const bool seen = seen_by_some(at + tid);
                sm.ks[buf][tid] = ksr * to_log2;
                sm.vs[buf][tid] = seen ? vsr : 0.f;
            }
        }
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float m = kNoMax, l = 0.f, ref = 0.f, ref_inv = 0.f;

    if (t0 < t1) {
        load_pages(t0);
        load_tile(t0);
        store_tile(t0, 0);
        if (t0 + 1 < t1) {
            load_pages(t0 + 1);
            load_tile(t0 + 1);
        }
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1, at = tiles.start(t);
        if (t + 2 < t1) load_pages(t + 2);
        f32x16 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int j = 0; j < 16; ++j) sc[u][j] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const u32x4 kk = *reinterpret_cast<const u32x4*>(&sm.k[buf][(2 * s + half) * Smem<D, I4>::kChunk + (32 * u + r32) * 16]);
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, kk), __builtin_bit_cast(f16x8, qf[s]), sc[u], 0, 0, 0);
            }
        }
        if constexpr (I4) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 s4 = *reinterpret_cast<const f32x4*>(&sm.ks[buf][32 * u + 8 * i + 4 * half]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sc[u][4 * i + j] *= s4[j];
                }
        }
        const float f_log2 = I4 ? 1.f : to_log2;
        const bool full = at + kW - 1 <= p_lo && (a.window == 0 || at > p_hi - a.window || at + kW <= tiles.sinks);
        if (!full) {
            // visible: t <= pos, and t > pos - window or t < sinks
            const int from = a.window ? pos - a.window + 1 : 0;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int p = at + 32 * u + 8 * (j >> 2) + 4 * half + (j & 3);
                    const bool seen = p <= pos && (p >= from || p < a.sinks);
                    sc[u][j] = seen ? sc[u][j] : -INFINITY;
                }
        }
        float top = sc[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, sc[u][j]);
        top *= f_log2;
        bool raise = top > m + kSlack;
        float wide = 0.f;
        if constexpr (I4) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 s4 = *reinterpret_cast<const f32x4*>(&sm.vs[buf][32 * u + 8 * i + 4 * half]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) wide = fmaxf(wide, s4[j]);
                }
            raise = raise || wide > 16.f * ref;
        }
        if (__any(raise)) {
            top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
            float f = exp2_fast(m - top);
            l *= f;
            m = top;
            if constexpr (I4) {
                wide = fmaxf(wide, __shfl_xor(wide, 32, 64));
                const float r = fmaxf(ref, __uint_as_float(__float_as_uint(wide) & 0x7F800000u));
                f *= ref == r ? 1.f : ref / r;
                ref = r;
                ref_inv = r > 0.f ? 1.f / r : 0.f;
            }
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= f;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 pw;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = sc[u][8 * s + j], e = exp2_fast(I4 ? x - m : fmaf(x, f_log2, -m));
                    sc[u][8 * s + j] = e;
                    l += e;
                }
                if constexpr (I4) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f32x4 s4 = *reinterpret_cast<const f32x4*>(&sm.vs[buf][32 * u + 16 * s + 8 * i + 4 * half]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[u][8 * s + 4 * i + j] *= s4[j] * ref_inv;
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) pw[j] = pack_f16(sc[u][8 * s + 2 * j], sc[u][8 * s + 2 * j + 1]);
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const u32x4 vv = *reinterpret_cast<const u32x4*>(&sm.v[buf][((2 * (2 * u + s) + half) * D + 32 * i + r32) * 16]);
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, vv), __builtin_bit_cast(f16x8, pw), o[i], 0, 0, 0);
                }
            }
        if (t + 1 < t1) store_tile(t + 1, buf ^ 1);
        if (t + 2 < t1) load_tile(t + 2);
        __syncthreads();
    }

    l += __shfl_xor(l, 32, 64);
    if (!valid) return;
    // slot 32 i + r of the values is d = 4 (slot % (D / 4)) + slot / (D / 4), and
    // the lane's rows r = 8 x + 4 half + y: 4 consecutive d for every (x, y)
    float f = 1.f;
    if constexpr (I4) f = ref;
    if (S == 1) f *= l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (D == 128 ? o[e % DT][4 * x + y] : o[e >> 1][4 * x + 8 * (e & 1) + y]) * f;
            const int d = 4 * (8 * x + 4 * half + y);
            if (S == 1) {
                *reinterpret_cast<u32x2*>(a.out + row * D + d) = u32x2{pack_f16(v[0], v[1]), pack_f16(v[2], v[3])};
            } else {
                *reinterpret_cast<f32x4*>(part + (row * S + split) * D + d) = f32x4{v[0], v[1], v[2], v[3]};
            }
        }
    if (S > 1 && half == 0) {
        ml[(row * S + split) * 2] = m;
        ml[(row * S + split) * 2 + 1] = l;
    }
}

struct Plan {
    int row_tiles;
    int S;
};

// The tiles are split where the workgroups number fewer than the compute
// units, into parts of at least four tiles, up to two workgroups a unit.
Plan plan_prefill(const KvView& c, const AttnArgs& a) {
    Plan p;
    const int64_t group = a.heads / c.kv_heads;
    p.row_tiles = static_cast<int>((a.max_q * group + kRows - 1) / kRows);
    const int64_t most = std::min<int64_t>(c.max_len, static_cast<int64_t>(c.width) << c.page_shift);
    int64_t tiles = (most + kW - 1) / kW;
    if (a.window) {
        const int64_t tokens = std::min<int64_t>(a.max_q, (kRows - 1) / group + 2);  // new tokens of a row tile
        const int64_t w = (static_cast<int64_t>(a.window) + tokens + kW - 2) / kW + 1 + (static_cast<int64_t>(a.sinks) + kW - 1) / kW;
        tiles = std::min(tiles, w);
    }
    const int64_t units = static_cast<int64_t>(c.B) * c.kv_heads * p.row_tiles;
    const int cu = device_cu_count();
    int64_t S = 1;
    if (units < cu) S = std::min<int64_t>((2 * cu + units - 1) / units, tiles / 4);
    p.S = static_cast<int>(std::min<int64_t>(std::max<int64_t>(S, 1), 128));
    return p;
}

int64_t blocks_of(const KvView& c, const Plan& p) {
    return static_cast<int64_t>(c.B) * c.kv_heads * p.row_tiles * p.S;
}

}  // namespace

int64_t attn_prefill_workspace(const KvView& c, const AttnArgs& a) {
    const Plan p = plan_prefill(c, a);
    if (blocks_of(c, p) > 0x7FFFFFFFll) return -1;
    return p.S == 1 ? 0 : a.T * a.heads * p.S * static_cast<int64_t>(c.D + 2) * 4;
}

hipError_t launch_attn_prefill(const KvView& c, const AttnArgs& a, hipStream_t stream) {
    const Plan p = plan_prefill(c, a);
    float* part = static_cast<float*>(a.workspace);
    float* ml = part + a.T * a.heads * p.S * c.D;
    auto run = [&](auto kernel, int lds, std::atomic<uint64_t>& done) {
        const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, done);
        if (e != hipSuccess) return e;
        kernel<<<static_cast<unsigned>(blocks_of(c, p)), kThreads, lds, stream>>>(c, a, p.S, p.row_tiles, part, ml);
        return hipGetLastError();
    };
    static std::atomic<uint64_t> done[4];
    hipError_t e;
    if (c.D == 128)
        e = c.i4 ? run(attn_prefill_kernel<128, true>, sizeof(Smem<128, true>), done[0])
                 : run(attn_prefill_kernel<128, false>, sizeof(Smem<128, false>), done[1]);
    else
        e = c.i4 ? run(attn_prefill_kernel<64, true>, sizeof(Smem<64, true>), done[2])
                 : run(attn_prefill_kernel<64, false>, sizeof(Smem<64, false>), done[3]);
    if (e != hipSuccess || p.S == 1) return e;
    return launch_attn_join(part, ml, a.T * a.heads, p.S, c.D, a.out, stream);
}

}  // namespace apex4
