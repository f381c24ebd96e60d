// Attention of packed new tokens over the paged cache (prompts, chunks of them,
// a few tokens at a time): causal, with or without a sliding window and first
// positions that stay visible.
//
// One pass over the positions with the running maximum and sum of the softmax.
// A workgroup takes 128 or 256 rows of one key head (a row is a new token and one
// of the query heads that share the key head, so that few tokens still fill it)
// and the tiles of 64 positions that any of them sees; a wave takes 32 rows,
// with q and the output sums in registers.
//   S^T = K Q^T   32 x 32 x 16 products: a lane holds 16 positions of one row
//                 in each of the tile's two halves, so the softmax needs no
//                 other lane but lane ^ 32, and that only when the maximum is
//                 raised (kSlack) and at the end;
//   O^T = V^T P^T the scores' layout, rounded to binary16, is the right operand
//                 as it stands: position 16 s + 8 (j / 4) + 4 h + j % 4 is
//                 element j of lane half h in step s.
// Keys and values go into LDS as they lie in a page, by loads that pass no
// register; only the 16-byte pieces of a position change places, so that neither
// the keys' reads nor the transposing reads of the values meet in a bank.  The
// loads of the next tile are in flight during a tile's products, and its first
// products run beside the tile's exponentials; two buffers, one barrier a tile.
// 4-bit codes become small integers in binary16 (exact) on their way into LDS,
// through registers; a position's scales multiply its scores and weights in 32
// bits.  The weights are rounded to binary16 for the second product (2^-11 of
// each), the sums of scores, weights and outputs are of 32 bits.
// With few rows and a long cache the tiles of a workgroup are cut into S parts,
// joined by the kernel that joins those of attn_decode.hip.
//
// Bound by the matrix cores and, next to them, the vector units: a tile's 32 products
// take a wave 1024 cycles of its SIMD's matrix core, its exponentials (16 cycles each),
// their arguments, maxima and sums about 830 of the vector unit.  A prompt of 8192
// tokens, 64 query heads of 128: 1.04 to 1.10 ms, 1000 to 1055 TFLOP/s of the 1343 that
// a product of 8192^3 reaches, at a clock that falls with the load (queries of zero,
// which cost less power: 0.85 ms).  No faster: three and four buffers, two halves of the
// waves half a step apart, 64 rows a wave, fragments read further ahead, wave
// priorities.  Codes: some 16 % more a tile, for putting them into LDS and for the scales
// (the prompt 1.24 to 1.26 ms; 2048 new tokens of 2 sequences of 8192 under a window of 1024: 207
// us, binary16 177); multiplications left out to see, and the conversion elsewhere in
// the step changed nothing.  Heads of 64: the prompt 0.61 ms, codes 0.97; the window 99
// and 160 us.
#include "attn_core.h"

namespace apex4 {
namespace {

using namespace attn;

constexpr int kShift = 6, kW = 1 << kShift;  // positions of a tile

// Keys and values of a tile lie in LDS as they lie in a binary16 page, a row of D
// values a position, but with the 16-byte pieces of a row exchanged (piece c at
// c ^ the numbers below), so that the 16 lanes that read at a time find theirs in
// different banks: 16 positions' piece c of the keys; and of the values 32
// bytes of 4 positions next to 32 other bytes of the same (the transposing read).
// Codes are written a piece of 4 (D = 64: 8) positions at a time, which the low bits
// of both numbers keep apart (1 % of the time over an int4 cache).
template <int D>
__device__ __forceinline__ int k_swizzle(int t) { return D == 128 ? (t & 15) : ((t >> 1) & 7); }
template <int D>
__device__ __forceinline__ int v_swizzle(int t) { return D == 128 ? 5 * (t & 3) : ((t & 2) << 1) ^ ((t >> 1) & 3); }

template <int D, bool I4, int kWaves>
struct Smem {
    uint8_t k[2][kW * D * 2];
    uint8_t v[2][kW * D * 2];
    // scales, the softmax's factor in the keys'; those of the keys of tile t are read in
    // step t, beside the writing of tile t + 2's: four slots
    float ks[4][I4 ? kW : 4];
    float vs[2][I4 ? kW : 4];
    float vl[2][I4 ? kW : 4];  // log2 of the values', for a row's maximum
    uint32_t vs_most[4];       // the largest of a tile's, as bits; a tile's slot is cleared two steps before it is written
};

typedef __attribute__((address_space(3))) uint8_t lds_u8;
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u8*)p));
}

// 16 bytes a lane from base + off straight into LDS at `to` + 16 lane.  The
// compiler does not see these loads: landed() waits for all of them.  (The wait
// states let M0, and a base that came out of a vector instruction, settle.)  M0 is
// among the clobbers, so that no setting of the compiler's own is taken to outlive the
// statement; it warns that it reserves the register, and so has none to save.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(uint32_t to, uint32_t off, const uint8_t* base) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off),
                 "s"(static_cast<uint64_t>(hi) << 32 | lo)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// 4 positions' value d for the lane's d: lanes 4 j + i of 16 point at 4 values
// each of position j, and the lane numbered n gets the n-th of the 16 of all four.
__device__ __forceinline__ u32x2 read_transposed(uint32_t at) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4*)static_cast<uintptr_t>(at)));
}
__device__ __forceinline__ u32x4 read_lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) u32x4*)static_cast<uintptr_t>(at);
}
__device__ __forceinline__ void write_lds(uint32_t at, u32x4 v) {
    *(__attribute__((address_space(3))) u32x4*)static_cast<uintptr_t>(at) = v;
}

template <int D, bool I4, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_prefill_kernel(KvView c, AttnArgs a, int S, int row_tiles,
                                                                   float* __restrict__ part, float* __restrict__ ml) {
    constexpr int kRows = 32 * kWaves;
    constexpr int KS = D / 16;        // products along d in the first
    constexpr int DT = D / 32;        // tiles of d in the second
    constexpr int kRow = 2 * D;       // bytes of a position in LDS
    constexpr int kTileBytes = kW * kRow;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem<D, I4, kWaves>& sm = *reinterpret_cast<Smem<D, I4, kWaves>*>(smem_raw);

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r32 = lane & 31, half = lane >> 5;
    uint32_t id = workgroup_number();
    const int h = static_cast<int>(id % c.kv_heads);  // workgroups of one key head on one XCD's L2 where the heads allow it
    id /= c.kv_heads;
    const int split = static_cast<int>(id % S);
    id /= S;
    // The longest sequences first (among 64 next to each other), and of each the last
    // rows, which see the most: what starts late is short.  (In the order given, six
    // ragged chunks took 137 us instead of 96.)
    int b = static_cast<int>(id / row_tiles);
    if (b >= c.B) return;
    const int from_last = static_cast<int>(id) - b * row_tiles;
    int q0, n, len;
    {
        const int first = b & ~63, many = min(c.B - first, 64), x = first + min(lane, many - 1);
        const int mine = cached_tokens(c, x), q_mine = a.q_start[x], n_mine = new_tokens(a, x);
        int rank = 0;
        for (int i = 0; i < many; ++i) {
            const int other = __builtin_amdgcn_readlane(mine, i);
            rank += other > mine || (other == mine && i < lane);
        }
        const int at = __builtin_ctzll(__ballot(lane < many && rank == b - first));  // one lane has each rank
        b = first + at;
        q0 = __builtin_amdgcn_readlane(q_mine, at);
        n = __builtin_amdgcn_readlane(n_mine, at);
        len = __builtin_amdgcn_readlane(mine, at);
    }
    const uint32_t group = a.group;

    // past max_q tokens nothing is computed; T heads and max_q heads are below 2^28
    const uint32_t rows = min(n, static_cast<int>(a.max_q)) * group;
    const int mt = static_cast<int>((rows + kRows - 1) / kRows) - 1 - from_last;
    if (mt < 0) return;
    const uint32_t R0 = mt * kRows;
    const int before = len - n;  // position of the sequence's first new token (negative: it has no place)
    const uint32_t tok0 = R0 / group;
    const int p_lo = before + static_cast<int>(tok0);
    const int p_hi = before + static_cast<int>(((R0 + kRows < rows ? R0 + kRows : rows) - 1) / group);
    const Tiles<kW> tiles(p_lo, p_hi, a.window, a.sinks);
    // the split's share of the tiles (below 2^24 of them, S below 2^8)
    const int t0 = S == 1 ? 0 : static_cast<uint32_t>(tiles.count) * split / static_cast<uint32_t>(S);
    const int t1 = S == 1 ? tiles.count : static_cast<uint32_t>(tiles.count) * (split + 1) / static_cast<uint32_t>(S);

    // the lane's row
    const uint32_t r_wave = R0 - tok0 * group + 32 * wave;  // of the tile's first token
    struct Row {
        int tok, head;
        bool valid;
    };
    auto row_of = [&](int r) {
        Row x;
        const uint32_t t = (r_wave + r) / group;
        x.tok = tok0 + t;
        x.head = h * group + (r_wave + r - t * group);
        x.valid = R0 + 32 * wave + r < rows && q0 >= 0 && q0 + x.tok < a.T;
        return x;
    };
    const bool idle = R0 + 32 * wave >= rows;  // a wave without rows only stages
    int pos;
    u32x4 qf[KS];  // right operand: d = 16 s + 8 half ..
    {
        const Row x = row_of(r32);
        pos = before + x.tok;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qf[s] = u32x4{0u, 0u, 0u, 0u};
            if (x.valid) qf[s] = *reinterpret_cast<const u32x4*>(a.q + (q0 + x.tok) * a.q_stride + x.head * D + 16 * s + 8 * half);
            if constexpr (I4) qf[s] = code_order(qf[s]);
        }
    }

    // Values that a thread could keep over the loop are made anew from this (a
    // few instructions a tile): the registers are worth more.
    auto anew = [](uint32_t x) {
        asm("" : "+v"(x));
        return static_cast<int>(x);
    };
    const float to_log2 = a.scale * kLog2e;
    const int page_mask = (1 << c.page_shift) - 1;
    const int64_t head_at = static_cast<int64_t>(h) << c.page_shift;
    const int64_t scale_at = (static_cast<int64_t>(c.kv_heads) << c.page_shift) * (D / 2);
    const uint32_t k_lds = lds_offset(sm.k), v_lds = lds_offset(sm.v);
    const uint32_t ks_lds = lds_offset(sm.ks), vs_lds = lds_offset(sm.vs), vl_lds = lds_offset(sm.vl);

    // positions that no row of the workgroup sees hold anything: their values,
    // times a weight of zero, must not count
    auto seen_by_some = [&](int t) { return t <= p_hi && (t >= tiles.lo || t < tiles.sinks); };
    // Which tiles have such positions (the last, and those at the end of the sinks and
    // the window's start), and which hold positions that some row does not see: by
    // numbers worked out once, for a step has no scalar instructions to spare.
    const int edge = tiles.n_sink + ((p_hi + 1) >> kShift) - tiles.first;
    auto at_edge = [&](int t) { return t >= edge || static_cast<uint32_t>(t - tiles.n_sink + 1) < 2u; };
    const int whole_to = tiles.n_sink + ((p_lo + 1) >> kShift) - tiles.first;
    const int whole_from = a.window ? tiles.n_sink + ((p_hi - a.window) >> kShift) + 1 - tiles.first : 0;
    const int whole_sinks = a.window ? tiles.sinks >> kShift : 0;
    auto late = [&](int t) { return t >= whole_to; };  // some of its positions are past some row
    auto early = [&](int t) { return t < whole_from && t >= whole_sinks; };  // or before its window
    // Staging.  begin_k/v(t) sends the loads of tile t out, end_k/v(t, buf) has it
    // in LDS before the next barrier.
    // binary16: every 1 KB that a wave copies is kPos positions of 16 (one page)
    constexpr int kPos = 1024 / kRow;          // 4 (D = 128) or 8
    constexpr int kCopies = kW / kPos / kWaves;  // 4 or 2
    constexpr int kPieces = kRow / 16;
    const int c_pos = lane / kPieces, c_slot = lane % kPieces;
    auto first_of = [&](int i) { return kPos * (kWaves * i + wave); };
    const uint32_t k_off = c_pos * kRow + 16 * (c_slot ^ k_swizzle<D>(kPos * wave + c_pos));
    const uint32_t v_off = c_pos * kRow + 16 * (c_slot ^ v_swizzle<D>(c_pos));
    // int4: a thread takes 16 bytes, 32 codes, of one position; the first four
    // waves the keys', the others the values'
    constexpr int kLanes = D / 32;
    static_assert(!I4 || kWaves == 8, "four waves for the keys, four for the values");
    const bool i_values = wave >= 4;
    const int i_pos = (tid & 255) / kLanes, i_part = tid % kLanes;
    const bool i_thread = i_pos < kW;
    u32x4 i_codes;
    uint16_t i_scale = 0;

    // The pages of what a wave, or a thread, loads of a tile: ids are looked up a
    // step before they are needed, and make the places of a tile's keys, then of its
    // values.
    constexpr int kIds = I4 ? 1 : kCopies;
    struct Ids {
        int page[kIds];
    };
    const bool one_page = c.page_shift >= 6;  // a tile lies in one page
    struct Places {
        int64_t at[kIds];
        int64_t scale;
    };
    typedef const __attribute__((address_space(4))) int32_t table_i32;
    const __attribute__((address_space(4))) uint8_t* table =
        (const __attribute__((address_space(4))) uint8_t*)(c.table + static_cast<int64_t>(b) * c.width);
    const uint32_t page_bytes = static_cast<uint32_t>(c.page_bytes);  // at most 2^30
    auto first = [&](int i) { return I4 ? i_pos & (kW - 1) : first_of(i); };
    auto look_up = [&](int t) {
        const int at = tiles.start(t);
        Ids r;
#pragma unroll
        for (int i = 0; i < kIds; ++i) {
            if (i && one_page) break;
            const uint32_t p = static_cast<uint32_t>(at + first(i)) >> c.page_shift, most = c.width - 1;
            r.page[i] = *reinterpret_cast<table_i32*>(table + 4 * (p < most ? p : most));  // below 2^22 bytes
        }
        return r;
    };
    // positions past the last page are masked, and read page 0
    auto places = [&](int t, const Ids& ids) {
        const int at = tiles.start(t);
        Places r;
#pragma unroll
        for (int i = 0; i < kIds; ++i) {
            if (i && one_page) {
                r.at[i] = r.at[0] + kPos * kWaves * kRow * i;
                continue;
            }
            const uint32_t p = static_cast<uint32_t>(ids.page[i]) < static_cast<uint32_t>(c.n_pages) ? ids.page[i] : 0;
            const uint32_t x = static_cast<uint32_t>(head_at) + ((at + first(i)) & page_mask);
            const uint64_t page = static_cast<uint64_t>(p) * page_bytes;
            r.at[i] = page + x * (I4 ? D / 2 : kRow);
            if constexpr (I4) r.scale = page + static_cast<uint32_t>(scale_at) + 2 * x;
        }
        return r;
    };
    // Sends out tile t's loads, and has what they brought in LDS before the next
    // barrier (values of positions that nobody sees as zeros).
    auto begin_copies = [&](int buf, const Places& at, const uint8_t* plane, uint32_t lds, uint32_t off) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(lds + buf * kTileBytes + first_of(i) * kRow, off, plane + at.at[i]);
    };
    auto clear_unseen = [&](int t, int buf) {  // a wave clears what it copied itself
        if (!at_edge(t)) return;
        const int at = tiles.start(t);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int x = first_of(i);
            if (!seen_by_some(at + x + c_pos)) write_lds(v_lds + buf * kTileBytes + x * kRow + 16 * lane, u32x4{0u, 0u, 0u, 0u});
        }
    };
    auto begin_codes = [&](const Places& at) {
        if (i_thread) {
            const uint8_t* plane = i_values ? c.v : c.k;
            i_codes = *reinterpret_cast<const u32x4*>(plane + at.at[0] + 16 * i_part);
            i_scale = *reinterpret_cast<const uint16_t*>(plane + at.scale);
        }
    };
    // A piece, 8 codes, stays in the order of codes_f16 (code i, code i + 4, ..): q has
    // the same (code_order), and of the values it shows in the rows of the sums.  The
    // tile's largest scale is an atomic maximum, the same whatever the order: every
    // wave waits for the values' four, and a reduction by shuffles and the values'
    // reordering had them take twice as long as the keys' (8192 tokens: 1270 us, 1200 so).
    const uint32_t least = __builtin_bit_cast(uint32_t, 0x1p-24f);  // a scale of zero leaves the sum of the weights alone to grow
    auto end_codes = [&](int t, int buf) {
        const int i_pos = (anew(tid) & 255) / kLanes, i_part = anew(tid) % kLanes;
        const bool i_thread = i_pos < kW;
        if (i_thread) {
            const uint32_t to = (i_values ? v_lds : k_lds) + buf * kTileBytes + i_pos * kRow;
            const int number = i_values ? v_swizzle<D>(i_pos) : k_swizzle<D>(i_pos);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[4];
                codes_f16(i_codes[j], w);
                write_lds(to + 16 * ((4 * i_part + j) ^ number), u32x4{w[0], w[1], w[2], w[3]});
            }
            if (i_part == 0) {
                const float x = half_of(i_scale, 0);
                if (!i_values) {
                    sm.ks[t & 3][i_pos] = x * to_log2;
                } else {
                    const float scale = seen_by_some(tiles.start(t) + i_pos) ? x : 0.f;
                    sm.vs[buf][i_pos] = scale;
                    sm.vl[buf][i_pos] = __builtin_amdgcn_logf(fmaxf(scale, 0x1p-24f));
                    atomicMax(&sm.vs_most[anew(t & 3)], __builtin_bit_cast(uint32_t, fmaxf(scale, 0.f)));  // not negative: bits are in order
                }
            }
        }
        if (tid == 256) sm.vs_most[(t + 1) & 3] = least;
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float m = kNoMax, l = 0.f;

    const uint32_t k_read = k_lds + r32 * kRow + 16 * (half ^ k_swizzle<D>(r32));
    // the transposing read: 16 lanes at 4 positions' 32 bytes of d = 32 i + 16 (lane / 16 % 2) ..
    const uint32_t v_read = v_lds + (4 * half + ((lane & 15) >> 2)) * kRow +
                            ((32 * ((lane >> 4) & 1) + 8 * (lane & 3)) ^ (16 * v_swizzle<D>(4 * half + ((lane & 15) >> 2))));

    // Fragments of the products, a quarter of a tile's at a time: KS / 4 steps of
    // d for both halves of the keys, one step of 16 positions for all values d.
    constexpr int KQ = KS / 4;
    struct KeyFrags {
        u32x4 f[KQ][2];
    };
    struct ValueFrags {
        u32x4 f[DT];
    };
    auto read_k = [&](int s, uint32_t base) {
        KeyFrags r;
#pragma unroll
        for (int i = 0; i < KQ; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u) r.f[i][u] = read_lds((base ^ (32 * (KQ * s + i))) + 32 * u * kRow);
        return r;
    };
    auto read_v = [&](int s, uint32_t base) {
        ValueFrags r;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const uint32_t p = (base ^ (64 * i)) + 16 * s * kRow;
            const u32x2 v0 = read_transposed(p), v1 = read_transposed(p + 8 * kRow);
            r.f[i] = u32x4{v0[0], v0[1], v1[0], v1[1]};
        }
        return r;
    };
    auto add_scores = [&](f32x16 (&sc)[2], int s, const KeyFrags& k) {
        if (s == 0) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[u][j] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < KQ; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, k.f[i][u]),
                                                               __builtin_bit_cast(f16x8, qf[KQ * s + i]), sc[u], 0, 0, 0);
    };

    // One tile, whose scores are in sc; the next one's products run into next
    // beside the exponentials.
    // Sending the loads out takes some hundred scalar instructions: in the midst of the
    // products they hide (a prompt of 8192 with 64 heads of 128: 1095 us after the third
    // quarter, 1117 at the step's beginning).  Heads of 64, three workgroups a compute
    // unit and shorter steps, want the loads early (ragged chunks: 96 us, 100 later), and
    // so do codes, which the step itself waits for.
    constexpr int kStage = I4 || D == 64 ? 0 : 3;
    Places next_v;  // tile t + 1's values
    Ids ids;        // of tile t + 2 (int4: of t + 1 where the thread stages values)
    auto step = [&](int t, f32x16 (&sc)[2], f32x16 (&next)[2], int buf) {
        const int at = tiles.start(t);
        const int staged = I4 && i_values ? t + 1 : t + 2;
        auto stage = [&] {
            const Places next_k = places(staged, ids);
            if constexpr (I4) {
                if (staged < t1) begin_codes(next_k);
            } else {
                if (t + 2 < t1) begin_copies(buf, next_k, c.k, k_lds, k_off);
                if (t + 1 < t1) begin_copies(buf ^ 1, next_v, c.v, v_lds, v_off);
                next_v = next_k;
            }
            ids = look_up(staged + 1);
        };
        if (kStage == 0 || idle) stage();
        if (!idle) {
            const uint32_t sb = 16 * (anew(tid) >> 5 & 1);
            if constexpr (I4) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 s4 = __builtin_bit_cast(f32x4, read_lds(ks_lds + sb + 4 * kW * (t & 3) + 128 * u + 32 * i));
#pragma unroll
                        for (int j = 0; j < 4; ++j) sc[u][4 * i + j] *= s4[j];
                    }
            }
            const float f_log2 = I4 ? 1.f : to_log2;
            // visible: t <= pos, and t > pos - window or t < sinks; as bounds of t less
            // the lane's first position
            if (late(t)) {
                const int last = pos - at - 4 * (anew(tid) >> 5 & 1);
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int p = 32 * u + 8 * (j >> 2) + (j & 3);
                        sc[u][j] = p <= last ? sc[u][j] : -INFINITY;
                    }
            }
            if (early(t)) {
                const int p0 = at + 4 * (anew(tid) >> 5 & 1), from = pos - a.window + 1 - p0, first = a.sinks - p0;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int p = 32 * u + 8 * (j >> 2) + (j & 3);
                        const bool seen = (p >= from) | (p < first);
                        sc[u][j] = seen ? sc[u][j] : -INFINITY;
                    }
            }
            float top = sc[0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = fmaxf(top, sc[u][j]);
            // how far the row's largest weight would be above 1, in units of log2: of scores
            // of any magnitude (differences are taken first, or inside one fma)
            float rise, most_vl = 0.f;
            if constexpr (I4) {
                // A bound of the scores plus log2 of their values' scales; where it passes
                // the slack, their maximum for each row.  The bound is none: its scale may
                // be that of a position without weight, or of one that the row does not
                // see, and under it the row's weights would fall below what binary16
                // holds.  (The windowed case above 203 -> 207 us; in the same branch as
                // the rescale 12 more, for the compiler then copies the output sums every
                // tile; with the logarithms taken here 4 more.)
                most_vl = __builtin_amdgcn_logf(__builtin_bit_cast(float, sm.vs_most[t & 3]));
                rise = (top - m) + most_vl;
                if (__any(rise > kHeadroom + kSlack)) {
                    most_vl = kNoMax;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const f32x4 vl = __builtin_bit_cast(f32x4, read_lds(vl_lds + sb + 4 * kW * buf + 32 * i));
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            most_vl = fmaxf(most_vl, (sc[i >> 2][4 * (i & 3) + j] - top) + vl[j]);
                    }
                    rise = (top - m) + most_vl;
                }
            } else {
                rise = fmaf(top, f_log2, -m);
            }
            // Only the rows that need it are raised: what a row gives does not depend on
            // what others of its wave see.
            if (const uint64_t over = __ballot(rise > kHeadroom + kSlack)) {
                top = I4 ? top + (most_vl - kHeadroom) : fmaf(top, f_log2, -kHeadroom);
                top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
                top = (over >> (anew(tid) & 31) & 0x100000001ull) ? top : m;
                const float f = exp2_fast(m - top);
                l *= f;
                m = top;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= f;
            }
            // the next tile's products (past the last tile: of whatever lies there, and
            // not used) a quarter at a time beside a quarter of the exponentials
            // A tile's weights are summed first: added one by one to the sum of a long
            // length, small ones would all be rounded the same way.
            float sum = 0.f;
            u32x4 pw[4];
            const uint32_t kb = anew(k_read + (buf ^ 1) * kTileBytes), vb = anew(v_read + buf * kTileBytes);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                add_scores(next, s, read_k(s, kb));
                if (s + 1 == kStage) stage();
                float e[8];
                f32x4 sv[2];
                if constexpr (I4) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) sv[i] = __builtin_bit_cast(f32x4, read_lds(vs_lds + sb + 4 * kW * buf + 64 * s + 32 * i));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = sc[s >> 1][8 * (s & 1) + j];
                    e[j] = exp2_fast(I4 ? x - m : fmaf(x, f_log2, -m));
                    if constexpr (I4) {
                        sum += e[j];
                        e[j] *= sv[j >> 2][j & 3];
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t p = pack_f16(e[2 * j], e[2 * j + 1]);
                    if constexpr (!I4) sum = add_pair(p, sum);  // the rounded weights: one large weight's rounding cancels
                    pw[s][j] = p;
                }
            }
            l += sum;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const ValueFrags vf = read_v(s, vb);
#pragma unroll
                for (int i = 0; i < DT; ++i)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, vf.f[i]), __builtin_bit_cast(f16x8, pw[s]), o[i], 0, 0, 0);
            }
        }
        if constexpr (I4) {
            if (staged < t1) end_codes(staged, i_values ? buf ^ 1 : buf);
        } else {
            landed();
            if (t + 1 < t1) clear_unseen(t + 1, buf ^ 1);
        }
        __syncthreads();
    };

    f32x16 s0[2], s1[2];
    if (t0 < t1) {
        ids = look_up(t0);
        if constexpr (I4) {
            next_v = places(t0, ids);
            begin_codes(next_v);
            if (tid < 4) sm.vs_most[tid] = least;
            __syncthreads();
            end_codes(t0, 0);
            if (!i_values && t0 + 1 < t1) {
                begin_codes(places(t0 + 1, look_up(t0 + 1)));
                end_codes(t0 + 1, 1);
            }
            ids = look_up(i_values ? t0 + 1 : t0 + 2);
        } else {
            const Ids ids1 = look_up(t0 + 1), ids2 = look_up(t0 + 2);
            next_v = places(t0, ids);
            begin_copies(0, next_v, c.k, k_lds, k_off);
            begin_copies(0, next_v, c.v, v_lds, v_off);
            next_v = places(t0 + 1, ids1);
            if (t0 + 1 < t1) begin_copies(1, next_v, c.k, k_lds, k_off);
            ids = ids2;
            landed();
            clear_unseen(t0, 0);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s) add_scores(s0, s, read_k(s, k_read));
        __syncthreads();  // the keys' first buffer is free
        for (int t = t0; t < t1; t += 2) {
            step(t, s0, s1, 0);
            if (t + 1 < t1) step(t + 1, s1, s0, 1);
        }
    }

    l += __shfl_xor(l, 32, 64);
    if (idle) return;
    const int ln = anew(tid) & 63, r = ln & 31, h8 = ln >> 5;
    const Row x = row_of(r);
    const int row = (q0 + x.tok) * a.heads + x.head;  // below 2^27 where it is valid
    // the lane's rows of the sums are d = 32 i + 8 k + 4 half + y, of codes in their order
    if (S == 1) {
        // through LDS (the tiles are used, a wave has 32 rows of it), so that a row goes out
        // in one piece.  (8 bytes a lane to 32 rows at a time: the windowed case above took 241
        // us, 226 so.)
        const float f = l != 0.f ? 1.f / l : 0.f;
        auto piece_of = [&](int r, int c) { return wave * 32 * kRow + r * kRow + 16 * (c ^ (D == 128 ? r & 15 : r >> 1 & 7)); };
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = o[i][4 * k + y] * f;
                uint8_t* to = smem_raw + piece_of(r, 4 * i + k);
                if constexpr (I4) {  // d = 8 k + 2 half, + 4, + 1, + 5
                    *reinterpret_cast<uint32_t*>(to + 4 * h8) = pack_f16(v[0], v[2]);
                    *reinterpret_cast<uint32_t*>(to + 8 + 4 * h8) = pack_f16(v[1], v[3]);
                } else {
                    *reinterpret_cast<u32x2*>(to + 8 * h8) = u32x2{pack_f16(v[0], v[1]), pack_f16(v[2], v[3])};
                }
            }
        const int mine = x.valid ? row : -1;
#pragma unroll
        for (int i = 0; i < kPieces / 2; ++i) {
            const int to_r = 64 / kPieces * i + ln / kPieces, c = ln % kPieces, to = __shfl(mine, to_r, 64);
            const u32x4 v = *reinterpret_cast<const u32x4*>(smem_raw + piece_of(to_r, c));
            if (to >= 0) *reinterpret_cast<u32x4*>(a.out + static_cast<int64_t>(to) * D + 8 * c) = v;
        }
        return;
    }
    if (!x.valid) return;
    const int64_t at = static_cast<int64_t>(row) * S + split;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float* to = part + at * D + 32 * i + 8 * k;
            const f32x4 v = {o[i][4 * k], o[i][4 * k + 1], o[i][4 * k + 2], o[i][4 * k + 3]};
            if constexpr (I4) {
                *reinterpret_cast<f32x2*>(to + 2 * h8) = f32x2{v[0], v[2]};
                *reinterpret_cast<f32x2*>(to + 4 + 2 * h8) = f32x2{v[1], v[3]};
            } else {
                *reinterpret_cast<f32x4*>(to + 4 * h8) = v;
            }
        }
    if (h8 == 0) {
        ml[at * 2] = m;
        ml[at * 2 + 1] = l;
    }
}

struct Plan {
    int waves;
    int row_tiles;
    int S;
};

// Eight waves (256 rows, half the staging a row) where that leaves four workgroups a
// compute unit of 12 tiles or more, and always for codes (64 query heads of 128 over 8
// key heads: 8192 tokens 1082 -> 1044 us, 2 x 2048 tokens of 8192 under a window of 1024
// 183 -> 177); four otherwise: two workgroups a unit hide each other's beginnings and
// even out the last round (4 x 1024 tokens, two a unit: 63 us, 68).  The
// tiles are split where the workgroups number fewer than the compute units, into
// parts of at least four tiles, as many as the units hold at once and no more (32
// rows of 7954 positions: 4 parts 94 us, 5 parts 120).
Plan plan_prefill(const KvView& c, const AttnArgs& a) {
    Plan p;
    const int64_t group = a.heads / c.kv_heads, cu = device_cu_count();
    const int64_t heads = static_cast<int64_t>(c.B) * c.kv_heads;
    const int64_t most = std::min<int64_t>(c.max_len, static_cast<int64_t>(c.width) << c.page_shift);
    int64_t tiles = (most + kW - 1) / kW;
    if (a.window) {
        const int64_t tokens = std::min<int64_t>(a.max_q, 255 / group + 2);  // new tokens of a row tile, at most
        const int64_t w = (static_cast<int64_t>(a.window) + tokens + kW - 2) / kW + 1 + (static_cast<int64_t>(a.sinks) + kW - 1) / kW;
        tiles = std::min(tiles, w);
    }
    p.waves = c.i4 || (c.D == 128 && tiles >= 12 && heads * ((a.max_q * group + 255) / 256) >= 4 * cu) ? 8 : 4;
    const int64_t rows = 32 * p.waves;
    p.row_tiles = static_cast<int>((a.max_q * group + rows - 1) / rows);
    const int64_t units = heads * p.row_tiles;
    int64_t S = 1;
    const int64_t held = p.waves == 8 ? cu : (c.D == 64 ? 3 : 2) * cu;  // workgroups that run at once
    if (units < cu) S = std::min<int64_t>(held / units, tiles / 4);
    p.S = static_cast<int>(std::min<int64_t>(std::max<int64_t>(S, 1), 128));
    return p;
}

// Rows (new tokens times the heads that share a key head) up to which the decode
// kernel, 16 at a time, is the faster one.  It reads the cache once for every 16 rows
// (from the L2 after the first), this one once, but this one makes codes binary16 in
// LDS by a workgroup whose products are few.  The decode kernel's time against this
// one's in us, 14 sequences of 7954 | 14 of 600 | 64 of 600; 8 key heads, 64 query heads
// unless 32 of each are said:
//   binary16, D = 128, 16 rows   94, 96 | 12, 17 | 27, 32     32 of each 360, 344 | 24, 28 | 121, 137
//                      32 rows  141, 97 | 15, 17 | 49, 33                523, 344 | 45, 28 | 186, 143
//             D = 64,  16 rows   42, 43 |  8, 14 | 17, 20                187, 158 | 15, 17 |  56,  71
//                      32 rows   76, 45 |  9, 13 | 27, 21                268, 158 | 25, 18 |  94,  74
//   int4,     D = 128, 64 rows   82, 109 | 13, 19 | 36, 50               291, 394 | 30, 46 | 113, 189
//                     128 rows  154, 115 | 21, 25 | 62, 54               526, 407 | 53, 49 | 221, 212
//             D = 64,  64 rows   53, 99  |  9, 18 | 24, 44               186, 356 | 22, 39 |  79, 169
//                     128 rows   94, 101 | 14, 22 | 42, 46               345, 356 | 38, 42 | 154, 174
bool few_rows(const KvView& c, const AttnArgs& a) { return a.max_q * (a.heads / c.kv_heads) <= (c.i4 ? 64 : 16); }

int64_t blocks_of(const KvView& c, const Plan& p) {
    return static_cast<int64_t>(c.B) * c.kv_heads * p.row_tiles * p.S;
}

template <int D, bool I4, int kWaves>
hipError_t run(const KvView& c, const AttnArgs& a, const Plan& p, float* part, float* ml, hipStream_t stream) {
    static std::atomic<uint64_t> done;
    constexpr int lds = sizeof(Smem<D, I4, kWaves>);
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(attn_prefill_kernel<D, I4, kWaves>), lds, done);
    if (e != hipSuccess) return e;
    attn_prefill_kernel<D, I4, kWaves><<<grid_of(blocks_of(c, p)), 64 * kWaves, lds, stream>>>(c, a, p.S, p.row_tiles, part, ml);
    return hipGetLastError();
}

}  // namespace

int64_t attn_prefill_workspace(const KvView& c, const AttnArgs& a) {
    if (few_rows(c, a)) return attn_decode_workspace(c, a);
    const Plan p = plan_prefill(c, a);
    if (blocks_of(c, p) > 0x7FFFFFFFll) return -1;
    return p.S == 1 ? 0 : a.T * a.heads * p.S * static_cast<int64_t>(c.D + 2) * 4;
}

hipError_t launch_attn_prefill(const KvView& c, const AttnArgs& a, hipStream_t stream) {
    if (few_rows(c, a)) return launch_attn_decode(c, a, stream);
    const Plan p = plan_prefill(c, a);
    float* part = static_cast<float*>(a.workspace);
    float* ml = part + a.T * a.heads * p.S * c.D;
    const auto kernel = c.D == 64 ? (c.i4 ? run<64, true, 8> : run<64, false, 4>)
                        : c.i4    ? run<128, true, 8>
                                  : (p.waves == 8 ? run<128, false, 8> : run<128, false, 4>);
    const hipError_t e = kernel(c, a, p, part, ml, stream);
    if (e != hipSuccess || p.S == 1) return e;
    return launch_attn_join(part, ml, a.T * a.heads, p.S, c.D, a.out, stream);
}

}  // namespace apex4
