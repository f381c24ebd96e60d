// Y = binary16(s_a s_w sum_k A W) of 8-bit codes, many rows.
//
// A workgroup takes BM x BN outputs and goes over K in stages of 128 bytes; rows of
// A and W are copied straight into LDS (16 bytes a lane, no register), two to six buffers.
// A wave owns TM x TN outputs as 32 x 32 blocks of v_mfma_i32_32x32x32_i8 (weights the
// rows, tokens the columns, so that a lane holds neighbouring channels of one token).  The
// sums are whole numbers below 2^31 in any order (K is bounded), so outputs do not depend on
// the tile: the sum to binary32, times s_a, times s_w, each rounded, and then to binary16.
//
// Many rows are bound by the matrix cores and the power that they draw: 4096 x 10240 of
// K 8192 292 to 303 us, by card, 2.3e15 operations a second at about 1.5 GHz; 8192^3 485 us with the matrix
// cores 0.70 busy.  Steps there: all loads in a burst behind the barrier 507 us (0.59 busy),
// spread among the products 502 (0.64), no branches in the loop and the barrier in the
// midst of the last step's products 485; stages of 64 bytes in four buffers 513, four waves
// of 128 x 128 instead of eight 538.
// A few hundred rows are bound by what one compute unit draws: 300 x 10240 of K 8192 takes 38
// us, 64 stages of 0.55 us, as many with 64 tiles as with 240.  Its loads alone take 35 to
// 40 (55 KB a us; 100 from a warm L2), its products and LDS reads alone 27 to 33.  No gain
// from: four waves or eight, three to five buffers, fragments read a whole stage ahead, K
// begun elsewhere by every tile; a wave that reads W ahead for the tiles that share it: 44 to 48.
// Not tried: larger tiles that each take a part of K, with partial sums to be added.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <atomic>
#include <type_traits>

#include "apex4_internal.h"
#include "quant8_core.h"

namespace apex4 {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
using quant8::u32x2;
typedef __attribute__((address_space(3))) uint8_t lds_u8;

constexpr int kStage = 128;                 // bytes of K a stage
constexpr uint32_t kNowhere = 0x7FFFFFFFu;  // past any buffer: such loads give zeros
constexpr int kRsrcFlags = 0x00027000;      // raw buffer descriptor, 32-bit data format

__device__ __forceinline__ i32x4 descriptor(const void* base, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    i32x4 r;
    r[0] = __builtin_amdgcn_readfirstlane(static_cast<int>(at));
    r[1] = __builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32) & 0xFFFF);
    r[2] = __builtin_amdgcn_readfirstlane(static_cast<int>(bytes));
    r[3] = kRsrcFlags;
    return r;
}

// 16 bytes a lane from the buffer straight into LDS at `to` + 16 lane.  The compiler does
// not see these loads; the wait before the barrier is for all of them.  (The wait states
// let M0 and the descriptor settle.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(uint32_t to, uint32_t off, i32x4 buffer, uint32_t soff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(buffer), "s"(soff)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

__device__ __forceinline__ i32x4 read_lds(uint32_t at) {
    return *(const __attribute__((address_space(3))) i32x4*)static_cast<uintptr_t>(at);
}

// A row's eight 16-byte pieces of a stage lie in LDS in another order, piece c at
// c ^ ((row / 2) % 8): the 16 rows that a read takes at a time find their pieces in
// different banks.
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

template <int N>
__device__ __forceinline__ void landed_but() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

// WM x WN waves; NB: stages in LDS.  AHEAD, for waves of one block and few of them on a compute
// unit: a step's one product is over before the next step's fragments arrive, so those of a
// whole stage are read at once while the stage before is multiplied.  With 64 x 32 tiles: 16
// rows of 8192 channels, K 8192, 17.5 -> 16.1 us, 4112 channels of K 28672 50 -> 42; 64 rows of
// 8192, bound by what a unit draws, 19.0 and 18.9.  Where several workgroups share a unit it
// gives nothing (27 rows of 57344, 32 x 64 tiles: 92 and 96).
template <int BM, int BN, int WM, int WN, int NB, bool AHEAD>
__global__ __launch_bounds__(64 * WM * WN) void w8a8_tile_kernel(const int8_t* __restrict__ A, const float* __restrict__ sa,
                                                                 const int8_t* __restrict__ W, const float* __restrict__ sw, int M,
                                                                 int N, int K, uint16_t* __restrict__ Y) {
    constexpr int kWaves = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 32, NI = TN / 32;
    constexpr int kRows = 8, KK = kStage / 32;  // rows of a load; products' steps
    constexpr int LA = BM / kRows / kWaves, LB = BN / kRows / kWaves;  // loads of a wave and stage
    static_assert(LA * kRows * kWaves == BM && LB * kRows * kWaves == BN && kRows * kWaves % 16 == 0, "whole loads");
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_u8*)smem));
    constexpr uint32_t kBufA = BM * kStage, kBufB = BN * kStage, kBuf = kBufA + kBufB;

    const int mt_count = (M + BM - 1) / BM, nt_count = (N + BN - 1) / BN;
    int mt, nt;
    {
        // each XCD (workgroups go round the eight of them) takes a run of tiles that share
        // rows and columns: bands of up to 8 m-tiles, n within
        const int T = mt_count * nt_count;
        const int x = blockIdx.x & 7, j = blockIdx.x >> 3;
        int t = x * (T >> 3) + min(x, T & 7) + j;
        const int band = t / (8 * nt_count), in = t - band * 8 * nt_count;
        const int rows = min(8, mt_count - band * 8);
        mt = band * 8 + in % rows;
        nt = in / rows;
    }
    const int m0 = mt * BM, n0 = nt * BN;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;

    const i32x4 bufA = descriptor(A + static_cast<int64_t>(m0) * K, static_cast<uint32_t>(min(BM, M - m0)) * static_cast<uint32_t>(K));
    const i32x4 bufB = descriptor(W + static_cast<int64_t>(n0) * K, static_cast<uint32_t>(min(BN, N - n0)) * static_cast<uint32_t>(K));
    const int lrow = wave * kRows + lane / 8;
    const int piece = lane % 8 ^ swizzle(lrow);  // the same for the rows of all loads: they are multiples of 16 apart
    const int stages = (K + kStage - 1) / kStage;
    uint32_t offA[LA], offB[LB];
#pragma unroll
    for (int j = 0; j < LA; ++j) offA[j] = static_cast<uint32_t>(lrow + j * kRows * kWaves) * static_cast<uint32_t>(K) + piece * 16;
#pragma unroll
    for (int j = 0; j < LB; ++j) offB[j] = static_cast<uint32_t>(lrow + j * kRows * kWaves) * static_cast<uint32_t>(K) + piece * 16;
    const bool past = (stages - 1) * kStage + piece * 16 >= K;  // the last stage's pieces behind K
    // load i of stage t: a wave's rows of A, or of W.  TAIL: the stage may be the last one
    // (pieces behind K give zeros), or behind it (nothing is read).
    auto fetch = [&](auto tail, int i, int t) {
        const uint32_t to = lds + t % NB * kBuf + wave * 1024;
        const bool none = tail.value && (t >= stages || (past && t == stages - 1));
        if (i < LA) copy_to_lds(to + i * 1024 * kWaves, none ? kNowhere : offA[i], bufA, t * kStage);
        else copy_to_lds(to + kBufA + (i - LA) * 1024 * kWaves, none ? kNowhere : offB[i - LA], bufB, t * kStage);
    };

    i32x16 acc[NI][MI];
#pragma unroll
    for (int n = 0; n < NI; ++n)
#pragma unroll
        for (int m = 0; m < MI; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] = 0;

    // fragment: row l32 of a block, bytes 32 k + 16 lh of the stage; blocks are a multiple of 32 rows apart
    const uint32_t rowA = lds + (wm * TM + l32) * kStage, rowB = lds + kBufA + (wn * TN + l32) * kStage;
    uint32_t at[KK];
#pragma unroll
    for (int k = 0; k < KK; ++k) at[k] = ((2 * k + lh) ^ swizzle(l32)) * 16;
    constexpr int L = LA + LB;
    const std::true_type yes;
    const std::false_type no;
    if constexpr (AHEAD) {
        static_assert(MI * NI == 1 && KK % 2 == 0 && (NB - 1) * L < 64, "one block, a count that the wait can hold");
        i32x4 f[2][2][KK];
        i32x16 odd;  // every other step's sums: a product does not wait for the one before
#pragma unroll
        for (int i = 0; i < 16; ++i) odd[i] = 0;
        auto read = [&](int set, int buffer) {
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                f[set][0][k] = read_lds(rowB + buffer * kBuf + at[k]);
                f[set][1][k] = read_lds(rowA + buffer * kBuf + at[k]);
            }
        };
        auto fetch_all = [&](auto tail, int t) {
#pragma unroll
            for (int i = 0; i < L; ++i) fetch(tail, i, t);
        };
        for (int t = 0; t < NB; ++t) fetch_all(yes, t);
        landed_but<(NB - 1) * L>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0, 0);
        int b = 0;
        // all of stage s is in registers, the next one has landed; stage s + NB takes its buffer
        auto stage = [&](auto tail, int set, int s) {
            b = b + 1 == NB ? 0 : b + 1;
            landed_but<(NB - 2) * L>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            read(set ^ 1, b);  // behind the last stage what the buffer holds, not used
            fetch_all(tail, s + NB);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KK; k += 2) {
                acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f[set][0][k], f[set][1][k], acc[0][0], 0, 0, 0);
                odd = __builtin_amdgcn_mfma_i32_32x32x32_i8(f[set][0][k + 1], f[set][1][k + 1], odd, 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        int s = 0;
        for (; s + 2 + NB < stages; s += 2) {  // stages up to s + 1 + NB are whole
            stage(no, 0, s);
            stage(no, 1, s + 1);
        }
        for (; s < stages; s += 2) {
            stage(yes, 0, s);
            if (s + 1 < stages) stage(yes, 1, s + 1);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][0][i] += odd[i];
    } else {
        i32x4 fa[2][MI], fb[2][NI];
        auto read = [&](int i, int set, int buffer, int k) {
            if (i < NI) fb[set][i] = read_lds(rowB + buffer * kBuf + i * 32 * kStage + at[k]);
            else fa[set][i - NI] = read_lds(rowA + buffer * kBuf + (i - NI) * 32 * kStage + at[k]);
        };
        // Products first .. last of a step with the fragments of `set`, and among them, evenly,
        // the reads of the next step's into the other set and loads from .. to of stage t.
        auto step = [&](auto tail, int first, int last, int set, int buffer, int k, int from, int to, int t) {
            constexpr int R = MI + NI;
            const int P = last - first, loads = to - from;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (k >= 0) {
#pragma unroll
                    for (int i = p * R / P; i < (p + 1) * R / P; ++i) read(i, set ^ 1, buffer, k);
                }
#pragma unroll
                for (int i = from + p * loads / P; i < from + (p + 1) * loads / P; ++i) fetch(tail, i, t);
                const int n = (first + p) % NI, m = (first + p) / NI;
                acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[set][n], fa[set][m], acc[n][m], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        constexpr int kFirst = (L + 1) / 2, P = MI * NI, kHalf = P / 2;
        for (int t = 0; t < NB; ++t) {
#pragma unroll
            for (int i = 0; i < L; ++i)
                if (t < NB - 1 || i < kFirst) fetch(yes, i, t);
        }
        landed_but<(NB - 2) * L + kFirst>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MI + NI; ++i) read(i, 0, 0, 0);
        int b = 0;
        // A stage: its steps but the last, half of that one's products, and then, when all of
        // the stage is read and the next one has landed, for every wave past the barrier, the
        // other half beside the next stage's first reads and the loads into the buffer that
        // became free.  (Products wait for neither: their fragments are there.)
        auto stage = [&](auto tail, int s) {
            const int b1 = b + 1 == NB ? 0 : b + 1;
#pragma unroll
            for (int k = 0; k < KK - 1; ++k) step(tail, 0, P, k & 1, b, k + 1, kFirst, k == 0 ? L : kFirst, s + NB - 1);
            step(tail, 0, kHalf, (KK - 1) & 1, b, -1, 0, 0, 0);
            landed_but<(NB - 2) * L>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            step(tail, kHalf, P, (KK - 1) & 1, b1, 0, 0, kFirst, s + NB);  // behind the last stage the reads are of what the buffer holds, not used
            b = b1;
        };
        int s = 0;
        for (; s < stages - NB - 1; ++s) stage(no, s);
        for (; s < stages; ++s) stage(yes, s);
    }
    landed_but<0>();  // LDS is no longer written when the workgroup gives it back

    // lane: token m, channels n .. n + 3 of each i / 4
    const bool whole = (N & 3) == 0;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
        const int m = m0 + wm * TM + mi * 32 + l32;
        if (m >= M) continue;
        const float a = sa[m];
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + wn * TN + ni * 32 + 8 * q + 4 * lh;
                if (n >= N) continue;
                uint16_t* y = Y + static_cast<int64_t>(m) * N + n;
                if (whole) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(sw + n);
                    uint32_t h[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[i] = quant8::result(acc[ni][mi][4 * q + i], a, w[i]);
                    *reinterpret_cast<u32x2*>(y) = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n + i < N) y[i] = static_cast<uint16_t>(quant8::result(acc[ni][mi][4 * q + i], a, sw[n + i]));
                }
            }
        }
    }
}

template <int BM, int BN, int WM, int WN, int NB, bool AHEAD = false>
hipError_t run_tile(const int8_t* A, const float* sa, const int8_t* W, const float* sw, int M, int N, int K, uint16_t* Y, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    constexpr int bytes = NB * (BM + BN) * kStage;
    const auto k = w8a8_tile_kernel<BM, BN, WM, WN, NB, AHEAD>;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void*>(k), bytes, done);
    if (e != hipSuccess) return e;
    const int64_t tiles = static_cast<int64_t>((M + BM - 1) / BM) * ((N + BN - 1) / BN);
    if (tiles * 64 * WM * WN > 0xFFFFFFFFll) return hipErrorInvalidValue;  // a grid holds less than 2^32 threads
    k<<<dim3(static_cast<unsigned>(tiles)), dim3(64 * WM * WN), bytes, st>>>(A, sa, W, sw, M, N, K, Y);
    return hipGetLastError();
}

}  // namespace

namespace {

// The forms: us for K = 8192 of a tile alone on its compute unit with nearly all others idle,
// and with all of them busy.  Tiles of 256 x 256 read the fewest bytes for their products, the
// others are for counts of tiles that leave units idle (4096 x 10240: 2.5 rounds of 256 x 256
// 333 to 357 us, 2 of 256 x 320 292 to 303; 300 x 57344: 128 x 256 200, 320 x 256 168; 1024 x 10240:
// 256 x 256 109, 256 x 192 100; 3000 x 8192: 128 x 256 222, 192 x 256 210; 768 x 8192 of K
// 28672: 128 x 256 200, 192 x 128 183; 200 x 8192: 128 x 128 39, 128 x 64 29).
struct Form {
    int bm, bn;
    double alone, full;
};
constexpr Form kForms[] = {{256, 256, 96, 123}, {256, 320, 106, 146}, {320, 256, 104, 142}, {256, 192, 80, 98}, {192, 256, 84, 101}, {128, 256, 57, 70},
                           {192, 128, 41, 55},  {128, 128, 38, 43},   {96, 128, 35, 37},    {128, 64, 28, 30},  {64, 128, 30, 30},   {64, 64, 20, 20}};
constexpr int kFormCount = sizeof(kForms) / sizeof(kForms[0]);

// Time of a form: whole rounds of a tile a unit, and a last one that takes the longer the more
// units it keeps busy (clock and memory are shared); a tile starts in 5 us and goes over K
// evenly.  For 70 to 4096 rows of 2048 to 57344 channels, K 4096 to 28672 (133 calls, each
// form timed on each, weights from memory), what it picks takes 0.2 % longer than the
// fastest form on average and 6 % at most (on the card that the forms' times are of 0.06 and 3
// %), and 0.88 of the library's int8 product without scales.
double cost_of(const Form& f, int64_t M, int64_t N, int64_t K, int cus) {
    const double tiles = static_cast<double>((M + f.bm - 1) / f.bm) * static_cast<double>((N + f.bn - 1) / f.bn);
    const double whole = static_cast<double>(static_cast<int64_t>(tiles / cus)), left = tiles / cus - whole, deep = static_cast<double>(K) / 8192.0;
    const double alone = 5.0 + (f.alone - 5.0) * deep, full = 5.0 + (f.full - 5.0) * deep;
    return whole * full + (left > 0 ? alone + (full - alone) * left : 0.0);
}

}  // namespace

// Up to 64 rows the weights' bytes bound the call: tiles of few rows, and as narrow as
// still gives no compute unit more than one (8192 channels, 32 and 64 rows: 64 x 32 tiles
// 16.5 and 18.9 us, 32 x 64 19.5 and 64 x 64 23.7; 57344 channels: 126 and 129, 89 and 99).
hipError_t launch_w8a8_tiles(const int8_t* A, const float* sa, const int8_t* W, const float* sw, int M, int N, int K, uint16_t* Y,
                             hipStream_t st) {
    const int cus = device_cu_count();
    if (M <= 64) {
        if ((N + 31) / 32 <= cus) return run_tile<64, 32, 2, 1, 6, true>(A, sa, W, sw, M, N, K, Y, st);
        if (M <= 32) return run_tile<32, 64, 1, 2, 6>(A, sa, W, sw, M, N, K, Y, st);
        return run_tile<64, 64, 2, 2, 5>(A, sa, W, sw, M, N, K, Y, st);
    }
    int best = 0;
    for (int i = 1; i < kFormCount; ++i)
        if (cost_of(kForms[i], M, N, K, cus) < cost_of(kForms[best], M, N, K, cus)) best = i;
    switch (best) {
        case 0: return run_tile<256, 256, 2, 4, 2>(A, sa, W, sw, M, N, K, Y, st);
        case 1: return run_tile<256, 320, 4, 2, 2>(A, sa, W, sw, M, N, K, Y, st);
        case 2: return run_tile<320, 256, 2, 4, 2>(A, sa, W, sw, M, N, K, Y, st);
        case 3: return run_tile<256, 192, 4, 2, 2>(A, sa, W, sw, M, N, K, Y, st);
        case 4: return run_tile<192, 256, 2, 4, 2>(A, sa, W, sw, M, N, K, Y, st);
        case 5: return run_tile<128, 256, 2, 4, 3>(A, sa, W, sw, M, N, K, Y, st);
        case 6: return run_tile<192, 128, 2, 4, 3>(A, sa, W, sw, M, N, K, Y, st);
        case 7: return run_tile<128, 128, 2, 4, 4>(A, sa, W, sw, M, N, K, Y, st);
        case 8: return run_tile<96, 128, 1, 4, 5>(A, sa, W, sw, M, N, K, Y, st);
        case 9: return run_tile<128, 64, 4, 2, 5>(A, sa, W, sw, M, N, K, Y, st);
        case 10: return run_tile<64, 128, 2, 4, 5>(A, sa, W, sw, M, N, K, Y, st);
        default: return run_tile<64, 64, 2, 2, 5>(A, sa, W, sw, M, N, K, Y, st);
    }
}

}  // namespace apex4
