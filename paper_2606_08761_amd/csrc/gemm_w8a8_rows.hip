// Y = binary16(s_a s_w sum_k A W) of 8-bit codes, few rows: the weights streamed once.
//
// The eight waves of a workgroup share 16 C channels and take the 128-byte pieces of K
// in turn, so that together they read each channel's row in runs of 1 KB; weights go from
// memory straight into the operands of v_mfma_i32_16x16x64_i8 (weights the rows, tokens
// the columns; 16 R tokens), D pieces ahead.  The waves' integer sums meet in LDS at the
// end: exact in any order.
//
// With SLOTS a single token is quantized by every workgroup itself, into LDS, while its first
// weights are on their way; otherwise the codes come from the quantizer's buffer.
//
// Bound by memory.  8192 x 8192: one row, quantized on the way, 14.3 us (67 MB, 4.7 TB/s; with
// the quantizer as a launch of its own 18).  Loads that give nothing still take their place
// among the others, so a wave asks for its own pieces alone (18.2 -> 15.0 us); a token in
// registers by two slots a thread (eight cost the weights theirs: 19.1).
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "apex4_internal.h"
#include "quant8_core.h"

namespace apex4 {
namespace {

using namespace quant8;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8, kThreads = 64 * kWaves, kPiece = 128;
constexpr int kMostFused = kThreads * 8 * 8;  // K of a token that is quantized on the way
constexpr uint32_t kNowhere = 0xFFFFFFFFu;  // past any buffer: such loads give zeros
constexpr int kRsrcFlags = 0x00027000;      // raw buffer descriptor, 32-bit data format

// SLOTS: of 8 values a thread, of a token that is quantized on the way; 0: none is.
template <int R, int C, int D, int SLOTS>
__global__ __launch_bounds__(kThreads) void w8a8_rows_kernel(const int8_t* __restrict__ A, const float* __restrict__ sa,
                                                             const uint16_t* __restrict__ x, const int8_t* __restrict__ W,
                                                             const float* __restrict__ sw, int M, int N, int K,
                                                             uint16_t* __restrict__ Y) {
    constexpr bool FUSED = SLOTS > 0;
    extern __shared__ __align__(16) uint8_t smem[];  // FUSED: the token's codes; then the sums
    __shared__ uint32_t red[FUSED ? kWaves : 1];
    const int n0 = blockIdx.x * 16 * C, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int rows = min(16 * C, N - n0), pieces = (K + kPiece - 1) / kPiece;
    const auto bufW = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(W) + static_cast<int64_t>(n0) * K, 0,
                                                        static_cast<uint32_t>(rows) * static_cast<uint32_t>(K), kRsrcFlags);
    const auto bufA = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(A), 0,
                                                        FUSED ? 0u : static_cast<uint32_t>(static_cast<int64_t>(M) * K), kRsrcFlags);
    i32x4 w[D][2][C], a[D][2][R];
    // piece p: channels' and tokens' bytes 64 h + 16 g of it; nothing behind K
    auto load = [&](int d, int p) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t k = static_cast<uint32_t>(p) * kPiece + 64 * h + 16 * g;
            const bool in = k < static_cast<uint32_t>(K);
#pragma unroll
            for (int c = 0; c < C; ++c)
                w[d][h][c] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                           bufW, in ? static_cast<uint32_t>(16 * c + l16) * static_cast<uint32_t>(K) + k : kNowhere, 0, 0));
            if constexpr (!FUSED) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    a[d][h][r] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                               bufA, in && 16 * r + l16 < M ? static_cast<uint32_t>(16 * r + l16) * static_cast<uint32_t>(K) + k : kNowhere, 0, 0));
            }
        }
    };
    // FUSED: the token first, since loads come back in order
    u32x4 v[FUSED ? SLOTS : 1];
    if constexpr (FUSED) {
        const u32x4* xr = reinterpret_cast<const u32x4*>(x);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            v[j] = u32x4{0u, 0u, 0u, 0u};
            if (tid + j * kThreads < K / 8) v[j] = xr[tid + j * kThreads];
        }
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (wave + d * kWaves < pieces) load(d, wave + d * kWaves);

    float s_token = 0.f;
    if constexpr (FUSED) {
        uint32_t am = 0;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            const uint32_t b = quant::absmax8_bits(make_uint4(v[j][0], v[j][1], v[j][2], v[j][3]));
            am = am > b ? am : b;
        }
        am = quant::group_max<64>(am);
        if (lane == 0) red[wave] = am;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) am = am > red[i] ? am : red[i];
        const Scale sc = scale_of(am);
        s_token = sc.s;
        auto put = [&](int i, u32x4 t) {  // whole pieces: zeros behind K
            // (RARE's branch takes 12 registers and with them one workgroup of four: 32000 channels
            // of K 4096 25.7 and 26.0 us)
            if (i < pieces * (kPiece / 8)) *reinterpret_cast<u32x2*>(smem + 8 * i) = codes8<(SLOTS > 2)>(t, sc);
        };
        if constexpr (SLOTS <= 2) {
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) put(tid + j * kThreads, v[j]);
        } else {  // read once more: kept, they take the registers of a second workgroup
#pragma unroll 1
            for (int i = tid; i < pieces * (kPiece / 8); i += kThreads) {
                u32x4 t = {0u, 0u, 0u, 0u};
                if (i < K / 8) t = reinterpret_cast<const u32x4*>(x)[i];
                put(i, t);
            }
        }
        __syncthreads();
    }

    i32x4 acc[C][R];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[c][r] = i32x4{0, 0, 0, 0};
    for (int p0 = wave; p0 < pieces; p0 += D * kWaves) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int p = p0 + d * kWaves;
            if (p >= pieces) break;  // uniform, as below: what would be loaded costs its issue even where nothing is read
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (FUSED) {
                    a[d][h][0] = *reinterpret_cast<const i32x4*>(smem + p * kPiece + 64 * h + 16 * g);
                }
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int r = 0; r < R; ++r) acc[c][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[d][h][c], a[d][h][r], acc[c][r], 0, 0, 0);
            }
            if (p + D * kWaves < pieces) load(d, p + D * kWaves);
        }
    }

    // the waves' sums: lane's token 16 r + l16, channels 16 c + 4 g .. + 3
    __syncthreads();  // the codes are read
    i32x4* sums = reinterpret_cast<i32x4*>(smem);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < R; ++r) sums[((wave * C + c) * R + r) * 64 + lane] = acc[c][r];
    __syncthreads();
    for (int u = tid; u < C * R * 64; u += kThreads) {
        i32x4 t = sums[u];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) t += sums[v * C * R * 64 + u];
        const int m = u / 64 % R * 16 + (u & 15), n = n0 + u / (64 * R) * 16 + (u >> 4 & 3) * 4;
        if (m >= M || n >= N) continue;
        const float s = FUSED ? s_token : sa[m];
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = result(t[i], s, sw[min(n + i, N - 1)]);
        uint16_t* y = Y + static_cast<int64_t>(m) * N + n;
        if ((N & 3) == 0) {
            *reinterpret_cast<u32x2*>(y) = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
        } else {
            for (int i = 0; i < 4 && n + i < N; ++i) y[i] = static_cast<uint16_t>(h[i]);
        }
    }
}

template <int R, int C, int D, int SLOTS>
hipError_t run(const int8_t* A, const float* sa, const uint16_t* x, const int8_t* W, const float* sw, int M, int N, int K, uint16_t* Y, hipStream_t st) {
    const int sums = kWaves * C * R * 64 * 16, codes = SLOTS ? (K + kPiece - 1) / kPiece * kPiece : 0;
    static_assert(kWaves * C * R * 64 * 16 <= 65536 && kMostFused <= 65536, "no more LDS than any launch may have");
    w8a8_rows_kernel<R, C, D, SLOTS><<<dim3(static_cast<unsigned>((N + 16 * C - 1) / (16 * C))), dim3(kThreads), sums > codes ? sums : codes, st>>>(
        A, sa, x, W, sw, M, N, K, Y);
    return hipGetLastError();
}

}  // namespace

// Up to 8 rows, and up to 24 where no compute unit gets more than one workgroup (1024 channels,
// K 8192, 16, 24 and 32 rows: 9.8, 12.7 and 14.6 us, tiles 14.6; 4096 of K 28672, 16, 24 and 32
// rows: 29.4, 42.9 and 49.2, tiles 42.6 to 43.3).
// One group of 16 channels a workgroup: two fill the chip with half as many waves (8 rows of
// 8192 and 57344 channels: 15.9 and 87.8 us, two groups 19.8 and 102).
bool w8a8_rows_fits(int64_t M, int64_t N) {
    if (N > 1 << 26) return false;  // a grid holds less than 2^32 threads
    return M <= 8 || (M <= 24 && N <= 16 * static_cast<int64_t>(device_cu_count()));
}
bool w8a8_fused_fits(int64_t M, int64_t N, int64_t K) { return M == 1 && N <= 1 << 26 && K <= kMostFused; }

hipError_t launch_w8a8_rows(const int8_t* A, const float* sa, const int8_t* W, const float* sw, int M, int N, int K, uint16_t* Y, hipStream_t st) {
    if (M <= 16) return run<1, 1, 4, 0>(A, sa, nullptr, W, sw, M, N, K, Y, st);
    return run<2, 1, 4, 0>(A, sa, nullptr, W, sw, M, N, K, Y, st);
}
hipError_t launch_w8a8_fused(const uint16_t* x, const int8_t* W, const float* sw, int N, int K, uint16_t* Y, hipStream_t st) {
    if (K <= kThreads * 16) return run<1, 1, 4, 2>(nullptr, nullptr, x, W, sw, 1, N, K, Y, st);
    return run<1, 1, 4, 8>(nullptr, nullptr, x, W, sw, 1, N, K, Y, st);
}

}  // namespace apex4
