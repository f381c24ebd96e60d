// Activations in 8 bits, one scale a token: S = max|x| / 127 in binary32 and codes
// clamp(round-half-even(x / S), -127, 127), taken on the exact quotient.
//
// Bound by memory (2 bytes read and 1 written a value): a workgroup of T threads takes a
// row and holds it in registers, U slots of 8 values a thread, all loads in flight
// together, so that it is read once.  Arithmetic:
//   S     max|x| (exact: magnitudes order like their bits) / 127, one correctly
//         rounded binary32 division a row;
//   t     x rcp(S), within 2^-15 of x / S (|t| <= 127, two roundings of 2^-23 each);
//   code  rint(t), then d = x - code S, one fma: exact wherever it decides, since x and
//         code S are multiples of the last place of S and |d| stays near S / 2, so d has
//         24 bits at most.  |d| > S / 2 (t was rounded across a border), or = S / 2 with an
//         odd code (a tie), moves the code by one.
// A row of zeros (or whose S is zero) gets zero codes; a row that holds an infinity or a
// NaN gets a scale that is one and zero codes, so that its products are NaN.
//
// 4096 rows of 8192: 18.4 us (101 MB, 5.5 TB/s); 300 rows 4.3 us, 16 rows 3.5, a launch mostly;
// 16 rows of 28672 5.3.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "apex4_internal.h"
#include "quant8_core.h"

namespace apex4 {
namespace {

using namespace quant8;

template <int T, int U>
__global__ __launch_bounds__(T) void quant8_kernel(const uint16_t* __restrict__ x, int64_t M, int slots, int8_t* __restrict__ q,
                                                   float* __restrict__ s) {
    __shared__ uint32_t red[T / 64];
    const int64_t row = static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x;
    if (row >= M) return;
    const u32x4* xr = reinterpret_cast<const u32x4*>(x) + row * slots;
    u32x2* qr = reinterpret_cast<u32x2*>(q) + row * slots;
    u32x4 v[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int i = static_cast<int>(threadIdx.x) + j * T;
        v[j] = u32x4{0u, 0u, 0u, 0u};
        if (i < slots) v[j] = xr[i];
    }
    uint32_t am = 0;
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const uint32_t a = quant::absmax8_bits(make_uint4(v[j][0], v[j][1], v[j][2], v[j][3]));
        am = am > a ? am : a;
    }
    am = quant::group_max<64>(am);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = am;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < T / 64; ++w) am = am > red[w] ? am : red[w];
    const Scale sc = scale_of(am);
    if (threadIdx.x == 0) s[row] = sc.s;
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int i = static_cast<int>(threadIdx.x) + j * T;
        if (i < slots) qr[i] = codes8<true>(v[j], sc);
    }
}

template <int T, int U>
hipError_t run(const uint16_t* x, int64_t M, int slots, int8_t* q, float* s, hipStream_t st) {
    constexpr int64_t kMost = 1 << 21;  // of the first dimension, which holds less than 2^32 threads
    const int64_t n = M < kMost ? M : kMost;
    quant8_kernel<T, U><<<dim3(static_cast<unsigned>(n), static_cast<unsigned>((M + n - 1) / n)), dim3(T), 0, st>>>(x, M, slots, q, s);
    return hipGetLastError();
}

}  // namespace

// K < 2^17: at most 16384 slots a row.  Two slots a thread keep more rows on a compute
// unit than four do, one leaves its threads too little to load (4096 rows of 8192: 512
// threads with two 18.4 us, 5.5 TB/s; 256 with four 20.6, 1024 with one 21.2; 300 rows 4.3, 5.3 and 4.2).
hipError_t launch_quantize8(const uint16_t* x, int64_t M, int64_t K, int8_t* q, float* s, hipStream_t st) {
    const int n = static_cast<int>(K / 8);
    if (n <= 64) return run<64, 1>(x, M, n, q, s, st);
    if (n <= 128) return run<128, 1>(x, M, n, q, s, st);
    if (n <= 256) return run<256, 1>(x, M, n, q, s, st);
    if (n <= 512) return run<256, 2>(x, M, n, q, s, st);
    if (n <= 1024) return run<512, 2>(x, M, n, q, s, st);
    if (n <= 4096) return run<1024, 4>(x, M, n, q, s, st);
    return run<1024, 16>(x, M, n, q, s, st);
}

}  // namespace apex4
