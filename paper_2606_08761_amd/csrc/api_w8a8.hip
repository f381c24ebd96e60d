// C ABI front end of the 8-bit linears: argument validation (before any HIP call), device
// check and dispatch.  See include/apex4.h for the contract.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4.h"
#include "apex4_internal.h"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool present(const void* p, int64_t rows) { return p != nullptr || rows == 0; }

int check_shape(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 1 || K < 32 || K % 32 != 0 || K >= 131072) return APEX4_ERR_SHAPE;
    if (M > 0x7FFFFFFF || N > 0x7FFFFFFF) return APEX4_ERR_SHAPE;
    // the kernels address a few rows of an operand with 32-bit byte offsets
    if (M * K > 0xFFFFFFFFll || N * K > 0xFFFFFFFFll) return APEX4_ERR_SHAPE;
    return APEX4_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? APEX4_OK : APEX4_ERR_LAUNCH; }

hipError_t gemm(const int8_t* A, const float* sa, const int8_t* W, const float* sw, int64_t M, int64_t N, int64_t K, void* Y,
                hipStream_t st) {
    const auto launch = apex4::w8a8_rows_fits(M, N) ? apex4::launch_w8a8_rows : apex4::launch_w8a8_tiles;
    return launch(A, sa, W, sw, static_cast<int>(M), static_cast<int>(N), static_cast<int>(K), static_cast<uint16_t*>(Y), st);
}

}  // namespace

using apex4::check_device;

extern "C" {

int apex4_quantize_act8(const void* x, int64_t M, int64_t K, int8_t* A_8, float* s_a, void* stream) {
    if (!present(x, M) || !present(A_8, M) || !present(s_a, M)) return APEX4_ERR_NULL;
    int rc = check_shape(M, 1, K);
    if (rc) return rc;
    if (!aligned16(x) || !aligned16(A_8) || !aligned16(s_a)) return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (M == 0) return APEX4_OK;
    return status_of(apex4::launch_quantize8(static_cast<const uint16_t*>(x), M, K, A_8, s_a, static_cast<hipStream_t>(stream)));
}

int apex4_w8a8_gemm(const int8_t* A_8, const float* s_a, const int8_t* W_8, const float* s_w, int64_t M, int64_t N, int64_t K,
                    void* Y, void* stream) {
    if (!present(A_8, M) || !present(s_a, M) || !W_8 || !s_w || !present(Y, M)) return APEX4_ERR_NULL;
    int rc = check_shape(M, N, K);
    if (rc) return rc;
    if (!aligned16(A_8) || !aligned16(s_a) || !aligned16(W_8) || !aligned16(s_w) || !aligned16(Y)) return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (M == 0) return APEX4_OK;
    return status_of(gemm(A_8, s_a, W_8, s_w, M, N, K, Y, static_cast<hipStream_t>(stream)));
}

int apex4_w8a8_linear(const void* x, const int8_t* W_8, const float* s_w, int64_t M, int64_t N, int64_t K, void* Y,
                      int8_t* A_8_work, float* s_a_work, void* stream) {
    if (!present(x, M) || !W_8 || !s_w || !present(Y, M) || !present(A_8_work, M) || !present(s_a_work, M)) return APEX4_ERR_NULL;
    int rc = check_shape(M, N, K);
    if (rc) return rc;
    if (!aligned16(x) || !aligned16(W_8) || !aligned16(s_w) || !aligned16(Y) || !aligned16(A_8_work) || !aligned16(s_a_work))
        return APEX4_ERR_ALIGN;
    if ((rc = check_device())) return rc;
    if (M == 0) return APEX4_OK;
    const auto st = static_cast<hipStream_t>(stream);
    if (apex4::w8a8_fused_fits(M, N, K))
        return status_of(apex4::launch_w8a8_fused(static_cast<const uint16_t*>(x), W_8, s_w, static_cast<int>(N), static_cast<int>(K),
                                                  static_cast<uint16_t*>(Y), st));
    const hipError_t e = apex4::launch_quantize8(static_cast<const uint16_t*>(x), M, K, A_8_work, s_a_work, st);
    return e == hipSuccess ? status_of(gemm(A_8_work, s_a_work, W_8, s_w, M, N, K, Y, st)) : APEX4_ERR_LAUNCH;
}

}  // extern "C"
