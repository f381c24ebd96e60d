// C ABI front end of sampling: argument validation (before any HIP call), device check
// and dispatch.  See include/apex4.h for the contract.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "apex4.h"
#include "apex4_internal.h"

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool present(const void* p, int64_t n) { return p != nullptr || n == 0; }

int check_shape(int type, int64_t B, int64_t V) {
    if (type != APEX4_LOGITS_FP16 && type != APEX4_LOGITS_FP32) return APEX4_ERR_SHAPE;
    return B < 0 || B > (1ll << 21) || V < 1 || V > (1ll << 18) ? APEX4_ERR_SHAPE : APEX4_OK;
}

}  // namespace

extern "C" int apex4_sample_workspace_size(int type, int64_t B, int64_t V, int64_t* bytes) {
    if (!bytes) return APEX4_ERR_NULL;
    int rc = check_shape(type, B, V);
    if (rc || (rc = apex4::check_device())) return rc;
    *bytes = apex4::sample_workspace(B, V);
    return APEX4_OK;
}

extern "C" int apex4_sample(const void* logits, int type, int64_t stride, int64_t B, int64_t V, const float* u,
                            const float* temperature, float temperature_all, const int32_t* top_k, int64_t top_k_all,
                            const float* top_p, float top_p_all, const float* min_p, float min_p_all, int32_t* tokens,
                            float* probs, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!present(logits, B) || !present(u, B) || !present(tokens, B)) return APEX4_ERR_NULL;
    int rc = check_shape(type, B, V);
    if (rc) return rc;
    if (stride < V || stride > (1ll << 40)) return APEX4_ERR_SHAPE;
    if (!aligned(logits, type == APEX4_LOGITS_FP16 ? 2 : 4) || !aligned(workspace, 16) || !aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) ||
        !aligned(min_p, 4) || !aligned(tokens, 4) || !aligned(probs, 4))
        return APEX4_ERR_ALIGN;
    if ((rc = apex4::check_device())) return rc;
    if (B == 0) return APEX4_OK;
    const int64_t need = apex4::sample_workspace(B, V);
    if (need > 0 && (!workspace || workspace_bytes < need)) return APEX4_ERR_WORKSPACE;
    apex4::SampleArgs a;
    a.logits = logits;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.tokens = tokens;
    a.probs = probs;
    a.workspace = workspace;
    a.stride = stride;
    a.V = static_cast<int>(V);
    a.top_k_all = top_k_all <= 0 || top_k_all > V ? 0 : static_cast<int>(top_k_all);
    a.temperature_all = temperature_all;
    a.top_p_all = top_p_all;
    a.min_p_all = min_p_all;
    const hipError_t e = apex4::launch_sample(a, B, type == APEX4_LOGITS_FP16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? APEX4_OK : APEX4_ERR_LAUNCH;
}
