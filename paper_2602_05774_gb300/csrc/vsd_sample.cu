// vsd_sample.cu -- the entry points of the filtered sampling (include/vsd_decode.h): sizes,
// argument checks and the launch (vsd_sample.cuh).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "vsd_fixed.cuh"
#include "vsd_sample.h"

namespace vsd {
namespace {

bool share_bytes(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + bn && y < x + an;
}

}  // namespace
}  // namespace vsd

using namespace vsd;

extern "C" {

size_t vsd_sample_filtered_workspace_bytes(int32_t R, int32_t V) {
    return R >= 1 && R <= (1 << 24) && V >= 1 && V <= (1 << 20) ? 256 : 0;
}

vsd_status vsd_sample_filtered(const void* logits, vsd_dtype dtype, int32_t R, int32_t V,
                               const vsd_policy* policy, const float* u,
                               vsd_filtered_outputs* out, void* ws, size_t ws_bytes,
                               void* stream) {
    const size_t need = vsd_sample_filtered_workspace_bytes(R, V);
    if (!logits || !policy || !out || need == 0) return VSD_ERR_INVALID_ARG;
    if (dtype != VSD_F32 && dtype != VSD_BF16) return VSD_ERR_INVALID_ARG;
    const size_t size = dtype == VSD_BF16 ? 2 : 4, bytes = (size_t)R * V * size, row = 4 * (size_t)R;
    if (((uintptr_t)logits | (uintptr_t)out->filtered) & (size - 1)) return VSD_ERR_INVALID_ARG;
    const vsd_policy& p = *policy;
    const void* in[] = {p.row_T, p.row_top_k, p.row_top_p, p.row_min_p, u};
    const void* res[] = {out->tokens, out->logq_tok, out->kept};
    for (const void* q : in)
        if ((uintptr_t)q & 3) return VSD_ERR_INVALID_ARG;
    for (const void* q : res)
        if ((uintptr_t)q & 3) return VSD_ERR_INVALID_ARG;
    if (!u && (out->tokens || out->logq_tok)) return VSD_ERR_INVALID_ARG;
    if (!p.row_T && !(p.T == 0.f || (p.T >= kMinT && p.T <= kMaxT))) return VSD_ERR_INVALID_ARG;
    if ((!p.row_top_p && p.top_p != p.top_p) || (!p.row_min_p && p.min_p != p.min_p))
        return VSD_ERR_INVALID_ARG;
    if (out->filtered != logits && share_bytes(out->filtered, bytes, logits, bytes))
        return VSD_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
        if (share_bytes(res[i], row, logits, bytes) || share_bytes(res[i], row, out->filtered, bytes))
            return VSD_ERR_INVALID_ARG;
        for (const void* q : in)
            if (share_bytes(res[i], row, q, row)) return VSD_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (share_bytes(res[i], row, res[j], row)) return VSD_ERR_INVALID_ARG;
    }
    for (const void* q : in)
        if (share_bytes(out->filtered, bytes, q, row)) return VSD_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need) return VSD_ERR_WORKSPACE;
    if (!u && !out->kept && !out->filtered) return VSD_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(ws, 0, 256, st) != cudaSuccess) return VSD_ERR_CUDA;
    const bool same = (((uintptr_t)logits ^ (uintptr_t)out->filtered) & 15) == 0;
    const SampleArgs a{p, u, *out, R, V, exp_shift(V), same, static_cast<int*>(ws)};
    const cudaError_t e = dtype == VSD_BF16 ? sample<__nv_bfloat16>(logits, a, st)
                                            : sample<float>(logits, a, st);
    return e == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

}  // extern "C"
