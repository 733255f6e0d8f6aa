// vsd_fp8.cu -- a matrix in e4m3 with a scale for each block of 128 columns, and the
// LM head's logits from two such matrices (include/vsd_decode.h).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "vsd_common.cuh"
#include "vsd_decode.h"

namespace vsd {
namespace {

constexpr int kBlock = 128;  // columns of a scale

__device__ __forceinline__ float f32_of(float x) { return x; }
__device__ __forceinline__ float f32_of(__nv_bfloat16 x) { return __bfloat162float(x); }

// The least power of two s with amax / s <= 448 = 1.75 2^8.
__device__ __forceinline__ float scale_of(float amax) {
    if (!(amax < INFINITY)) return NAN;
    if (amax == 0.f) return 1.f;
    const uint32_t b = __float_as_uint(amax);
    int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u);
    return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

template <typename T>
__global__ void __launch_bounds__(256)
    k_quantize(const T* x, int R, int H, int rows, __nv_fp8_e4m3* q, float* scale) {
    __shared__ uint32_t amax;
    const int64_t r0 = (int64_t)blockIdx.y * rows;
    const int h0 = blockIdx.x * kBlock, nr = (int)min((int64_t)rows, R - r0), nh = min(kBlock, H - h0);
    if (threadIdx.x == 0) amax = 0;
    __syncthreads();
    uint32_t m = 0;
    for (int i = threadIdx.x; i < nr * nh; i += blockDim.x)
        m = max(m, __float_as_uint(f32_of(x[(r0 + i / nh) * H + h0 + i % nh])) & 0x7FFFFFFFu);
    atomicMax(&amax, m);
    __syncthreads();
    const float s = scale_of(__uint_as_float(amax));
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
    for (int i = threadIdx.x; i < nr * nh; i += blockDim.x) {
        const int64_t at = (r0 + i / nh) * H + h0 + i % nh;
        q[at] = __nv_fp8_e4m3(f32_of(x[at]) / s);
    }
}

constexpr int kTile = 64, kStep = 32;

__global__ void __launch_bounds__(256)
    k_head_fp8(const __nv_fp8_e4m3* hidden, const float* hs, const __nv_fp8_e4m3* weight,
               const float* ws, int R, int V, int H, __nv_bfloat16* logits) {
    __shared__ float A[kStep][kTile + 1], B[kStep][kTile + 1];
    const int64_t r0 = (int64_t)blockIdx.y * kTile, v0 = (int64_t)blockIdx.x * kTile;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16, nk = (H + kBlock - 1) / kBlock;
    float acc[4][4] = {};
    for (int kb = 0; kb < nk; ++kb) {
        float part[4][4] = {};
        for (int h0 = kb * kBlock; h0 < min(H, (kb + 1) * kBlock); h0 += kStep) {
            __syncthreads();
            for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
                const int row = i / kStep, k = i % kStep;
                const bool in = h0 + k < H;
                A[k][row] = in && r0 + row < R ? float(hidden[(r0 + row) * H + h0 + k]) : 0.f;
                B[k][row] = in && v0 + row < V ? float(weight[(v0 + row) * H + h0 + k]) : 0.f;
            }
            __syncthreads();
            for (int k = 0; k < kStep; ++k)
                for (int i = 0; i < 4; ++i)
                    for (int j = 0; j < 4; ++j)
                        part[i][j] = fmaf(A[k][ty + 16 * i], B[k][tx + 16 * j], part[i][j]);
        }
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) {
                const int64_t r = r0 + ty + 16 * i, v = v0 + tx + 16 * j;
                if (r < R && v < V)
                    acc[i][j] = fmaf(part[i][j], hs[r * nk + kb] * ws[(v / kBlock) * nk + kb], acc[i][j]);
            }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + ty + 16 * i, v = v0 + tx + 16 * j;
            if (r < R && v < V) logits[r * V + v] = __float2bfloat16_rn(acc[i][j]);
        }
}

bool share_bytes(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + bn && y < x + an;
}
bool sizes_ok(int R, int H) {
    return R >= 1 && R <= (1 << 24) && H >= 16 && H <= (1 << 20) && H % 16 == 0;
}

}  // namespace
}  // namespace vsd

using namespace vsd;

extern "C" {

vsd_status vsd_quantize_fp8(const void* x, vsd_dtype dtype, int32_t R, int32_t H,
                            int32_t block_rows, void* q, float* scale, void* stream) {
    if (!x || !q || !scale || !sizes_ok(R, H)) return VSD_ERR_INVALID_ARG;
    if (dtype != VSD_F32 && dtype != VSD_BF16) return VSD_ERR_INVALID_ARG;
    if (block_rows != 1 && block_rows != kBlock) return VSD_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uintptr_t)q) & 15) || ((uintptr_t)scale & 3)) return VSD_ERR_INVALID_ARG;
    const size_t n = (size_t)R * H, xb = n * (dtype == VSD_BF16 ? 2 : 4);
    const int nr = (R + block_rows - 1) / block_rows, nh = (H + kBlock - 1) / kBlock;
    const size_t sb = 4 * (size_t)nr * nh;
    if (share_bytes(x, xb, q, n) || share_bytes(x, xb, scale, sb) || share_bytes(q, n, scale, sb))
        return VSD_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 grid(nh, nr);
    __nv_fp8_e4m3* out = static_cast<__nv_fp8_e4m3*>(q);
    if (dtype == VSD_BF16)
        k_quantize<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(x), R, H, block_rows, out, scale);
    else
        k_quantize<<<grid, 256, 0, st>>>(static_cast<const float*>(x), R, H, block_rows, out, scale);
    return cudaGetLastError() == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

vsd_status vsd_lmhead_logits_fp8(const void* hidden, const float* hidden_scale,
                                 const void* weight, const float* weight_scale, int32_t R,
                                 int32_t V, int32_t H, void* logits, void* ws, size_t ws_bytes,
                                 void* stream) {
    if (!hidden || !hidden_scale || !weight || !weight_scale || !logits || !sizes_ok(R, H))
        return VSD_ERR_INVALID_ARG;
    if (V < 1 || V > (1 << 20)) return VSD_ERR_INVALID_ARG;
    if ((((uintptr_t)hidden | (uintptr_t)weight) & 15) || ((uintptr_t)logits & 1) ||
        (((uintptr_t)hidden_scale | (uintptr_t)weight_scale) & 3))
        return VSD_ERR_INVALID_ARG;
    const size_t nk = (H + kBlock - 1) / kBlock, ob = 2 * (size_t)R * V;
    if (share_bytes(logits, ob, hidden, (size_t)R * H) || share_bytes(logits, ob, weight, (size_t)V * H) ||
        share_bytes(logits, ob, hidden_scale, 4 * nk * R) ||
        share_bytes(logits, ob, weight_scale, 4 * nk * ((V + kBlock - 1) / kBlock)))
        return VSD_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < 256) return VSD_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(ws, 0, 4, st) != cudaSuccess) return VSD_ERR_CUDA;
    k_head_fp8<<<dim3((V + kTile - 1) / kTile, (R + kTile - 1) / kTile), 256, 0, st>>>(
        static_cast<const __nv_fp8_e4m3*>(hidden), hidden_scale, static_cast<const __nv_fp8_e4m3*>(weight),
        weight_scale, R, V, H, static_cast<__nv_bfloat16*>(logits));
    return cudaGetLastError() == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

}  // extern "C"
