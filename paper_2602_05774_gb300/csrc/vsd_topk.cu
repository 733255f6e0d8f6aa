// vsd_topk.cu -- distillation from a teacher's top logits on logits in hand:
//
//   q_r = softmax(x_r / T),  l_r = sum_k p_rk (log p_rk - log q_r(id_rk)),
//   grad_rv = a_r (q_r(v) - sum_k p_rk [v = id_rk]),  a_r = scale w_r / (T sum w).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_launch.h"
#include "vsd_loss.h"

namespace vsd {
namespace {

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct TopkWs {
    size_t status, done, zero_end, nrows, wsum, wmax, n, id, p, plogp, w, rowmap, rowinv, total;
};

TopkWs topk_ws(int R, int K) {
    TopkWs w;
    const size_t r = (size_t)R, rk = r * (size_t)K;
    size_t o = 0;
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o = up256(o + bytes);
        return at;
    };
    w.status = take(256);
    w.done = take(256);
    w.zero_end = o;
    w.nrows = take(4);
    w.wsum = take(8);
    w.wmax = take(4);
    w.n = take(4 * r);
    w.id = take(4 * rk);
    w.p = take(4 * rk);
    w.plogp = take(4 * r);
    w.w = take(4 * r);
    w.rowmap = take(4 * r);
    w.rowinv = take(4 * r);
    w.total = o;
    return w;
}

template <typename U> U* at(void* ws, size_t off) {
    return reinterpret_cast<U*>(static_cast<char*>(ws) + off);
}

__device__ __forceinline__ float get(const float* x, size_t v) { return x[v]; }
__device__ __forceinline__ float get(const __nv_bfloat16* x, size_t v) { return __bfloat162float(x[v]); }
__device__ __forceinline__ void put(float* x, size_t v, float f) { x[v] = f; }
__device__ __forceinline__ void put(__nv_bfloat16* x, size_t v, float f) { x[v] = __float2bfloat16_rn(f); }

__global__ void k_topk_targets(TargetIn in, Targets tg, float* row_loss, float* logz) {
    const int lane = threadIdx.x & 31;
    const int r = (int)((blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5);
    if (r < in.R) target_row(in, tg, r, lane);
    __shared__ int last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(tg.done, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    scan_rows(tg, in.R, row_loss, logz);
}

// One block per row.
template <typename T>
__global__ void __launch_bounds__(256)
    k_topk(const T* logits, int V, int K, Targets tg, float c, float Tq, float grad_scale,
           float* row_loss, float* logz, T* grad) {
    const int r = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = logits + (size_t)r * V;
    T* g = grad ? grad + (size_t)r * V : nullptr;
    const int n = tg.n[r];
    if (n < 0) {
        if (g) for (int v = threadIdx.x; v < V; v += 256) put(g, v, 0.f);
        return;
    }
    __shared__ float red[8];
    __shared__ double dred[8];
    __shared__ float slse;
    __shared__ float xs[kMaxTeacher];
    float m = -INFINITY;
    for (int v = threadIdx.x; v < V; v += 256) m = fmaxf(m, get(x, v));
    m = warp_max(m);
    if (lane == 0) red[warp] = m;
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = fmaxf(m, red[w]);
    __syncthreads();
    float s = 0.f;
    for (int v = threadIdx.x; v < V; v += 256) {
        const float f = get(x, v);
        s += m > -INFINITY ? ex2((f - m) * c) : (f == f ? 0.f : f);
    }
    s = warp_sum(s);
    if (lane == 0) red[warp] = s;
    const int32_t* id = tg.id + (size_t)r * K;
    const float* p = tg.p + (size_t)r * K;
    double dot = 0.0;
    for (int k = threadIdx.x; k < n; k += 256) {
        xs[k] = get(x, id[k]);
        dot += (double)p[k] * ((double)xs[k] - (double)m);
    }
    dot = warp_sum(dot);
    if (lane == 0) dred[warp] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        dot = 0.0;
        for (int w = 0; w < 8; ++w) s += red[w], dot += dred[w];
        const double ls = log((double)s), lz = (double)m / (double)Tq + ls;
        if (!isfinite(lz)) atomicOr(tg.status, VSD_STATUS_BAD_ROW);
        logz[r] = (float)lz;
        row_loss[r] = (float)((double)tg.plogp[r] + ls - dot / (double)Tq);
        slse = (float)(ls * kLog2e);
    }
    __syncthreads();
    if (!g) return;
    const float l = slse;
    const float a = (float)((double)grad_scale * (double)tg.w[r] / (*tg.wsum * (double)Tq));
    for (int v = threadIdx.x; v < V; v += 256) put(g, v, a * ex2((get(x, v) - m) * c - l));
    __syncthreads();
    for (int k = threadIdx.x; k < n; k += 256)
        put(g, id[k], a * (ex2((xs[k] - m) * c - l) - p[k]));
}

// The weighted mean of the rows' losses, in row order.
__global__ void k_mean_loss(Targets tg, int R, const float* row_loss, float* loss) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ double part[32];
    double sum = 0.0;
    for (int r = threadIdx.x; r < R; r += blockDim.x)
        if (tg.n[r] >= 0 && tg.w[r] != 0.f) sum += (double)tg.w[r] * (double)row_loss[r];
    sum = warp_sum(sum);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += part[w];
        *loss = (float)(sum / *tg.wsum);
    }
}

}  // namespace

bool topk_shape_ok(int R, int V, int K) {
    return R >= 1 && R <= (1 << 24) && V >= 1 && V <= (1 << 20) && K >= 1 && K <= kMaxTeacher;
}

size_t topk_workspace_bytes(int R, int V, int K) {
    return topk_shape_ok(R, V, K) ? topk_ws(R, K).total : 0;
}

cudaError_t topk_distill(const void* logits, bool bf16, const TargetIn& in, float T,
                         float grad_scale, const vsd_loss_outputs& out, void* ws,
                         cudaStream_t st) {
    const TopkWs w = topk_ws(in.R, in.K);
    Targets tg{at<int32_t>(ws, w.n), at<int32_t>(ws, w.id), at<float>(ws, w.p),
               at<float>(ws, w.plogp), at<float>(ws, w.w), at<int32_t>(ws, w.rowmap),
               at<int32_t>(ws, w.rowinv), at<int32_t>(ws, w.nrows), at<double>(ws, w.wsum),
               at<float>(ws, w.wmax), at<int32_t>(ws, w.done), at<int32_t>(ws, w.status)};
    const float c = (float)(kLog2e / (double)T);
    cudaError_t e = cudaMemsetAsync(ws, 0, w.zero_end, st);
    if (e != cudaSuccess) return e;
    k_topk_targets<<<(in.R + 7) / 8, 256, 0, st>>>(in, tg, out.row_loss, out.logz);
    if (bf16)
        k_topk<__nv_bfloat16><<<in.R, 256, 0, st>>>(
            static_cast<const __nv_bfloat16*>(logits), in.V, in.K, tg, c, T, grad_scale,
            out.row_loss, out.logz, static_cast<__nv_bfloat16*>(out.grad));
    else
        k_topk<float><<<in.R, 256, 0, st>>>(static_cast<const float*>(logits), in.V, in.K, tg, c, T,
                                            grad_scale, out.row_loss, out.logz,
                                            static_cast<float*>(out.grad));
    k_mean_loss<<<1, 1024, 0, st>>>(tg, in.R, out.row_loss, out.loss);
    return cudaGetLastError();
}

}  // namespace vsd
