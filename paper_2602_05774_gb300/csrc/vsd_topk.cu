// vsd_topk.cu -- distillation from a teacher's top logits on logits in hand:
//
//   q_r = softmax(x_r / T),  l_r = sum_k p_rk (log p_rk - log q_r(id_rk)),
//   grad_rv = a_r (q_r(v) - sum_k p_rk [v = id_rk]),  a_r = scale w_r / (T sum w).
//
// The rows' targets first (vsd_target.cuh), then one pass over the logits
// (vsd_rowloss.cuh), which starts loading while the targets are made.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_launch.h"
#include "vsd_loss.h"
#include "vsd_rowloss.cuh"

namespace vsd {
namespace {

struct TopkWs {
    size_t status, done, zero_end, nrows, wsum, wmax, kappa, unit, share, n, id, p, plogp, w, part,
        total;
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
    w.kappa = take(4);
    w.unit = take(4);
    w.share = take(4);
    w.n = take(4 * r);
    w.id = take(4 * rk);
    w.p = take(4 * rk);
    w.plogp = take(4 * r);
    w.w = take(4 * r);
    w.part = take(8 * (r / 4 + 1));
    w.total = o;
    return w;
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
    RowArgs a{};
    a.tg = Targets{ws_at<int32_t>(ws, w.n), ws_at<int32_t>(ws, w.id), ws_at<float>(ws, w.p),
                   ws_at<float>(ws, w.plogp), ws_at<float>(ws, w.w), ws_at<double>(ws, w.part),
                   nullptr, nullptr, ws_at<int32_t>(ws, w.nrows), ws_at<double>(ws, w.wsum),
                   ws_at<float>(ws, w.wmax), ws_at<float>(ws, w.kappa), ws_at<float>(ws, w.unit),
                   ws_at<float>(ws, w.share), ws_at<int32_t>(ws, w.done),
                   ws_at<int32_t>(ws, w.status)};
    a.rows = in.R;
    a.V = in.V;
    a.K = in.K;
    a.ldx = a.ldg = in.V;
    a.gcols = in.V;
    a.row_loss = out.row_loss;
    a.logz = out.logz;
    a.same_align = (((uintptr_t)logits ^ (uintptr_t)out.grad) & 15) == 0;
    cudaError_t e = launch_targets(in, a.tg, (double)grad_scale / (double)T, out.row_loss,
                                   out.logz, w.zero_end, st);
    if (e != cudaSuccess) return e;
    if (bf16)
        e = launch_row_loss<__nv_bfloat16, __nv_bfloat16, false>(
            static_cast<const __nv_bfloat16*>(logits), static_cast<__nv_bfloat16*>(out.grad), a,
            T, 1.f, resident_clusters, st);
    else
        e = launch_row_loss<float, float, false>(static_cast<const float*>(logits),
                                                 static_cast<float*>(out.grad), a, T, 1.f,
                                                 resident_clusters, st);
    if (e != cudaSuccess) return e;
    return launch_dep(true, k_mean_loss, dim3(1), 1024, 0, 1, st, a.tg, in.R, out.row_loss,
                      out.loss);
}

}  // namespace vsd
