// vsd_loss.h -- host-side launchers of the supervised losses: the LM-head
// losses (vsd_lmloss.cu) and distillation on logits in hand (vsd_topk.cu).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include "vsd.h"
#include "vsd_target.cuh"

namespace vsd {

// Workspaces: arrays at multiples of 256 bytes.
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
template <typename U> U* ws_at(void* ws, size_t off) {
    return reinterpret_cast<U*>(static_cast<char*>(ws) + off);
}

// Sizes of an LM-head loss call.
struct LmLossShape {
    int R, V, H, K;
    bool dh, dw;  // gradients asked for
    int piece;    // vocabulary columns at a time, 0: the library's choice
};
bool lmloss_shape_ok(const LmLossShape& s);
size_t lmloss_workspace_bytes(const LmLossShape& s);
cudaError_t lmloss(const LmLossShape& s, const void* hidden, const void* weight,
                   const TargetIn& in, float T, float grad_scale, const vsd_loss_outputs& out,
                   void* ws, cudaStream_t stream);

bool topk_shape_ok(int R, int V, int K);
size_t topk_workspace_bytes(int R, int V, int K);
cudaError_t topk_distill(const void* logits, bool bf16, const TargetIn& in, float T,
                         float grad_scale, const vsd_loss_outputs& out, void* ws,
                         cudaStream_t stream);

}  // namespace vsd
