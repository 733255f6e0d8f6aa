// vsd_sample.h -- host-side launchers of the filtered sampling, one for each type of
// logits (vsd_sample_f32.cu, vsd_sample_bf16.cu).
#pragma once

#include <cuda_runtime.h>

#include "vsd_decode.h"

namespace vsd {

constexpr float kMinT = 0x1p-64f, kMaxT = 0x1p64f;

struct SampleArgs {
    vsd_policy policy;
    const float* u;
    vsd_filtered_outputs out;
    int R, V, shift;
    bool same_align;     // filtered rows start where logits rows do, modulo 16 bytes
    int* status;
};

// Of logits of type T, rows V elements apart.
template <typename T>
cudaError_t sample(const void* logits, const SampleArgs& a, cudaStream_t st);

}  // namespace vsd
