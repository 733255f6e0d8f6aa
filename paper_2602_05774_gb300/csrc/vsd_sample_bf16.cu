// vsd_sample_bf16.cu -- filtered sampling of bf16 logits.
#include "vsd_sample.cuh"

template cudaError_t vsd::sample<__nv_bfloat16>(const void*, const vsd::SampleArgs&, cudaStream_t);
