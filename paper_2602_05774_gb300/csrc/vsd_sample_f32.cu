// vsd_sample_f32.cu -- filtered sampling of float logits.
#include "vsd_sample.cuh"

template cudaError_t vsd::sample<float>(const void*, const vsd::SampleArgs&, cudaStream_t);
