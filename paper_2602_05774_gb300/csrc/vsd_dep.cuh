// vsd_dep.cuh -- kernels that begin before the one ahead of them has ended, and
// bounded waits.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "vsd_common.cuh"

namespace vsd {

// Programmatic dependent launch: a kernel started this way may begin before
// the one ahead of it in the stream has ended, and reads what that one wrote
// only after dep_wait().  Every kernel of a chain calls dep_wait(), so each
// one's end implies the end of all before it.
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The kernel after this one may be brought in.
__device__ __forceinline__ void dep_launch() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// early: whether it may.  A persistent grid of clusters that fills the GPU may
// not: placed around the blocks of the kernel before, not all of its clusters
// would fit at once, and the rest would run after them.
template <typename... P, typename... A>
cudaError_t launch_dep(bool early, void (*kern)(P...), dim3 grid, int threads, size_t smem,
                       int cluster, cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    unsigned n = 0;
    if (early) {
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = (unsigned)cluster;
        at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = at;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

// Waits until done(), at most until give_up() or for limit_ns; whether done()
// held.  The clock is read once in 256 tries: reading it is slow,
// and a warp that reads it is late for what it waits for.
template <typename Done, typename GiveUp>
__device__ __forceinline__ bool bounded_wait(Done done, GiveUp give_up, uint64_t limit_ns) {
    uint64_t t0 = 0;
    for (uint32_t n = 1;; ++n) {
        if (done()) return true;
        if (n & 255u) continue;
        if (give_up()) return false;
        const uint64_t now = global_timer_ns();
        if (t0 == 0) t0 = now;
        else if (now - t0 > limit_ns) return false;
    }
}

}  // namespace vsd
