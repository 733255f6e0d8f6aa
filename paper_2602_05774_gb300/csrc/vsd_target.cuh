// vsd_target.cuh -- the target distributions of the supervised losses: per row
// either a label or a teacher's top logits, turned into a short sorted list of
// (token, probability), and the list of rows that count.
//
//   p_k = softmax over the row's valid entries of teacher_k / T
//   plogp = sum_k p_k log p_k
//
// A row is counted when its label is not the ignored one, or when it has a
// teacher entry with a finite logit, and its weight is finite and >= 0.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "vsd.h"
#include "vsd_common.cuh"

namespace vsd {

constexpr int kMaxTeacher = 128;  // entries of a teacher row: four per lane of a warp

// Programmatic dependent launch: a kernel started this way may begin before
// the one ahead of it in the stream has ended, and reads what that one wrote
// only after dep_wait().  Every kernel of a chain calls dep_wait(), so each
// one's end implies the end of all before it.
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The kernel after this one may be brought in.
__device__ __forceinline__ void dep_launch() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t launch_dep(void (*kern)(P...), dim3 grid, int threads, size_t smem, int cluster,
                       cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

// What a call says about its targets (device pointers).
struct TargetIn {
    const int32_t* labels;     // [R], or null: ids and logits below
    int32_t ignore;            // the label that is not counted
    const int32_t* ids;        // [R][K], negative: no entry
    const void* teacher;       // [R][K] of float or bf16
    int teacher_bf16;
    const float* row_weight;   // [R], or null: 1
    int R, V, K;
    float invT;
};

// The targets in the workspace.  Lists are per original row; the entries of a
// row are distinct tokens in ascending order (probabilities of equal ids added).
struct Targets {
    int32_t* n;       // [R] entries of the list; -1: the row is not counted
    int32_t* id;      // [R][K]
    float* p;         // [R][K]
    float* plogp;     // [R]
    float* w;         // [R] the row's weight
    int32_t* rowmap;  // [R] i-th counted row, in row order
    int32_t* rowinv;  // [R] its inverse, -1: not counted
    int32_t* nrows;   // counted rows
    double* wsum;     // sum of their weights, 1 where that is 0
    float* wmax;      // the largest of them
    int32_t* done;    // block counter, 0 at the start
    int32_t* status;
};

__device__ __forceinline__ float teacher_logit(const TargetIn& in, size_t i) {
    if (in.teacher_bf16)
        return __uint_as_float(
            (uint32_t)__ldg(static_cast<const unsigned short*>(in.teacher) + i) << 16);
    return __ldg(static_cast<const float*>(in.teacher) + i);
}

// The target of one row, by one warp; kPer entries of the list per lane.
template <int kPer>
__device__ __forceinline__ void target_row(const TargetIn& in, const Targets& tg, int r,
                                           int lane) {
    constexpr unsigned kAll = 0xffffffffu;
    const float w = in.row_weight ? __ldg(in.row_weight + r) : 1.f;
    int bits = (w >= 0.f && isfinite(w)) ? 0 : VSD_STATUS_BAD_ROW;
    const size_t base = (size_t)r * in.K;
    if (in.labels) {
        const int lab = __ldg(in.labels + r);
        bool counted = lab != in.ignore && !bits;
        if (lab != in.ignore && (lab < 0 || lab >= in.V)) {
            bits |= VSD_STATUS_BAD_TOKEN;
            counted = false;
        }
        if (lane == 0) {
            tg.n[r] = counted ? 1 : -1;
            tg.id[base] = counted ? lab : 0;
            tg.p[base] = 1.f;
            tg.plogp[r] = 0.f;
            tg.w[r] = w;
            if (bits) atomicOr(tg.status, bits);
        }
        return;
    }
    int id[kPer];
    float t[kPer];
    float m = -INFINITY;
    bool bad = false, far = false;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int k = lane + 32 * j;
        id[j] = -1;
        t[j] = -INFINITY;
        if (k < in.K) {
            const int v = __ldg(in.ids + base + k);
            if (v >= in.V) far = true;
            if (v >= 0 && v < in.V) {
                id[j] = v;
                t[j] = teacher_logit(in, base + k);
                if (!(t[j] < INFINITY)) bad = true;  // NaN or +inf
            }
        }
        m = fmaxf(m, t[j]);
    }
    if (__any_sync(kAll, bad)) bits |= VSD_STATUS_BAD_ROW;
    if (__any_sync(kAll, far)) bits |= VSD_STATUS_BAD_TOKEN;
    m = warp_max(m);
    const bool counted = m > -INFINITY && !(bits & VSD_STATUS_BAD_ROW);
    int n = 0;
    float plogp = 0.f;
    if (counted) {  // (one outcome for the warp)
        float e[kPer], z = 0.f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            e[j] = id[j] >= 0 ? expf((t[j] - m) * in.invT) : 0.f;
            if (!(e[j] > 0.f)) id[j] = -1;  // no mass: not in the list
            z += e[j];
        }
        z = warp_sum(z);
        const float lz = logf(z);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (id[j] >= 0) plogp += e[j] / z * ((t[j] - m) * in.invT - lz);
        plogp = warp_sum(plogp);
        // the mass of equal ids is added at the first of them, whose place is
        // the number of distinct smaller ids
        float p[kPer];
        bool first[kPer];
        int rank[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) p[j] = 0.f, first[j] = id[j] >= 0, rank[j] = 0;
#pragma unroll
        for (int jo = 0; jo < kPer; ++jo) {
            if (32 * jo >= in.K) break;
            for (int o = 0; o < 32; ++o) {
                const int oid = __shfl_sync(kAll, id[jo], o);
                const float oe = __shfl_sync(kAll, e[jo], o);
                if (oid < 0) continue;
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (id[j] == oid) {
                        p[j] += oe;
                        if (o + 32 * jo < lane + 32 * j) first[j] = false;
                    }
            }
        }
#pragma unroll
        for (int jo = 0; jo < kPer; ++jo) {
            if (32 * jo >= in.K) break;
            for (int o = 0; o < 32; ++o) {
                const int oid = __shfl_sync(kAll, first[jo] ? id[jo] : -1, o);
                if (oid < 0) continue;
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (oid < id[j]) ++rank[j];
            }
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (first[j]) {
                tg.id[base + rank[j]] = id[j];
                tg.p[base + rank[j]] = p[j] / z;
            }
            n += __popc(__ballot_sync(kAll, first[j]));
        }
    }
    if (lane == 0) {
        tg.n[r] = counted ? n : -1;
        tg.plogp[r] = plogp;
        tg.w[r] = w;
        if (bits) atomicOr(tg.status, bits);
    }
}

// The list of counted rows, the sum and the largest of their weights, by one
// block.  Each thread takes a run of rows; the runs' counts and sums are
// combined in thread order, so the result does not depend on timing.
__device__ __forceinline__ void scan_rows(const Targets& tg, int R, float* row_loss,
                                          float* logz) {
    __shared__ int cnt[32];
    __shared__ double sum[32];
    __shared__ float top[32];
    const int nt = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = (R + nt - 1) / nt;
    const int64_t r0 = (int64_t)threadIdx.x * per;
    const int64_t r1 = min((int64_t)R, r0 + per);
    int c = 0;
    double ws = 0.0;
    float wm = 0.f;
    for (int64_t b = r0; b < r1; b += 8) {  // (eight rows' loads at a time)
        int n[8];
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = b + i < r1 ? ld_cg(tg.n + b + i) : -1;
            w[i] = b + i < r1 ? ld_cg(tg.w + b + i) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n[i] >= 0) {
                ++c;
                ws += (double)w[i];
                wm = fmaxf(wm, w[i]);
            }
    }
    int inc = c;
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
    }
    const double wsw = warp_sum(ws);
    if (lane == 31) cnt[warp] = inc;
    wm = warp_max(wm);
    if (lane == 0) sum[warp] = wsw, top[warp] = wm;
    __syncthreads();
    int at = inc - c;
    for (int i = 0; i < warp; ++i) at += cnt[i];
    for (int64_t b = r0; b < r1; b += 8) {
        int n[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = b + i < r1 ? ld_cg(tg.n + b + i) : -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (b + i >= r1) break;
            const int r = (int)(b + i);
            const bool on = n[i] >= 0;
            if (tg.rowinv) tg.rowinv[r] = on ? at : -1;
            if (on) {
                if (tg.rowmap) tg.rowmap[at] = r;
                ++at;
            } else {
                row_loss[r] = 0.f;
                logz[r] = 0.f;
            }
        }
    }
    if (threadIdx.x == 0) {
        int total = 0;
        double s = 0.0;
        for (int i = 0; i < nt / 32; ++i) total += cnt[i], s += sum[i], wm = fmaxf(wm, top[i]);
        *tg.nrows = total;
        *tg.wsum = s > 0.0 ? s : 1.0;
        *tg.wmax = wm;
    }
}

// Rows packed for the LM-head losses: counted rows of hidden [R][H], in order,
// then zero rows up to a multiple of 64; rows not counted get a zero gradient.
// Nothing is packed where every row counts.
struct RowGather {
    const __nv_bfloat16* hidden;  // null: nothing to do
    __nv_bfloat16* packed;
    __nv_bfloat16* d_hidden;      // may be null
    int H;                        // a multiple of 8
};
// One block's share of the rows.
__device__ __forceinline__ void gather_rows(const RowGather& g, int R, const Targets& tg,
                                            int block, int blocks) {
    const int n = *(const volatile int*)tg.nrows;
    if (n == R) return;
    const int vecs = g.H / 8;
    const int64_t step = (int64_t)blocks * blockDim.x, t0 = (int64_t)block * blockDim.x + threadIdx.x;
    const int64_t end = (int64_t)((n + 63) / 64 * 64) * vecs;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
    for (int64_t t = t0; t < end; t += step) {
        const int i = (int)(t / vecs), v = (int)(t - (int64_t)i * vecs);
        reinterpret_cast<uint4*>(g.packed)[t] =
            i < n ? __ldg(reinterpret_cast<const uint4*>(
                              g.hidden + (size_t)ld_cg(tg.rowmap + i) * g.H) + v)
                  : zero;
    }
    if (!g.d_hidden) return;
    for (int64_t t = t0; t < (int64_t)R * vecs; t += step)
        if (ld_cg(tg.rowinv + (int)(t / vecs)) < 0) reinterpret_cast<uint4*>(g.d_hidden)[t] = zero;
}
// Elements up to which the block that makes the targets packs the rows too.
constexpr int64_t kInlineGather = 32768;

// Whether a call's targets are made by a single block, which then also clears
// the status word and the counters: one launch less where latency counts.  Each
// of its 32 warps takes up to 32 labels, or two teacher lists.
inline bool targets_in_one_block(const TargetIn& in) { return in.R <= (in.labels ? 1024 : 64); }

namespace {

// All rows' targets, then (the last block to finish) the list of counted rows.
template <int kPer, bool kOneBlock>
__global__ void __launch_bounds__(kOneBlock ? 1024 : 256)
    k_targets(TargetIn in, Targets tg, float* row_loss, float* logz, RowGather g) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    dep_launch();
    if (kOneBlock) {
        if (threadIdx.x < 4) tg.done[threadIdx.x] = 0;
        if (threadIdx.x == 0) *tg.status = 0;
        __syncthreads();
        for (int r = warp; r < in.R; r += 32) target_row<kPer>(in, tg, r, lane);
        __syncthreads();
    } else {
        const int r = (int)(blockIdx.x * 8 + warp);
        if (r < in.R) target_row<kPer>(in, tg, r, lane);
        __shared__ int last;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(tg.done, 1) == (int)gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
    }
    scan_rows(tg, in.R, row_loss, logz);
    if (kOneBlock && g.hidden) {
        __syncthreads();
        gather_rows(g, in.R, tg, 0, 1);
    }
}

// `zero_bytes` of the workspace from its start (status word, counters) are
// cleared, then the targets made.
inline cudaError_t launch_targets(const TargetIn& in, const Targets& tg, float* row_loss,
                                  float* logz, size_t zero_bytes, cudaStream_t st,
                                  const RowGather& g = RowGather{}) {
    const int per = in.labels || in.K <= 32 ? 1 : in.K <= 64 ? 2 : 4;
    if (targets_in_one_block(in)) {
        auto k = per == 1 ? k_targets<1, true> : per == 2 ? k_targets<2, true> : k_targets<4, true>;
        k<<<1, 1024, 0, st>>>(in, tg, row_loss, logz, g);
        return cudaGetLastError();
    }
    cudaError_t e = cudaMemsetAsync(tg.status, 0, zero_bytes, st);
    if (e != cudaSuccess) return e;
    auto k = per == 1 ? k_targets<1, false> : per == 2 ? k_targets<2, false> : k_targets<4, false>;
    k<<<(unsigned)((in.R + 7) / 8), 256, 0, st>>>(in, tg, row_loss, logz, g);
    return cudaGetLastError();
}

}  // namespace

}  // namespace vsd
