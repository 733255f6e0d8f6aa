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

#include <algorithm>

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
// row are in ascending order of their tokens (equal ones next to each other).
struct Targets {
    int32_t* n;       // [R] entries of the list; -1: the row is not counted
    int32_t* id;      // [R][K]
    float* p;         // [R][K]
    float* plogp;     // [R]
    float* w;         // [R] the row's weight
    double* part;     // [R / 4 + 1] scratch where rowmap is null
    int32_t* rowmap;  // [R] i-th counted row, in row order; null: no list is made
    int32_t* rowinv;  // [R] its inverse, -1: not counted
    int32_t* nrows;   // counted rows
    double* wsum;     // sum of their weights, 1 where that is 0
    float* wmax;      // the largest of them
    float* kappa;     // a constant of the call times wmax / wsum
    float* unit;      // about 1 / wsum: a power of two, by which weights and their
                      // sum may be multiplied without rounding
    float* share;     // that constant / (wsum unit)
    int32_t* done;    // block counter, 0 at the start
    int32_t* status;
};

// The power of two, within what a float and its inverse reach.
__device__ __forceinline__ void put_share(const Targets& tg, double scale, double wsum) {
    const double unit = ldexp(1.0, -max(-126, min(126, ilogb(wsum))));
    *tg.unit = (float)unit;
    *tg.share = (float)(scale / (wsum * unit));
}

__device__ __forceinline__ float teacher_logit(const TargetIn& in, size_t i) {
    if (in.teacher_bf16)
        return __uint_as_float(
            (uint32_t)__ldg(static_cast<const unsigned short*>(in.teacher) + i) << 16);
    return __ldg(static_cast<const float*>(in.teacher) + i);
}

// The target of one teacher row, by one warp; kPer entries of the list per lane.
// Returns the row's weight, or -1 where the row does not count.
template <int kPer>
__device__ __forceinline__ float target_row(const TargetIn& in, const Targets& tg, int r,
                                           int lane) {
    constexpr unsigned kAll = 0xffffffffu;
    const float w = in.row_weight ? __ldg(in.row_weight + r) : 1.f;
    int bits = (w >= 0.f && isfinite(w)) ? 0 : VSD_STATUS_BAD_ROW;
    const size_t base = (size_t)r * in.K;
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
            const float x = teacher_logit(in, base + k);  // (loaded beside the id)
            if (v >= in.V) far = true;
            if (v >= 0 && v < in.V) {
                id[j] = v;
                t[j] = x;
                if (!(x < INFINITY)) bad = true;  // NaN or +inf
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
        // an entry's place: the number of entries before it by (id, position),
        // packed into one key (an absent entry has the largest)
        static_assert(kMaxTeacher == 128, "seven bits of position");
        uint32_t key[kPer];
        int rank[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            key[j] = id[j] >= 0 ? (uint32_t)id[j] << 7 | (uint32_t)(lane + 32 * j) : 0xffffffffu;
            rank[j] = 0;
        }
#pragma unroll
        for (int jo = 0; jo < kPer; ++jo) {
            if (32 * jo >= in.K) break;
#pragma unroll 8
            for (int o = 0; o < 32; ++o) {
                const uint32_t other = __shfl_sync(kAll, key[jo], o);
#pragma unroll
                for (int j = 0; j < kPer; ++j) rank[j] += other < key[j];
            }
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (id[j] >= 0) {
                tg.id[base + rank[j]] = id[j];
                tg.p[base + rank[j]] = e[j] / z;
            }
            n += __popc(__ballot_sync(kAll, id[j] >= 0));
        }
    }
    if (lane == 0) {
        tg.n[r] = counted ? n : -1;
        tg.plogp[r] = plogp;
        tg.w[r] = w;
        if (bits) atomicOr(tg.status, bits);
    }
    return counted ? w : -1.f;
}

// The list of counted rows, the sum and the largest of their weights, by one
// block of whole warps.  A thread takes a run of rows, 16 at a time; the runs'
// counts and sums are combined in an order that timing does not change.
// look(b, n, w): flags (n >= 0) and weights of rows b .. b + 15 that the thread
// owns.
template <int kBatch, typename Look>
__device__ __forceinline__ void scan_rows(const Targets& tg, int R, double scale, float* row_loss,
                                          float* logz, Look look) {
    __shared__ int cnt[32];
    __shared__ double sum[32];
    __shared__ float top[32];
    const int nt = blockDim.x, nw = nt / 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = (R + nt - 1) / nt;
    const int64_t r0 = min((int64_t)R, (int64_t)threadIdx.x * per);
    const int64_t r1 = min((int64_t)R, r0 + per);
    int c = 0;
    double ws = 0.0;
    float wm = 0.f;
    uint32_t mask = 0;  // the last batch's flags
    auto batch = [&](int64_t b) {
        int n[kBatch];
        float w[kBatch];
        look(b, r1, n, w);
        mask = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (n[i] >= 0) {
                mask |= 1u << i;
                ++c;
                ws += (double)w[i];
                wm = fmaxf(wm, w[i]);
            }
    };
    for (int64_t b = r0; b < r1; b += kBatch) batch(b);
    int inc = c;
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
    }
    int at = inc - c;
    ws = warp_sum(ws);
    wm = warp_max(wm);
    if (lane == 31) cnt[warp] = inc;
    if (lane == 0) sum[warp] = ws, top[warp] = wm;
    __syncthreads();
    // every warp: the count of the warps before it
    int others = lane < nw ? cnt[lane] : 0;
    const int all = __reduce_add_sync(0xffffffffu, others);
    at += __reduce_add_sync(0xffffffffu, lane < warp ? others : 0);
    if (warp == 0) {
        ws = warp_sum(lane < nw ? sum[lane] : 0.0);
        wm = warp_max(lane < nw ? top[lane] : 0.f);
        if (lane == 0) {
            ws = ws > 0.0 ? ws : 1.0;
            *tg.nrows = all;
            *tg.wsum = ws;
            *tg.wmax = wm;
            *tg.kappa = (float)(scale * (double)wm / ws);
            put_share(tg, scale, ws);
        }
    }
    for (int64_t b = r0; b < r1; b += kBatch) {
        if (per > kBatch) batch(b);  // (else still held)
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (b + i >= r1) break;
            const int r = (int)(b + i);
            const bool on = mask >> i & 1;
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
}

// Whether a call's targets are made by a single block, which then also clears
// the status word and the counters: one launch less where latency counts.  A
// thread takes up to 8 labels, or a warp two teacher lists.
inline bool targets_in_one_block(const TargetIn& in) { return in.R <= (in.labels ? 8192 : 64); }

namespace {

// The targets of up to kBatch labels from row b on, to r1; all loads first.
template <int kBatch>
__device__ __forceinline__ void label_rows(const TargetIn& in, const Targets& tg, int64_t b,
                                           int64_t r1, int (&n)[kBatch], float (&w)[kBatch],
                                           int* bits) {
    int lab[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) lab[i] = __ldg(in.labels + min(b + i, r1 - 1));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
        w[i] = in.row_weight ? __ldg(in.row_weight + min(b + i, r1 - 1)) : 1.f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
        n[i] = -1;
        if (b + i >= r1) continue;
        const bool bad_w = !(w[i] >= 0.f && isfinite(w[i]));
        const bool far = lab[i] != in.ignore && (lab[i] < 0 || lab[i] >= in.V);
        if (bad_w) *bits |= VSD_STATUS_BAD_ROW;
        if (far) *bits |= VSD_STATUS_BAD_TOKEN;
        n[i] = lab[i] != in.ignore && !far && !bad_w ? 1 : -1;
        tg.n[b + i] = n[i];
        tg.id[b + i] = n[i] > 0 ? lab[i] : 0;
        tg.p[b + i] = 1.f;
        tg.plogp[b + i] = 0.f;
        tg.w[b + i] = w[i];
    }
}

// All rows' targets, then (the last block to finish) the list of counted rows.
// kPer: entries of a teacher row per lane, or the batch of labels of a thread.
template <int kPer, bool kLabels, bool kOneBlock>
__global__ void __launch_bounds__(1024)
    k_targets(TargetIn in, Targets tg, double scale, float* row_loss, float* logz) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ float ws[8];
    __shared__ double sums[8];
    dep_launch();
    int bits = 0;
    auto made = [&](int64_t b, int64_t r1, int (&n)[16], float (&w)[16]) {  // by any block
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = ld_cg(tg.n + min(b + i, r1 - 1));
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = ld_cg(tg.w + min(b + i, r1 - 1));
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (b + i >= r1) n[i] = -1;
    };
    if constexpr (kOneBlock) {
        if (threadIdx.x < 4) tg.done[threadIdx.x] = 0;
        if (threadIdx.x == 0) *tg.status = 0;
        __syncthreads();
        if constexpr (kLabels) {
            scan_rows<kPer>(tg, in.R, scale, row_loss, logz,
                            [&](int64_t b, int64_t r1, int (&n)[kPer], float (&w)[kPer]) {
                                label_rows<kPer>(in, tg, b, r1, n, w, &bits);
                            });
            if (bits) atomicOr(tg.status, bits);
        } else {
            for (int r = warp; r < in.R; r += blockDim.x / 32) target_row<kPer>(in, tg, r, lane);
            __syncthreads();
            scan_rows<16>(tg, in.R, scale, row_loss, logz, made);
        }
    } else {
        if constexpr (kLabels) {
            const int64_t r = blockIdx.x * (int64_t)256 + threadIdx.x;
            int n[1];
            float w[1];
            if (r < in.R) label_rows<1>(in, tg, r, r + 1, n, w, &bits);
            if (bits) atomicOr(tg.status, bits);
        } else {
            const int64_t r = blockIdx.x * (int64_t)(blockDim.x / 32) + warp;
            const float w = r < in.R ? target_row<kPer>(in, tg, (int)r, lane) : -1.f;
            if (!tg.rowmap) {  // no list: the blocks' sums are enough
                if (lane == 0) {
                    ws[warp] = w;
                    if (r < in.R && w < 0.f) row_loss[r] = logz[r] = 0.f;
                }
                __syncthreads();
                if (threadIdx.x == 0) {
                    double sum = 0.0;
                    for (int i = 0; i < (int)blockDim.x / 32; ++i)
                        if (ws[i] > 0.f) sum += (double)ws[i];
                    tg.part[blockIdx.x] = sum;
                }
            }
        }
        __shared__ int last;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(tg.done, 1) == (int)gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        if (tg.rowmap) {
            scan_rows<16>(tg, in.R, scale, row_loss, logz, made);
            return;
        }
        double sum = 0.0;
        for (int b = threadIdx.x; b < (int)gridDim.x; b += blockDim.x) sum += ld_cg(tg.part + b);
        sum = warp_sum(sum);
        if (lane == 0) sums[warp] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.0;
            for (int i = 0; i < (int)blockDim.x / 32; ++i) sum += sums[i];
            sum = sum > 0.0 ? sum : 1.0;
            *tg.wsum = sum;
            put_share(tg, scale, sum);
        }
    }
}

// `zero_bytes` of the workspace from its start (status word, counters) are
// cleared, then the targets made; scale: of kappa.
inline cudaError_t launch_targets(const TargetIn& in, const Targets& tg, double scale,
                                  float* row_loss, float* logz, size_t zero_bytes, cudaStream_t st) {
    const int per = in.K <= 32 ? 1 : in.K <= 64 ? 2 : 4;
    if (targets_in_one_block(in)) {
        // threads: a label each while they reach, then four at a time; a warp per list
        const int threads = in.labels ? (in.R <= 256 ? 256 : 1024)
                                      : std::max(64, std::min(1024, 32 * in.R));
        auto k = in.labels ? (in.R <= 1024 ? k_targets<1, true, true> : k_targets<4, true, true>)
                 : per == 1 ? k_targets<1, false, true>
                 : per == 2 ? k_targets<2, false, true>
                            : k_targets<4, false, true>;
        return launch_dep(false, k, dim3(1), threads, 0, 1, st, in, tg, scale, row_loss, logz);
    }
    cudaError_t e = cudaMemsetAsync(tg.status, 0, zero_bytes, st);
    if (e != cudaSuccess) return e;
    auto k = in.labels  ? k_targets<1, true, false>
             : per == 1 ? k_targets<1, false, false>
             : per == 2 ? k_targets<2, false, false>
                        : k_targets<4, false, false>;
    const int threads = in.labels ? 256 : 128, rows = in.labels ? 256 : 4;  // of a block
    return launch_dep(false, k, dim3((unsigned)((in.R + rows - 1) / rows)), threads, 0, 1, st, in,
                      tg, scale, row_loss, logz);
}

}  // namespace

}  // namespace vsd
