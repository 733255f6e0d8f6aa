// vsd_rowloss.cuh -- softmax, loss and gradient of rows of logits in memory,
// each row read once:
//
//   (m, s) = (max x, sum 2^{(x - m) c}),  c = log2(e) / T,
//   l = plogp + ln s - sum_k p_k (x_{id_k} - m) / T,  log Z = m / T + ln s,
//   g_v = a (2^{(x_v - m) c} / s - sum_k p_k [v = id_k]).
//
// Bound by memory: one read of the row, one write of its gradient.  A cluster of
// up to 8 blocks holds a row in shared memory between the two, a segment each
// (bulk copies, four barriers so that the first part is worked on while the rest
// arrives); the blocks' partial sums meet in distributed shared memory.  Small
// segments keep several blocks on an SM, so that some load while others wait
// for their cluster or write.  A row too long for the cluster is read twice, in
// rounds.  A row that does not start on 16 bytes is laid out from the vector
// boundary below it; its ragged first and last vectors are filled element by
// element.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_target.cuh"

namespace vsd {
namespace {

#ifndef ROW_T
#define ROW_T 128
#endif
#ifndef ROW_SEG
#define ROW_SEG 32768
#endif
constexpr int kRowThreads = ROW_T;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kRowBars = 4;
constexpr int kSegBytes = ROW_SEG;    // a block's segment, where the cluster reaches over the row
constexpr int kSegMax = 200 << 10;  // at most
constexpr uint64_t kRowWaitNs = 2000000000ull;

struct RowArgs {
    Targets tg;
    int rows, V, K, rounds;
    int vper;            // vectors of a block's segment
    int64_t ldx, ldg;    // row pitches in elements
    int gcols;           // columns of a gradient row that are written (zero from V on)
    float c, invT;
    float *row_loss, *logz;
    bool same_align;     // gradient rows start where logits rows do, modulo 16 bytes
};

template <typename T> __device__ __forceinline__ float row_value(T x);
template <> __device__ __forceinline__ float row_value(float x) { return x; }
template <> __device__ __forceinline__ float row_value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void row_put(float* x, float f) { *x = f; }
__device__ __forceinline__ void row_put(__nv_bfloat16* x, float f) { *x = __float2bfloat16_rn(f); }

// N gradient elements, N sizeof(TO) = 8 or 16 bytes.
template <int N> __device__ __forceinline__ void row_store(float* g, const float* o) {
    static_assert(N == 4, "a 16-byte vector of floats");
    *reinterpret_cast<float4*>(g) = make_float4(o[0], o[1], o[2], o[3]);
}
template <int N> __device__ __forceinline__ void row_store(__nv_bfloat16* g, const float* o) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(o[2 * i], o[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    if (N == 8) *reinterpret_cast<uint4*>(g) = make_uint4(w[0], w[1], w[2 % (N / 2)], w[3 % (N / 2)]);
    else *reinterpret_cast<uint2*>(g) = make_uint2(w[0], w[1]);
}

// LM: the rows are the LM head's packed ones (row i is original row rowmap[i],
// there are *nrows of them, rows up to the next multiple of 64 are zeroed) and
// the gradient is scaled for the products (top, see there).
template <typename TI, typename TO, bool LM>
__global__ void __launch_bounds__(kRowThreads)
    k_row_loss(const TI* logits, TO* grad, RowArgs a, float top) {
    constexpr int PV = Traits<TI>::kPerVec;
    extern __shared__ __align__(128) unsigned char row_smem[];
    uint4* seg = reinterpret_cast<uint4*>(row_smem);
    __shared__ uint64_t bars[kRowBars];
    __shared__ float2 part[kRowWarps], cpart[kMaxCluster];
    __shared__ float xs[kMaxTeacher];
    uint32_t rank, C;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int i = (int)(blockIdx.x / C);
    const int V = a.V;
    const TI* x = logits + (size_t)i * a.ldx;
    const int off = (int)(((uintptr_t)x / sizeof(TI)) % PV);
    const int nvec = (V + off + PV - 1) / PV;
    const int in0 = off ? 1 : 0, in1 = (V + off) / PV;  // whole vectors
    const int stride = (int)C * a.vper;
    dep_launch();
    if (tid == 0) {
        for (int b = 0; b < kRowBars; ++b) mbar_init(&bars[b], 1);
        mbar_init_fence();
    }
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    // vectors v0 .. v1 - 1 of the row are this block's in round rd; quarter q of
    // them is counted on barrier q
    const int vq = (a.vper + kRowBars - 1) / kRowBars;
    auto load = [&](int rd) {
        const int v0 = rd * stride + (int)rank * a.vper, v1 = min(nvec, v0 + a.vper);
        if (tid == 0) {
            const uint64_t pol = policy_evict_first();
            for (int q = 0; q < kRowBars; ++q) {
                const int b = max(v0 + q * vq, in0), e = min(min(v0 + (q + 1) * vq, v0 + a.vper), in1);
                const uint32_t bytes = e > b ? 16u * (uint32_t)(e - b) : 0u;
                mbar_expect_tx(&bars[q], bytes);
                if (bytes)
                    bulk_g2s(seg + (b - v0), x + ((int64_t)b * PV - off), bytes, &bars[q], pol);
            }
        }
        // the ragged ends
        if (warp == 1 && lane < 2 * PV) {
            const int v = lane < PV ? 0 : nvec - 1, el = lane % PV;
            const int col = v * PV - off + el;
            if (v >= v0 && v < v1 && (v < in0 || v >= in1)) {
                TI* d = reinterpret_cast<TI*>(seg + (v - v0)) + el;
                if (col >= 0 && col < V) *d = x[col];
                else row_put(d, -INFINITY);
            }
        }
    };
    if (!LM) {
        load(0);  // (these logits were there before the targets' kernel began)
        dep_wait();
    } else {
        dep_wait();
    }
    if (LM) {  // the kernel before this one stored the logits (all rows' space may be read)
        if (tid == 0) asm volatile("fence.proxy.async;" ::: "memory");
        load(0);
    }
    const int n_rows = LM ? *(const volatile int*)a.tg.nrows : a.rows;
    const bool real = i < n_rows;
    const int r = LM ? (real ? a.tg.rowmap[i] : 0) : i;
    const int n = real ? a.tg.n[r] : -1;
    const int32_t* id = a.tg.id + (size_t)r * a.K;
    const float* p = a.tg.p + (size_t)r * a.K;
    TO* g = grad ? grad + (size_t)i * a.ldg : nullptr;
    __syncthreads();  // the barriers and the ragged ends are set
    bool ok = true;
    auto arrived = [&](int q, int rd) {
        if (mbar_try_wait(&bars[q], rd & 1)) return;
        const uint64_t t0 = global_timer_ns();
        while (!mbar_try_wait(&bars[q], rd & 1))
            if (global_timer_ns() - t0 > kRowWaitNs) {
                ok = false;
                atomicOr(a.tg.status, VSD_STATUS_TIMEOUT);
                return;
            }
    };
    float M = 0.f, S = 1.f;
    int loads = 0;  // of this block so far
    if (n >= 0) {
        // the target logits (read before any gradient is written, used after)
        const float xv = tid < n ? row_value(x[id[tid]]) : 0.f;
        float m = -INFINITY, s = 0.f;
        for (int rd = 0; rd < a.rounds; ++rd) {
            if (rd) {
                __syncthreads();  // the segment has been read
                if (tid == 0) fence_proxy_async();
                load(rd);
                __syncthreads();
            }
            const int v0 = rd * stride + (int)rank * a.vper, cnt = min(nvec, v0 + a.vper) - v0;
            for (int q = 0; q < kRowBars; ++q) {
                arrived(q, loads);
                const int e = min((q + 1) * vq, cnt);
                for (int j = q * vq + tid; j < e; j += 4 * kRowThreads) {
                    uint4 b[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        b[u] = j + u * kRowThreads < e
                                   ? seg[j + u * kRowThreads]
                                   : make_uint4(Traits<TI>::kNegInf, Traits<TI>::kNegInf,
                                                Traits<TI>::kNegInf, Traits<TI>::kNegInf);
                    const float nm = fmaxf(fmaxf(fmaxf(vec_max<TI>(b[0]), vec_max<TI>(b[1])),
                                                 fmaxf(vec_max<TI>(b[2]), vec_max<TI>(b[3]))), m);
                    const float z = nm > -INFINITY ? nm : 0.f;  // (a NaN still reaches the sum)
                    const uint64_t z2 = f2(z, z), c2 = f2(a.c, a.c);
                    uint64_t acc = f2(0.f, 0.f);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        uint64_t v[PV / 2];
                        vec_pairs<TI>(b[u], v);
#pragma unroll
                        for (int w = 0; w < PV / 2; ++w) acc = f2add(acc, f2_mass(v[w], z2, c2));
                    }
                    float lo, hi;
                    f2split(acc, lo, hi);
                    s = s * ex2((m - z) * a.c) + (lo + hi);
                    m = nm;
                }
            }
            ++loads;
        }
        if (tid < n) xs[tid] = xv;
        const float wm = warp_max(m), wz = wm > -INFINITY ? wm : 0.f;
        s = warp_sum(s * ex2(((m > -INFINITY ? m : wz) - wz) * a.c));
        if (lane == 0) part[warp] = make_float2(wm, s);
        __syncthreads();
        auto join = [&](const float2* e, int cnt) {
            M = e[0].x;
            for (int k = 1; k < cnt; ++k) M = fmaxf(M, e[k].x);
            S = 0.f;
            const float z = M > -INFINITY ? M : 0.f;  // (a part without mass adds 0, or its NaN)
            for (int k = 0; k < cnt; ++k) S += e[k].y * ex2((e[k].x - z) * a.c);
        };
        join(part, kRowWarps);
        if (C > 1) {
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // the others have begun
            if (tid < (int)C) {
                uint32_t dst;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(dst) : "r"(smem_u32(&cpart[rank])), "r"(tid));
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};"
                             :: "r"(dst), "f"(M), "f"(S) : "memory");
            }
            asm volatile("barrier.cluster.arrive.release.aligned;\n\t"
                         "barrier.cluster.wait.acquire.aligned;" ::: "memory");
            join(cpart, (int)C);
        }
    } else {
        // (copies of a row that does not count land before the block may exit)
        for (int q = 0; q < kRowBars; ++q) arrived(q, 0);
        if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    const float inv = 1.f / S;
    float coef = 0.f;
    if (n >= 0) {
        const float w = a.tg.w[r];
        if (LM) {
            const float wm = *a.tg.wmax;
            coef = wm > 0.f ? top * (w / wm) : 0.f;
        } else {
            coef = w * *a.tg.share;
        }
    }
    if (g && (!LM || i < (n_rows + 63) / 64 * 64)) {
        const bool on = n >= 0;
        const float cs = coef * inv;
        const uint64_t m2 = f2(M, M), c2 = f2(a.c, a.c), cs2 = f2(cs, cs);
        for (int rd = 0; rd < a.rounds; ++rd) {
            if (on && a.rounds > 1) {
                __syncthreads();
                if (tid == 0) fence_proxy_async();
                load(rd);
                __syncthreads();
                for (int q = 0; q < kRowBars; ++q) arrived(q, loads);
                ++loads;
            }
            const int v0 = rd * stride + (int)rank * a.vper, cnt = min(nvec, v0 + a.vper) - v0;
#pragma unroll 4
            for (int j = tid; j < cnt; j += kRowThreads) {
                uint64_t v[PV / 2];
                vec_pairs<TI>(on ? seg[j] : make_uint4(0u, 0u, 0u, 0u), v);
                float o[PV];
#pragma unroll
                for (int w = 0; w < PV / 2; ++w) {
                    float lo, hi;
                    f2split(f2mul(f2_mass(v[w], m2, c2), cs2), lo, hi);
                    o[2 * w] = on ? lo : 0.f;
                    o[2 * w + 1] = on ? hi : 0.f;
                }
                const int e0 = (v0 + j) * PV - off;
                if (a.same_align && e0 >= 0 && e0 + PV <= V) {
                    row_store<PV>(g + e0, o);
                } else {
#pragma unroll
                    for (int w = 0; w < PV; ++w)
                        if (e0 + w >= 0 && e0 + w < V) row_put(g + e0 + w, o[w]);
                }
            }
        }
        if (LM && rank == C - 1)
            for (int v = V + tid; v < a.gcols; v += kRowThreads) row_put(g + v, 0.f);
        __syncthreads();
        if (tid < n && (tid == 0 || id[tid - 1] != id[tid])) {
            // the target entries this block wrote as dense ones; equal tokens add
            const int v = id[tid], j = (v + off) / PV % stride;
            if (j / a.vper == (int)rank) {
                float q = p[tid];
                for (int k = tid + 1; k < n && id[k] == v; ++k) q += p[k];
                row_put(g + v, coef * (ex2((xs[tid] - M) * a.c) * inv - q));
            }
        }
    }
    // the row's loss
    if (rank != 0 || warp != 0 || n < 0) return;
    float dot = 0.f;
    for (int k = lane; k < n; k += 32) dot = fmaf(p[k], xs[k] - M, dot);
    dot = warp_sum(dot);
    if (lane == 0) {
        const float l = logf(S), lz = fmaf(M, a.invT, l);
        if (!isfinite(lz)) atomicOr(a.tg.status, VSD_STATUS_BAD_ROW);
        a.logz[r] = lz;
        a.row_loss[r] = a.tg.plogp[r] + (l - dot * a.invT);
    }
}

// The weighted mean of the rows' losses, in row order, by one block.
__global__ void __launch_bounds__(1024) k_mean_loss(Targets tg, int R, const float* row_loss,
                                                    float* loss) {
    __shared__ double part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    dep_launch();
    dep_wait();
    double sum = 0.0;
    for (int64_t b = threadIdx.x; b < R; b += 1024 * 4) {
        float w[4], l[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t r = min(b + u * 1024, (int64_t)R - 1);
            const bool on = ld_cg(tg.n + r) >= 0 && b + u * 1024 < R;
            w[u] = on ? ld_cg(tg.w + r) : 0.f;
            l[u] = ld_cg(row_loss + r);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (w[u] != 0.f) sum += (double)w[u] * (double)l[u];
    }
    sum = warp_sum(sum);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        sum = warp_sum(lane < (int)blockDim.x / 32 ? part[lane] : 0.0);
        if (lane == 0) *loss = (float)(sum / *tg.wsum);
    }
}

// Launches `rows` rows (a.rounds and a.vper are set here).
template <typename TI, typename TO, bool LM>
cudaError_t launch_row_loss(const TI* logits, TO* grad, RowArgs a, int64_t rows, float top,
                            int sms, cudaError_t (*smem_opt_in)(const void*, size_t),
                            cudaStream_t st) {
    constexpr int PV = Traits<TI>::kPerVec;
    const int64_t need = ((int64_t)a.V + 2 * PV - 2) / PV;  // vectors, whatever the offset
    int64_t C = 1;
    while (C < kMaxCluster && C * kSegBytes < 16 * need) C *= 2;
    // few rows: spread each over more SMs, while a thread has a vector
    while (C < kMaxCluster && rows * C < 2 * sms && C * kRowThreads < need) C *= 2;
    const int64_t vper = std::min<int64_t>((need + C - 1) / C, kSegMax / 16);
    a.vper = (int)vper;
    a.rounds = (int)((need + C * vper - 1) / (C * vper));
    const size_t smem = (size_t)vper * 16;
    auto k = k_row_loss<TI, TO, LM>;
    cudaError_t e = smem_opt_in((const void*)k, smem);
    if (e != cudaSuccess) return e;
    return launch_dep(k, dim3((unsigned)(rows * C)), kRowThreads, smem, (int)C, st, logits, grad, a,
                      top);
}

}  // namespace
}  // namespace vsd
