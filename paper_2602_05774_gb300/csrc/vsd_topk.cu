// vsd_topk.cu -- distillation from a teacher's top logits on logits in hand:
//
//   q_r = softmax(x_r / T),  l_r = sum_k p_rk (log p_rk - log q_r(id_rk)),
//   grad_rv = a_r (q_r(v) - sum_k p_rk [v = id_rk]),  a_r = scale w_r / (T sum w).
//
// Bound by memory: a row is read once and its gradient written once.  The row
// is held in registers between the two, 16 vectors of 16 bytes per thread at
// most, by one block or by a cluster of up to 8 whose partial sums meet in
// shared memory; a longer row (over 262144 bf16 or 131072 float32 logits) is
// read twice.  A row that does not start on 16 bytes is read from the vector
// boundary below it, its two ragged ends element by element.
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

constexpr int kRowThreads = 256;
constexpr int kMaxCluster = 8;
constexpr int kMaxVecs = 16;

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct TopkWs {
    size_t status, done, zero_end, nrows, wsum, wmax, n, id, p, plogp, w, total;
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
    w.total = o;
    return w;
}

template <typename U> U* at(void* ws, size_t off) {
    return reinterpret_cast<U*>(static_cast<char*>(ws) + off);
}

__device__ __forceinline__ uint32_t raw_of(const float* x) { return *reinterpret_cast<const uint32_t*>(x); }
__device__ __forceinline__ uint32_t raw_of(const __nv_bfloat16* x) {
    return *reinterpret_cast<const unsigned short*>(x);
}
__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ float value_of(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* x, float f) { *x = f; }
__device__ __forceinline__ void put(__nv_bfloat16* x, float f) { *x = __float2bfloat16_rn(f); }

// (not the read-only path: the gradient may overwrite the logits)
__device__ __forceinline__ uint4 ld_once(const void* p, uint64_t pol) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p), "l"(pol) : "memory");
    return r;
}

// Vector j of a row that starts `off` elements past a vector boundary:
// elements j PV - off .. + PV - 1, -inf outside [0, V).
template <typename T>
__device__ __forceinline__ uint4 load_vec(const T* x, int V, int j, int off, uint64_t pol) {
    constexpr int PV = Traits<T>::kPerVec;
    const int e0 = j * PV - off;
    if (e0 >= 0 && e0 + PV <= V) return ld_once(x + e0, pol);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Traits<T>::kNegInf;
    if (e0 < V) {
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            const int v = e0 + i;
            if (v >= 0 && v < V) {
                if (PV == 4) w[i & 3] = raw_of(x + v);
                else w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xFFFFu) | raw_of(x + v) << 16
                                         : (w[i >> 1] & 0xFFFF0000u) | raw_of(x + v);
            }
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T> __device__ __forceinline__ uint4 pack_vec(const float* g);
template <> __device__ __forceinline__ uint4 pack_vec<float>(const float* g) {
    return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]),
                      __float_as_uint(g[3]));
}
template <> __device__ __forceinline__ uint4 pack_vec<__nv_bfloat16>(const float* g) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * i], g[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct TopkArgs {
    Targets tg;
    int R, V, K, rounds;
    float c, T, grad_scale;
    float *row_loss, *logz, *loss;
    bool same_align;  // gradient rows start where logits rows do, modulo 16 bytes
};

// One row per cluster.  Thread t of CTA b holds vectors (b NV + k) 256 + t of a
// round, k < NV.
template <typename T, int NV>
__global__ void __launch_bounds__(kRowThreads)
    k_topk(const T* logits, T* grad, TopkArgs a) {
    constexpr int PV = Traits<T>::kPerVec;
    constexpr int kWarpsN = kRowThreads / 32;
    __shared__ float2 part[kWarpsN], cpart[kMaxCluster];
    __shared__ float xs[kMaxTeacher];
    __shared__ int last;
    uint32_t rank, C;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = (int)(blockIdx.x / C);
    const int V = a.V;
    const T* x = logits + (size_t)r * V;
    const int off = (int)(((uintptr_t)x / sizeof(T)) % PV);
    const int nvec = (V + off + PV - 1) / PV;
    const int per_round = (int)C * NV * kRowThreads;
    const int j0 = (int)rank * NV * kRowThreads + tid;
    const uint64_t pol = policy_evict_first();
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    uint4 buf[NV];
    auto load = [&](int rd) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int j = rd * per_round + j0 + k * kRowThreads;
            buf[k] = j < nvec ? load_vec(x, V, j, off, pol)
                              : make_uint4(Traits<T>::kNegInf, Traits<T>::kNegInf,
                                           Traits<T>::kNegInf, Traits<T>::kNegInf);
        }
    };
    load(0);  // (the logits were there before the kernel that makes the targets began)
    dep_wait();
    const int n = a.tg.n[r];
    const int32_t* id = a.tg.id + (size_t)r * a.K;
    const float* p = a.tg.p + (size_t)r * a.K;
    T* g = grad ? grad + (size_t)r * V : nullptr;
    float M = 0.f, S = 1.f;
    if (n >= 0) {
        if (tid < n) xs[tid] = value_of(x[id[tid]]);  // (before any gradient is written)
        float m = -INFINITY, s = 0.f;
        for (int rd = 0; rd < a.rounds; ++rd) {
            if (rd) load(rd);
            float gm = vec_max<T>(buf[0]);
#pragma unroll
            for (int k = 1; k < NV; ++k) gm = fmaxf(gm, vec_max<T>(buf[k]));
            const float nm = fmaxf(m, gm);
            const float z = nm > -INFINITY ? nm : 0.f;  // (a NaN still reaches the sum)
            const uint64_t z2 = f2(z, z), c2 = f2(a.c, a.c);
            uint64_t acc = f2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                uint64_t v[PV / 2];
                vec_pairs<T>(buf[k], v);
#pragma unroll
                for (int i = 0; i < PV / 2; ++i) acc = f2add(acc, f2_mass(v[i], z2, c2));
            }
            float lo, hi;
            f2split(acc, lo, hi);
            s = (rd ? s * ex2((m - z) * a.c) : 0.f) + (lo + hi);
            m = nm;
        }
        const float wm = warp_max(m), wz = wm > -INFINITY ? wm : 0.f;
        s = warp_sum(s * ex2(((m > -INFINITY ? m : wz) - wz) * a.c));
        if (lane == 0) part[warp] = make_float2(wm, s);
        __syncthreads();
        auto join = [&](const float2* e, int cnt) {
            M = e[0].x;
            for (int i = 1; i < cnt; ++i) M = fmaxf(M, e[i].x);
            S = 0.f;
            const float z = M > -INFINITY ? M : 0.f;  // (a part without mass adds 0, or its NaN)
            for (int i = 0; i < cnt; ++i) S += e[i].y * ex2((e[i].x - z) * a.c);
        };
        join(part, kWarpsN);
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
    } else if (C > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    const float inv = 1.f / S;
    const float coef = n >= 0 ? (float)((double)a.grad_scale * (double)a.tg.w[r] /
                                        (*a.tg.wsum * (double)a.T))
                              : 0.f;
    if (g) {
        const bool on = n >= 0;
        const float cs = coef * inv;
        const uint64_t m2 = f2(M, M), c2 = f2(a.c, a.c), cs2 = f2(cs, cs);
        for (int rd = 0; rd < a.rounds; ++rd) {
            if (a.rounds > 1) load(rd);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int j = rd * per_round + j0 + k * kRowThreads;
                if (j >= nvec) break;
                uint64_t v[PV / 2];
                vec_pairs<T>(buf[k], v);
                float o[PV];
#pragma unroll
                for (int i = 0; i < PV / 2; ++i) {
                    float lo, hi;
                    f2split(f2mul(f2_mass(v[i], m2, c2), cs2), lo, hi);
                    o[2 * i] = on ? lo : 0.f;
                    o[2 * i + 1] = on ? hi : 0.f;
                }
                const int e0 = j * PV - off;
                if (a.same_align && e0 >= 0 && e0 + PV <= V) {
                    *reinterpret_cast<uint4*>(g + e0) = pack_vec<T>(o);
                } else {
#pragma unroll
                    for (int i = 0; i < PV; ++i)
                        if (e0 + i >= 0 && e0 + i < V) put(g + e0 + i, o[i]);
                }
            }
        }
        __syncthreads();
        if (tid < n) {  // the target entries this CTA wrote as dense ones
            const int j = (id[tid] + off) / PV % per_round;
            if (j / (NV * kRowThreads) == (int)rank)
                put(g + id[tid], coef * (ex2((xs[tid] - M) * a.c) * inv - p[tid]));
        }
    }
    // the row's loss, then (the last row) their weighted mean in row order
    if (rank == 0) {
        if (warp == 0 && n >= 0) {
            double dot = 0.0;
            for (int k = lane; k < n; k += 32)
                dot += (double)p[k] * ((double)value_of(xs[k]) - (double)M);
            dot = warp_sum(dot);
            if (lane == 0) {
                const double l = log((double)S), lz = (double)M / (double)a.T + l;
                if (!isfinite(lz)) atomicOr(a.tg.status, VSD_STATUS_BAD_ROW);
                a.logz[r] = (float)lz;
                a.row_loss[r] = (float)((double)a.tg.plogp[r] + l - dot / (double)a.T);
            }
        }
        if (tid == 0) {
            __threadfence();
            last = atomicAdd(a.tg.done + 1, 1) == a.R - 1;
        }
        __syncthreads();
        if (!last) return;
        __threadfence();
        double sum = 0.0;
        for (int b = tid; b < a.R; b += kRowThreads * 4) {
            float w[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int q = b + i * kRowThreads;
                const bool on = q < a.R && ld_cg(a.tg.n + q) >= 0;
                w[i] = on ? ld_cg(a.tg.w + q) : 0.f;
                l[i] = on ? ld_cg(a.row_loss + q) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (w[i] != 0.f) sum += (double)w[i] * (double)l[i];
        }
        __shared__ double dpart[kWarpsN];
        sum = warp_sum(sum);
        if (lane == 0) dpart[warp] = sum;
        __syncthreads();
        if (tid == 0) {
            sum = 0.0;
            for (int i = 0; i < kWarpsN; ++i) sum += dpart[i];
            *a.loss = (float)(sum / *a.tg.wsum);
        }
    }
}

template <typename T>
cudaError_t launch_rows(const T* logits, T* grad, TopkArgs a, cudaStream_t st) {
    constexpr int PV = Traits<T>::kPerVec;
    const int64_t need = ((int64_t)a.V + 2 * PV - 2) / PV;  // vectors, whatever the offset
    int64_t C = 1;
    while (C < kMaxCluster && C * kRowThreads * kMaxVecs < need) C *= 2;
    // few rows: spread each over more SMs, while a thread has a vector
    while (C < kMaxCluster && a.R * C < 2 * device_sm_count() && C * kRowThreads < need) C *= 2;
    int nv = 1;
    while (nv < kMaxVecs && C * kRowThreads * nv < need) nv *= 2;
    a.rounds = (int)((need + C * kRowThreads * nv - 1) / (C * kRowThreads * nv));
    auto k = nv == 1   ? k_topk<T, 1>
             : nv == 2 ? k_topk<T, 2>
             : nv == 4 ? k_topk<T, 4>
             : nv == 8 ? k_topk<T, 8>
                       : k_topk<T, 16>;
    return launch_dep(k, dim3((unsigned)(a.R * C)), kRowThreads, 0, (int)C, st, logits, grad, a);
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
    TopkArgs a{};
    a.tg = Targets{at<int32_t>(ws, w.n), at<int32_t>(ws, w.id), at<float>(ws, w.p),
                   at<float>(ws, w.plogp), at<float>(ws, w.w), nullptr, nullptr,
                   at<int32_t>(ws, w.nrows), at<double>(ws, w.wsum), at<float>(ws, w.wmax),
                   at<int32_t>(ws, w.done), at<int32_t>(ws, w.status)};
    a.R = in.R;
    a.V = in.V;
    a.K = in.K;
    a.c = (float)(kLog2e / (double)T);
    a.T = T;
    a.grad_scale = grad_scale;
    a.row_loss = out.row_loss;
    a.logz = out.logz;
    a.loss = out.loss;
    a.same_align = (((uintptr_t)logits ^ (uintptr_t)out.grad) & 15) == 0;
    cudaError_t e = launch_targets(in, a.tg, out.row_loss, out.logz, w.zero_end, st);
    if (e != cudaSuccess) return e;
    if (bf16)
        return launch_rows(static_cast<const __nv_bfloat16*>(logits),
                           static_cast<__nv_bfloat16*>(out.grad), a, st);
    return launch_rows(static_cast<const float*>(logits), static_cast<float*>(out.grad), a, st);
}

}  // namespace vsd
