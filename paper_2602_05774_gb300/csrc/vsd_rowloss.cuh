// vsd_rowloss.cuh -- softmax, loss and gradient of rows of logits in memory,
// each row read once:
//
//   (m, s) = (max x, sum 2^{(x - m) c}),  c = log2(e) / T,
//   l = plogp + ln s - sum_k p_k (x_{id_k} - m) / T,  log Z = m / T + ln s,
//   g_v = a (2^{(x_v - m) c} / s - sum_k p_k [v = id_k]).
//
// Bound by memory: one read of the row, one write of its gradient.  A cluster of
// up to 8 blocks holds a row in shared memory between the two, a segment each;
// the blocks' partial sums meet in distributed shared memory.  The clusters are
// persistent, several to an SM, so that some load while others sum or write.
// 4096 x 128256 bf16: 0.36 ms a call, 5.8 TB/s (0.85 of a copy); instruction issue
// is 61 % busy beside it.  A row too long for the cluster is read twice, in
// rounds.  A row that does not start on 16 bytes is laid out from the vector
// boundary below it; its ragged first and last vectors are filled element by
// element.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include <type_traits>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_target.cuh"

namespace vsd {
namespace {

constexpr int kRowThreads = 128;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kSegBytes = 32768;    // a block's segment, where the cluster reaches over the row
constexpr int kSegMax = 200 << 10;  // at most
constexpr uint64_t kRowWaitNs = 2000000000ull;
static_assert(kRowThreads >= kMaxTeacher, "a thread per target entry");

struct RowArgs {
    Targets tg;
    int rows, V, K, rounds;
    int vper;            // vectors of a block's segment, whole rounds of its threads
    bool by4;            // rounds of four vectors
    int64_t ldx, ldg;    // row pitches in elements
    int gcols;           // columns of a gradient row that are written (zero from V on)
    float c;
    float invT, invT_lo; // 1 / T and what its rounding left
    float *row_loss, *logz;
    bool same_align;     // gradient rows start where logits rows do, modulo 16 bytes
};

template <typename T> __device__ __forceinline__ float row_value(T x);
template <> __device__ __forceinline__ float row_value(float x) { return x; }
template <> __device__ __forceinline__ float row_value(__nv_bfloat16 x) {
    return __bfloat162float(x);
}
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
    if (N == 8)
        *reinterpret_cast<uint4*>(g) = make_uint4(w[0], w[1], w[2 % (N / 2)], w[3 % (N / 2)]);
    else
        *reinterpret_cast<uint2*>(g) = make_uint2(w[0], w[1]);
}

// LM: the rows are the LM head's packed ones (row i is original row rowmap[i],
// there are *nrows of them, rows up to the next multiple of 64 are zeroed) and
// the gradient is scaled for the products (top, see there).
template <typename TI, typename TO, bool LM>
__global__ void __launch_bounds__(kRowThreads)
    k_row_loss(const TI* logits, TO* grad, RowArgs a, float top) {
    constexpr int PV = Traits<TI>::kPerVec;
    extern __shared__ __align__(128) unsigned char row_smem[];
    __shared__ uint64_t bar, xbars[2];
    __shared__ float2 part[kRowWarps], cpart[2][kMaxCluster];
    __shared__ float xs[2][kMaxTeacher], ps[2][kMaxTeacher];
    __shared__ int ids[2][kMaxTeacher];
    __shared__ int dead;  // a wait of this block ran out
    uint4* seg = reinterpret_cast<uint4*>(row_smem);
    uint32_t rank, C;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int V = a.V, stride = (int)C * a.vper;
    const int first = (int)(blockIdx.x / C), step = (int)(gridDim.x / C);
    const uint4 none = make_uint4(Traits<TI>::kNegInf, Traits<TI>::kNegInf, Traits<TI>::kNegInf,
                                  Traits<TI>::kNegInf);
    dep_launch();
    if (tid == 0) {
        mbar_init(&bar, 1);
        mbar_init(&xbars[0], 1);
        mbar_init(&xbars[1], 1);
        dead = 0;
        mbar_init_fence();
    }
    __syncwarp();  // (the barrier is one instruction of the whole warp)
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    auto row_of = [&](int i) { return logits + (size_t)i * a.ldx; };
    auto off_of = [&](const TI* x) { return (int)(((uintptr_t)x / sizeof(TI)) % PV); };
    // Once a wait has run out the results are void: the thread waits and copies
    // no more, after one more wait for what it had in flight (before a wait for
    // other blocks none of its copies are).
    bool lost = false;
    auto wait_bounded = [&](uint64_t* b, uint32_t parity) {
        auto done = [&] { return mbar_try_wait(b, parity); };
        if (lost || bounded_wait(done, [&] { return *(volatile int*)&dead != 0; }, kRowWaitNs))
            return;
        lost = true;
        if (!*(volatile int*)&dead) {
            dead = 1;
            atomicOr(a.tg.status, VSD_STATUS_TIMEOUT);
        }
        if (tid == 0) bounded_wait(done, [] { return false; }, kRowWaitNs);
    };
    // vectors rd stride + rank vper .. of row i, and -inf in the segment's rest
    // (all of it the first time: a later row's part is at most a vector shorter)
    auto load = [&](int i, int rd, bool all) {
        const TI* x = row_of(i);
        const int off = off_of(x), nvec = (V + off + PV - 1) / PV;
        const int in0 = off ? 1 : 0, in1 = (V + off) / PV;  // whole vectors
        const int v0 = rd * stride + (int)rank * a.vper, v1 = min(nvec, v0 + a.vper);
        if (tid == 0 && !lost) {
            const int lo = max(v0, in0), hi = min(v1, in1);
            const uint32_t bytes = hi > lo ? 16u * (uint32_t)(hi - lo) : 0u;
            mbar_expect_tx(&bar, bytes);
            if (bytes)
                bulk_g2s(seg + (lo - v0), x + ((int64_t)lo * PV - off), bytes, &bar,
                         policy_evict_first());
        }
        if (warp == 1 && lane < 2 * PV) {  // the ragged ends
            const int v = lane < PV ? 0 : nvec - 1, el = lane % PV;
            const int col = v * PV - off + el;
            if (v >= v0 && v < v1 && (v < in0 || v >= in1)) {
                TI* d = reinterpret_cast<TI*>(seg + (v - v0)) + el;
                if (col >= 0 && col < V) *d = x[col];
                else row_put(d, -INFINITY);
            }
        }
        const int cnt = max(v1 - v0, 0);
        if (all || a.rounds > 1) {
            for (int j = cnt + tid; j < a.vper; j += kRowThreads) seg[j] = none;
        } else if (tid == 2 && cnt < a.vper) {
            seg[cnt] = none;
        }
    };
    uint32_t phase = 0;  // parity of the next load
    auto arrived = [&]() {
        wait_bounded(&bar, phase);
        phase ^= 1u;
    };
    int rows = a.rows, n_rows = a.rows;
    if (LM) {  // the kernel before this one stored the logits
        dep_wait();
        if (tid == 0) asm volatile("fence.proxy.async;" ::: "memory");
        n_rows = *(const volatile int*)a.tg.nrows;
        rows = (n_rows + 63) / 64 * 64;
    }
    // (logits in hand were there before the targets' kernel began: the first rows
    // are loaded and summed while it runs)
    if (first < rows) load(first, 0, true);
    __syncwarp();
    if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // all have begun

    // A row's target: thread k holds entry k.  Looked up for the next row while
    // one is worked on (first the entry, then its logit).
    int r = 0, n = -1, my_id = 0;
    float my_p = 0.f, w = 0.f, plogp = 0.f, xv = 0.f, scale = 0.f, unit = 1.f;
    auto look = [&](int i) {
        n = -1;
        if (i >= n_rows) return;
        r = LM ? a.tg.rowmap[i] : i;
        if (tid < a.K) {
            my_id = a.tg.id[(size_t)r * a.K + tid];
            my_p = a.tg.p[(size_t)r * a.K + tid];
        }
        n = a.tg.n[r];
        w = a.tg.w[r];
        plogp = a.tg.plogp[r];
    };
    // (read before the cluster writes any of the row's gradient, used after)
    auto look_logit = [&](int i) { xv = tid < n ? row_value(row_of(i)[my_id]) : 0.f; };

    for (int i = first, it = 0; i < rows; i += step, ++it) {
        const int par = it & 1;
        const TI* x = row_of(i);
        const int off = off_of(x), nvec = (V + off + PV - 1) / PV;
        float m = -INFINITY, s = 0.f;
        // N of the segment's vectors, N rounds of threads apart
        auto take = [&](int j, auto count) {
            constexpr int N = decltype(count)::value;
            uint4 q[N];
#pragma unroll
            for (int u = 0; u < N; ++u) q[u] = seg[j + u * kRowThreads];
            float nm = vec_max<TI>(q[0]);
#pragma unroll
            for (int u = 1; u < N; ++u) nm = fmaxf(nm, vec_max<TI>(q[u]));
            nm = fmaxf(nm, m);
            const float z = nm > -INFINITY ? nm : 0.f;  // (a NaN still reaches the sum)
            const uint64_t z2 = f2(z, z), c2 = f2(a.c, a.c);
            uint64_t acc[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
            for (int u = 0; u < N; ++u) {
                uint64_t v[PV / 2];
                vec_pairs<TI>(q[u], v);
#pragma unroll
                for (int e = 0; e < PV / 2; ++e)
                    acc[e & 1] = f2add(acc[e & 1], f2_mass(v[e], z2, c2));
            }
            float lo, hi;
            f2split(f2add(acc[0], acc[1]), lo, hi);
            s = s * ex2((m - z) * a.c) + (lo + hi);
            m = nm;
        };
        for (int rd = 0; rd < a.rounds; ++rd) {
            if (rd) {
                __syncthreads();  // the segment has been read
                if (tid == 0) fence_proxy_async();
                load(i, rd, false);
            }
            __syncthreads();  // what the threads wrote of the segment
            arrived();
            if (a.by4)
                for (int j = tid; j < a.vper; j += 4 * kRowThreads)
                    take(j, std::integral_constant<int, 4>());
            else
                for (int j = tid; j < a.vper; j += kRowThreads)
                    take(j, std::integral_constant<int, 1>());
        }
        if (it == 0) {
            if (!LM) dep_wait();
            scale = LM ? *a.tg.wmax : *a.tg.share;
            if (!LM) unit = *a.tg.unit;
            look(i);
            look_logit(i);
        }
        // this row's target
        const int row = r, cnt_n = n;
        const float row_w = w, row_plogp = plogp;
        if (tid < cnt_n) {
            xs[par][tid] = xv;
            ps[par][tid] = my_p;
            ids[par][tid] = my_id;
        }
        const float wm = warp_max(m), wz = wm > -INFINITY ? wm : 0.f;
        s = warp_sum(s * ex2(((m > -INFINITY ? m : wz) - wz) * a.c));
        if (lane == 0) part[warp] = make_float2(wm, s);
        __syncthreads();
        if (i + step < rows) look(i + step);
        float M, S;
        auto join = [&](const float2* e, int cnt) {
            M = e[0].x;
            for (int k = 1; k < cnt; ++k) M = fmaxf(M, e[k].x);
            S = 0.f;
            const float z = M > -INFINITY ? M : 0.f;  // (a part without mass adds 0, or its NaN)
            for (int k = 0; k < cnt; ++k) S += e[k].y * ex2((e[k].x - z) * a.c);
        };
        join(part, kRowWarps);
        if (C > 1) {
            // every block's pair to every block, counted in bytes on the
            // receiver's barrier (a cluster barrier would also wait for this
            // block's gradient stores); two sets, as a block may be a row ahead
            // of one still reading
            if (tid == 0 && !lost) mbar_expect_tx(&xbars[par], 8u * C);
            if (tid < (int)C && !lost) {
                uint32_t dst, bar;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(dst) : "r"(smem_u32(&cpart[par][rank])), "r"(tid));
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                             : "=r"(bar) : "r"(smem_u32(&xbars[par])), "r"(tid));
                asm volatile(
                    "st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];"
                    :: "r"(dst), "l"(f2(M, S)), "r"(bar) : "memory");
            }
            wait_bounded(&xbars[par], (uint32_t)it >> 1 & 1);
            join(cpart[par], (int)C);
        }
        const float inv = 1.f / S;
        const bool on = cnt_n >= 0;
        const float coef = !on ? 0.f : LM ? (scale > 0.f ? top * (row_w / scale) : 0.f)
                                          : row_w * unit * scale;
        TO* g = grad ? grad + (size_t)i * a.ldg : nullptr;
        if (g) {
            const float cs = coef * inv;
            const uint64_t m2 = f2(M, M), c2 = f2(a.c, a.c), cs2 = f2(cs, cs);
            for (int rd = 0; rd < a.rounds; ++rd) {
                if (a.rounds > 1) {
                    __syncthreads();
                    if (tid == 0) fence_proxy_async();
                    load(i, rd, false);
                    __syncthreads();
                    arrived();
                }
                const int v0 = rd * stride + (int)rank * a.vper;
                const int cnt = min(nvec, v0 + a.vper) - v0;
                auto vec = [&](int j, float (&o)[PV]) {
                    uint64_t v[PV / 2];
                    vec_pairs<TI>(seg[j], v);
#pragma unroll
                    for (int e = 0; e < PV / 2; ++e)
                        f2split(f2mul(f2_mass(v[e], m2, c2), cs2), o[2 * e], o[2 * e + 1]);
                };
                // whole vectors, then the ragged ends (or all) by element
                const int lo = max(0, (off ? 1 : 0) - v0);
                const int hi = a.same_align ? min(cnt, (V + off) / PV - v0) : lo;
                TO* gv = g + (int64_t)v0 * PV - off;
                if (on) {
#pragma unroll 4
                    for (int j = lo + tid; j < hi; j += kRowThreads) {
                        float o[PV];
                        vec(j, o);
                        row_store<PV>(gv + j * PV, o);
                    }
                } else {
                    const float o[PV] = {};
                    for (int j = lo + tid; j < hi; j += kRowThreads) row_store<PV>(gv + j * PV, o);
                }
                for (int j = tid; j < cnt; j += kRowThreads) {
                    if (j >= lo && j < hi) {  // (only the ends are left)
                        j += (hi - 1 - j) / kRowThreads * kRowThreads;
                        continue;
                    }
                    float o[PV] = {};
                    if (on) vec(j, o);
                    const int e0 = (v0 + j) * PV - off;
#pragma unroll
                    for (int e = 0; e < PV; ++e)
                        if (e0 + e >= 0 && e0 + e < V) row_put(g + e0 + e, o[e]);
                }
            }
            if (LM && rank == C - 1)
                for (int v = V + tid; v < a.gcols; v += kRowThreads) row_put(g + v, 0.f);
        }
        __syncthreads();  // the segment has been read
        if (i + step < rows) {
            if (tid == 0) fence_proxy_async();
            load(i + step, 0, false);
        }
        if (i + step < rows) look_logit(i + step);
        if (g && tid < cnt_n && (tid == 0 || ids[par][tid - 1] != ids[par][tid])) {
            // the target entries this block wrote as dense ones; equal tokens add
            const int v = ids[par][tid], j = (v + off) / PV % stride;
            if (j / a.vper == (int)rank) {
                float q = ps[par][tid];
                for (int k = tid + 1; k < cnt_n && ids[par][k] == v; ++k) q += ps[par][k];
                row_put(g + v, coef * (ex2((xs[par][tid] - M) * a.c) * inv - q));
            }
        }
        // the row's loss
        if (rank == 0 && warp == 0 && on) {
            float dot = 0.f;
            for (int k = lane; k < cnt_n; k += 32) dot = fmaf(ps[par][k], xs[par][k] - M, dot);
            dot = warp_sum(dot);
            if (lane == 0) {
                const float l = logf(S);
                const float lz = fmaf(M, a.invT, fmaf(fmaxf(M, -FLT_MAX), a.invT_lo, l));
                if (!isfinite(lz)) atomicOr(a.tg.status, VSD_STATUS_BAD_ROW);
                a.logz[row] = lz;
                a.row_loss[row] = row_plogp + (l - dot * a.invT);
            }
        }
    }
    // (a cluster without rows still waits for the kernels before)
    if (!LM && first >= rows) dep_wait();
    // no block ends while another may write to it
    if (C > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
}

// A sum in two floats: what the additions to hi round off is exact and goes to lo, so
// that it holds some 2^-45 of its terms.  (Where hi is not finite, lo is NaN.)
struct Sum2 {
    float hi = 0.f, lo = 0.f;
    __device__ __forceinline__ void add(float x, float rest) {
        const float s = hi + x, b = s - hi;
        lo += ((hi - (s - b)) + (x - b)) + rest;
        hi = s;
    }
    __device__ __forceinline__ void warp() {
#pragma unroll
        for (int o = 16; o; o >>= 1)
            add(__shfl_xor_sync(0xffffffffu, hi, o), __shfl_xor_sync(0xffffffffu, lo, o));
    }
};

// The weighted mean of the rows' losses, in row order, by one block, rounded once.  (With
// sums in 64 bits a call on 32 x 1024 logits takes 16.2 us as a graph, 14.9 so; on 768 x
// 32000 35.6 and 31.7.)
__global__ void __launch_bounds__(1024) k_mean_loss(Targets tg, int R, const float* row_loss,
                                                    float* loss) {
    __shared__ float2 part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    dep_launch();
    dep_wait();
    const float unit = *tg.unit;
    Sum2 sum;
    for (int64_t b = threadIdx.x; b < R; b += 1024 * 4) {
        float w[4], l[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t r = min(b + u * 1024, (int64_t)R - 1);
            const bool on = ld_cg(tg.n + r) >= 0 && b + u * 1024 < R;
            w[u] = on ? ld_cg(tg.w + r) * unit : 0.f;
            l[u] = ld_cg(row_loss + r);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (w[u] != 0.f) {
                const float x = w[u] * l[u];
                sum.add(x, fmaf(w[u], l[u], -x));
            }
    }
    sum.warp();
    if (lane == 0) part[warp] = make_float2(sum.hi, sum.lo);
    __syncthreads();
    if (warp == 0) {
        const double all = *tg.wsum * (double)unit;  // 1 .. 2, or a power of two beyond
        const float d = (float)all, d_lo = (float)(all - (double)d);
        sum.hi = part[lane].x;
        sum.lo = part[lane].y;
        sum.warp();
        if (lane == 0) {
            // (hi + lo) / (d + d_lo): the quotient of the first parts, and the rest's
            const float q = sum.hi / d, rest = (fmaf(-q, d, sum.hi) + sum.lo - q * d_lo) / d;
            *loss = isfinite(rest) ? q + rest : q;
        }
    }
}

// Launches a.rows rows at temperature T (a.c, a.invT, a.vper, a.by4 and a.rounds are
// set here).
// resident: clusters of a kernel's blocks of so many threads and bytes that can
// be resident at once.
template <typename TI, typename TO, bool LM>
cudaError_t launch_row_loss(const TI* logits, TO* grad, RowArgs a, float T, float top,
                            int (*resident)(const void*, int, size_t, int),
                            cudaStream_t st) {
    constexpr int PV = Traits<TI>::kPerVec;
    a.c = (float)(kLog2e / (double)T);
    a.invT = 1.f / T;
    a.invT_lo = (float)(1.0 / (double)T - (double)a.invT);
    const int64_t need = ((int64_t)a.V + 2 * PV - 2) / PV;  // vectors, whatever the offset
    int64_t C = 1;
    while (C < kMaxCluster && C * kSegBytes < 16 * need) C *= 2;
    int64_t vper = std::min<int64_t>((need + C - 1) / C, kSegMax / 16);
    // four vectors a thread at a time (4096 x 128256 bf16, the loss alone: 7 % less
    // time than with one), one where a segment has no more than two
    a.by4 = vper > 2 * kRowThreads;
    const int64_t unit = kRowThreads * (a.by4 ? 4 : 1);
    vper = (vper + unit - 1) / unit * unit;
    a.vper = (int)vper;
    a.rounds = (int)((need + C * vper - 1) / (C * vper));
    auto k = k_row_loss<TI, TO, LM>;
    const size_t smem = (size_t)vper * 16;
    const int64_t clusters = resident((const void*)k, kRowThreads, smem, (int)C);
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    return launch_dep(a.rows <= clusters, k,
                      dim3((unsigned)(std::min<int64_t>(clusters, a.rows) * C)), kRowThreads, smem,
                      (int)C, st, logits, grad, a, top);
}

}  // namespace
}  // namespace vsd
