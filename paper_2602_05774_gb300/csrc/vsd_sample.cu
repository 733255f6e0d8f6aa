// vsd_sample.cu -- one token a row from what temperature, top-k, top-p and min-p
// leave of a distribution, and the logits these leave (include/vsd_decode.h).
//
// Every filter keeps a first part of the tokens in the order (logit falling, id
// rising), so what is kept is one place in that order: a logit, and how many of the
// tokens that equal it.  Masses are whole numbers (vsd_fixed.cuh).
//
// One block a row; a filter's place is found by bisection of the logits' ordered
// bits, each step one pass over the row.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "vsd_common.cuh"
#include "vsd_decode.h"
#include "vsd_fixed.cuh"

namespace vsd {
namespace {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr float kMinT = 0x1p-64f, kMaxT = 0x1p64f;

struct SampleArgs {
    vsd_policy policy;
    const float* u;
    vsd_filtered_outputs out;
    int V, shift;
    int* status;
};

__constant__ ExpParts kExpParts = make_exp_parts();

__device__ __forceinline__ float value_of(float x) { return x + 0.f; }  // (-0 is 0)
__device__ __forceinline__ float value_of(__nv_bfloat16 x) { return __bfloat162float(x) + 0.f; }
__device__ __forceinline__ void put_none(float* x) { *x = -INFINITY; }
__device__ __forceinline__ void put_none(__nv_bfloat16* x) {
    *reinterpret_cast<unsigned short*>(x) = 0xFF80u;
}
// Bits whose order is the logits'.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007FFFFFu;

template <typename U> __device__ __forceinline__ U block_sum(U v, U* part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    U s = 0;
    for (int i = 0; i < kSampleWarps; ++i) s += part[i];
    return s;
}

// floor(f w) for 0 <= f < 1
__device__ __forceinline__ uint64_t share_of(uint64_t w, float f) {
    if (!(f > 0.f)) return 0;
    int e;
    const float m = frexpf(f, &e);  // f = m 2^e
    const uint64_t k = (uint64_t)(m * 16777216.f);
    const int sh = 24 - e;          // f = k 2^-sh, sh >= 24
    const uint64_t hi = __umul64hi(w, k), lo = w * k;
    if (sh >= 128) return 0;
    return sh >= 64 ? hi >> (sh - 64) : hi << (64 - sh) | lo >> sh;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) k_sample(const T* logits, SampleArgs a) {
    __shared__ uint64_t tab[kExpTab];
    __shared__ uint64_t part[kSampleThreads];
    __shared__ int chosen, limit;
    const int tid = threadIdx.x, V = a.V;
    const int64_t r = blockIdx.x;
    const T* x = logits + r * V;
    for (int j = tid; j < kExpTab; j += kSampleThreads) tab[j] = exp_entry(kExpParts, j);
    auto row = [&](const float* p, float v) { return p ? p[r] : v; };
    const float Tr = row(a.policy.row_T, a.policy.T), top_p = row(a.policy.row_top_p, a.policy.top_p),
                min_p = row(a.policy.row_min_p, a.policy.min_p);
    const int top_k = a.policy.row_top_k ? a.policy.row_top_k[r] : a.policy.top_k;
    const bool ok_par = (Tr == 0.f || (Tr >= kMinT && Tr <= kMaxT)) && top_p == top_p && min_p == min_p;
    // the maximum, the live tokens
    uint32_t top = 0;
    int live = 0;
    bool bad = false;
    for (int v = tid; v < V; v += kSampleThreads) {
        const float f = value_of(x[v]);
        bad |= !(f < INFINITY);
        live += f > -INFINITY;
        top = max(top, key_of(f));
    }
    live = (int)block_sum((uint64_t)live, part);
    bad = __syncthreads_or(bad);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((tid & 31) == 0) part[tid >> 5] = top;
    __syncthreads();
    for (int i = 0; i < kSampleWarps; ++i) top = max(top, (uint32_t)part[i]);
    T* filt = a.out.filtered ? static_cast<T*>(a.out.filtered) + r * V : nullptr;
    if (bad || live == 0 || !ok_par) {
        if (tid == 0) {
            atomicOr(a.status, (bad || live == 0 ? VSD_STATUS_BAD_ROW : 0) |
                                   (ok_par ? 0 : VSD_STATUS_BAD_PARAM));
            if (a.out.tokens) a.out.tokens[r] = -1;
            if (a.out.logq_tok) a.out.logq_tok[r] = NAN;
            if (a.out.kept) a.out.kept[r] = 0;
        }
        if (filt)
            for (int v = tid; v < V; v += kSampleThreads) put_none(filt + v);
        return;
    }
    const float m = of_key(top);
    const ExpScale sc = exp_scale(Tr > 0.f ? Tr : 1.f, a.shift);
    auto mass_of = [&](uint32_t k) { return exp_fixed(of_key(k), m, sc, tab); };
    auto count_from = [&](uint32_t k) {
        int n = 0;
        for (int v = tid; v < V; v += kSampleThreads) n += key_of(value_of(x[v])) >= k;
        return (int)block_sum((uint64_t)n, part);
    };
    auto mass_from = [&](uint32_t k) {
        uint64_t s = 0;
        for (int v = tid; v < V; v += kSampleThreads) {
            const uint32_t q = key_of(value_of(x[v]));
            if (q >= k) s += mass_of(q);
        }
        return block_sum(s, part);
    };
    // The place of the kept tokens' last: all above `cut` and `ties` of those at it.
    uint32_t cut = kKeyNegInf + 1;
    int ties = V;
    int kept = live;
    // the n-th token's place
    auto place = [&](int n) {
        uint32_t lo = kKeyNegInf + 1, hi = top;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo + 1) / 2;
            if (count_from(mid) >= n) lo = mid;
            else hi = mid - 1;
        }
        cut = lo;
        ties = n - (lo == 0xFFFFFFFFu ? 0 : count_from(lo + 1));
        kept = n;
    };
    if (Tr == 0.f) {
        place(1);
    } else {
        if (top_k > 0 && top_k < live) place(top_k);
        int n = kept;
        if (top_p < 1.f) {
            const uint64_t above = mass_from(cut + 1), at = mass_of(cut);
            const uint64_t all = kept == live ? mass_from(cut) : above + at * (uint64_t)ties;
            // C >= p W, a whole number C
            uint64_t goal = share_of(all, top_p);
            if (share_of(all, top_p) == 0) goal = 1;
            else {
                // rounded up unless exact
                int e;
                const uint64_t kk = (uint64_t)(frexpf(top_p, &e) * 16777216.f);
                const int sh = 24 - e;
                const uint64_t back_hi = __umul64hi(all, kk), back_lo = all * kk;
                const bool whole = sh >= 64 ? (back_lo == 0 && (sh == 64 || (back_hi << (128 - sh)) == 0))
                                            : (back_lo << (64 - sh)) == 0;
                if (!whole) ++goal;
            }
            uint32_t lo = cut, hi = top;
            auto mass_in = [&](uint32_t k) { return k == cut ? all : mass_from(k); };
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                if (mass_in(mid) >= goal) lo = mid;
                else hi = mid - 1;
            }
            const uint64_t before = mass_from(lo + 1), each = mass_of(lo);
            const int count_before = count_from(lo + 1);
            const uint64_t t = (goal - before + each - 1) / each;
            n = count_before + (int)t;
        }
        if (min_p > 0.f) {
            const double thr = (double)m + (double)Tr * log((double)fminf(min_p, 1.f));
            const uint32_t k = key_of(value_of(__double2float_ru(thr)));
            n = min(n, count_from(max(k, kKeyNegInf + 1)));
        }
        if (n < kept) place(n);
    }
    // ids up to `limit` among those at the cut
    if (tid == 0) limit = V;
    __syncthreads();
    const int seg = (V + kSampleThreads - 1) / kSampleThreads;
    const int v0 = min(V, tid * seg), v1 = min(V, v0 + seg);
    {
        int n = 0;
        for (int v = v0; v < v1; ++v) n += key_of(value_of(x[v])) == cut;
        part[tid] = n;
        __syncthreads();
        uint64_t before = 0;
        for (int i = 0; i < tid; ++i) before += part[i];
        if ((int64_t)before < ties && (int64_t)(before + n) >= ties) {
            int left = ties - (int)before;
            for (int v = v0; v < v1; ++v)
                if (key_of(value_of(x[v])) == cut && --left == 0) limit = v;
        }
        __syncthreads();
    }
    const int lim = limit;
    auto is_kept = [&](uint32_t k, int v) { return k > cut || (k == cut && v <= lim); };
    if (a.u) {
        const float u = a.u[r];
        uint64_t s = 0;
        int last = -1, first = V;
        for (int v = v0; v < v1; ++v) {
            const uint32_t k = key_of(value_of(x[v]));
            if (is_kept(k, v)) {
                s += mass_of(k);
                last = v;
                first = min(first, v);
            }
        }
        __syncthreads();
        part[tid] = s;
        if (tid == 0) chosen = -1;
        __syncthreads();
        uint64_t before = 0, all = 0;
        for (int i = 0; i < kSampleThreads; ++i) {
            if (i == tid) before = all;
            all += part[i];
        }
        if (u >= 1.f) {
            if (last >= 0) atomicMax(&chosen, last);
        } else if (!(u >= 0.f)) {
            if (tid == 0) chosen = V;
            __syncthreads();
            if (first < V) atomicMin(&chosen, first);
        } else {
            const uint64_t goal = share_of(all, u);
            if (before <= goal && goal < before + s) {
                uint64_t c = before;
                for (int v = v0; v < v1; ++v) {
                    const uint32_t k = key_of(value_of(x[v]));
                    if (!is_kept(k, v)) continue;
                    c += mass_of(k);
                    if (c > goal) {
                        chosen = v;
                        break;
                    }
                }
            }
        }
        __syncthreads();
        if (tid == 0) {
            if (a.out.tokens) a.out.tokens[r] = chosen;
            if (a.out.logq_tok) {
                const float f = value_of(x[chosen]);
                a.out.logq_tok[r] = Tr == 0.f ? 0.f
                    : (float)(((double)f - (double)m) / (double)Tr -
                              log((double)all * exp2((double)(a.shift - 62))));
            }
        }
    }
    if (tid == 0 && a.out.kept) a.out.kept[r] = kept;
    if (filt) {
        __syncthreads();
        for (int v = tid; v < V; v += kSampleThreads) {
            const T raw = x[v];
            if (is_kept(key_of(value_of(raw)), v)) filt[v] = raw;
            else put_none(filt + v);
        }
    }
}

bool share_bytes(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + bn && y < x + an;
}

}  // namespace
}  // namespace vsd

using namespace vsd;

extern "C" {

size_t vsd_sample_filtered_workspace_bytes(int32_t R, int32_t V) {
    return R >= 1 && R <= (1 << 24) && V >= 1 && V <= (1 << 20) ? 256 : 0;
}

vsd_status vsd_sample_filtered(const void* logits, vsd_dtype dtype, int32_t R, int32_t V,
                               const vsd_policy* policy, const float* u,
                               vsd_filtered_outputs* out, void* ws, size_t ws_bytes,
                               void* stream) {
    const size_t need = vsd_sample_filtered_workspace_bytes(R, V);
    if (!logits || !policy || !out || need == 0) return VSD_ERR_INVALID_ARG;
    if (dtype != VSD_F32 && dtype != VSD_BF16) return VSD_ERR_INVALID_ARG;
    const size_t size = dtype == VSD_BF16 ? 2 : 4, bytes = (size_t)R * V * size, row = 4 * (size_t)R;
    if (((uintptr_t)logits | (uintptr_t)out->filtered) & (size - 1)) return VSD_ERR_INVALID_ARG;
    const vsd_policy& p = *policy;
    const void* in[] = {p.row_T, p.row_top_k, p.row_top_p, p.row_min_p, u};
    const void* res[] = {out->tokens, out->logq_tok, out->kept};
    for (const void* q : in)
        if ((uintptr_t)q & 3) return VSD_ERR_INVALID_ARG;
    for (const void* q : res)
        if ((uintptr_t)q & 3) return VSD_ERR_INVALID_ARG;
    if (!u && (out->tokens || out->logq_tok)) return VSD_ERR_INVALID_ARG;
    if (!p.row_T && !(p.T == 0.f || (p.T >= kMinT && p.T <= kMaxT))) return VSD_ERR_INVALID_ARG;
    if ((!p.row_top_p && p.top_p != p.top_p) || (!p.row_min_p && p.min_p != p.min_p))
        return VSD_ERR_INVALID_ARG;
    if (out->filtered != logits && share_bytes(out->filtered, bytes, logits, bytes))
        return VSD_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
        if (share_bytes(res[i], row, logits, bytes) || share_bytes(res[i], row, out->filtered, bytes))
            return VSD_ERR_INVALID_ARG;
        for (const void* q : in)
            if (share_bytes(res[i], row, q, row)) return VSD_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (share_bytes(res[i], row, res[j], row)) return VSD_ERR_INVALID_ARG;
    }
    for (const void* q : in)
        if (share_bytes(out->filtered, bytes, q, row)) return VSD_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need) return VSD_ERR_WORKSPACE;
    if (!u && !out->kept && !out->filtered) return VSD_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(ws, 0, 256, st) != cudaSuccess) return VSD_ERR_CUDA;
    const SampleArgs a{p, u, *out, V, exp_shift(V), static_cast<int*>(ws)};
    if (dtype == VSD_BF16)
        k_sample<<<R, kSampleThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(logits), a);
    else
        k_sample<<<R, kSampleThreads, 0, st>>>(static_cast<const float*>(logits), a);
    return cudaGetLastError() == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

}  // extern "C"
