// vsd_lmloss.cu -- the LM head's supervised losses without keeping the logits:
//
//   x = hidden . W^T,  q_r = softmax(x_r / T),
//   l_r = sum_k p_rk (log p_rk - log q_r(id_rk)),
//   G_rv = a_r (q_r(v) - sum_k p_rk [v = id_rk]),   a_r = scale w_r / (T sum w),
//   d_hidden = G . W,  d_weight = G^T . hidden.
//
// The rows that count are gathered first (a row not counted costs nothing and
// cannot spread a NaN).  A first sweep over pieces of the vocabulary takes each
// row's maximum, sum of exponentials and target logits; the rows' losses and
// log-partitions follow; a second sweep makes each piece's logits again, turns
// them into G (bf16) and adds the piece's products.
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

typedef __nv_bfloat16 bf16;

constexpr int kRowPad = 256;     // the workspace's rows are a multiple of this
constexpr int kPieceUnit = 256;  // a piece's columns are a multiple of this

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct LmWs {
    size_t status, done, zero_end, nrows, wsum, n, id, p, plogp, w, rowmap, rowinv, lse2, coef, xk,
        tab, hid, X, G, dh, total;
    int rpad, piece, npiece;
};

LmWs lm_ws(const LmLossShape& s) {
    LmWs w;
    const size_t R = (size_t)s.R, RK = R * (size_t)s.K;
    w.rpad = (int)round_up(s.R, kRowPad);
    const int64_t vpad = round_up(s.V, kPieceUnit);
    int64_t piece = s.piece ? round_up(s.piece, kPieceUnit)
                            : round_up(std::max<int64_t>(1, (64ll << 20) / w.rpad), kPieceUnit);
    w.piece = (int)std::min(piece, vpad);
    w.npiece = (int)((s.V + (int64_t)w.piece - 1) / w.piece);
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
    w.n = take(4 * R);
    w.id = take(4 * RK);
    w.p = take(4 * RK);
    w.plogp = take(4 * R);
    w.w = take(4 * R);
    w.rowmap = take(4 * R);
    w.rowinv = take(4 * R);
    w.lse2 = take(4 * (size_t)w.rpad);
    w.coef = take(4 * (size_t)w.rpad);
    w.xk = take(4 * RK);
    w.tab = take(8 * (size_t)w.rpad * w.npiece);
    w.hid = take(2 * (size_t)w.rpad * s.H);
    w.X = take(4 * (size_t)w.rpad * w.piece);
    const bool grads = s.dh || s.dw;
    w.G = take(grads ? 2 * (size_t)w.rpad * w.piece : 0);
    w.dh = take(grads ? 4 * (size_t)w.rpad * s.H : 0);
    w.total = o;
    return w;
}

template <typename U> U* at(void* ws, size_t off) {
    return reinterpret_cast<U*>(static_cast<char*>(ws) + off);
}

// ------------------------------------------------------------ rows
// The rows' targets, then (the last block to finish) the list of counted rows.
__global__ void k_targets(TargetIn in, Targets tg, float* row_loss, float* logz) {
    const int lane = threadIdx.x & 31;
    const int r = (int)((blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5);
    if (r < in.R) target_row(in, tg, r, lane);
    __shared__ int last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(tg.done, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    scan_rows(tg, in.R, row_loss, logz);
}

// Counted rows of hidden, packed; the rows up to the next multiple of kRowPad
// are zero.
__global__ void k_gather(const bf16* hidden, int H, Targets tg, bf16* hid) {
    const int n = *tg.nrows;
    const int end = (n + kRowPad - 1) / kRowPad * kRowPad;
    const int vecs = H / 8;
    for (int i = blockIdx.x; i < end; i += gridDim.x) {
        uint4* dst = reinterpret_cast<uint4*>(hid + (size_t)i * H);
        const uint4* src =
            i < n ? reinterpret_cast<const uint4*>(hidden + (size_t)tg.rowmap[i] * H) : nullptr;
        for (int v = threadIdx.x; v < vecs; v += blockDim.x)
            dst[v] = src ? src[v] : make_uint4(0u, 0u, 0u, 0u);
    }
}

// ------------------------------------------------------------ products
// C[m][n] (+)= sum_k A(m, k) B(k, n) in fp32, 64 x 64 tiles, 16 x 16 threads.
struct MatA { const bf16* p; int64_t sm, sk; };
template <typename OUT, bool ADD>
__global__ void __launch_bounds__(256)
    k_product(MatA a, MatA b, OUT* c, int64_t ldc, int M, int N, int K, const int* m_dev,
              const int* k_dev) {
    if (m_dev) M = min(M, *m_dev);
    if (k_dev) K = min(K, *k_dev);
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
    if (m0 >= M || n0 >= N) return;
    __shared__ float sa[16][65], sb[16][65];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int i = threadIdx.x; i < 1024; i += 256) {
            // neighbouring threads along the contiguous index of each operand
            const int ka = a.sk == 1 ? (i & 15) : (i >> 6), ma = a.sk == 1 ? (i >> 4) : (i & 63);
            const int kb = b.sk == 1 ? (i & 15) : (i >> 6), nb = b.sk == 1 ? (i >> 4) : (i & 63);
            sa[ka][ma] = (m0 + ma < M && k0 + ka < K)
                             ? __bfloat162float(a.p[(m0 + ma) * a.sm + (k0 + ka) * a.sk]) : 0.f;
            sb[kb][nb] = (n0 + nb < N && k0 + kb < K)
                             ? __bfloat162float(b.p[(n0 + nb) * b.sm + (k0 + kb) * b.sk]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < M && n < N) {
                OUT* o = c + m * ldc + n;
                if constexpr (sizeof(OUT) == 2) *o = __float2bfloat16_rn(acc[i][j]);
                else *o = ADD ? *o + acc[i][j] : acc[i][j];
            }
        }
}

// ------------------------------------------------------------ statistics

// One block per counted row: (max, sum 2^{(x - max) c}) of the piece's logits
// and the target logits in it.
__global__ void k_piece_stats(const float* X, int64_t ldx, int v0, int cols, int K, Targets tg,
                              float c, float2* tab, float* xk) {
    const int i = blockIdx.x;
    if (i >= *tg.nrows) return;
    const float* x = X + (size_t)i * ldx;
    __shared__ float red[8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float m = -INFINITY;
    for (int v = threadIdx.x; v < cols; v += blockDim.x) m = fmaxf(m, x[v]);
    m = warp_max(m);
    if (lane == 0) red[warp] = m;
    __syncthreads();
    for (int w = 0; w < 8; ++w) m = fmaxf(m, red[w]);
    __syncthreads();
    float s = 0.f;
    for (int v = threadIdx.x; v < cols; v += blockDim.x)
        s += m > -INFINITY ? ex2((x[v] - m) * c) : (x[v] == x[v] ? 0.f : x[v]);
    s = warp_sum(s);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < 8; ++w) s += red[w];
    if (threadIdx.x == 0) tab[i] = make_float2(m, s);
    const int r = tg.rowmap[i], n = tg.n[r];
    const int32_t* id = tg.id + (size_t)r * K;
    for (int k = threadIdx.x; k < n; k += blockDim.x)
        if (id[k] >= v0 && id[k] < v0 + cols) xk[(size_t)i * K + k] = x[id[k] - v0];
}

// One warp per counted row: its log-partition, loss and gradient coefficient;
// the last block to finish sums the losses in row order.
__global__ void k_rows(const float2* tab, int ntab, int64_t stride, Targets tg, int K, float c,
                       float T, float grad_scale, const float* xk, float* lse2, float* coef,
                       float* row_loss, float* logz, float* loss, int R) {
    const int n_rows = *tg.nrows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = (int)((blockIdx.x * (int64_t)blockDim.x + threadIdx.x) >> 5);
    if (i < n_rows) {
        float m = -INFINITY;
        for (int t = lane; t < ntab; t += 32) m = fmaxf(m, tab[t * stride + i].x);
        m = warp_max(m);
        float s = 0.f;
        for (int t = lane; t < ntab; t += 32) {
            const float2 e = tab[t * stride + i];
            // (a part of no mass has maximum -inf and sum 0, or NaN)
            s += e.x > -INFINITY ? e.y * ex2((e.x - m) * c) : e.y;
        }
        s = warp_sum(s);
        const int r = tg.rowmap[i], n = tg.n[r];
        double dot = 0.0;
        for (int k = lane; k < n; k += 32)
            dot += (double)tg.p[(size_t)r * K + k] * (double)xk[(size_t)i * K + k];
        dot = warp_sum(dot);
        if (lane == 0) {
            const double lz = (double)m / (double)T + log((double)s);
            if (!isfinite(lz)) atomicOr(tg.status, VSD_STATUS_BAD_ROW);
            logz[r] = (float)lz;
            row_loss[r] = (float)((double)tg.plogp[r] + lz - dot / (double)T);
            lse2[i] = (float)(lz * kLog2e);
            coef[i] = (float)((double)grad_scale * (double)tg.w[r] / (*tg.wsum * (double)T));
        }
    }
    __shared__ int last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(tg.done + 1, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    double sum = 0.0;
    for (int r = threadIdx.x; r < R; r += blockDim.x)
        if (tg.rowinv[r] >= 0 && tg.w[r] != 0.f) sum += (double)tg.w[r] * (double)ld_cg(row_loss + r);
    __shared__ double part[8];
    sum = warp_sum(sum);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < (int)blockDim.x / 32; ++w) sum += part[w];
        *loss = (float)(sum / *tg.wsum);
    }
}

// G of a piece from its logits, one block per row (the rows up to the next
// multiple of kRowPad and the columns up to ldg are zero).
__global__ void k_make_g(const float* X, int64_t ldx, int v0, int cols, int K, Targets tg, float c,
                         const float* lse2, const float* coef, bf16* G, int64_t ldg) {
    const int i = blockIdx.x;
    const int n_rows = *tg.nrows;
    if (i >= (n_rows + kRowPad - 1) / kRowPad * kRowPad) return;
    bf16* g = G + (size_t)i * ldg;
    const bool on = i < n_rows;
    const float a = on ? coef[i] : 0.f, l = on ? lse2[i] : 0.f;
    const float* x = X + (size_t)i * ldx;
    for (int v = threadIdx.x; v < ldg; v += blockDim.x)
        g[v] = __float2bfloat16_rn(on && v < cols ? a * ex2(fmaf(x[v], c, -l)) : 0.f);
    if (!on) return;
    __syncthreads();
    const int r = tg.rowmap[i], n = tg.n[r];
    const int32_t* id = tg.id + (size_t)r * K;
    for (int k = threadIdx.x; k < n; k += blockDim.x) {
        const int v = id[k] - v0;
        if (v >= 0 && v < cols)
            g[v] = __float2bfloat16_rn(a * (ex2(fmaf(x[v], c, -l)) - tg.p[(size_t)r * K + k]));
    }
}

// d_hidden in the caller's rows: one rounding of the fp32 sums, zero in rows
// not counted.
__global__ void k_dh_out(const float* dh, int H, Targets tg, bf16* out) {
    const int r = blockIdx.x, i = tg.rowinv[r];
    for (int h = threadIdx.x; h < H; h += blockDim.x)
        out[(size_t)r * H + h] = __float2bfloat16_rn(i >= 0 ? dh[(size_t)i * H + h] : 0.f);
}

}  // namespace

bool lmloss_shape_ok(const LmLossShape& s) {
    return s.R >= 1 && s.R <= (1 << 24) && s.V >= 1 && s.V <= (1 << 20) && s.H >= 8 &&
           s.H <= (1 << 20) && s.H % 8 == 0 && s.K >= 1 && s.K <= kMaxTeacher && s.piece >= 0;
}

size_t lmloss_workspace_bytes(const LmLossShape& s) {
    return lmloss_shape_ok(s) ? lm_ws(s).total : 0;
}

cudaError_t lmloss(const LmLossShape& s, const void* hidden, const void* weight,
                   const TargetIn& in, float T, float grad_scale, const vsd_loss_outputs& out,
                   void* ws, cudaStream_t st) {
    const LmWs w = lm_ws(s);
    const int R = s.R, V = s.V, H = s.H, K = s.K;
    Targets tg{at<int32_t>(ws, w.n), at<int32_t>(ws, w.id), at<float>(ws, w.p),
               at<float>(ws, w.plogp), at<float>(ws, w.w), at<int32_t>(ws, w.rowmap),
               at<int32_t>(ws, w.rowinv), at<int32_t>(ws, w.nrows), at<double>(ws, w.wsum),
               at<int32_t>(ws, w.done), at<int32_t>(ws, w.status)};
    bf16* hid = at<bf16>(ws, w.hid);
    float* X = at<float>(ws, w.X);
    bf16* G = at<bf16>(ws, w.G);
    float2* tab = at<float2>(ws, w.tab);
    float *xk = at<float>(ws, w.xk), *lse2 = at<float>(ws, w.lse2), *coef = at<float>(ws, w.coef),
          *dh = at<float>(ws, w.dh);
    const bf16* W = static_cast<const bf16*>(weight);
    const float c = (float)(kLog2e / (double)T);
    cudaError_t e = cudaMemsetAsync(ws, 0, w.zero_end, st);
    if (e != cudaSuccess) return e;
    k_targets<<<(R + 7) / 8, 256, 0, st>>>(in, tg, out.row_loss, out.logz);
    k_gather<<<std::min(w.rpad, 4 * device_sm_count()), 256, 0, st>>>(
        static_cast<const bf16*>(hidden), H, tg, hid);
    auto logits = [&](int v0, int cols) {
        const dim3 grid((cols + 63) / 64, (R + 63) / 64);
        k_product<float, false><<<grid, 256, 0, st>>>(MatA{hid, H, 1}, MatA{W + (size_t)v0 * H, H, 1},
                                                      X, w.piece, R, cols, H, tg.nrows, nullptr);
    };
    for (int q = 0; q < w.npiece; ++q) {
        const int v0 = q * w.piece, cols = std::min(w.piece, V - v0);
        logits(v0, cols);
        k_piece_stats<<<R, 256, 0, st>>>(X, w.piece, v0, cols, K, tg, c, tab + (size_t)q * w.rpad, xk);
    }
    k_rows<<<(R + 7) / 8, 256, 0, st>>>(tab, w.npiece, w.rpad, tg, K, c, T, grad_scale, xk, lse2,
                                        coef, out.row_loss, out.logz, out.loss, R);
    if (s.dh || s.dw) {
        for (int q = 0; q < w.npiece; ++q) {
            const int v0 = q * w.piece, cols = std::min(w.piece, V - v0);
            logits(v0, cols);
            k_make_g<<<w.rpad, 256, 0, st>>>(X, w.piece, v0, cols, K, tg, c, lse2, coef, G, w.piece);
            if (s.dw) {
                const dim3 grid((H + 63) / 64, (cols + 63) / 64);
                k_product<bf16, false><<<grid, 256, 0, st>>>(
                    MatA{G, 1, w.piece}, MatA{hid, 1, H}, static_cast<bf16*>(out.d_weight) + (size_t)v0 * H,
                    H, cols, H, w.rpad, nullptr, tg.nrows);
            }
            if (s.dh) {
                const dim3 grid((H + 63) / 64, (R + 63) / 64);
                const MatA a{G, w.piece, 1}, b{W + (size_t)v0 * H, 1, H};
                if (q == 0) k_product<float, false><<<grid, 256, 0, st>>>(a, b, dh, H, R, H, cols, tg.nrows, nullptr);
                else k_product<float, true><<<grid, 256, 0, st>>>(a, b, dh, H, R, H, cols, tg.nrows, nullptr);
            }
        }
        if (s.dh) k_dh_out<<<R, 256, 0, st>>>(dh, H, tg, static_cast<bf16*>(out.d_hidden));
    }
    return cudaGetLastError();
}

}  // namespace vsd
