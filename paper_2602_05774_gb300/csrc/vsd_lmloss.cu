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
#include <string.h>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_launch.h"
#include "vsd_loss.h"
#include "vsd_pair.cuh"

namespace vsd {
namespace {

typedef __nv_bfloat16 bf16;

constexpr int kRowPad = 256;     // the workspace's rows are a multiple of this
constexpr int kPieceUnit = 256;  // a piece's columns are a multiple of this
// Bytes of a piece's G: about the L2, so that the products read it from there.
constexpr int64_t kPieceBytes = 128ll << 20;
constexpr int64_t kKeepBytes = 64ll << 20;
constexpr int64_t kPairsHint = 152;  // d_hidden jobs wanted: two for each pair of SMs
// The operand G is scaled so that the largest weight sits at the top of a
// binade (1.984 ..), where bf16's relative rounding error is least: a row's
// target entries are near -w before the draft has learned them, and they
// dominate the products.  The outputs take the factor back in fp32 (kappa).
constexpr float kTopMantissa = 1.984375f;

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct LmWs {
    size_t status, done, zero_end, nrows, wsum, wmax, kappa, n, id, p, plogp, w, rowmap, rowinv,
        lse2, coef, xk, tab, hid, X, G, dh, total;
    int rpad, piece, npiece, split;
    bool keep;  // the logits are kept (one piece)
};

LmWs lm_ws(const LmLossShape& s) {
    LmWs w;
    const size_t R = (size_t)s.R, RK = R * (size_t)s.K;
    const bool grads = s.dh || s.dw;
    w.rpad = (int)round_up(s.R, kRowPad);
    const int64_t vpad = round_up(s.V, kPieceUnit);
    const int64_t most = std::max<int64_t>(1, kPieceBytes / (2 * (int64_t)w.rpad * kPieceUnit));
    // few rows: the whole vocabulary's logits (4 bytes) and G (2) fit the space
    // of the weight, or are small; they are made once
    const int64_t whole = 6 * (int64_t)w.rpad * vpad;
    w.keep = grads && (s.piece ? s.piece >= s.V : true) && w.rpad <= 65280 &&  // (a grid's rows)
             whole <= std::max<int64_t>(2 * (int64_t)s.V * s.H, kKeepBytes);
    int64_t units = vpad / kPieceUnit, per;
    if (s.piece) {
        per = std::min(units, round_up(s.piece, kPieceUnit) / kPieceUnit);
    } else {
        const int64_t pieces = w.keep ? 1 : (units + most - 1) / most;
        per = (units + pieces - 1) / pieces;  // pieces of about the same size
    }
    w.piece = (int)(per * kPieceUnit);
    w.npiece = (int)((units + per - 1) / per);
    // parts of a piece's columns in d_hidden: enough jobs for every pair, each
    // of 8 K blocks at least
    const int64_t tiles = (int64_t)(w.rpad / kRowPad) * ((s.H + kRowPad - 1) / kRowPad);
    w.split = (int)std::max<int64_t>(1, std::min<int64_t>((kPairsHint + tiles - 1) / tiles,
                                                          w.piece / 512));
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
    w.kappa = take(4);
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
    w.tab = take(8 * (size_t)w.rpad * (size_t)units);
    w.hid = take(2 * (size_t)w.rpad * s.H);
    w.X = take(w.keep ? 4 * (size_t)w.rpad * w.piece : 0);
    w.G = take(grads ? 2 * (size_t)w.rpad * w.piece : 0);
    w.dh = take(s.dh ? 4 * (size_t)w.rpad * s.H * w.split : 0);
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

// Counted rows of hidden, packed; the rows up to the next K block of d_weight
// are zero.
__global__ void k_gather(const bf16* hidden, int H, Targets tg, bf16* hid) {
    const int n = *tg.nrows;
    const int end = (n + 63) / 64 * 64;
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
// All products run as 256 x 256 tiles of a CTA pair, K in blocks of 64 through
// a ring of kStages stages; the accumulator of one tile is read back while the
// next one is computed (2 x 256 TMEM columns).  Per CTA:
//   warp 0     TMA producer: its half of A and of B (16 KB each) per K block,
//              counted on the leader's barrier;
//   warp 1     the leader's MMA issuer (one thread, for both CTAs);
//   warps 2-5  epilogue: 32 rows each, tcgen05.ld, then what the product is for:
//     logits   A = hidden rows, B = weight rows, both K-major.  kStats: per row
//              and tile (max, sum 2^{(x - max) c}) and the target logits in the
//              tile (kKeep: the logits too).  kGrad: G, rounded to bf16.
//     d_hidden A = G (K-major), B = weight (MN-major, as it lies): fp32 sums,
//              added up over the pieces of the vocabulary by TMA.
//     d_weight A = G (MN-major), B = hidden (MN-major): one rounding to bf16.
// What is stored goes through 4 KB of swizzled shared memory per warp (double
// buffered) and a TMA store.  Every wait is bounded: one that runs out sets
// VSD_STATUS_TIMEOUT, and the pair winds down, waits for its copies and MMAs
// in flight and frees its tensor memory.
namespace tc = vsd_pair;

constexpr int BT = 256, BK = 64;
constexpr int kPairThreads = 192;
constexpr int kHalfBytes = 128 * BK * 2;       // one operand's half tile: 16 KB
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kPairStages = 6;
constexpr int kBoxBytes = 64 * BK * 2;         // an MN-major half is two 64-column boxes
constexpr int kOutBytes = 4096;                // 32 rows x 128 bytes
constexpr uint32_t kTmemAll = 2 * BT;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kGroupM = 16;                    // M tiles that share B tiles in L2

struct PairBars {
    uint64_t full[kPairStages];   // leader: both CTAs' bytes landed
    uint64_t empty[kPairStages];  // the MMAs reading the stage are done
    uint64_t acc_full[2];
    uint64_t acc_empty[2];        // leader: 8 epilogue warps
    uint64_t drain;
    uint32_t tmem_base;
    int err;
};
constexpr size_t kPairSmem =
    1024 + (size_t)kPairStages * kStageBytes + 8 * kOutBytes + sizeof(PairBars);

enum { kStats = 0, kKeep = 1, kGrad = 2, kProd = 3 };

struct PairMaps {
    CUtensorMap a, b, o;        // logits: hidden, weight, stored tiles
    CUtensorMap gk, gt, wt, ht; // products: G K- and MN-major, weight and hidden MN-major
    CUtensorMap dw, dh;
};
struct PairArgs {
    Targets tg;
    int K;                 // entries of a target list
    int H, V, v0, cols;    // this piece: columns v0 .. v0 + cols - 1
    int nkh;               // K blocks of the hidden size
    int64_t rpad;
    float c;
    float2* tab;
    float* xk;
    const float *lse2, *coef, *kappa;
    int split, first;      // d_hidden: parts of the piece's columns; first piece
    int want_dh, want_dw;
};

struct Job {
    int kind;  // 0 logits, 1 d_hidden, 2 d_weight
    int m0, n0, kb0, kb1, part;
};

// The pair's jobs.  Logits: tiles with M fastest within groups of kGroupM M
// tiles (the rows of a group stay in L2 while the weight streams by).
// Products: the long d_hidden jobs first, dealt round; where they leave some
// pairs one short, those take d_weight jobs of the same length before the rest
// is dealt round.
template <int MODE> struct Jobs {
    int i, c, C, mt, nt, total;
    int dh, dw, kdh, kp, kr, r, L, fill, step;
    __device__ Jobs(const PairArgs& a, int n_rows) {
        c = blockIdx.x >> 1;
        C = gridDim.x >> 1;
        i = 0;
        mt = (n_rows + BT - 1) / BT;
        if (MODE != kProd) {
            nt = (a.cols + BT - 1) / BT;
            total = mt * nt;
            return;
        }
        nt = (a.H + BT - 1) / BT;
        kp = (a.cols + BK - 1) / BK;   // K blocks of the piece
        kr = (n_rows + BK - 1) / BK;   // K blocks of the rows
        kdh = (kp + a.split - 1) / a.split;
        dh = a.want_dh ? mt * nt * a.split : 0;
        dw = a.want_dw ? (a.cols + BT - 1) / BT * nt : 0;
        r = dh % C;
        L = r && kr ? (kdh + kr / 2) / kr : 0;
        fill = min(dw, (C - r) * L);
        step = 0;
    }
    __device__ bool next(Job& j) {
        if (MODE != kProd) {
            const int t = c + i * C;
            if (t >= total) return false;
            ++i;
            const int g = t / (kGroupM * nt), u = t - g * kGroupM * nt;
            const int mg = min(kGroupM, mt - g * kGroupM);
            j = Job{0, (g * kGroupM + u % mg) * BT, u / mg * BT, 0, 0, 0};
            return true;
        }
        if (step == 0) {
            const int t = c + i * C;
            if (t < dh) {
                ++i;
                const int s = t / (mt * nt), u = t - s * mt * nt;
                j = Job{1, u % mt * BT, u / mt * BT, min(kp, s * kdh), min(kp, (s + 1) * kdh), s};
                return true;
            }
            step = 1;
            i = 0;
        }
        int t;
        if (step == 1) {
            t = (c - r) * L + i;
            if (c >= r && i < L && t < fill) {
                ++i;
                j = Job{2, t / nt * BT, t % nt * BT, 0, kr, 0};
                return true;
            }
            step = 2;
            i = 0;
        }
        t = fill + c + i * C;
        if (t >= dw) return false;
        ++i;
        j = Job{2, t / nt * BT, t % nt * BT, 0, kr, 0};
        return true;
    }
};

__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, PairBars* sb,
                                          int* status) {
    if (tc::try_wait_cluster(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        if (tc::try_wait_cluster(bar, parity)) return true;
        if (*(volatile int*)&sb->err) return false;
        if (global_timer_ns() - t0 > kWaitNs) {
            sb->err = 1;
            atomicOr(status, VSD_STATUS_TIMEOUT);
            return false;
        }
    }
}
__device__ __forceinline__ void drain_pair(uint64_t* bar, uint32_t parity) {
    const uint64_t t0 = global_timer_ns();
    while (!tc::try_wait_cluster(bar, parity))
        if (global_timer_ns() - t0 > kWaitNs) return;
}

// First place of a list not below v.
__device__ __forceinline__ int lower_bound(const int32_t* id, int n, int v) {
    int lo = 0;
    while (lo < n) {
        const int mid = (lo + n) >> 1;
        if (__ldg(id + mid) < v) lo = mid + 1; else n = mid;
    }
    return lo;
}

// A row's target list, for one epilogue thread.
struct RowList {
    const int32_t* id;
    const float* p;
    int n;
    __device__ RowList(const PairArgs& a, int row, bool on) {
        const int r = on ? __ldg(a.tg.rowmap + row) : 0;
        id = a.tg.id + (size_t)r * a.K;
        p = a.tg.p + (size_t)r * a.K;
        n = on ? __ldg(a.tg.n + r) : 0;
    }
};

// 32 accumulators as floats, -inf from column `lim` on.
__device__ __forceinline__ void read32(uint32_t taddr, int lim, float (&f)[32]) {
    uint32_t u[32];
    tc::tmem_ld32(taddr, u);
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(u[i]);
    if (lim < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i >= lim) f[i] = -INFINITY;
    }
}

// The warp's staging buffers: `use` counts its stores.
struct Stage {
    unsigned char* buf;
    int use, lane;
    __device__ unsigned char* acquire() {
        if (lane == 0) tc::bulk_wait_read<1>();  // the store before last has read its buffer
        __syncwarp();
        return buf + (use & 1) * kOutBytes;
    }
    __device__ void store(const CUtensorMap* map, int x, int y, bool inside, bool add = false) {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            if (inside) {
                if (add) tc::add_2d(map, x, y, buf + (use & 1) * kOutBytes);
                else tc::store_2d(map, x, y, buf + (use & 1) * kOutBytes);
            }
            tc::bulk_commit();
        }
        ++use;
    }
};

// Row `lane` of a staged box: 16-byte chunk j sits at chunk j ^ (row % 8).
__device__ __forceinline__ uint4* chunk_at(unsigned char* box, int lane, int j) {
    return reinterpret_cast<uint4*>(box + lane * 128) + (j ^ (lane & 7));
}

template <bool KEEP>
__device__ __forceinline__ void stats_tile(const PairArgs& a, const PairMaps& maps, const Job& j,
                                           int row0, int lane, int n_rows, uint32_t taddr,
                                           Stage& out) {
    const int row = row0 + lane;
    const bool on = row < n_rows;
    float m = -INFINITY, s = 0.f;
#pragma unroll 1
    for (int cc = 0; cc < BT / 32; ++cc) {
        float f[32];
        read32(taddr + 32u * cc, a.cols - j.n0 - 32 * cc, f);
        float gm = f[0];
#pragma unroll
        for (int i = 1; i < 32; ++i) gm = fmaxf(gm, f[i]);
        const float nm = fmaxf(m, gm);
        if (nm > -INFINITY) {
            const float b = -nm * a.c;
            float t0 = 0.f, t1 = 0.f;
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                t0 += ex2(fmaf(f[i], a.c, b));
                t1 += ex2(fmaf(f[i + 1], a.c, b));
            }
            s = s * ex2((m - nm) * a.c) + (t0 + t1);
            m = nm;
        } else {  // nothing but -inf and NaN: a NaN has to reach the sum
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (f[i] != f[i]) s = f[i];
        }
        if (KEEP) {
            unsigned char* box = out.acquire();
#pragma unroll
            for (int v = 0; v < 8; ++v)
                *chunk_at(box, lane, v) =
                    make_uint4(__float_as_uint(f[4 * v]), __float_as_uint(f[4 * v + 1]),
                               __float_as_uint(f[4 * v + 2]), __float_as_uint(f[4 * v + 3]));
            out.store(&maps.o, j.n0 + 32 * cc, row0, row0 < n_rows);
        }
    }
    if (on) a.tab[(int64_t)(j.n0 / BT) * a.rpad + row] = make_float2(m, s);
    // the target logits in this tile: the warp reads each wanted column once
    const RowList list(a, row, on);
    const int lo = a.v0 + j.n0, hi = lo + min(BT, a.cols - j.n0);
    int k = lower_bound(list.id, list.n, lo);
    int id = k < list.n ? __ldg(list.id + k) : hi;
    for (;;) {
        const unsigned want = __ballot_sync(0xffffffffu, id < hi);
        if (!want) break;
        const int col = __shfl_sync(0xffffffffu, id, __ffs(want) - 1);
        const float x = tc::tmem_ld1(taddr + (uint32_t)(col - lo));
        if (id == col) {
            a.xk[(size_t)row * a.K + k] = x;
            ++k;
            id = k < list.n ? __ldg(list.id + k) : hi;
        }
    }
}

__device__ __forceinline__ void grad_tile(const PairArgs& a, const PairMaps& maps, const Job& j,
                                          int row0, int lane, int n_rows, uint32_t taddr,
                                          Stage& out) {
    const int row = row0 + lane;
    const bool on = row < n_rows;
    const float cf = on ? __ldg(a.coef + row) : 0.f, l = on ? __ldg(a.lse2 + row) : 0.f;
    const RowList list(a, row, on);
    const int lo = a.v0 + j.n0;
    int k = lower_bound(list.id, list.n, lo);
    // rows up to the next K block of d_weight are written (zero past the last)
    const bool inside = row0 < (n_rows + BK - 1) / BK * BK;
#pragma unroll 1
    for (int g = 0; g < BT / 64; ++g) {
        unsigned char* box = out.acquire();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[32];
            read32(taddr + 64u * g + 32u * h, a.cols - j.n0 - 64 * g - 32 * h, f);
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float lo_ = on ? cf * ex2(fmaf(f[2 * i], a.c, -l)) : 0.f;
                const float hi_ = on ? cf * ex2(fmaf(f[2 * i + 1], a.c, -l)) : 0.f;
                w[i] = tc::pack_bf16(__float_as_uint(lo_), __float_as_uint(hi_));
            }
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *chunk_at(box, lane, 4 * h + v) =
                    make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
        }
        const int base = lo + 64 * g;
        while (k < list.n) {
            const int col = __ldg(list.id + k) - base;
            if (col >= 64) break;
            const float x = __ldg(a.xk + (size_t)row * a.K + k);
            reinterpret_cast<bf16*>(chunk_at(box, lane, col >> 3))[col & 7] =
                __float2bfloat16_rn(cf * (ex2(fmaf(x, a.c, -l)) - __ldg(list.p + k)));
            ++k;
        }
        out.store(&maps.o, j.n0 + 64 * g, row0, inside);
    }
}

__device__ __forceinline__ void dh_tile(const PairArgs& a, const PairMaps& maps, const Job& j,
                                        int row0, int lane, int n_rows, uint32_t taddr,
                                        Stage& out) {
    const bool none = j.kb0 == j.kb1;
    if (none && !a.first) return;  // nothing to add
#pragma unroll 1
    for (int g = 0; g < BT / 32; ++g) {
        unsigned char* box = out.acquire();
        uint32_t u[32];
        tc::tmem_ld32(taddr + 32u * g, u);
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *chunk_at(box, lane, v) =
                none ? make_uint4(0u, 0u, 0u, 0u)
                     : make_uint4(u[4 * v], u[4 * v + 1], u[4 * v + 2], u[4 * v + 3]);
        const int x = j.n0 + 32 * g;
        out.store(&maps.dh, x, (int)(j.part * a.rpad) + row0, x < a.H && row0 < n_rows, !a.first);
    }
}

__device__ __forceinline__ void dw_tile(const PairArgs& a, const PairMaps& maps, const Job& j,
                                        int row0, int lane, uint32_t taddr, Stage& out) {
    const bool none = j.kb0 == j.kb1;
    const float s = none ? 0.f : __ldg(a.kappa);
#pragma unroll 1
    for (int g = 0; g < BT / 64; ++g) {
        unsigned char* box = out.acquire();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t u[32];
            tc::tmem_ld32(taddr + 64u * g + 32u * h, u);
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                w[i] = none ? 0u
                            : tc::pack_bf16(__float_as_uint(s * __uint_as_float(u[2 * i])),
                                            __float_as_uint(s * __uint_as_float(u[2 * i + 1])));
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *chunk_at(box, lane, 4 * h + v) =
                    make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
        }
        const int x = j.n0 + 64 * g, y = a.v0 + row0;
        out.store(&maps.dw, x, y, x < a.H && y < a.V);
    }
}

template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    k_pair(const __grid_constant__ PairMaps maps, const PairArgs a) {
    extern __shared__ unsigned char dsm_raw[];
    unsigned char* dsm = dsm_raw + ((1024u - (smem_u32(dsm_raw) & 1023u)) & 1023u);
    unsigned char* outs = dsm + kPairStages * kStageBytes;
    PairBars* sb = reinterpret_cast<PairBars*>(outs + 8 * kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)tc::cluster_rank();
    int* status = a.tg.status;
    const int n_rows = __ldg(a.tg.nrows);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(&sb->full[s], 1);
            mbar_init(&sb->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sb->acc_full[b], 1);
            mbar_init(&sb->acc_empty[b], 8);
        }
        mbar_init(&sb->drain, 1);
        sb->err = 0;
        mbar_init_fence();
    }
    if (warp == 1) tc::tmem_alloc_pair(&sb->tmem_base, kTmemAll);
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after();
    const uint32_t tmem = sb->tmem_base;
    Jobs<MODE> jobs(a, n_rows);
    Job j;

    if (warp == 0) {
        // ------------------------------------------------------ TMA producer
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            while (ok && !*(volatile int*)&sb->err && jobs.next(j)) {
                const int kb1 = MODE == kProd ? j.kb1 : a.nkh;
                for (int kb = j.kb0; kb < kb1; ++kb) {
                    const int s = (int)(it % kPairStages);
                    const uint32_t round = it / kPairStages;
                    if (round > 0 && !wait_pair(&sb->empty[s], (round - 1) & 1u, sb, status)) {
                        ok = false;
                        break;
                    }
                    unsigned char* A = dsm + s * kStageBytes;
                    unsigned char* B = A + kHalfBytes;
                    const uint32_t bar = tc::leader_addr(&sb->full[s]);
                    if (rank == 0) mbar_expect_tx(&sb->full[s], 2 * kStageBytes);
                    if (MODE != kProd) {
                        tc::load_2d(A, &maps.a, kb * BK, j.m0 + 128 * rank, bar);
                        tc::load_2d(B, &maps.b, kb * BK, a.v0 + j.n0 + 128 * rank, bar);
                    } else {
                        const int n = j.n0 + 128 * rank;
                        if (j.kind == 1) {
                            tc::load_2d(A, &maps.gk, kb * BK, j.m0 + 128 * rank, bar);
                            tc::load_2d(B, &maps.wt, n, a.v0 + kb * BK, bar);
                            tc::load_2d(B + kBoxBytes, &maps.wt, n + 64, a.v0 + kb * BK, bar);
                        } else {
                            const int m = j.m0 + 128 * rank;
                            tc::load_2d(A, &maps.gt, m, kb * BK, bar);
                            tc::load_2d(A + kBoxBytes, &maps.gt, m + 64, kb * BK, bar);
                            tc::load_2d(B, &maps.ht, n, kb * BK, bar);
                            tc::load_2d(B + kBoxBytes, &maps.ht, n + 64, kb * BK, bar);
                        }
                    }
                    ++it;
                }
            }
            // the copies still in flight have landed before the pair may exit
            if (rank == 0)
                for (uint32_t i = it > (uint32_t)kPairStages ? it - kPairStages : 0; i < it; ++i)
                    drain_pair(&sb->full[i % kPairStages], (i / kPairStages) & 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------ MMA issuer
        if (lane == 0 && rank == 0) {
            uint32_t it = 0;
            int lt = 0;
            bool ok = true;
            for (; ok && !*(volatile int*)&sb->err && jobs.next(j); ++lt) {
                const int buf = lt & 1;
                const uint32_t use = (uint32_t)lt >> 1;
                if (use > 0 && !wait_pair(&sb->acc_empty[buf], (use - 1) & 1u, sb, status)) break;
                tc::tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * BT);
                const bool amn = MODE == kProd && j.kind == 2, bmn = MODE == kProd;
                const uint32_t idesc = tc::idesc_bf16(256, BT) | (amn ? 1u << 15 : 0u) |
                                       (bmn ? 1u << 16 : 0u);
                const int kb1 = MODE == kProd ? j.kb1 : a.nkh;
                for (int kb = j.kb0; kb < kb1; ++kb) {
                    const int s = (int)(it % kPairStages);
                    if (!wait_pair(&sb->full[s], (it / kPairStages) & 1u, sb, status)) {
                        ok = false;
                        break;
                    }
                    tc::tc_fence_after();
                    const uint32_t A = smem_u32(dsm + s * kStageBytes), B = A + kHalfBytes;
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k)
                        tc::mma_pair(d,
                                     amn ? tc::desc_mn(A + 2048u * k, kBoxBytes)
                                         : tc::sdesc_sw128(A + 32u * k),
                                     bmn ? tc::desc_mn(B + 2048u * k, kBoxBytes)
                                         : tc::sdesc_sw128(B + 32u * k),
                                     idesc, (kb != j.kb0 || k != 0) ? 1u : 0u);
                    tc::commit_pair(&sb->empty[s]);
                    ++it;
                }
                if (!ok) break;
                tc::commit_pair(&sb->acc_full[buf]);
            }
            tc::commit_pair(&sb->drain);  // every MMA issued is done once it arrives
            drain_pair(&sb->drain, 0);
        }
    } else {
        // ------------------------------------------------------ epilogue
        const int q = warp & 3;  // TMEM lanes 32q .. 32q + 31
        Stage out{outs + (warp - 2) * 2 * kOutBytes, 0, lane};
        for (int lt = 0; jobs.next(j); ++lt) {
            const int buf = lt & 1;
            const uint32_t use = (uint32_t)lt >> 1;
            if (!__all_sync(0xffffffffu, wait_pair(&sb->acc_full[buf], use & 1u, sb, status)))
                break;
            tc::tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * BT);
            const int row0 = j.m0 + 128 * rank + 32 * q;
            if (MODE == kStats) stats_tile<false>(a, maps, j, row0, lane, n_rows, taddr, out);
            if (MODE == kKeep) stats_tile<true>(a, maps, j, row0, lane, n_rows, taddr, out);
            if (MODE == kGrad) grad_tile(a, maps, j, row0, lane, n_rows, taddr, out);
            if (MODE == kProd) {
                if (j.kind == 1) dh_tile(a, maps, j, row0, lane, n_rows, taddr, out);
                else dw_tile(a, maps, j, row0, lane, taddr, out);
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::arrive_remote(tc::leader_addr(&sb->acc_empty[buf]));
        }
        if (lane == 0) tc::bulk_wait_all();
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_free_pair(tmem, kTmemAll);
    }
}

// One warp per counted row: its log-partition, loss and gradient coefficient;
// the last block to finish sums the losses in row order.
__global__ void k_rows(const float2* tab, int ntab, int64_t stride, Targets tg, int K, float c,
                       float T, float grad_scale, const float* xk, float* lse2, float* coef,
                       float* kappa, float* row_loss, float* logz, float* loss, int R) {
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
            const float wm = *tg.wmax;
            coef[i] = wm > 0.f ? kTopMantissa * (tg.w[r] / wm) : 0.f;
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
        *kappa = (float)((double)grad_scale * (double)*tg.wmax /
                         ((double)kTopMantissa * *tg.wsum * (double)T));
    }
}

// G from logits that were kept, 2048 columns of a row per block; rows up to the
// next K block of d_weight and columns up to ldg are written, zero where there
// is no logit.
constexpr int kMakeCols = 2048;
__global__ void __launch_bounds__(256)
    k_make_g(const float* X, int64_t ldx, int V, int K, Targets tg, float c, const float* lse2,
             const float* coef, const float* xk, bf16* G, int64_t ldg) {
    const int i = blockIdx.y, n_rows = *tg.nrows;
    if (i >= (n_rows + BK - 1) / BK * BK) return;
    const int c0 = blockIdx.x * kMakeCols, v = c0 + threadIdx.x * 8;
    bf16* g = G + (size_t)i * ldg;
    const bool on = i < n_rows;
    const float a = on ? coef[i] : 0.f, l = on ? lse2[i] : 0.f;
    if (v < ldg) {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (on && v < V) {  // (ldx is a multiple of 256: the loads stay in the row)
            const float4* x = reinterpret_cast<const float4*>(X + (size_t)i * ldx + v);
            const float4 x0 = x[0], x1 = x[1];
            const float f[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = v + 2 * e < V ? a * ex2(fmaf(f[2 * e], c, -l)) : 0.f;
                const float hi = v + 2 * e + 1 < V ? a * ex2(fmaf(f[2 * e + 1], c, -l)) : 0.f;
                w[e] = tc::pack_bf16(__float_as_uint(lo), __float_as_uint(hi));
            }
        }
        *reinterpret_cast<uint4*>(g + v) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (!on) return;
    __syncthreads();
    const int r = tg.rowmap[i], n = tg.n[r];
    const int32_t* id = tg.id + (size_t)r * K;
    for (int k = threadIdx.x; k < n; k += blockDim.x)
        if (id[k] >= c0 && id[k] < c0 + kMakeCols)
            g[id[k]] = __float2bfloat16_rn(
                a * (ex2(fmaf(xk[(size_t)i * K + k], c, -l)) - tg.p[(size_t)r * K + k]));
}

// d_hidden in the caller's rows: the parts added in order, one rounding, zero
// in rows not counted.
__global__ void k_dh_out(const float* dh, int split, int64_t rpad, int H, Targets tg,
                         const float* kappa, bf16* out) {
    const int r = blockIdx.x, i = tg.rowinv[r];
    const float s = *kappa;
    for (int h = threadIdx.x * 8; h < H; h += blockDim.x * 8) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (i >= 0) {
            float f[8] = {};
            for (int q = 0; q < split; ++q) {
                const float4* p =
                    reinterpret_cast<const float4*>(dh + ((size_t)q * rpad + i) * H + h);
                const float4 x = p[0], y = p[1];
                f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
                f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
            }
            uint32_t* o = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[e] = tc::pack_bf16(__float_as_uint(s * f[2 * e]), __float_as_uint(s * f[2 * e + 1]));
        }
        *reinterpret_cast<uint4*>(out + (size_t)r * H + h) = w;
    }
}

}  // namespace

bool lmloss_shape_ok(const LmLossShape& s) {
    return s.R >= 1 && s.R <= (1 << 24) && s.V >= 1 && s.V <= (1 << 20) && s.H >= 8 &&
           s.H <= (1 << 20) && s.H % 8 == 0 && s.K >= 1 && s.K <= kMaxTeacher && s.piece >= 0;
}

size_t lmloss_workspace_bytes(const LmLossShape& s) {
    return lmloss_shape_ok(s) ? lm_ws(s).total : 0;
}

template <int MODE>
static cudaError_t launch_pair(const PairMaps& maps, const PairArgs& a, int64_t jobs,
                               cudaStream_t st) {
    cudaError_t e = ensure_dyn_smem((const void*)k_pair<MODE>, kPairSmem);
    if (e != cudaSuccess) return e;
    const int64_t pairs = std::max<int64_t>(1, std::min<int64_t>(jobs, device_sm_count() / 2));
    k_pair<MODE><<<(unsigned)(2 * pairs), kPairThreads, kPairSmem, st>>>(maps, a);
    return cudaGetLastError();
}

cudaError_t lmloss(const LmLossShape& s, const void* hidden, const void* weight,
                   const TargetIn& in, float T, float grad_scale, const vsd_loss_outputs& out,
                   void* ws, cudaStream_t st) {
    const LmWs w = lm_ws(s);
    const int R = s.R, V = s.V, H = s.H, K = s.K;
    Targets tg{at<int32_t>(ws, w.n), at<int32_t>(ws, w.id), at<float>(ws, w.p),
               at<float>(ws, w.plogp), at<float>(ws, w.w), at<int32_t>(ws, w.rowmap),
               at<int32_t>(ws, w.rowinv), at<int32_t>(ws, w.nrows), at<double>(ws, w.wsum),
               at<float>(ws, w.wmax), at<int32_t>(ws, w.done), at<int32_t>(ws, w.status)};
    bf16* hid = at<bf16>(ws, w.hid);
    float* X = at<float>(ws, w.X);
    bf16* G = at<bf16>(ws, w.G);
    float2* tab = at<float2>(ws, w.tab);
    float *xk = at<float>(ws, w.xk), *lse2 = at<float>(ws, w.lse2), *coef = at<float>(ws, w.coef),
          *kappa = at<float>(ws, w.kappa), *dh = at<float>(ws, w.dh);
    const float c = (float)(kLog2e / (double)T);
    // rows of the packed hidden states that may be read: up to a K block
    const int64_t hrows = round_up(R, BK);
    PairMaps maps;
    memset(&maps, 0, sizeof(maps));
    using vsd_lm::make_map_sw128;
    bool ok = make_map_sw128(&maps.a, hid, false, hrows, H, H, 128) &&
              make_map_sw128(&maps.b, weight, false, V, H, H, 128);
    if (s.dh || s.dw)
        ok = ok && make_map_sw128(&maps.gk, G, false, w.rpad, w.piece, w.piece, 128) &&
             make_map_sw128(&maps.gt, G, false, w.rpad, w.piece, w.piece, BK) &&
             make_map_sw128(&maps.wt, weight, false, V, H, H, BK) &&
             make_map_sw128(&maps.ht, hid, false, hrows, H, H, BK);
    if (w.keep) ok = ok && make_map_sw128(&maps.o, X, true, w.rpad, w.piece, w.piece, 32);
    else if (s.dh || s.dw)
        ok = ok && make_map_sw128(&maps.o, G, false, w.rpad, w.piece, w.piece, 32);
    if (s.dw) ok = ok && make_map_sw128(&maps.dw, out.d_weight, false, V, H, H, 32);
    if (s.dh)
        ok = ok && make_map_sw128(&maps.dh, dh, true, (int64_t)w.rpad * w.split, H, H, 32);
    if (!ok) return cudaErrorInvalidValue;

    PairArgs a{};
    a.tg = tg;
    a.K = K;
    a.H = H;
    a.V = V;
    a.v0 = 0;
    a.cols = V;
    a.nkh = (H + BK - 1) / BK;
    a.rpad = w.rpad;
    a.c = c;
    a.tab = tab;
    a.xk = xk;
    a.lse2 = lse2;
    a.coef = coef;
    a.kappa = kappa;
    a.split = w.split;
    a.want_dh = s.dh;
    a.want_dw = s.dw;

    cudaError_t e = cudaMemsetAsync(ws, 0, w.zero_end, st);
    if (e != cudaSuccess) return e;
    k_targets<<<(R + 7) / 8, 256, 0, st>>>(in, tg, out.row_loss, out.logz);
    k_gather<<<std::min(w.rpad, 4 * device_sm_count()), 256, 0, st>>>(
        static_cast<const bf16*>(hidden), H, tg, hid);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const int64_t mt = w.rpad / kRowPad, units = (V + kPieceUnit - 1) / kPieceUnit;
    const int64_t ht = (H + BT - 1) / BT;
    e = w.keep ? launch_pair<kKeep>(maps, a, mt * units, st)
               : launch_pair<kStats>(maps, a, mt * units, st);
    if (e != cudaSuccess) return e;
    k_rows<<<(R + 7) / 8, 256, 0, st>>>(tab, (int)units, w.rpad, tg, K, c, T, grad_scale, xk, lse2,
                                        coef, kappa, out.row_loss, out.logz, out.loss, R);
    if ((e = cudaGetLastError()) != cudaSuccess || !(s.dh || s.dw)) return e;
    for (int q = 0; q < w.npiece; ++q) {
        a.v0 = q * w.piece;
        a.cols = std::min(w.piece, V - a.v0);
        a.first = q == 0;
        const int64_t nu = (a.cols + kPieceUnit - 1) / kPieceUnit;
        if (w.keep) {
            const dim3 grid((unsigned)((w.piece + kMakeCols - 1) / kMakeCols), (unsigned)hrows);
            k_make_g<<<grid, 256, 0, st>>>(X, w.piece, V, K, tg, c, lse2, coef, xk, G, w.piece);
            e = cudaGetLastError();
        } else {
            e = launch_pair<kGrad>(maps, a, mt * nu, st);
        }
        if (e != cudaSuccess) return e;
        e = launch_pair<kProd>(maps, a, (s.dh ? mt * ht * w.split : 0) + (s.dw ? nu * ht : 0), st);
        if (e != cudaSuccess) return e;
    }
    if (s.dh) {
        k_dh_out<<<R, 256, 0, st>>>(dh, w.split, w.rpad, H, tg, kappa,
                                    static_cast<bf16*>(out.d_hidden));
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace vsd
