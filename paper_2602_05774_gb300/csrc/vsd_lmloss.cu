// vsd_lmloss.cu -- the LM head's supervised losses without keeping the logits:
//
//   x = hidden . W^T,  q_r = softmax(x_r / T),
//   l_r = sum_k p_rk (log p_rk - log q_r(id_rk)),
//   G_rv = a_r (q_r(v) - sum_k p_rk [v = id_rk]),   a_r = scale w_r / (T sum w),
//   d_hidden = G . W,  d_weight = G^T . hidden.
//
// The rows that count are gathered first (a row not counted costs nothing and
// cannot spread a NaN).  A first sweep over the vocabulary takes each row's
// maximum, sum of exponentials and target logits; the rows' losses and
// log-partitions follow; a second sweep makes the logits again, piece by piece,
// turns them into G (bf16) and adds the piece's products.  Few rows' logits are
// kept and made once.
//
// Bound by the tensor cores for many rows (4096 x 32000 x 4096 with gradients:
// 2.51 to 2.57 ms from GPU to GPU for 4.29 TFLOP, 1.67 to 1.71 PFLOP/s, where
// cuBLAS sustains 1.69), by memory for few (48 x 128256 x 4096: 0.54 ms for the
// weight read twice and its gradient written, 3.15 GB).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>
#include <string.h>

#include "vsd.h"
#include "vsd_common.cuh"
#include "vsd_launch.h"
#include "vsd_loss.h"
#include "vsd_pair.cuh"
#include "vsd_rowloss.cuh"

namespace vsd {
namespace {

typedef __nv_bfloat16 bf16;

constexpr int kRowPad = 256;     // the workspace's rows are a multiple of this
constexpr int BK = 64;           // K block of the products
constexpr int kPieceUnit = 256;  // a piece's columns are a multiple of this
// Bytes of a piece's G: about the L2.  The time hardly depends on it (4096 x 32000
// x 4096 with pieces of 8192, 16128 and 32000 columns: within the 5 % that the power
// limit moves them).
constexpr int64_t kPieceBytes = 128ll << 20;
constexpr int64_t kKeepBytes = 64ll << 20;
// Pairs of SMs, of the part these kernels are built for: the plan and the workspace's
// size go by it on any device, and no launch has more.
constexpr int64_t kPairs = 76;
// The tensor cores' running sum truncates: up to 1e-7 of it a step of 16 where the
// terms have one sign (5.2 % after 2^19 steps).  Longer sums than these, in K blocks,
// are cut into parts that are added up in fp32: the gradient's logits at 8192 hidden
// elements (5e-5 of a logit), products at 65536 rows or columns (4e-4, a fifth of
// their rounding to bf16).
constexpr int kLongLogits = 128, kLongProd = 1024;
constexpr int64_t kCarry = 8 * 32 * 128;  // a CTA's sums so far: the epilogue's part of a tile
constexpr int kStoreCost = 5;    // K blocks of time that storing a d_weight tile takes at least
// The operand G is scaled so that the largest weight sits at the top of a
// binade (1.984 ..), where bf16's relative rounding error is least: a row's
// target entries are near -w before the draft has learned them, and they
// dominate the products.  The outputs take the factor back in fp32 (kappa).
constexpr float kTopMantissa = 1.984375f;

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct LmWs {
    size_t status, done, zero_end, nrows, wsum, wmax, kappa, unit, share, n, id, p, plogp, w,
        rowmap, rowinv, top, coef, coefs, xk, tab, part, hid, X, G, dh, carry, total;
    int rpad, hrows, piece, npiece, split;  // rows padded to a tile, to a K block
    bool keep;  // the logits are kept (one piece)
    bool cut_grad, cut_prod;  // long sums are cut into parts
};

LmWs lm_ws(const LmLossShape& s) {
    LmWs w;
    const size_t R = (size_t)s.R, RK = R * (size_t)s.K;
    const bool grads = s.dh || s.dw;
    w.rpad = (int)round_up(s.R, kRowPad);
    w.hrows = (int)round_up(s.R, BK);
    const int64_t vpad = round_up(s.V, kPieceUnit);
    const int64_t most = std::max<int64_t>(1, kPieceBytes / (2 * (int64_t)w.hrows * kPieceUnit));
    // few rows: the whole vocabulary's logits (4 bytes) and G (2) fit the space
    // of the weight, or are small; they are made once (48 x 128256 x 4096: 540 us,
    // 714 with two sweeps; 1000 x 32000 x 4096: 528 and 637)
    const int64_t whole = 6 * (int64_t)w.hrows * vpad;
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
    // parts of a piece's columns in d_hidden where its tiles are few: the least
    // time by 0.3 us a K block (its own rounds, or where d_weight's jobs fill in
    // the pairs' share of all and part of a job), 6 us for the launch that adds
    // parts up and, for a part, 0.1 us and its bytes' way out and back at 6 TB/s;
    // each part of 8 K blocks at least.  (d_hidden alone, and with the best of nine
    // other numbers of parts: 48 x 128256 x 4096 353 us and 348, 300 x 32000 x 4096 201
    // and 201, 777 x 32003 x 2056 306 and 306, 40 x 60000 x 264 47 and 48, 1000 x 128256
    // x 1024 531 and 527; in one part 696, 256, 358, 270 and 913)
    const int64_t ht = (s.H + kRowPad - 1) / kRowPad, tiles = (int64_t)(w.rpad / kRowPad) * ht;
    w.split = 1;
    if (tiles < 2 * kPairs) {
        const int64_t kp = w.piece / BK, kr = std::max(w.hrows / BK, kStoreCost);
        const double share = (double)(tiles * kp + per * ht * kr) / kPairs;
        const double part_us = 0.1 + 8e-6 / 6.0 * (double)w.hrows * s.H;
        double best = 1e30;
        for (int64_t n = 1; n <= kPairs && (n == 1 || kp >= 8 * n); ++n) {
            const double job = (double)((kp + n - 1) / n);
            const double blocks = s.dw ? std::max(job, share + 0.25 * job)
                                       : job * (double)((tiles * n + kPairs - 1) / kPairs);
            const double us = 0.3 * blocks + (n > 1 ? 6.0 + part_us * (double)n : 0.0);
            if (us < best) best = us, w.split = (int)n;
        }
    }
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
    w.unit = take(4);
    w.share = take(4);
    w.n = take(4 * R);
    w.id = take(4 * RK);
    w.p = take(4 * RK);
    w.plogp = take(4 * R);
    w.w = take(4 * R);
    w.rowmap = take(4 * R);
    w.rowinv = take(4 * R);
    w.top = take(4 * (size_t)w.rpad);
    w.coef = take(4 * (size_t)w.rpad);
    w.coefs = take(4 * (size_t)w.rpad);
    w.xk = take(4 * RK);
    w.tab = take(8 * (size_t)w.rpad * (size_t)units * 2);
    w.part = take(8 * R);
    w.hid = take(2 * (size_t)w.hrows * s.H);
    w.X = take(w.keep ? 4 * (size_t)w.hrows * w.piece : 0);
    w.G = take(grads ? 2 * (size_t)w.hrows * w.piece : 0);
    w.dh = take(s.dh ? 4 * (size_t)w.rpad * s.H * w.split : 0);
    w.cut_grad = grads && !w.keep && (s.H + BK - 1) / BK > kLongLogits;
    w.cut_prod = (s.dw && w.hrows / BK > kLongProd) ||
                 (s.dh && (w.piece / BK + w.split - 1) / w.split > kLongProd);
    w.carry = take(w.cut_grad || w.cut_prod ? 4 * kCarry * 2 * kPairs : 0);
    w.total = o;
    return w;
}

// ------------------------------------------------------------ rows
// Counted rows of hidden, packed; the rows up to the next K block of d_weight
// are zero (where every row counts the products read hidden itself).  Rows not
// counted get a zero gradient.
__global__ void __launch_bounds__(256)
    k_gather(const bf16* hidden, int R, int H, Targets tg, bf16* hid, bf16* d_hidden) {
    dep_launch();
    dep_wait();
    const int n = *(const volatile int*)tg.nrows;
    if (n == R) return;
    const int vecs = H / 8;
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    const int64_t t0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t end = (int64_t)((n + BK - 1) / BK * BK) * vecs;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 4
    for (int64_t t = t0; t < end; t += step) {
        const int i = (int)(t / vecs), v = (int)(t - (int64_t)i * vecs);
        reinterpret_cast<uint4*>(hid)[t] =
            i < n ? __ldg(reinterpret_cast<const uint4*>(hidden + (size_t)tg.rowmap[i] * H) + v)
                  : zero;
    }
    if (!d_hidden) return;
    for (int64_t t = t0; t < (int64_t)R * vecs; t += step)
        if (tg.rowinv[t / vecs] < 0) reinterpret_cast<uint4*>(d_hidden)[t] = zero;
}

// ------------------------------------------------------------ products
// All products run as 256 x 256 tiles of a CTA pair, K in blocks of 64 through
// a ring of kStages stages; the accumulator of one tile is read back while the
// next one is computed (2 x 256 TMEM columns).  Per CTA:
//   warp 0     TMA producer: its half of A and of B (16 KB each) per K block,
//              counted on the leader's barrier;
//   warp 1     the leader's MMA issuer (one thread, for both CTAs);
//   warps 4-11 epilogue: 32 rows x 128 columns each, tcgen05.ld, then what the
//              product is for:
//     logits   A = hidden rows, B = weight rows, both K-major.  kStats: per row
//              and half tile (max, sum 2^{(x - max) c}) and the target logits
//              in it.  kKeep: the logits themselves, fp32.  Both sum K in parts
//              of 512 that are added up in the epilogue's registers (round to
//              nearest: the tensor cores' truncation grows with the steps).
//              kGrad: G, rounded to bf16.  Its epilogue has no registers for
//              that; its sums are cut at kLongLogits.
//     d_hidden A = G (K-major), B = weight (MN-major, as it lies): fp32 sums,
//              added up over the pieces of the vocabulary by TMA.
//     d_weight A = G (MN-major), B = hidden (MN-major): one rounding to bf16.
//              Both products' sums are cut at kLongProd.
// A cut sum is carried from part to part in the workspace, 16 KB a warp (CUT: an
// instance of its own; the registers it takes cost 48 x 128256 x 4096 546 to 558 us).
// What is stored goes through 4 KB of swizzled shared memory per warp and a TMA
// store.  Every wait is bounded: one that runs out sets VSD_STATUS_TIMEOUT, and
// the pair winds down, waits for its copies and MMAs in flight and frees its
// tensor memory.
namespace tc = vsd_pair;

constexpr int BT = 256;
constexpr int kTileWarps = 8;                  // epilogue warps of a tile
constexpr int kHalfN = BT / 2;                 // columns of an epilogue warp
constexpr int kSumBlocks = 8;                  // K blocks of a partial sum, at most
// Registers per thread of the kernels that add partial sums: launched with 168,
// of which the first warpgroup gives up what the two epilogue groups take
// (128 (40 + 232 + 232) = 384 * 168).
constexpr int kRegsFew = 40, kRegsMany = 232;
static_assert(kRegsFew + 2 * kRegsMany <= 3 * 168, "the launch's registers");
constexpr int kHalfBytes = 128 * BK * 2;       // one operand's half tile: 16 KB
constexpr int kBoxBytes = 64 * BK * 2;         // an MN-major half is two 64-column boxes
constexpr int kOutBytes = 4096;                // 32 rows x 128 bytes
constexpr int kMaxStages = 9;
constexpr uint32_t kTmemAll = 2 * BT;
constexpr uint64_t kWaitNs = 2000000000ull;
constexpr int kGroupM = 16;                    // M tiles that share B tiles in L2
static_assert(kCarry == kTileWarps * 32 * kHalfN, "a CTA's accumulator");

struct PairBars {
    uint64_t full[kMaxStages];    // leader: both CTAs' bytes landed
    uint64_t empty[kMaxStages];   // the MMAs reading the stage are done
    uint64_t acc_full[2];
    uint64_t acc_empty[2];        // leader: the epilogue warps of both CTAs
    uint64_t drain;
    uint32_t tmem_base;
    int err;
};
// kStats1: kStats where one partial sum spans the hidden size (1715 x 105611 x
// 104: 371 us a step, 393 with kStats)
enum { kStats = 0, kKeep = 1, kGrad = 2, kProd = 3, kStats1 = 4 };

// Few rows (NF = 64 or 128 at most): the products with the rows' side are turned
// round, so that the weight's side is the 256-wide M of the tile and the rows
// are its N, and no part of the tile is empty:
//     logits^T  A = weight rows (K-major), B = hidden rows (K-major)
//     d_hidden^T  A = weight (MN-major, M = hidden size), B = G rows (K-major)
// What the tile costs then is bringing the weight in.  NF = 0: rows are M.
template <int MODE, int NF> struct PairCfg {
    static constexpr bool kFew = NF > 0;
    // Epilogues that exponentiate take as long as some ten K blocks: two sets of
    // warps, one for each accumulator, for the gradient and for kStats1 (1715 x
    // 105611 x 104: 371 us; 400 with one set for the gradient, 399 for kStats1).
    // kStats and kKeep have no registers for it; the products gain more from the
    // stage it costs (3 % of a step of 300 x 32000 x 4096).
    static constexpr int kSets = MODE == kGrad || MODE == kStats1 ? 2 : 1;
    static constexpr int kThreads = 32 * (4 + kSets * kTileWarps);
    static constexpr int kFewB = NF / 2 * BK * 2;  // the rows' half of a turned stage
    static constexpr int kStageBytes = MODE == kKeep && kFew ? kHalfBytes + kFewB : 2 * kHalfBytes;
    static constexpr int kStages =
        MODE == kKeep && kFew ? (NF == 64 ? 9 : 8) : kSets == 2 ? 5 : 6;
    static constexpr size_t kSmem =
        1024 + (size_t)kStages * kStageBytes + kSets * kTileWarps * kOutBytes +
        sizeof(PairBars);
    static_assert(kStages <= kMaxStages && kSmem <= 232448, "shared memory");
};

struct PairMaps {
    CUtensorMap a, a0, b, o;         // logits: packed rows, hidden, weight; stored tiles
    CUtensorMap gk, gt, wt, ht, ht0; // products: G K- and MN-major; MN-major the weight,
                                     // the packed rows, hidden
    CUtensorMap dh;
};
struct PairArgs {
    Targets tg;
    int R, K;              // rows of the call, entries of a target list
    int H, V, v0, cols;    // this piece: columns v0 .. v0 + cols - 1
    int nkh, part;         // K blocks of the hidden size, of an uncut sum
    float* carry;
    int64_t rpad;
    float c;
    float2* tab;
    float* xk;
    const float *top, *coef, *coefs, *kappa;  // a row's largest logit, coefficient, the same / S
    int split;             // d_hidden: parts of the piece's columns
    int first, last;       // first and last piece
    int want_dh, want_dw;
    float* dh;             // sums of the pieces so far, [split][rpad][H]
    const float* row_loss; // for the mean, written by the first product that has `loss`
    float* loss;
    float* X;              // kept logits
    int64_t ldx;
    bf16 *d_hidden, *d_weight;
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
template <int MODE, bool FEW> struct Jobs {
    int i, c, C, mt, nt, total;
    int dh, dw, kdh, kp, kr, r, L, fill, step;
    __device__ Jobs(const PairArgs& a, int n_rows) {
        c = blockIdx.x >> 1;
        C = gridDim.x >> 1;
        i = 0;
        mt = (n_rows + BT - 1) / BT;
        if (MODE != kProd) {
            nt = (a.cols + BT - 1) / BT;
            total = mt * nt;  // (few rows: mt is 1, or 0 where no row counts)
            return;
        }
        nt = (a.H + BT - 1) / BT;
        kp = (a.cols + BK - 1) / BK;   // K blocks of the piece
        kr = (n_rows + BK - 1) / BK;   // K blocks of the rows
        kdh = (kp + a.split - 1) / a.split;
        dh = a.want_dh ? mt * nt * a.split : 0;
        dw = a.want_dw ? (a.cols + BT - 1) / BT * nt : 0;
        r = dh % C;
        const int cost = max(kr, kStoreCost);
        L = r ? (kdh + cost / 2) / cost : 0;
        fill = min(dw, (C - r) * L);
        step = 0;
    }
    __device__ bool next(Job& j) {
        if (MODE != kProd) {
            const int t = c + i * C;
            if (t >= total) return false;
            ++i;
            if (FEW) {
                j = Job{0, t * BT, 0, 0, 0, 0};
                return true;
            }
            const int g = t / (kGroupM * nt), u = t - g * kGroupM * nt;
            const int mg = min(kGroupM, mt - g * kGroupM);
            j = Job{0, (g * kGroupM + u % mg) * BT, u / mg * BT, 0, 0, 0};
            return true;
        }
        // steps 0: d_hidden, 1: the d_weight jobs in place of one, 2: the rest
        for (; step < 3; ++step, i = 0) {
            if (step == 0) {
                const int t = c + i * C;
                if (t < dh) {
                    ++i;
                    const int s = t / (mt * nt), u = t - s * mt * nt;
                    j = Job{1, (FEW ? u : u % mt) * BT, FEW ? 0 : u / mt * BT, min(kp, s * kdh),
                            min(kp, (s + 1) * kdh), s};
                    return true;
                }
                continue;
            }
            const int t = step == 1 ? (c - r) * L + i : fill + c + i * C;
            if (step == 1 ? c >= r && i < L && t < fill : t < dw) {
                ++i;
                j = Job{2, t / nt * BT, t % nt * BT, 0, kr, 0};
                return true;
            }
        }
        return false;
    }
};

__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, PairBars* sb,
                                          int* status) {
    if (bounded_wait([&] { return tc::try_wait_cluster(bar, parity); },
                     [&] { return *(volatile int*)&sb->err != 0; }, kWaitNs))
        return true;
    if (!*(volatile int*)&sb->err) {
        sb->err = 1;
        atomicOr(status, VSD_STATUS_TIMEOUT);
    }
    return false;
}
__device__ __forceinline__ void drain_pair(uint64_t* bar, uint32_t parity) {
    bounded_wait([&] { return tc::try_wait_cluster(bar, parity); }, [] { return false; }, kWaitNs);
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

// A row's target list, for one epilogue thread: entry k is the first from token
// `lo` on, next its token.  (Made before the tile's accumulator is waited for.)
struct RowList {
    const int32_t* id;
    const float* p;
    int n, k, next;
    __device__ RowList(const PairArgs& a, int row, bool on, int lo) {
        const int r = on ? __ldg(a.tg.rowmap + row) : 0;
        id = a.tg.id + (size_t)r * a.K;
        p = a.tg.p + (size_t)r * a.K;
        n = on ? __ldg(a.tg.n + r) : 0;
        k = lower_bound(id, n, lo);
        next = k < n ? __ldg(id + k) : INT_MAX;
    }
};

// 32 accumulators of a lane, with the sum of the parts before, if any (element i of
// carry at 32 i; kCarryStep on from one 32 columns to the next).
constexpr int kCarryStep = 32 * 32;
__device__ __forceinline__ void sum32(uint32_t taddr, const float* carry, uint32_t (&u)[32]) {
    __syncwarp();  // (tensor memory is read by whole warps)
    tc::tmem_ld32(taddr, u);
    if (carry) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            u[i] = __float_as_uint(__uint_as_float(u[i]) + carry[32 * i]);
    }
}
__device__ __forceinline__ const float* carried(const float* carry, int g) {
    return carry ? carry + g * kCarryStep : nullptr;
}

// 32 accumulators as floats, -inf from column `lim` on.
__device__ __forceinline__ void read32(uint32_t taddr, const float* carry, int lim,
                                       float (&f)[32]) {
    uint32_t u[32];
    sum32(taddr, carry, u);
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = i < lim ? __uint_as_float(u[i]) : -INFINITY;
}

// The warp's staging buffer.
struct Stage {
    unsigned char* buf;
    int lane;
    __device__ unsigned char* acquire() {
        if (lane == 0) tc::bulk_wait_read<0>();  // the last store has read it
        __syncwarp();
        return buf;
    }
    __device__ void store(const CUtensorMap* map, int x, int y, bool inside, bool add = false) {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            if (inside) {
                if (add) tc::add_2d(map, x, y, buf);
                else tc::store_2d(map, x, y, buf);
            }
            tc::bulk_commit();
        }
    }
};

// Row `lane` of a staged box: 16-byte chunk j sits at chunk j ^ (row % 8).
__device__ __forceinline__ uint4* chunk_at(unsigned char* box, int lane, int j) {
    return reinterpret_cast<uint4*>(box + lane * 128) + (j ^ (lane & 7));
}

// n0: the warp's first column of the piece; x: its row's 128 logits.
__device__ __forceinline__ void keep_tile(const PairMaps& maps, int n0, int row0, int lane,
                                          int n_rows, const float (&x)[kHalfN], Stage& out) {
#pragma unroll
    for (int g = 0; g < kHalfN / 32; ++g) {
        unsigned char* box = out.acquire();
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *chunk_at(box, lane, v) = make_uint4(
                __float_as_uint(x[32 * g + 4 * v]), __float_as_uint(x[32 * g + 4 * v + 1]),
                __float_as_uint(x[32 * g + 4 * v + 2]), __float_as_uint(x[32 * g + 4 * v + 3]));
        out.store(&maps.o, n0 + 32 * g, row0, row0 < n_rows);
    }
}

// sum 2^{(x - z) c} of N logits.  The difference is taken first, as it is exact near
// the maximum z: a product z c rounded by itself is off by half an ulp of z c, which
// the table's z would not know of.
template <int N> __device__ __forceinline__ float masses(const float (&x)[N], float z, float c) {
    const uint64_t z2 = f2(z, z), c2 = f2(c, c);
    uint64_t t[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
    for (int i = 0; i < N; i += 2)
        t[i >> 1 & 1] = f2add(t[i >> 1 & 1], f2_mass(f2(x[i], x[i + 1]), z2, c2));
    float lo, hi;
    f2split(f2add(t[0], t[1]), lo, hi);
    return lo + hi;
}

__device__ __forceinline__ void stats_tile(const PairArgs& a, int n0, int row0, int lane,
                                           int n_rows, float (&x)[kHalfN], const RowList& list,
                                           Stage& out) {
    const int row = row0 + lane;
    const bool on = row < n_rows;
    const int lim = a.cols - n0;
    // the target logits among these columns, each read back by its own row's
    // thread from shared memory (a register array cannot be indexed)
    const int lo = a.v0 + n0, hi = lo + min(kHalfN, lim);
    int k = list.k, id = min(list.next, hi);
#pragma unroll
    for (int g = 0; g < kHalfN / 32; ++g) {
        const int end = min(lo + 32 * (g + 1), hi);
        if (!__any_sync(0xffffffffu, id < end)) continue;
        unsigned char* box = out.acquire();
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *chunk_at(box, lane, v) = make_uint4(
                __float_as_uint(x[32 * g + 4 * v]), __float_as_uint(x[32 * g + 4 * v + 1]),
                __float_as_uint(x[32 * g + 4 * v + 2]), __float_as_uint(x[32 * g + 4 * v + 3]));
        while (id < end) {
            const int col = id - lo - 32 * g;
            a.xk[(size_t)row * a.K + k] =
                reinterpret_cast<const float*>(chunk_at(box, lane, col >> 2))[col & 3];
            ++k;
            id = k < list.n ? __ldg(list.id + k) : hi;
        }
    }
    if (lim < kHalfN) {
#pragma unroll
        for (int i = 0; i < kHalfN; ++i)
            if (i >= lim) x[i] = -INFINITY;
    }
    float m0 = x[0], m1 = x[1];
#pragma unroll
    for (int i = 2; i < kHalfN; i += 2) m0 = fmaxf(m0, x[i]), m1 = fmaxf(m1, x[i + 1]);
    const float m = fmaxf(m0, m1);
    const float s = masses(x, m > -INFINITY ? m : 0.f, a.c);  // (a NaN still reaches the sum)
    if (on) a.tab[(int64_t)(n0 / kHalfN) * a.rpad + row] = make_float2(m, s);
}

// The same straight from the accumulator, 32 columns at a time with a running
// maximum; it is handed back once read.
template <typename Release>
__device__ __forceinline__ void stats1_tile(const PairArgs& a, int n0, int row0, int lane,
                                            int n_rows, uint32_t taddr, const RowList& list,
                                            Stage& out, Release release) {
    const int row = row0 + lane;
    const int lim = a.cols - n0;
    const int lo = a.v0 + n0, hi = lo + min(kHalfN, lim);
    int k = list.k, id = min(list.next, hi);
    float m = -INFINITY, s = 0.f;
#pragma unroll 1
    for (int g = 0; g < kHalfN / 32; ++g) {
        float f[32];
        read32(taddr + 32u * g, nullptr, lim - 32 * g, f);
        if (g == kHalfN / 32 - 1) release();
        const int end = min(lo + 32 * (g + 1), hi);
        if (__any_sync(0xffffffffu, id < end)) {
            unsigned char* box = out.buf;
#pragma unroll
            for (int v = 0; v < 8; ++v)
                *chunk_at(box, lane, v) = make_uint4(
                    __float_as_uint(f[4 * v]), __float_as_uint(f[4 * v + 1]),
                    __float_as_uint(f[4 * v + 2]), __float_as_uint(f[4 * v + 3]));
            while (id < end) {
                const int col = id - lo - 32 * g;
                a.xk[(size_t)row * a.K + k] =
                    reinterpret_cast<const float*>(chunk_at(box, lane, col >> 2))[col & 3];
                ++k;
                id = k < list.n ? __ldg(list.id + k) : hi;
            }
        }
        float m0 = f[0], m1 = f[1];
#pragma unroll
        for (int i = 2; i < 32; i += 2) m0 = fmaxf(m0, f[i]), m1 = fmaxf(m1, f[i + 1]);
        const float nm = fmaxf(fmaxf(m0, m1), m);
        const float z = nm > -INFINITY ? nm : 0.f;  // (a NaN still reaches the sum)
        s = s * ex2((m - z) * a.c) + masses(f, z, a.c);
        m = nm;
    }
    if (row < n_rows) a.tab[(int64_t)(n0 / kHalfN) * a.rpad + row] = make_float2(m, s);
}

// The row's G = cs 2^{(x - z) c} - cf p, with z the row's largest logit and cs = cf / S
// (by difference here too: 2^{x c - lse} would round the log-partition).
__device__ __forceinline__ void grad_tile(const PairArgs& a, const PairMaps& maps, int n0,
                                          int row0, int lane, int n_rows, uint32_t taddr,
                                          const float* carry, const RowList& list, float cf,
                                          float cs, float z, Stage& out) {
    const int row = row0 + lane;
    const bool on = row < n_rows;
    const uint64_t z2 = f2(z, z), c2 = f2(a.c, a.c), cs2 = f2(cs, cs);
    const int lo = a.v0 + n0;
    int k = list.k;
    // rows up to the next K block of d_weight are written (zero past the last)
    const bool inside = row0 < (n_rows + BK - 1) / BK * BK;
#pragma unroll 1
    for (int g = 0; g < kHalfN / 64; ++g) {
        unsigned char* box = out.acquire();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[32];
            read32(taddr + 64u * g + 32u * h, carried(carry, 2 * g + h),
                   a.cols - n0 - 64 * g - 32 * h, f);
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float e0, e1;
                f2split(f2mul(f2_mass(f2(f[2 * i], f[2 * i + 1]), z2, c2), cs2), e0, e1);
                w[i] = on ? tc::pack_bf16(__float_as_uint(e0), __float_as_uint(e1)) : 0u;
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
            float p = __ldg(list.p + k++);
            while (k < list.n && __ldg(list.id + k) == base + col) p += __ldg(list.p + k++);
            reinterpret_cast<bf16*>(chunk_at(box, lane, col >> 3))[col & 7] =
                __float2bfloat16_rn(fmaf(cs, ex2((x - z) * a.c), -(cf * p)));
        }
        out.store(&maps.o, n0 + 64 * g, row0, inside);
    }
}

// d_hidden in one part and the last piece: the earlier pieces' sums are added
// here, rounded once and stored in the caller's row.
__device__ __forceinline__ void dh_last_tile(const PairArgs& a, bool none, int n0, int row,
                                             int n_rows, uint32_t taddr, const float* carry) {
    const bool on = row < n_rows;
    const float s = none ? 0.f : __ldg(a.kappa);
    const float* part = a.dh + (size_t)row * a.H;
    bf16* o = a.d_hidden + (size_t)(on ? __ldg(a.tg.rowmap + row) : 0) * a.H;
#pragma unroll 1
    for (int g = 0; g < kHalfN / 32; ++g) {
        uint32_t u[32];
        sum32(taddr + 32u * g, carried(carry, g), u);
        const int x = n0 + 32 * g;
        if (!on) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            if (x + 8 * v >= a.H) break;
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = none ? 0.f : __uint_as_float(u[8 * v + i]);
            if (!a.first) {
                const float4* q = reinterpret_cast<const float4*>(part + x + 8 * v);
                const float4 y = ld_cg(q), z = ld_cg(q + 1);
                f[0] += y.x; f[1] += y.y; f[2] += y.z; f[3] += y.w;
                f[4] += z.x; f[5] += z.y; f[6] += z.z; f[7] += z.w;
            }
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = tc::pack_bf16(__float_as_uint(s * f[2 * i]),
                                     __float_as_uint(s * f[2 * i + 1]));
            *reinterpret_cast<uint4*>(o + x + 8 * v) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

__device__ __forceinline__ void dh_tile(const PairArgs& a, const PairMaps& maps, const Job& j,
                                        int n0, int row0, int lane, int n_rows, uint32_t taddr,
                                        const float* carry, Stage& out) {
    const bool none = j.kb0 == j.kb1;
    if (a.last && a.split == 1) {
        dh_last_tile(a, none, n0, row0 + lane, n_rows, taddr, carry);
        return;
    }
    if (none && !a.first) return;  // nothing to add
#pragma unroll 1
    for (int g = 0; g < kHalfN / 32; ++g) {
        unsigned char* box = out.acquire();
        uint32_t u[32];
        sum32(taddr + 32u * g, carried(carry, g), u);
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *chunk_at(box, lane, v) =
                none ? make_uint4(0u, 0u, 0u, 0u)
                     : make_uint4(u[4 * v], u[4 * v + 1], u[4 * v + 2], u[4 * v + 3]);
        const int x = n0 + 32 * g;
        out.store(&maps.dh, x, (int)(j.part * a.rpad) + row0, x < a.H && row0 < n_rows, !a.first);
    }
}

// The turned tiles: this thread's row of the tile is column `col` of the output,
// u the accumulators of rows i0 .. i0 + 31.
__device__ __forceinline__ void few_keep_tile(const PairArgs& a, int col, int i0, int n_rows,
                                              const float* u) {
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (i0 + c < n_rows) a.X[(size_t)(i0 + c) * a.ldx + col] = u[c];
}
__device__ __forceinline__ void few_dh_tile(const PairArgs& a, const Job& j, int col, int i0,
                                            int n_rows, uint32_t taddr, const float* carry) {
    uint32_t u[32];
    sum32(taddr, carry, u);
    if (col >= a.H) return;
    if (a.split == 1) {
        const float s = __ldg(a.kappa);
#pragma unroll
        for (int c = 0; c < 32; ++c)
            if (i0 + c < n_rows)
                a.d_hidden[(size_t)__ldg(a.tg.rowmap + i0 + c) * a.H + col] =
                    __float2bfloat16_rn(s * __uint_as_float(u[c]));
        return;
    }
    float* o = a.dh + ((size_t)j.part * a.rpad + i0) * a.H + col;
    const bool none = j.kb0 == j.kb1;
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (i0 + c < n_rows) o[(size_t)c * a.H] = none ? 0.f : __uint_as_float(u[c]);
}

// The accumulator is read and handed back first, so that the next product runs
// while this one is stored: an SM's stores leave at 32 bytes a cycle at most.
template <typename Release>
__device__ __forceinline__ void dw_tile(const PairArgs& a, const Job& j, int n0, int row0,
                                        int lane, uint32_t taddr, const float* carry,
                                        unsigned char* box, Release release) {
    const bool none = j.kb0 == j.kb1;
    const float s = none ? 0.f : __ldg(a.kappa);
    uint32_t w[kHalfN / 2];
#pragma unroll
    for (int g = 0; g < kHalfN / 32; ++g) {
        uint32_t u[32];
        sum32(taddr + 32u * g, carried(carry, g), u);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            w[16 * g + i] = none ? 0u
                                 : tc::pack_bf16(__float_as_uint(s * __uint_as_float(u[2 * i])),
                                                 __float_as_uint(s * __uint_as_float(u[2 * i + 1])));
    }
    release();
#pragma unroll
    for (int g = 0; g < kHalfN / 64; ++g) {
        __syncwarp();  // the box has been read
#pragma unroll
        for (int v = 0; v < 8; ++v)
            *chunk_at(box, lane, v) = make_uint4(w[32 * g + 4 * v], w[32 * g + 4 * v + 1],
                                                 w[32 * g + 4 * v + 2], w[32 * g + 4 * v + 3]);
        __syncwarp();
        const int x = n0 + 64 * g + 8 * (lane & 7);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int rr = 4 * i + (lane >> 3), y = a.v0 + row0 + rr;
            const uint4 v = *chunk_at(box, rr, lane & 7);
            if (x < a.H && y < a.V)
                *reinterpret_cast<uint4*>(a.d_weight + (size_t)y * a.H + x) = v;
        }
    }
}

// The weighted mean of the rows' losses, in row order, by one warp.
__device__ __forceinline__ void mean_loss(const PairArgs& a, int n_rows, int lane) {
    double sum = 0.0;
    for (int b = lane; b < n_rows; b += 32 * 8) {
        float w[8], l[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int r = b + 32 * u < n_rows ? __ldg(a.tg.rowmap + b + 32 * u) : -1;
            w[u] = r >= 0 ? __ldg(a.tg.w + r) : 0.f;
            l[u] = r >= 0 ? ld_cg(a.row_loss + r) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (w[u] != 0.f) sum += (double)w[u] * (double)l[u];
    }
    sum = warp_sum(sum);
    if (lane == 0) *a.loss = (float)(sum / *a.tg.wsum);
}

// The first warpgroup's share of the register split, in each of its roles.
template <bool kSplit> __device__ __forceinline__ void give_registers() {
    if (kSplit) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kRegsFew));
}

template <int MODE, int NF, bool CUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairCfg<MODE, NF>::kThreads, 1)
    k_pair(const __grid_constant__ PairMaps maps, const PairArgs a) {
    using Cfg = PairCfg<MODE, NF>;
    constexpr bool kFew = Cfg::kFew;
    constexpr int kPairStages = Cfg::kStages, kStageBytes = Cfg::kStageBytes;
    extern __shared__ unsigned char dsm_raw[];
    unsigned char* dsm = dsm_raw + ((1024u - (smem_u32(dsm_raw) & 1023u)) & 1023u);
    unsigned char* outs = dsm + kPairStages * kStageBytes;
    PairBars* sb = reinterpret_cast<PairBars*>(outs + Cfg::kSets * kTileWarps * kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)tc::cluster_rank();
    int* status = a.tg.status;
    dep_launch();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(&sb->full[s], 1);
            mbar_init(&sb->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sb->acc_full[b], 1);
            mbar_init(&sb->acc_empty[b], 2 * kTileWarps);
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
    dep_wait();
    const int n_rows = *(const volatile int*)a.tg.nrows;
    const bool all = n_rows == a.R;  // hidden as it is
    // sums cut for the epilogue's registers
    constexpr bool kParts = MODE == kStats || MODE == kKeep;
    constexpr bool kSplitRegs = kParts && !kFew;
    Jobs<MODE, kFew> jobs(a, n_rows);
    Job j;
    if (warp == 0) {
        give_registers<kSplitRegs>();
        // ------------------------------------------------------ TMA producer
        if (lane == 0) {
            // what earlier kernels stored is read through the async proxy
            asm volatile("fence.proxy.async;" ::: "memory");
            const CUtensorMap* ma = all ? &maps.a0 : &maps.a;
            const CUtensorMap* mh = all ? &maps.ht0 : &maps.ht;
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
                    if (rank == 0) {
                        const bool turned = kFew && (MODE == kKeep || j.kind == 1);
                        mbar_expect_tx(&sb->full[s],
                                       2 * (kHalfBytes + (turned ? Cfg::kFewB : kHalfBytes)));
                    }
                    if (MODE == kKeep && kFew) {
                        tc::load_2d(A, &maps.b, kb * BK, j.m0 + 128 * rank, bar);
                        tc::load_2d(B, ma, kb * BK, NF / 2 * rank, bar);
                    } else if (MODE != kProd) {
                        tc::load_2d(A, ma, kb * BK, j.m0 + 128 * rank, bar);
                        tc::load_2d(B, &maps.b, kb * BK, a.v0 + j.n0 + 128 * rank, bar);
                    } else {
                        const int n = j.n0 + 128 * rank;
                        if (kFew && j.kind == 1) {
                            const int m = j.m0 + 128 * rank;
                            tc::load_2d(A, &maps.wt, m, a.v0 + kb * BK, bar);
                            tc::load_2d(A + kBoxBytes, &maps.wt, m + 64, a.v0 + kb * BK, bar);
                            tc::load_2d(B, &maps.gk, kb * BK, NF / 2 * rank, bar);
                        } else if (j.kind == 1) {
                            tc::load_2d(A, &maps.gk, kb * BK, j.m0 + 128 * rank, bar);
                            tc::load_2d(B, &maps.wt, n, a.v0 + kb * BK, bar);
                            tc::load_2d(B + kBoxBytes, &maps.wt, n + 64, a.v0 + kb * BK, bar);
                        } else {
                            const int m = j.m0 + 128 * rank;
                            tc::load_2d(A, &maps.gt, m, kb * BK, bar);
                            tc::load_2d(A + kBoxBytes, &maps.gt, m + 64, kb * BK, bar);
                            tc::load_2d(B, mh, n, kb * BK, bar);
                            tc::load_2d(B + kBoxBytes, mh, n + 64, kb * BK, bar);
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
        give_registers<kSplitRegs>();
        // ------------------------------------------------------ MMA issuer
        if (lane == 0 && rank == 0) {
            const uint32_t ring = smem_u32(dsm);
            uint32_t it = 0;
            int lt = 0;
            bool ok = true;
            while (ok && !*(volatile int*)&sb->err && jobs.next(j)) {
                const bool turned = kFew && (MODE == kKeep || j.kind == 1);
                const bool amn = MODE == kProd && (kFew || j.kind == 2);
                const bool bmn = MODE == kProd && !turned;
                const uint32_t idesc = (turned ? tc::idesc_bf16(256, NF) : tc::idesc_bf16(256, BT)) |
                                       (amn ? 1u << 15 : 0u) | (bmn ? 1u << 16 : 0u);
                // descriptors of stage 0; a stage and a K step add to the address
                // field (16-byte units), which never carries out of it
                const uint64_t a0 = amn ? tc::desc_mn(ring, kBoxBytes) : tc::sdesc_sw128(ring);
                const uint64_t b0 = bmn ? tc::desc_mn(ring + kHalfBytes, kBoxBytes)
                                        : tc::sdesc_sw128(ring + kHalfBytes);
                const uint32_t ka = amn ? 2048u >> 4 : 32u >> 4;
                const uint32_t kbs = bmn ? 2048u >> 4 : 32u >> 4;
                const uint32_t alo = (uint32_t)a0, ahi = (uint32_t)(a0 >> 32);
                const uint32_t blo = (uint32_t)b0, bhi = (uint32_t)(b0 >> 32);
                const int kb1 = MODE == kProd ? j.kb1 : a.nkh;
                int kb = j.kb0;
                do {  // (a job without K blocks hands on its accumulator unread)
                    const int end = kParts || CUT ? min(kb1, kb + a.part) : kb1;
                    const int buf = lt & 1;
                    const uint32_t use = (uint32_t)lt >> 1;
                    if (use > 0 && !wait_pair(&sb->acc_empty[buf], (use - 1) & 1u, sb, status)) {
                        ok = false;
                        break;
                    }
                    tc::tc_fence_after();
                    const uint32_t d = tmem + (uint32_t)(buf * BT);
                    uint32_t more = 0;
                    for (; kb < end; ++kb) {
                        const int s = (int)(it % kPairStages);
                        if (!wait_pair(&sb->full[s], (it / kPairStages) & 1u, sb, status)) {
                            ok = false;
                            break;
                        }
                        tc::tc_fence_after();
                        const uint32_t at = (uint32_t)s * (kStageBytes >> 4);
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k) {
                            tc::mma_pair(d, (uint64_t)ahi << 32 | (alo + at + ka * k),
                                         (uint64_t)bhi << 32 | (blo + at + kbs * k), idesc, more);
                            more = 1;
                        }
                        tc::commit_pair(&sb->empty[s]);
                        ++it;
                    }
                    if (!ok) break;
                    tc::commit_pair(&sb->acc_full[buf]);
                    ++lt;
                } while (kb < kb1);
            }
            tc::commit_pair(&sb->drain);  // every MMA issued is done once it arrives
            drain_pair(&sb->drain, 0);
        }
    } else if (warp < 4) {
        give_registers<kSplitRegs>();
        if (MODE == kProd && a.loss && blockIdx.x == 0 && warp == 2) mean_loss(a, n_rows, lane);
    } else {
        // ------------------------------------------------------ epilogue
        if (kSplitRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kRegsMany));
        const int q = warp & 3;               // TMEM lanes 32q .. 32q + 31
        const int h0 = ((warp - 4) >> 2 & 1) * kHalfN;  // its columns of the tile
        const int set = (warp - 4) / kTileWarps;  // its accumulator, where there are two sets
        Stage out{outs + (warp - 4) * kOutBytes, lane};
        const uint32_t empty = tc::leader_addr(&sb->acc_empty[0]);
        int lt = 0;
        auto ready = [&]() {
            const bool ok = __all_sync(0xffffffffu, wait_pair(&sb->acc_full[lt & 1],
                                                              ((uint32_t)lt >> 1) & 1u, sb, status));
            tc::tc_fence_after();
            return ok;
        };
        auto release = [&]() {
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::arrive_remote(empty + 8u * (lt & 1));
            ++lt;
        };
        auto acc_addr = [&](int col) {
            return tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)((lt & 1) * BT + col);
        };
        const int f0 = ((warp - 4) >> 2 & 1) * (NF / 2);  // its rows of a turned tile
        while (jobs.next(j)) {
            if (Cfg::kSets == 2 && CUT) {  // (one set takes all parts: its phases in a row)
                if (set) break;
            } else if (Cfg::kSets == 2 && (lt & 1) != set) {
                ++lt;
                continue;
            }
            const int row0 = j.m0 + 128 * rank + 32 * q, n0 = j.n0 + h0;
            const float* carry = nullptr;
            if constexpr (CUT) {  // all parts but a sum's last
                const bool turned = kFew && j.kind == 1;
                const int len = MODE == kGrad ? a.nkh : j.kb1 - j.kb0;
                float* mine = a.carry + (int64_t)(blockIdx.x * kTileWarps + warp - 4) *
                                            (kHalfN * 32) + lane;
                bool ok = true;
                for (int kb = a.part; kb < len; kb += a.part) {
                    if (!(ok = ready())) break;
#pragma unroll 1
                    for (int g = 0; g < (turned ? NF / 64 : kHalfN / 32); ++g) {
                        uint32_t u[32];
                        sum32(acc_addr((turned ? f0 : h0) + 32 * g), carried(carry, g), u);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            mine[g * kCarryStep + 32 * i] = __uint_as_float(u[i]);
                    }
                    carry = mine;
                    release();
                }
                if (!ok) break;
            }
            if (MODE == kKeep && kFew) {
                float x[kFew ? NF / 2 : 1];
                bool ok = true;
                for (int kb = 0; ok && kb < a.nkh; kb += a.part) {
                    if (!(ok = ready())) break;
#pragma unroll
                    for (int g = 0; g < NF / 64; ++g) {
                        uint32_t u[32];
                        tc::tmem_ld32(acc_addr(f0 + 32 * g), u);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            x[32 * g + i] = kb ? x[32 * g + i] + __uint_as_float(u[i])
                                               : __uint_as_float(u[i]);
                    }
                    release();
                }
                if (!ok) break;
#pragma unroll
                for (int g = 0; g < NF / 64; ++g)
                    few_keep_tile(a, row0 + lane, f0 + 32 * g, n_rows, x + 32 * g);
            } else if (kParts) {
                const RowList list(a, row0 + lane, MODE == kStats && row0 + lane < n_rows,
                                   a.v0 + n0);
                float x[kHalfN];
                bool ok = true;
                for (int kb = 0; ok && kb < a.nkh; kb += a.part) {
                    if (!(ok = ready())) break;
                    const uint32_t t = acc_addr(h0);
#pragma unroll
                    for (int g = 0; g < kHalfN / 32; ++g) {
                        uint32_t u[32];
                        tc::tmem_ld32(t + 32u * g, u);
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            x[32 * g + i] = kb ? x[32 * g + i] + __uint_as_float(u[i])
                                               : __uint_as_float(u[i]);
                    }
                    release();
                }
                if (!ok) break;
                if (MODE == kKeep) keep_tile(maps, n0, row0, lane, n_rows, x, out);
                else stats_tile(a, n0, row0, lane, n_rows, x, list, out);
            } else if (MODE == kStats1) {
                const RowList list(a, row0 + lane, row0 + lane < n_rows, a.v0 + n0);
                if (!ready()) break;
                stats1_tile(a, n0, row0, lane, n_rows, acc_addr(h0), list, out, release);
            } else if (MODE == kGrad) {
                const int row = row0 + lane;
                const bool on = row < n_rows;
                const RowList list(a, row, on, a.v0 + n0);
                const float cf = on ? __ldg(a.coef + row) : 0.f;
                const float cs = on ? __ldg(a.coefs + row) : 0.f, z = on ? __ldg(a.top + row) : 0.f;
                if (!ready()) break;
                grad_tile(a, maps, n0, row0, lane, n_rows, acc_addr(h0), carry, list, cf, cs, z,
                          out);
                release();
            } else {
                if (!ready()) break;
                const uint32_t t = acc_addr(h0);
                if (kFew && j.kind == 1) {
#pragma unroll
                    for (int g = 0; g < NF / 64; ++g)
                        few_dh_tile(a, j, row0 + lane, f0 + 32 * g, n_rows, acc_addr(f0 + 32 * g),
                                    carried(carry, g));
                } else if (n0 >= a.H) {
                    // no column of the output
                } else if (j.kind == 1) {
                    dh_tile(a, maps, j, n0, row0, lane, n_rows, t, carry, out);
                } else {
                    // (a TMA store may still read the box)
                    if (!kFew && a.want_dh) out.acquire();
                    dw_tile(a, j, n0, row0, lane, t, carry, out.buf, release);
                    continue;
                }
                release();
            }
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

// kRowsOf counted rows per block, 256 / kRowsOf threads each: log-partition,
// loss and gradient coefficient.  A thread takes every (256 / kRowsOf)-th part
// and list entry of its row (consecutive threads: consecutive rows, so a read
// fills its 32-byte sectors).  Latency bounds it: 9 us at 4096 rows x 250 parts, about
// half of what 32 rows to a block take.  With `loss` the blocks' weighted losses are added
// in block order by the last block to finish.
constexpr int kRowsOf = 8;
__global__ void __launch_bounds__(256)
    k_rows(const float2* tab, int ntab, int64_t stride, Targets tg, int K, float c, double invT,
           const float* xk, float* top, float* coef, float* coefs, float* row_loss, float* logz,
           double* part, float* loss) {
    constexpr int RB = kRowsOf;
    constexpr int P = 256 / RB;
    __shared__ float2 ms[8][RB];
    __shared__ double dots[8][RB], wl[8];
    __shared__ int last;
    dep_launch();
    dep_wait();
    const int n_rows = *(const volatile int*)tg.nrows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int q = threadIdx.x % RB, pt = threadIdx.x / RB;
    const int i = blockIdx.x * RB + q;
    const bool on = i < n_rows;
    const double wsum = *tg.wsum;
    const float wm = *tg.wmax;
    if (blockIdx.x * RB < n_rows) {
        float m = -INFINITY, s = 0.f;
        double dot = 0.0;
        const int r = on ? tg.rowmap[i] : 0;
        auto join = [&](const float2* e, int n) {
            float nm = m;
            for (int u = 0; u < n; ++u) nm = fmaxf(nm, e[u].x);
            const float z = nm > -INFINITY ? nm : 0.f;
            s *= ex2((m - z) * c);
            for (int u = 0; u < n; ++u) s += e[u].y * ex2((e[u].x - z) * c);
            m = nm;
        };
        const int n = on ? tg.n[r] : 0;
        const float plogp = on ? tg.plogp[r] : 0.f, w = on ? tg.w[r] : 0.f;
        if (on)
            for (int t = pt; t < ntab; t += 8 * P) {  // (eight parts' loads at a time)
                float2 e[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    e[u] = t + u * P < ntab ? ld_cg(tab + (t + u * P) * stride + i)
                                            : make_float2(-INFINITY, 0.f);
                join(e, 8);
            }
        // sum p x as ref + sum p (x - ref) with the first entry's logit ref: the
        // probabilities add up to 1 only to a float's rounding, which x would multiply
        const float x0 = on ? xk[(size_t)i * K] : 0.f;
        const double ref = x0 > -INFINITY ? (double)x0 : 0.0;
        for (int k = pt; k < n; k += P)
            dot += (double)tg.p[(size_t)r * K + k] * ((double)xk[(size_t)i * K + k] - ref);
#pragma unroll
        for (int o = RB; o < 32; o <<= 1) {
            const float2 e = make_float2(__shfl_xor_sync(0xffffffffu, m, o),
                                         __shfl_xor_sync(0xffffffffu, s, o));
            join(&e, 1);
            dot += __shfl_xor_sync(0xffffffffu, dot, o);
        }
        if (lane < RB) ms[warp][q] = make_float2(m, s), dots[warp][q] = dot;
        __syncthreads();
        if (warp == 0) {
            double wloss = 0.0;
            if (lane < RB && on) {
                float2 e[7];
#pragma unroll
                for (int u = 1; u < 8; ++u) e[u - 1] = ms[u][q], dot += dots[u][q];
                join(e, 7);
                const double l = (double)logf(s), lz = (double)m * invT + l;
                if (!isfinite(lz)) atomicOr(tg.status, VSD_STATUS_BAD_ROW);
                const float rl =
                    (float)((double)plogp + l + (((double)m - ref) - dot) * invT);
                logz[r] = (float)lz;
                row_loss[r] = rl;
                const float cf = wm > 0.f ? kTopMantissa * (w / wm) : 0.f;
                top[i] = m;
                coef[i] = cf;
                coefs[i] = cf / s;
                if (w != 0.f) wloss = (double)w * (double)rl;
            }
            wloss = warp_sum(wloss);
            if (lane == 0) part[blockIdx.x] = wloss;
        }
    }
    if (!loss) return;
    if (threadIdx.x == 0) {
        __threadfence();
        last = gridDim.x == 1 || atomicAdd(tg.done + 1, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int nb = (n_rows + RB - 1) / RB;
    double sum = 0.0;
    for (int b = threadIdx.x; b < nb; b += 256) sum += ld_cg(part + b);
    sum = warp_sum(sum);
    if (lane == 0) wl[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int u = 0; u < 8; ++u) sum += wl[u];
        *loss = (float)(sum / wsum);
    }
}

// d_hidden of several parts, in the caller's rows: the parts added in a fixed
// order, one rounding (rows not counted are zero already).  A block takes 256
// columns of a row; warp q every eighth part from q on.
__global__ void __launch_bounds__(256)
    k_dh_out(const float* dh, int split, int64_t rpad, int H, Targets tg, const float* kappa,
             bf16* out) {
    __shared__ float4 sum[8][2][32];
    dep_launch();
    dep_wait();
    const int r = blockIdx.x, i = tg.rowinv[r];
    const float s = *kappa;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int h = blockIdx.y * 256 + lane * 8;
    if (i < 0) return;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
    auto add = [](float4& a, const float4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; };
    if (h < H) {
#pragma unroll 4
        for (int q = warp; q < split; q += 8) {
            const float4* p = reinterpret_cast<const float4*>(dh + ((size_t)q * rpad + i) * H + h);
            add(x, p[0]);
            add(y, p[1]);
        }
    }
    sum[warp][0][lane] = x;
    sum[warp][1][lane] = y;
    __syncthreads();
    if (warp || h >= H) return;
    for (int q = 1; q < 8; ++q) add(x, sum[q][0][lane]), add(y, sum[q][1][lane]);
    const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w[e] = tc::pack_bf16(__float_as_uint(s * f[2 * e]), __float_as_uint(s * f[2 * e + 1]));
    *reinterpret_cast<uint4*>(out + (size_t)r * H + h) = make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace

bool lmloss_shape_ok(const LmLossShape& s) {
    return s.R >= 1 && s.R <= (1 << 24) && s.V >= 1 && s.V <= (1 << 20) && s.H >= 8 &&
           s.H <= (1 << 20) && s.H % 8 == 0 && s.K >= 1 && s.K <= kMaxTeacher && s.piece >= 0;
}

size_t lmloss_workspace_bytes(const LmLossShape& s) {
    return lmloss_shape_ok(s) ? lm_ws(s).total : 0;
}

template <int MODE, int NF = 0, bool CUT = false>
static cudaError_t launch_pair(const PairMaps& maps, const PairArgs& a, int64_t jobs,
                               cudaStream_t st) {
    constexpr size_t smem = PairCfg<MODE, NF>::kSmem;
    cudaError_t e = ensure_dyn_smem((const void*)k_pair<MODE, NF, CUT>, smem);
    if (e != cudaSuccess) return e;
    const int64_t most = std::min<int64_t>(kPairs, device_sm_count() / 2);
    const int64_t pairs = std::max<int64_t>(1, std::min(jobs, most));
    return launch_dep(true, k_pair<MODE, NF, CUT>, dim3((unsigned)(2 * pairs)),
                      PairCfg<MODE, NF>::kThreads, smem, 1, st, maps, a);
}

cudaError_t lmloss(const LmLossShape& s, const void* hidden, const void* weight,
                   const TargetIn& in, float T, float grad_scale, const vsd_loss_outputs& out,
                   void* ws, cudaStream_t st) {
    const LmWs w = lm_ws(s);
    const int R = s.R, V = s.V, H = s.H, K = s.K;
    const bool grads = s.dh || s.dw;
    Targets tg{ws_at<int32_t>(ws, w.n), ws_at<int32_t>(ws, w.id), ws_at<float>(ws, w.p),
               ws_at<float>(ws, w.plogp), ws_at<float>(ws, w.w), nullptr,
               ws_at<int32_t>(ws, w.rowmap), ws_at<int32_t>(ws, w.rowinv),
               ws_at<int32_t>(ws, w.nrows), ws_at<double>(ws, w.wsum), ws_at<float>(ws, w.wmax),
               ws_at<float>(ws, w.kappa), ws_at<float>(ws, w.unit), ws_at<float>(ws, w.share),
               ws_at<int32_t>(ws, w.done), ws_at<int32_t>(ws, w.status)};
    bf16* hid = ws_at<bf16>(ws, w.hid);
    float* X = ws_at<float>(ws, w.X);
    bf16* G = ws_at<bf16>(ws, w.G);
    float2* tab = ws_at<float2>(ws, w.tab);
    float *xk = ws_at<float>(ws, w.xk), *top = ws_at<float>(ws, w.top),
          *coef = ws_at<float>(ws, w.coef), *coefs = ws_at<float>(ws, w.coefs),
          *kappa = ws_at<float>(ws, w.kappa), *dh = ws_at<float>(ws, w.dh);
    const float c = (float)(kLog2e / (double)T);
    const int64_t hrows = w.hrows;
    PairMaps maps;
    memset(&maps, 0, sizeof(maps));
    using vsd_lm::make_map_sw128;
    // few rows: turned products (128256 x 4096: 540 us at 48 rows, 549 not turned;
    // 589 and 600 at 100)
    const int nf = !w.keep ? 0 : R <= 64 ? 64 : R <= 128 ? 128 : 0;
    const int rbox = nf ? nf / 2 : 128;                              // rows of a K-major half tile
    bool ok = make_map_sw128(&maps.a, hid, false, hrows, H, H, rbox) &&
              make_map_sw128(&maps.a0, hidden, false, R, H, H, rbox) &&
              make_map_sw128(&maps.b, weight, false, V, H, H, 128);
    if (grads)
        ok = ok && make_map_sw128(&maps.gk, G, false, hrows, w.piece, w.piece, rbox) &&
             make_map_sw128(&maps.gt, G, false, hrows, w.piece, w.piece, BK) &&
             make_map_sw128(&maps.wt, weight, false, V, H, H, BK) &&
             make_map_sw128(&maps.ht, hid, false, hrows, H, H, BK) &&
             make_map_sw128(&maps.ht0, hidden, false, R, H, H, BK);
    if (w.keep) ok = ok && make_map_sw128(&maps.o, X, true, hrows, w.piece, w.piece, 32);
    else if (grads) ok = ok && make_map_sw128(&maps.o, G, false, hrows, w.piece, w.piece, 32);
    if (s.dh)
        ok = ok && make_map_sw128(&maps.dh, dh, true, (int64_t)w.rpad * w.split, H, H, 32);
    if (!ok) return cudaErrorInvalidValue;

    PairArgs a{};
    a.tg = tg;
    a.R = R;
    a.K = K;
    a.H = H;
    a.V = V;
    a.v0 = 0;
    a.cols = V;
    a.nkh = (H + BK - 1) / BK;
    const int parts = (a.nkh + kSumBlocks - 1) / kSumBlocks;
    a.part = (a.nkh + parts - 1) / parts;  // parts of about the same size
    a.rpad = w.rpad;
    a.c = c;
    a.tab = tab;
    a.xk = xk;
    a.top = top;
    a.coef = coef;
    a.coefs = coefs;
    a.kappa = kappa;
    a.split = w.split;
    a.want_dh = s.dh;
    a.want_dw = s.dw;
    a.dh = dh;
    a.row_loss = out.row_loss;
    a.carry = ws_at<float>(ws, w.carry);
    a.X = X;
    a.ldx = w.piece;
    a.d_hidden = static_cast<bf16*>(out.d_hidden);
    a.d_weight = static_cast<bf16*>(out.d_weight);

    const double scale = (double)grad_scale / ((double)kTopMantissa * (double)T);
    cudaError_t e = launch_targets(in, tg, scale, out.row_loss, out.logz, w.zero_end, st);
    if (e == cudaSuccess)
        e = launch_dep(true, k_gather,
                       dim3((unsigned)std::min<int64_t>(hrows, 4 * device_sm_count())), 256, 0, 1,
                       st, static_cast<const bf16*>(hidden), R, H, tg, hid,
                       static_cast<bf16*>(out.d_hidden));
    if (e != cudaSuccess) return e;
    const int64_t mt = w.rpad / kRowPad, units = (V + kPieceUnit - 1) / kPieceUnit;
    const int64_t ht = (H + BT - 1) / BT;
    e = nf == 64    ? launch_pair<kKeep, 64>(maps, a, units, st)
        : nf == 128 ? launch_pair<kKeep, 128>(maps, a, units, st)
        : w.keep    ? launch_pair<kKeep>(maps, a, mt * units, st)
        : parts == 1 ? launch_pair<kStats1>(maps, a, mt * units, st)
                     : launch_pair<kStats>(maps, a, mt * units, st);
    if (e != cudaSuccess) return e;
    if (w.keep) {  // losses and G from the kept logits, a row at a time
        RowArgs ra{};
        ra.tg = tg;
        ra.rows = (int)hrows;
        ra.V = V;
        ra.K = K;
        ra.ldx = ra.ldg = w.piece;
        ra.gcols = w.piece;
        ra.row_loss = out.row_loss;
        ra.logz = out.logz;
        ra.same_align = true;
        e = launch_row_loss<float, bf16, true>(X, G, ra, T, kTopMantissa, resident_clusters, st);
    } else {
        e = launch_dep(true, k_rows, dim3((unsigned)((R + kRowsOf - 1) / kRowsOf)), 256, 0, 1, st,
                       tab, (int)(2 * units), (int64_t)w.rpad, tg, K, c, 1.0 / (double)T, xk, top,
                       coef, coefs, out.row_loss, out.logz, ws_at<double>(ws, w.part),
                       grads ? nullptr : out.loss);
    }
    if (e != cudaSuccess || !grads) return e;
    for (int q = 0; q < w.npiece; ++q) {
        a.v0 = q * w.piece;
        a.cols = std::min(w.piece, V - a.v0);
        a.first = q == 0;
        a.last = q == w.npiece - 1;
        a.loss = q == 0 ? out.loss : nullptr;
        const int64_t nu = (a.cols + kPieceUnit - 1) / kPieceUnit;
        a.part = kLongLogits;
        if (!w.keep) {
            e = w.cut_grad ? launch_pair<kGrad, 0, true>(maps, a, mt * nu, st)
                           : launch_pair<kGrad>(maps, a, mt * nu, st);
            if (e != cudaSuccess) return e;
        }
        a.part = kLongProd;
        const int64_t jobs = (s.dh ? mt * ht * w.split : 0) + (s.dw ? nu * ht : 0);
        if (w.cut_prod)
            e = nf == 64    ? launch_pair<kProd, 64, true>(maps, a, jobs, st)
                : nf == 128 ? launch_pair<kProd, 128, true>(maps, a, jobs, st)
                            : launch_pair<kProd, 0, true>(maps, a, jobs, st);
        else
            e = nf == 64    ? launch_pair<kProd, 64>(maps, a, jobs, st)
                : nf == 128 ? launch_pair<kProd, 128>(maps, a, jobs, st)
                            : launch_pair<kProd>(maps, a, jobs, st);
        if (e != cudaSuccess) return e;
    }
    if (s.dh && w.split > 1) {
        e = launch_dep(true, k_dh_out, dim3((unsigned)R, (unsigned)((H + 255) / 256)), 256, 0, 1,
                       st, dh, w.split, (int64_t)w.rpad, H, tg, kappa,
                       static_cast<bf16*>(out.d_hidden));
    }
    return e;
}

}  // namespace vsd
