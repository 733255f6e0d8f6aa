// vsd_fp8.cu -- a matrix in e4m3 with a scale for each block of 128 columns, and the
// LM head's logits from two such matrices (include/vsd_decode.h).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "vsd_common.cuh"
#include "vsd_decode.h"
#include "vsd_dep.cuh"
#include "vsd_launch.h"
#include "vsd_pair.cuh"

namespace vsd {
namespace {

constexpr int kBlock = 128;  // columns of a scale

// ------------------------------------------------------------ quantizing
// s = 2^ceil(log2(amax / 448)), q = x / s, an exact product with 2^-log2(s) rounded once.
// Bound by memory: one read, one write of half or a quarter of it.  A block of 128 or of
// 128 x 128 stays in registers between its largest magnitude and its quotients, so x is
// read once: 32000 x 4096 float32 by 128 rows takes 94 us, 7.0 TB/s (478 with a second
// read); 4096 x 4096 bf16 by rows 17, of which the host's call is 15.

// The least power of two s with amax / s <= 448 = 1.75 2^8, and its reciprocal; amax by
// its bits (NaN is above infinity).
__device__ __forceinline__ float scale_of(uint32_t amax, float& inv) {
    if (amax >= 0x7F800000u) return inv = NAN;
    if (amax == 0) return inv = 1.f;
    const int e = max((int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u), -126);
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}
// The largest magnitude of a vector, by its bits.
template <typename T> __device__ __forceinline__ uint32_t vec_amax(const uint4& q);
template <> __device__ __forceinline__ uint32_t vec_amax<float>(const uint4& q) {
    constexpr uint32_t m = 0x7FFFFFFFu;
    return max(max(q.x & m, q.y & m), max(q.z & m, q.w & m));
}
template <> __device__ __forceinline__ uint32_t vec_amax<__nv_bfloat16>(const uint4& q) {
    constexpr uint32_t m = 0x7FFF0000u;
    const uint32_t hi = max(max(q.x & m, q.y & m), max(q.z & m, q.w & m));
    const uint32_t lo = max(max(q.x << 16 & m, q.y << 16 & m), max(q.z << 16 & m, q.w << 16 & m));
    return max(hi, lo);
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
// A vector of x to 4 or 8 bytes of q.
__device__ __forceinline__ void put_vec(__nv_fp8_e4m3* q, const uint4& v, float inv, float) {
    float f[4];
    unpack<float>(v, f);
    *reinterpret_cast<uint32_t*>(q) = e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
}
__device__ __forceinline__ void put_vec(__nv_fp8_e4m3* q, const uint4& v, float inv, __nv_bfloat16) {
    float f[8];
    unpack<__nv_bfloat16>(v, f);
    *reinterpret_cast<uint2*>(q) = make_uint2(e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                                              e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
}

constexpr int kQuantThreads = 256;

// A scale for each row and 128 columns: kGroup lanes hold a block, kMany blocks each.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads)
    k_quantize_rows(const T* x, int64_t R, int H, __nv_fp8_e4m3* q, float* scale) {
    constexpr int PV = Traits<T>::kPerVec, kGroup = kBlock / PV, kMany = 4;
    const int nk = (H + kBlock - 1) / kBlock, lane = threadIdx.x % kGroup;
    const int64_t units = R * nk, groups = (int64_t)gridDim.x * (kQuantThreads / kGroup);
    // (whole warps go round together: w is the unit of a warp's first group)
    const int sub = threadIdx.x % 32 / kGroup;
    const int first = threadIdx.x / kGroup - sub;
    for (int64_t w = (int64_t)blockIdx.x * (kQuantThreads / kGroup) + first; w < units;
         w += groups * kMany) {
        const int64_t u0 = w + sub;
        uint4 v[kMany];
        int64_t at[kMany];
#pragma unroll
        for (int i = 0; i < kMany; ++i) {
            const int64_t u = u0 + i * groups, r = u / nk;
            const int col = (int)(u - r * nk) * kBlock + lane * PV;
            at[i] = u < units && col < H ? r * H + col : -1;
            v[i] = at[i] >= 0 ? *reinterpret_cast<const uint4*>(x + at[i]) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kMany; ++i) {
            uint32_t m = vec_amax<T>(v[i]);
            // (a group is a warp or half of one; all its lanes come here)
#pragma unroll
            for (int o = kGroup / 2; o; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
            float inv;
            const float s = scale_of(m, inv);
            const int64_t u = u0 + i * groups;
            if (at[i] >= 0) put_vec(q + at[i], v[i], inv, T());
            if (lane == 0 && u < units) scale[u] = s;
        }
    }
}

// A scale for 128 x 128: a block of threads holds it in registers.
template <typename T>
__global__ void __launch_bounds__(kQuantThreads, 3)
    k_quantize_blocks(const T* x, int64_t R, int H, __nv_fp8_e4m3* q, float* scale) {
    constexpr int PV = Traits<T>::kPerVec, kGroup = kBlock / PV;        // lanes of a row
    constexpr int kStep = kQuantThreads / kGroup, kMany = kBlock / kStep;  // rows at a time
    __shared__ uint32_t part[kQuantThreads / 32];
    const int64_t r0 = (int64_t)blockIdx.y * kBlock + threadIdx.x / kGroup;
    const int col = blockIdx.x * kBlock + threadIdx.x % kGroup * PV;
    uint4 v[kMany];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kMany; ++i) {
        const int64_t r = r0 + i * kStep;
        v[i] = r < R && col < H ? *reinterpret_cast<const uint4*>(x + r * H + col)
                                : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kMany; ++i) m = max(m, vec_amax<T>(v[i]));
    m = __reduce_max_sync(0xffffffffu, m);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 32; ++i) m = max(m, part[i]);
    float inv;
    const float s = scale_of(m, inv);
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
#pragma unroll
    for (int i = 0; i < kMany; ++i) {
        const int64_t r = r0 + i * kStep;
        if (r < R && col < H) put_vec(q + r * H + col, v[i], inv, T());
    }
}

template <typename T>
cudaError_t quantize(const T* x, int R, int H, int block_rows, __nv_fp8_e4m3* q, float* scale,
                     cudaStream_t st) {
    const int nk = (H + kBlock - 1) / kBlock;
    if (block_rows == 1) {
        constexpr int kPer = 4 * kQuantThreads * Traits<T>::kPerVec / kBlock;  // a block's at a time
        const int64_t blocks = ((int64_t)R * nk + kPer - 1) / kPer;
        const int most = 16 * device_sm_count();
        k_quantize_rows<T><<<(int)std::min<int64_t>(blocks, most), kQuantThreads, 0, st>>>(
            x, R, H, q, scale);
        return cudaGetLastError();
    }
    // (a grid's second dimension ends at 65535)
    constexpr int kMost = 65535;
    for (int64_t b = 0; b * kBlock < R; b += kMost) {
        const int64_t rows = std::min<int64_t>(R - b * kBlock, (int64_t)kMost * kBlock);
        k_quantize_blocks<T><<<dim3(nk, (int)((rows + kBlock - 1) / kBlock)), kQuantThreads, 0, st>>>(
            x + b * kBlock * H, rows, H, q + b * kBlock * H, scale + b * nk);
    }
    return cudaGetLastError();
}

// ------------------------------------------------------------ the head
// logits = hidden . weight^T on the tensor cores by pairs of CTAs (tcgen05,
// kind::f8f6f4, cta_group::2).  A K block is a scale's 128 columns: one 128-byte
// row of a swizzled tile, four MMAs.  Each K block gets an accumulator of its own
// (two or four, in turn), which the epilogue takes from tensor memory, multiplies by the
// block's scales and adds to the sums in its registers in fp32 while the next ones are
// computed.  (One accumulator over all of K would need scales that are the same for all
// blocks.)  Per CTA:
//   warp 0     TMA producer: its half of A and of B, counted on the leader's barrier;
//   warp 1     the leader's MMA issuer (one thread, for both CTAs);
//   warps 4-11 epilogue: 32 lanes and half of the columns each.
// Two forms:
//   NF = 0     many rows: A = 256 rows, B = 256 tokens.  A lane is a row and a warp's
//              128 columns share a scale of the weight, so a sum costs one FMA; stored
//              through 4 KB of shared memory a warp.
//   NF > 0     at most NF rows: A = tokens (2 `high` of them, see below), B = the
//              rows, so that nothing but the weight is brought in; a lane is a token
//              and a column a row, whose scales are in shared memory throughout.
// What bounds them, and what they measured (one GB300, the rows' form by its count):
//   NF = 0     the epilogue: 128 x 256 fp32 from tensor memory a K block and CTA, 64
//              FMAs of two each a thread.  4096 x 32000 x 4096: 390 to 445 us as power
//              allows (2.4 to 2.75 PFLOP/s), 322 without the epilogue.  2 % of that asks each
//              K block whether a lane has a product of scales that is no normal
//              number (NF > 0 asks once, in front).
//   NF > 0     memory: 8 x 128256 x 4096 in 87 us, 6.1 TB/s.
// Either by rows, V = 128256, H = 4096 (us; NF the least that holds them):
//   rows       1*    8    32    64   100   128      (* V = 32000)
//   NF > 0    25    87    87    89    98    99
//   NF = 0    44   132   102   104   106   108
// At 8 rows NF = 64 takes 89 us and 128 takes 95: so three sizes.  The scales of more than
// 128 rows would have to come in with the tiles.
// Every wait is bounded: one that runs out sets VSD_STATUS_TIMEOUT, and the pair winds
// down, waits for its copies and MMAs in flight and frees its tensor memory.
namespace tc = vsd_pair;
using bf16 = __nv_bfloat16;

constexpr int kEpilogueWarps = 8;
constexpr int kHeadThreads = 32 * (4 + kEpilogueWarps);
constexpr int kHalfBytes = 128 * kBlock;  // one operand's half tile: 16 KB
constexpr int kOutBytes = 4096;           // 32 rows x 64 columns of bf16
constexpr int kMaxStages = 16, kMaxAcc = 4;
constexpr size_t kSmemMost = 232448;
constexpr int kFewBlocks = 128;           // K blocks whose scales the turned form holds:
                                          // 64 KB, which leave it six stages
constexpr int kGroupM = 16;               // row tiles that share weight tiles in L2
constexpr uint64_t kWaitNs = 2000000000ull;
// Registers a thread: launched with 168, of which the first warpgroup gives up what
// the two epilogue groups take (128 (24 + 240 + 240) = 384 * 168).
constexpr int kRegsFew = 24, kRegsMany = 240;
static_assert(kRegsFew + 2 * kRegsMany <= 3 * 168, "the launch's registers");

struct HeadBars {
    uint64_t full[kMaxStages];   // leader: both CTAs' bytes landed
    uint64_t done[kMaxStages];   // the MMAs reading the stage are done: it is free, and
                                 // their accumulator holds the K block
    uint64_t acc_empty[kMaxAcc]; // leader: the epilogue warps of both CTAs
    uint64_t drain;
    uint32_t tmem_base;
    int err;
    uint32_t end[4];             // NF > 0: least and largest scale of the rows, and of the
                                 // weight's blocks (their magnitudes' bits)
};

template <int NF> struct HeadCfg {
    static constexpr int kN = NF ? NF : 256;      // columns of an accumulator
    static constexpr int kCols = kN / 2;          // of an epilogue warp
    static constexpr int kBBytes = kN / 2 * kBlock;
    static constexpr int kAcc = NF ? kMaxAcc : 2;  // K blocks whose accumulators there are
    static constexpr uint32_t kTmem = kAcc * kN;
    static constexpr size_t kOuts = NF ? 0 : kEpilogueWarps * kOutBytes;
    // everything but the ring; a turned tile of fewer than 128 tokens reads on behind its
    // last stage
    __host__ __device__ static constexpr size_t rest(int nk) {
        return 1024 + kOuts + sizeof(HeadBars) + (NF ? 4 * (size_t)NF * nk + kHalfBytes : 0);
    }
    __host__ __device__ static constexpr int stage(int high) { return high * kBlock + kBBytes; }
    __host__ __device__ static constexpr int stages(int high, int nk) {
        const int n = (int)((kSmemMost - rest(nk)) / (size_t)stage(high));
        return n < kMaxStages ? n : kMaxStages;
    }
};
// (a stage's next `done` comes after the epilogue has seen the one before: by then the
// accumulator of as many K blocks before has been handed back)
static_assert(HeadCfg<0>::stages(128, 0) == 6 &&
                  HeadCfg<128>::stages(128, kFewBlocks) >= HeadCfg<128>::kAcc,
              "shared memory, and at least as many stages as accumulators");

struct HeadMaps {
    CUtensorMap a, b, o;
};
struct HeadArgs {
    const float *hs, *ws;  // scales of the rows and of the weight
    int R, V, nk;
    int high;              // rows of A's half tile: NF > 0: tokens, a multiple of 8; else 128
    int stages;
    bool boxes;            // the logits' rows can be stored by TMA
    bf16* out;
    int* status;
};

// A place in the ring of stages.
struct Ring {
    int slot;
    uint32_t round;
    int stages;
    __device__ void next() {
        if (++slot == stages) slot = 0, ++round;
    }
};

// The pair's tiles.  Many rows: row tiles fastest within groups of kGroupM (their rows
// stay in L2 while the weight streams by).
template <int NF> struct HeadJobs {
    int t, C, mt, nt, total;
    __device__ HeadJobs(const HeadArgs& a) {
        t = blockIdx.x >> 1;
        C = gridDim.x >> 1;
        if (NF) {
            mt = nt = 0;
            total = (a.V + 2 * a.high - 1) / (2 * a.high);
        } else {
            mt = (a.R + 255) / 256;
            nt = (a.V + 255) / 256;
            total = mt * nt;
        }
    }
    __device__ bool next(const HeadArgs& a, int& m0, int& n0) {
        if (t >= total) return false;
        if (NF) {
            m0 = t * 2 * a.high;
            n0 = 0;
        } else {
            const int g = t / (kGroupM * nt), u = t - g * kGroupM * nt;
            const int mg = min(kGroupM, mt - g * kGroupM);
            m0 = (g * kGroupM + u % mg) * 256;
            n0 = u / mg * 256;
        }
        t += C;
        return true;
    }
};

__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, HeadBars* sb,
                                          int* status) {
    if (bounded_wait([&] { return mbar_try_wait(bar, parity); },
                     [&] { return *(volatile int*)&sb->err != 0; }, kWaitNs))
        return true;
    if (!*(volatile int*)&sb->err) {
        sb->err = 1;
        atomicOr(status, VSD_STATUS_TIMEOUT);
    }
    return false;
}
// The same by a whole warp, with one outcome for all its lanes.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, HeadBars* sb,
                                          int* status) {
    return __all_sync(0xffffffffu, wait_pair(bar, parity, sb, status));
}
// One lane of a converged warp.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void drain_pair(uint64_t* bar, uint32_t parity) {
    bounded_wait([&] { return mbar_try_wait(bar, parity); }, [] { return false; }, kWaitNs);
}

// Instruction descriptor, kind::f8f6f4: fp32 accumulator, e4m3 operands, K-major.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// One step of the pair over 32 K elements, issued by one thread of the leader.
__device__ __forceinline__ void mma_pair_fp8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                             uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        :: "r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 16 consecutive fp32 columns of this thread's TMEM lane, there after a
// tmem_arrived() of the same registers.
__device__ __forceinline__ void tmem_ask(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32"
        " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
// (the registers are operands, so that no use of them moves up past the wait)
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                   "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                   "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
// Two products and sums in one instruction, each rounded once.
__device__ __forceinline__ uint64_t f2fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) {
    return f2(__uint_as_float(lo), __uint_as_float(hi));
}

// A block's sum u is at most 2^25, and 2^-18 or more where it is not 0: h w u may be
// within a float's range although h w is not, or is no normal number.
__device__ __forceinline__ bool usual(float s) { return fabsf(s) >= FLT_MIN && fabsf(s) <= FLT_MAX; }
// h w = first . second; (1, h w) where h w is a normal number.  Else the larger and the
// smaller of them, brought nearer by powers of two: u first is a normal number, and second
// one or less than 2^-126 where h w u is below 2^-115 (off by 2^-139 then); past a float's
// range it is its end (u first is 2^30 then, or 0).
__device__ __forceinline__ void split_scales(float h, float w, float& first, float& second) {
    const float s = h * w;
    const bool swap = fabsf(w) > fabsf(h);
    const float large = swap ? w : h, little = swap ? h : w;
    const bool over = fabsf(s) > 1.f;
    const float end = little * 0x1p40f;
    first = over ? large * 0x1p-40f : little * 0x1p56f;
    second = over ? (fabsf(end) > FLT_MAX ? copysignf(FLT_MAX, end) : end) : large * 0x1p-56f;
    if (usual(s)) first = 1.f, second = s;
}

// The warp's 32 rows x 128 columns, through its box of 32 x 64 (16-byte chunk j of row
// i at chunk j ^ (i % 8)).
__device__ __forceinline__ void store_rows(const HeadArgs& a, const CUtensorMap* map, int row0,
                                           int col0, int lane, const uint64_t (&x)[64],
                                           unsigned char* box) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        if (lane == 0) tc::bulk_wait_read<0>();  // the last store has read the box
        __syncwarp();
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t p = x[32 * g + 4 * v + i];
                w[i] = tc::pack_bf16((uint32_t)p, (uint32_t)(p >> 32));
            }
            *(reinterpret_cast<uint4*>(box + lane * 128) + (v ^ (lane & 7))) =
                make_uint4(w[0], w[1], w[2], w[3]);
        }
        const int col = col0 + 64 * g;
        if (a.boxes) {
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (row0 < a.R && col < a.V) tc::store_2d(map, col, row0, box);
                tc::bulk_commit();
            }
        } else {  // rows at any 2-byte address
            __syncwarp();
            unsigned short* o = reinterpret_cast<unsigned short*>(a.out) + (size_t)row0 * a.V + col;
            const int rows = min(32, a.R - row0), cols = a.V - col;
            auto word = [&](int i) {  // columns 2 lane and 2 lane + 1 of row i
                return *reinterpret_cast<const uint32_t*>(
                    box + i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + 4 * (lane & 3));
            };
            if (cols >= 64) {
                // at an odd address a lane stores columns 2 lane + 1 and 2 lane + 2 as a
                // word, lanes 0 and 31 the row's two ends
                const int end = lane ? 63 : 0;
                auto put = [&](int i, bool odd) {
                    const uint32_t w = word(i);
                    if (odd) {
                        const uint32_t after = __shfl_down_sync(0xffffffffu, w, 1);
                        if (lane < 31)
                            *reinterpret_cast<uint32_t*>(o + 2 * lane + 1) = __funnelshift_r(w, after, 16);
                        if (lane == 0 || lane == 31) o[end] = (unsigned short)(lane ? w >> 16 : w);
                    } else {
                        *reinterpret_cast<uint32_t*>(o + 2 * lane) = w;
                    }
                    o += a.V;
                };
                const bool odd = (uintptr_t)o >> 1 & 1, turns = a.V & 1;
                if (rows < 32) {
                    for (int i = 0; i < rows; ++i) put(i, odd != (turns && i & 1));
                } else if (!turns && !odd) {
#pragma unroll 8
                    for (int i = 0; i < 32; ++i) put(i, false);
                } else {
                    if (odd) put(0, true);
                    const int i0 = odd ? 1 : 0;
                    if (turns) {
#pragma unroll 4
                        for (int i = i0; i < 31; i += 2) put(i, false), put(i + 1, true);
                        if (odd) put(31, false);
                    } else {
                        for (int i = i0; i < 32; ++i) put(i, true);
                    }
                }
            } else {
                for (int i = 0; i < rows; ++i, o += a.V) {
                    const uint32_t w = word(i);
                    if (2 * lane < cols) o[2 * lane] = (unsigned short)w;
                    if (2 * lane + 1 < cols) o[2 * lane + 1] = (unsigned short)(w >> 16);
                }
            }
            __syncwarp();
        }
    }
}

// NF > 0: whether a product of a row's scale and one of this CTA's tokens' may be no
// normal number, by the ends of both.  By the epilogue warps, while the first tiles come.
template <int NF>
__device__ __forceinline__ bool scales_apart(const HeadArgs& a, HeadBars* sb, const float* row_scale,
                                             int rank) {
    const int tid = threadIdx.x - 128, nt = 32 * kEpilogueWarps;
    uint32_t end[4] = {0x7F800000u, 0, 0x7F800000u, 0};  // by their bits; 0 is left out
    auto add = [](float s, uint32_t& least, uint32_t& most) {
        const uint32_t b = __float_as_uint(fabsf(s));
        least = min(least, b - 1 < 0x7F800000u ? b : least);
        most = max(most, b);
    };
    for (int i = tid; i < NF * a.nk; i += nt) add(row_scale[i], end[0], end[1]);
    // a tile's tokens are of two blocks at most
    const HeadJobs<NF> jobs(a);
    const int tiles = (jobs.total - jobs.t + jobs.C - 1) / jobs.C, last = (a.V - 1) / kBlock;
    const int64_t n = (int64_t)tiles * 2 * a.nk;
    for (int64_t i0 = tid; i0 < n; i0 += 4 * nt) {
        float w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = min(i0 + k * nt, n - 1);
            const int t = (int)(i / (2 * a.nk)), j = (int)(i - (int64_t)t * 2 * a.nk);
            const int m0 = (jobs.t + t * jobs.C) * 2 * a.high + a.high * rank;
            const int b = min(min(m0, a.V - 1) / kBlock + (j >= a.nk), last);
            w[k] = __ldg(a.ws + (size_t)b * a.nk + (j >= a.nk ? j - a.nk : j));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) add(w[k], end[2], end[3]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        end[k] = k & 1 ? __reduce_max_sync(0xffffffffu, end[k]) : __reduce_min_sync(0xffffffffu, end[k]);
        if (threadIdx.x % 32 == 0) {
            if (k & 1) atomicMax(&sb->end[k], end[k]);
            else atomicMin(&sb->end[k], end[k]);
        }
    }
    asm volatile("bar.sync 1, %0;" :: "n"(32 * kEpilogueWarps) : "memory");
    const volatile uint32_t* e = sb->end;
    return !(__uint_as_float(e[0]) * __uint_as_float(e[2]) >= FLT_MIN &&
             __uint_as_float(e[1]) * __uint_as_float(e[3]) <= FLT_MAX);
}

template <int NF>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kHeadThreads, 1)
    k_head_fp8(const __grid_constant__ HeadMaps maps, const HeadArgs a) {
    using Cfg = HeadCfg<NF>;
    constexpr int kN = Cfg::kN, kAcc = Cfg::kAcc;
    const int high = NF ? a.high : 128, stages = NF ? a.stages : Cfg::stages(128, 0);
    const int stage_bytes = Cfg::stage(high), a_bytes = high * kBlock;
    extern __shared__ unsigned char dsm_raw[];
    unsigned char* dsm = dsm_raw + ((1024u - (smem_u32(dsm_raw) & 1023u)) & 1023u);
    HeadBars* sb = reinterpret_cast<HeadBars*>(dsm + stages * stage_bytes + (NF ? kHalfBytes : Cfg::kOuts));
    unsigned char* outs = dsm + stages * stage_bytes;
    float* row_scale = reinterpret_cast<float*>(sb + 1);  // NF > 0: [nk][NF]
    static_assert(sizeof(HeadBars) % 16 == 0, "vectors of scales");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)tc::cluster_rank();
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *a.status = 0;  // (set, if ever, after the limit of a wait)
        for (int s = 0; s < stages; ++s) {
            mbar_init(&sb->full[s], 1);
            mbar_init(&sb->done[s], 1);
        }
        for (int b = 0; b < kAcc; ++b) mbar_init(&sb->acc_empty[b], 2 * kEpilogueWarps);
        mbar_init(&sb->drain, 1);
        sb->err = 0;
        sb->end[0] = sb->end[2] = 0x7F800000u;
        sb->end[1] = sb->end[3] = 0;
        mbar_init_fence();
    }
    if (NF)
        for (int i = threadIdx.x; i < NF * a.nk; i += kHeadThreads) {
            const int n = i / a.nk, kb = i - n * a.nk;
            row_scale[kb * NF + n] = n < a.R ? a.hs[(size_t)n * a.nk + kb] : 0.f;
        }
    if (warp == 1) tc::tmem_alloc_pair(&sb->tmem_base, Cfg::kTmem);
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    tc::tc_fence_after();
    const uint32_t tmem = sb->tmem_base;
    HeadJobs<NF> jobs(a);
    int m0, n0;
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kRegsFew));
        // ------------------------------------------------------ TMA producer
        Ring at{0, 0, stages};
        uint32_t it = 0;
        bool ok = true;
        while (ok && jobs.next(a, m0, n0)) {
            for (int kb = 0; kb < a.nk; ++kb, ++it, at.next()) {
                if (at.round > 0 &&
                    !(ok = wait_warp(&sb->done[at.slot], (at.round - 1) & 1u, sb, a.status)))
                    break;
                if (elected()) {
                    unsigned char* A = dsm + at.slot * stage_bytes;
                    const uint32_t bar = tc::leader_addr(&sb->full[at.slot]);
                    if (rank == 0) mbar_expect_tx(&sb->full[at.slot], 2 * stage_bytes);
                    tc::load_2d(A, &maps.a, kb * kBlock, m0 + high * rank, bar);
                    tc::load_2d(A + a_bytes, &maps.b, kb * kBlock, n0 + kN / 2 * rank, bar);
                }
                __syncwarp();
            }
        }
        // the copies still in flight have landed before the pair may exit
        if (rank == 0)
            for (uint32_t i = it > (uint32_t)stages ? it - stages : 0; i < it; ++i)
                drain_pair(&sb->full[i % stages], (i / stages) & 1u);
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kRegsFew));
        // ------------------------------------------------------ MMA issuer
        if (rank == 0) {
            const uint32_t ring = smem_u32(dsm);
            // descriptors of stage 0; a stage and a K step add to the address field
            // (16-byte units), which never carries out of it
            const uint64_t a0 = tc::sdesc_sw128(ring), b0 = tc::sdesc_sw128(ring + a_bytes);
            Ring at{0, 0, stages};
            uint32_t it = 0;
            bool ok = true;
            while (ok && jobs.next(a, m0, n0)) {
                for (int kb = 0; kb < a.nk; ++kb, ++it, at.next()) {
                    const uint32_t buf = it % kAcc, use = it / kAcc;
                    if ((use > 0 && !(ok = wait_warp(&sb->acc_empty[buf], (use - 1) & 1u, sb,
                                                     a.status))) ||
                        !(ok = wait_warp(&sb->full[at.slot], at.round & 1u, sb, a.status)))
                        break;
                    tc::tc_fence_after();
                    if (elected()) {
                        const uint64_t off = (uint32_t)(at.slot * stage_bytes) >> 4;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_pair_fp8(tmem + buf * kN, a0 + off + 2 * k, b0 + off + 2 * k,
                                         idesc_e4m3(256, kN), k != 0);
                        tc::commit_pair(&sb->done[at.slot]);
                    }
                    __syncwarp();
                }
            }
            // every MMA issued is done once it arrives
            if (elected()) tc::commit_pair(&sb->drain);
            __syncwarp();
            drain_pair(&sb->drain, 0);
        }
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kRegsFew));
    } else {
        // ------------------------------------------------------ epilogue
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kRegsMany));
        constexpr int kCols = Cfg::kCols, kStep = 16;
        const int q = warp & 3;                          // TMEM lanes 32q .. 32q + 31
        const int h0 = ((warp - 4) >> 2) * kCols;        // its columns of the tile
        const uint32_t empty = tc::leader_addr(&sb->acc_empty[0]);
        // The tiles; split: by two factors throughout (NF > 0).
        auto tiles = [&](auto split) {
            Ring at{0, 0, stages};
            uint32_t it = 0;
            bool ok = true;
            while (ok && jobs.next(a, m0, n0)) {
                const int in = 32 * q + lane;
                const int top = m0 + high * rank + in;       // this lane's row (NF = 0) or token
                // scales: of the lane (`lane_s`), and of the warp's columns
                const float* lane_s = NF ? a.ws + (size_t)(min(top, a.V - 1) / kBlock) * a.nk
                                         : a.hs + (size_t)min(top, a.R - 1) * a.nk;
                const float* col_s =
                    NF ? nullptr : a.ws + (size_t)(min(n0 + h0, a.V - 1) / kBlock) * a.nk;
                uint64_t x[kCols / 2];  // columns 2i and 2i + 1
#pragma unroll
                for (int i = 0; i < kCols / 2; ++i) x[i] = 0;
                float ls = __ldg(lane_s), cs = NF ? 0.f : __ldg(col_s);
                // NF = 0: whether a lane's product is no normal number
                bool apart = NF == 0 && __any_sync(0xffffffffu, !usual(ls * cs));
                for (int kb = 0; kb < a.nk; ++kb, ++it, at.next()) {
                    const float s = NF ? ls : ls * cs;
                    if (kb + 1 < a.nk) {
                        ls = __ldg(lane_s + kb + 1);
                        if (!NF) cs = __ldg(col_s + kb + 1);
                    }
                    const int buf = (int)(it % kAcc);
                    const uint64_t s2 = f2(s, s);
                    uint64_t c2[NF ? kCols / 2 : 1];  // the products of the two sides' scales
                    if constexpr (NF != 0 && !split.value) {
                        const float4* c = reinterpret_cast<const float4*>(row_scale + kb * NF + h0);
#pragma unroll
                        for (int i = 0; i < kCols / 4; ++i) {
                            c2[2 * i] = f2mul(f2(c[i].x, c[i].y), s2);
                            c2[2 * i + 1] = f2mul(f2(c[i].z, c[i].w), s2);
                        }
                    }
                    if (!(ok = wait_warp(&sb->done[at.slot], at.round & 1u, sb, a.status))) break;
                    tc::tc_fence_after();
                    const uint32_t t = tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * kN + h0);
                    bool next_apart = false;
                    auto take = [&](auto twice) {
                        float first = 1.f, second = s;
                        if constexpr (NF == 0 && twice.value)
                            split_scales(__ldg(lane_s + kb), __ldg(col_s + kb), first, second);
                        uint32_t u[2][kStep];
                        tmem_ask(t, u[0]);
#pragma unroll
                        for (int g = 0; g < kCols / kStep; ++g) {
                            tmem_arrived(u[g & 1]);
                            if (g + 1 < kCols / kStep) {
                                tmem_ask(t + (uint32_t)(kStep * (g + 1)), u[(g + 1) & 1]);
                            } else {  // all of it is in registers
                                tc::tc_fence_before();
                                __syncwarp();
                                if (lane == 0) tc::arrive_remote(empty + 8u * buf);
                                // (the next scales have come by now; asked for in front of
                                // their wait: 454 us, not 409)
                                if (NF == 0) next_apart = __any_sync(0xffffffffu, !usual(ls * cs));
                            }
#pragma unroll
                            for (int i = 0; i < kStep / 2; ++i) {
                                const int c = kStep / 2 * g + i;
                                uint64_t v = pair_of(u[g & 1][2 * i], u[g & 1][2 * i + 1]);
                                uint64_t by = NF || twice.value ? 0 : s2;
                                if constexpr (twice.value) {
                                    float first1 = first, second1 = second;
                                    if constexpr (NF != 0) {
                                        const float* h = row_scale + kb * NF + h0 + 2 * c;
                                        split_scales(h[0], s, first, second);
                                        split_scales(h[1], s, first1, second1);
                                    }
                                    v = f2mul(v, f2(first, first1));
                                    by = f2(second, second1);
                                } else if constexpr (NF != 0) {
                                    by = c2[c];
                                }
                                x[c] = f2fma(v, by, x[c]);
                            }
                        }
                    };
                    if constexpr (NF != 0) take(split);
                    else if (apart) take(std::true_type{});
                    else take(std::false_type{});
                    apart = next_apart;
                }
                if (!ok) break;
                if constexpr (NF == 0) {
                    store_rows(a, &maps.o, m0 + 128 * rank + 32 * q, n0 + h0, lane, x,
                               outs + (warp - 4) * kOutBytes);
                } else if (in < high && top < a.V) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        if (h0 + c < a.R)
                            a.out[(size_t)(h0 + c) * a.V + top] = __float2bfloat16_rn(
                                __uint_as_float((uint32_t)(x[c / 2] >> (c & 1 ? 32 : 0))));
                }
                __syncwarp();
            }
        };
        if constexpr (NF == 0) tiles(std::false_type{});
        else if (scales_apart<NF>(a, sb, row_scale, rank)) tiles(std::true_type{});
        else tiles(std::false_type{});
        if (NF == 0 && lane == 0) tc::bulk_wait_all();
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_free_pair(tmem, Cfg::kTmem);
    }
}

// ---------------------------------------------------------------- host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Tensor map of a row-major matrix of `size`-byte elements (1: e4m3, 2: bf16) in boxes
// of 128 bytes x box_rows with the 128-byte swizzle; reads past its edges give zero.
bool make_map(CUtensorMap* m, const void* base, int size, int64_t rows, int64_t cols,
              int box_rows) {
    static const EncodeTiledFn enc = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000,
                                                         cudaEnableDefault, &q) == cudaSuccess &&
                        q == cudaDriverEntryPointSuccess;
        return ok ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)cols * size};
    const cuuint32_t box[2] = {128u / size, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(m, size == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
               const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NF>
cudaError_t launch_head(const HeadMaps& maps, HeadArgs a, int64_t jobs, int most,
                        cudaStream_t st) {
    cudaError_t e = ensure_dyn_smem((const void*)k_head_fp8<NF>, kSmemMost);
    if (e != cudaSuccess) return e;
    a.stages = HeadCfg<NF>::stages(a.high, NF ? a.nk : 0);
    const size_t smem = HeadCfg<NF>::rest(NF ? a.nk : 0) + (size_t)a.stages * HeadCfg<NF>::stage(a.high);
    const int pairs = (int)std::min<int64_t>(jobs, most);
    k_head_fp8<NF><<<2 * pairs, kHeadThreads, smem, st>>>(maps, a);
    return cudaGetLastError();
}

cudaError_t head_fp8(const void* hidden, const void* weight, int H, HeadArgs a, cudaStream_t st) {
    const int most = std::max(1, device_sm_count() / 2);
    a.nk = (H + kBlock - 1) / kBlock;
    a.high = 128;
    HeadMaps maps;
    memset(&maps, 0, sizeof(maps));
    const int nf = a.nk > kFewBlocks ? 0 : a.R <= 32 ? 32 : a.R <= 64 ? 64 : a.R <= 128 ? 128 : 0;
    if (nf == 0) {
        a.boxes = a.V % 8 == 0 && ((uintptr_t)a.out & 15) == 0;
        if (!make_map(&maps.a, hidden, 1, a.R, H, 128) || !make_map(&maps.b, weight, 1, a.V, H, 128) ||
            (a.boxes && !make_map(&maps.o, a.out, 2, a.R, a.V, 32)))
            return cudaErrorInvalidValue;
        const int64_t jobs = (int64_t)((a.R + 255) / 256) * ((a.V + 255) / 256);
        return launch_head<0>(maps, a, jobs, most, st);
    }
    // the tiles' height with the least time: a K block takes what its bytes do at a
    // pair's share of the memory (43.7 bytes a ns and CTA, 6.6 TB/s over 152), 300 ns at
    // least.  (32000 tokens, 1 and 128 rows: 24.5 and 33.8 us, 25.5 and 35.1 at 128
    // throughout; 128256: no difference.)
    double best = 1e30;
    for (int high = 128; high >= 64; high -= 8) {
        const int64_t tiles = (a.V + 2 * high - 1) / (2 * high);
        const double ns = (double)((tiles + most - 1) / most) * std::max(300.0, high * kBlock / 43.7);
        if (ns < best) best = ns, a.high = high;
    }
    if (!make_map(&maps.a, weight, 1, a.V, H, a.high) || !make_map(&maps.b, hidden, 1, a.R, H, nf / 2))
        return cudaErrorInvalidValue;
    const int64_t jobs = (a.V + 2 * a.high - 1) / (2 * a.high);
    return nf == 32   ? launch_head<32>(maps, a, jobs, most, st)
           : nf == 64 ? launch_head<64>(maps, a, jobs, most, st)
                      : launch_head<128>(maps, a, jobs, most, st);
}

bool share_bytes(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + bn && y < x + an;
}
bool sizes_ok(int R, int H) {
    return R >= 1 && R <= (1 << 24) && H >= 16 && H <= (1 << 20) && H % 16 == 0;
}

}  // namespace
}  // namespace vsd

using namespace vsd;

extern "C" {

vsd_status vsd_quantize_fp8(const void* x, vsd_dtype dtype, int32_t R, int32_t H,
                            int32_t block_rows, void* q, float* scale, void* stream) {
    if (!x || !q || !scale || !sizes_ok(R, H)) return VSD_ERR_INVALID_ARG;
    if (dtype != VSD_F32 && dtype != VSD_BF16) return VSD_ERR_INVALID_ARG;
    if (block_rows != 1 && block_rows != kBlock) return VSD_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uintptr_t)q) & 15) || ((uintptr_t)scale & 3)) return VSD_ERR_INVALID_ARG;
    const size_t n = (size_t)R * H, xb = n * (dtype == VSD_BF16 ? 2 : 4);
    const int nr = (R + block_rows - 1) / block_rows, nh = (H + kBlock - 1) / kBlock;
    const size_t sb = 4 * (size_t)nr * nh;
    if (share_bytes(x, xb, q, n) || share_bytes(x, xb, scale, sb) || share_bytes(q, n, scale, sb))
        return VSD_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    __nv_fp8_e4m3* out = static_cast<__nv_fp8_e4m3*>(q);
    const cudaError_t e =
        dtype == VSD_BF16
            ? quantize(static_cast<const __nv_bfloat16*>(x), R, H, block_rows, out, scale, st)
            : quantize(static_cast<const float*>(x), R, H, block_rows, out, scale, st);
    return e == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

vsd_status vsd_lmhead_logits_fp8(const void* hidden, const float* hidden_scale,
                                 const void* weight, const float* weight_scale, int32_t R,
                                 int32_t V, int32_t H, void* logits, void* ws, size_t ws_bytes,
                                 void* stream) {
    if (!hidden || !hidden_scale || !weight || !weight_scale || !logits || !sizes_ok(R, H))
        return VSD_ERR_INVALID_ARG;
    if (V < 1 || V > (1 << 20)) return VSD_ERR_INVALID_ARG;
    if ((((uintptr_t)hidden | (uintptr_t)weight) & 15) || ((uintptr_t)logits & 1) ||
        (((uintptr_t)hidden_scale | (uintptr_t)weight_scale) & 3))
        return VSD_ERR_INVALID_ARG;
    const size_t nk = (H + kBlock - 1) / kBlock, ob = 2 * (size_t)R * V;
    if (share_bytes(logits, ob, hidden, (size_t)R * H) || share_bytes(logits, ob, weight, (size_t)V * H) ||
        share_bytes(logits, ob, hidden_scale, 4 * nk * R) ||
        share_bytes(logits, ob, weight_scale, 4 * nk * ((V + kBlock - 1) / kBlock)))
        return VSD_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < 256) return VSD_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    HeadArgs args{};
    args.hs = hidden_scale;
    args.ws = weight_scale;
    args.R = R;
    args.V = V;
    args.out = static_cast<bf16*>(logits);
    args.status = static_cast<int*>(ws);
    return head_fp8(hidden, weight, H, args, st) == cudaSuccess ? VSD_OK : VSD_ERR_CUDA;
}

}  // extern "C"
