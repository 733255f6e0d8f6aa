// vsd_sample.cuh -- one token a row from what temperature, top-k, top-p and min-p
// leave of a distribution, and the logits these leave (include/vsd_decode.h).
//
// Every filter keeps a first part of the tokens in the order (logit falling, id
// rising), so what is kept is one place in that order: a logit, and the last id kept
// among those that equal it.  Masses that a decision hangs on are whole numbers
// (vsd_fixed.cuh): sums of them are exact, in whatever order threads add them.
//
// A block works on a row, two blocks to an SM.  Bound by memory where the filters leave
// few tokens: the row comes from memory once, and from L2 for the passes after the
// first.  Bound by instructions where a nucleus is wide: 75 for an exact mass, 8 for an
// approximate one.  A row takes as few of these steps as decide it:
//
//   top      the maximum, and a bound `lo` that enough of the threads' first maxima
//            reach (kWant over the row).
//   list     the tokens from `lo` on, sorted; a prefix sum of their masses gives every
//            filter's place and the draw.  A nucleus also needs the mass of all others,
//            a sum of approximate exponentials (2^-17 off at most): where that leaves
//            the place open, it is made finer (2^-20), then exact.
//   bracket  a nucleus past the list: a histogram of approximate masses over 1024
//            steps of the logit brackets its place, first of a quarter of the row, then
//            of all of it; the tokens in the bracket are listed, and the mass above it
//            is summed exactly.  A list that overflows is bracketed within its bounds.
//   search   whatever these leave open (large k, thousands of equal logits, rows that
//            begin with more masked tokens than a round of loads): bisection
//            of the logits' ordered bits, exact counts and masses each step.
//
// At 4096 x 128256 bf16 (1.05 GB, 158 us at the copy's rate), us: greedy 245, top_k 50
// 410, top_p 0.8 806 and 0.95 1630 (nuclei of 3500 tokens).  8 rows: 15 greedy, 27 with
// top_k 50, 113 with top_p 0.95: one block's latency.  Measured against it: blocks of 256
// with lists of 2048, three to an SM (greedy 198, top_p 0.95 a fifth slower); blocks of
// 1024 where there is a row an SM at most (8 x 128256: 2 us more for greedy and top_k, a
// seventh less for wide nuclei); a cluster of 8 a row (four times as long for the 4096
// rows, by its barriers).
//
// Where the kept tokens are not all in the list, the exact sums are also kept by region
// of the row; the draw finds the region, then the token in it.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "vsd_common.cuh"
#include "vsd_fixed.cuh"
#include "vsd_launch.h"
#include "vsd_sample.h"

namespace vsd {
namespace {

constexpr int kSampleThreads = 512;
constexpr int kList = 4096;
constexpr int kPlaceBits = 12;           // of a place in it
constexpr int kBins = 1024;
// A list's length aimed at, where top-k does not say.  (256, 768, 1600, 2800: top_p 0.95 of
// 4096 x 128256 in 2642, 2248, 2097, 2736 us when it was set, and settings of all kinds at
// 512 x 32000 in 131, 119, 228, 226: 32000 is two rounds, of which the first then lists
// all.)
constexpr int kWant = 768;
constexpr int kDeep = 8;                 // vectors of a lane in a long row's regions
constexpr int kRegions = (1 << 18) / (32 * kDeep) + 1;
// Vectors of a row whose regions are one deep: no more than one round of a block's loads,
// so that all its warps have some.
constexpr int kShort = 2048;
static_assert(kList == 1 << kPlaceBits && kList % 1024 == 0 && kBins % 1024 == 0, "whole rounds");


__constant__ ExpParts kExpParts = make_exp_parts();

__device__ __forceinline__ float float_of(float x) { return x; }
__device__ __forceinline__ float float_of(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T none_of();
template <> __device__ __forceinline__ float none_of<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __nv_bfloat16 none_of<__nv_bfloat16>() {
    return __ushort_as_bfloat16(0xFF80u);
}
// Bits whose order is the logits' (-0 as 0).
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
constexpr uint32_t kKeyNone = 0x007FFFFFu;  // of -inf

// The largest element of a vector, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <typename T> __device__ __forceinline__ float vec_max_nan(const uint4& v);
template <> __device__ __forceinline__ float vec_max_nan<float>(const uint4& v) {
    return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)),
                   max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
}
template <> __device__ __forceinline__ float vec_max_nan<__nv_bfloat16>(const uint4& v) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
    return max_nan(__low2float(m), __high2float(m));
}

// Element e of a vector.
template <typename T> __device__ __forceinline__ float element(const uint4& q, int e);
template <> __device__ __forceinline__ float element<float>(const uint4& q, int e) {
    return __uint_as_float(e & 2 ? (e & 1 ? q.w : q.z) : (e & 1 ? q.y : q.x));
}
template <> __device__ __forceinline__ float element<__nv_bfloat16>(const uint4& q, int e) {
    const uint32_t w = e & 4 ? (e & 2 ? q.w : q.z) : (e & 2 ? q.y : q.x);
    return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
}

// For each element of q whether it is from `lo` on: all bits of its place set, or none.
// (lo: a value of the type)
template <typename T> __device__ __forceinline__ uint4 mask_from(const uint4& q, float lo);
template <> __device__ __forceinline__ uint4 mask_from<float>(const uint4& q, float lo) {
    auto one = [&](uint32_t w) { return __uint_as_float(w) >= lo ? ~0u : 0u; };
    return make_uint4(one(q.x), one(q.y), one(q.z), one(q.w));
}
template <> __device__ __forceinline__ uint4 mask_from<__nv_bfloat16>(const uint4& q, float lo) {
    const __nv_bfloat162 l = __float2bfloat162_rn(lo);
    auto two = [&](uint32_t w) { return __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w), l); };
    return make_uint4(two(q.x), two(q.y), two(q.z), two(q.w));
}
// q with -inf where the mask is set.
template <typename T> __device__ __forceinline__ uint4 cleared(const uint4& q, const uint4& m) {
    constexpr uint32_t n = Traits<T>::kNegInf;
    return make_uint4((q.x & ~m.x) | (n & m.x), (q.y & ~m.y) | (n & m.y), (q.z & ~m.z) | (n & m.z),
                      (q.w & ~m.w) | (n & m.w));
}
// The mask's elements as bits.
template <typename T> __device__ __forceinline__ uint32_t bits_of(const uint4& m);
template <> __device__ __forceinline__ uint32_t bits_of<float>(const uint4& m) {
    return (m.x & 1u) | (m.y & 2u) | (m.z & 4u) | (m.w & 8u);
}
template <> __device__ __forceinline__ uint32_t bits_of<__nv_bfloat16>(const uint4& m) {
    auto two = [](uint32_t w, uint32_t b) { return (w & b) | (w >> 16 & b << 1); };
    return two(m.x, 1u) | two(m.y, 4u) | two(m.z, 16u) | two(m.w, 64u);
}
// The lowest finite value of the type.
template <typename T> __device__ __forceinline__ float lowest_of();
template <> __device__ __forceinline__ float lowest_of<float>() { return -FLT_MAX; }
template <> __device__ __forceinline__ float lowest_of<__nv_bfloat16>() {
    return __uint_as_float(0xFF7F0000u);
}
// The nearest value of the type at or below, or above; down, the lowest finite one at least
// (from -inf on, tokens without mass and what pads a row's ends would be listed).
template <typename T> __device__ __forceinline__ float down_to(float v);
template <> __device__ __forceinline__ float down_to<float>(float v) { return fmaxf(v, -FLT_MAX); }
template <> __device__ __forceinline__ float down_to<__nv_bfloat16>(float v) {
    return fmaxf(__bfloat162float(__float2bfloat16_rd(v)), lowest_of<__nv_bfloat16>());
}
template <typename T> __device__ __forceinline__ float up_to(float v);
template <> __device__ __forceinline__ float up_to<float>(float v) { return v; }
template <> __device__ __forceinline__ float up_to<__nv_bfloat16>(float v) {
    return __bfloat162float(__float2bfloat16_ru(v));
}

// f w in whole numbers for 0 <= f < 1: rounded down, or up.
__device__ __forceinline__ uint64_t share_of(uint64_t w, float f, bool up) {
    if (!(f > 0.f)) return 0;
    int e;
    const uint64_t k = (uint64_t)(frexpf(f, &e) * 16777216.f);  // f = k 2^-sh
    const int sh = 24 - e;                                       // 24 at least
    const uint64_t hi = __umul64hi(w, k), lo = w * k;
    uint64_t q, rest;
    if (sh >= 128) q = 0, rest = hi | lo;
    else if (sh > 64) q = hi >> (sh - 64), rest = lo | hi << (128 - sh);
    else if (sh == 64) q = hi, rest = lo;
    else q = hi << (64 - sh) | lo >> sh, rest = lo << (64 - sh);
    return q + (up && rest ? 1 : 0);
}

__device__ __forceinline__ uint64_t warp_sum_u64(uint64_t v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint64_t warp_scan_u64(uint64_t v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t n = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += n;
    }
    return v;
}

// What is decided about a row.
enum { kDone = 0, kExactTail = 1, kBracket = 2, kSearch = 3, kOverflow = 4, kAbove = 5 };
struct Decision {
    int what;
    float cut;       // tokens above it are kept, and those at it up to id `limit`
    int limit, kept;
    int token;       // the token drawn, or -1
    uint64_t all, listed;  // the kept tokens' mass; for a bracket, the whole and the list's
    int bin0, bin1;    // of the bracket
};


// 128 bits of a logits row (which may be written later, by this block alone).
__device__ __forceinline__ uint4 ld_row(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// A region is `depth` vectors, one after another in the row, of which a warp sums the
// masses: 32 kDeep, or 32 in short rows, so that all warps have some.
template <typename T> struct Sampler {
    static constexpr int PV = Traits<T>::kPerVec;
    static constexpr int NT = kSampleThreads, kWarps = NT / 32;
    static constexpr int kLoad = 4;  // vectors of a lane in flight
    static constexpr int kQueue = 32 + 32 * PV;  // tokens of a warp that wait for their masses
    static_assert(kWarps * kQueue * sizeof(float) <= kList * sizeof(uint64_t) &&
                      kWarps * kQueue * sizeof(uint16_t) <= kList * sizeof(uint32_t) &&
                      32 * kDeep * PV <= 65536,
                  "in the masses' place, and the orders'");

    struct Shared {
        uint64_t tab[kExpTab];
        uint64_t list[kList];      // (key, ~id)
        uint64_t mass[kList];      // of the sorted list
        uint32_t order[kList];     // ids and places in the list; a histogram
        uint64_t region[kRegions];
        uint64_t part[kWarps], value;
        Decision dec;
        int count, token, next;
    };

    const SampleArgs& a;
    Shared& s;
    int tid, lane, warp;
    // of the row
    const T* x;
    int off, nvec;  // elements before x in its first vector; vectors
    int depth;
    float m, T_, c, base;  // (base: where a histogram's bins begin)
    float above_from;      // of the list at hand
    bool by_min;           // whether min_p is on: tokens as far below the first one as
    float far, far_lo;     // T ln(1 / min_p), in two floats, or nearer have it
    ExpScale sc;

    __device__ Sampler(const SampleArgs& args, Shared& sh) : a(args), s(sh) {
        tid = threadIdx.x;
        lane = tid & 31;
        warp = tid >> 5;
    }

    __device__ __forceinline__ uint64_t block_sum(uint64_t v) { return group_sum<NT>(v); }
    // The sum of v over the threads before this one, and over all.
    __device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t& all) {
        return group_scan<NT>(v, all);
    }
    // The same by the first G threads.
    template <int G> __device__ __forceinline__ void sync() {
        if (G == 32) __syncwarp();
        else if (G < NT) asm volatile("bar.sync 1, %0;" :: "n"(G) : "memory");
        else __syncthreads();
    }
    template <int G> __device__ __forceinline__ uint64_t group_scan(uint64_t v, uint64_t& all) {
        const uint64_t incl = warp_scan_u64(v, lane);
        if (G == 32) {
            all = __shfl_sync(0xffffffffu, incl, 31);
            return incl - v;
        }
        sync<G>();
        if (lane == 31) s.part[warp] = incl;
        sync<G>();
        uint64_t before = incl - v;
        all = 0;
#pragma unroll
        for (int i = 0; i < G / 32; ++i) {
            if (i < warp) before += s.part[i];
            all += s.part[i];
        }
        return before;
    }
    template <int G> __device__ __forceinline__ uint64_t group_sum(uint64_t v) {
        v = warp_sum_u64(v);
        if (G == 32) return v;
        sync<G>();
        if (lane == 0) s.part[warp] = v;
        sync<G>();
        uint64_t t = 0;
#pragma unroll
        for (int i = 0; i < G / 32; ++i) t += s.part[i];
        return t;
    }

    // ------------------------------------------------------------ the row
    __device__ __forceinline__ void open(const T* row) {
        x = row;
        off = (int)(((uintptr_t)x / sizeof(T)) % PV);
        nvec = (a.V + off + PV - 1) / PV;
        depth = nvec <= kShort ? 32 : 32 * kDeep;
    }
    // Brings a row into L2.
    __device__ __forceinline__ void bring(const T* row) const {
        for (int64_t i = (int64_t)tid * 128; i < (int64_t)a.V * (int64_t)sizeof(T); i += NT * 128)
            asm volatile("prefetch.global.L2 [%0];" :: "l"(reinterpret_cast<const char*>(row) + i));
    }
    // Vector j of the row, -inf where it reaches past it.
    __device__ __forceinline__ uint4 vec(int j) const {
        const int first = id_of(j);
        if (first >= 0 && first + PV <= a.V) return ld_row(x + first);
        T e[PV];
#pragma unroll
        for (int i = 0; i < PV; ++i)
            e[i] = first + i >= 0 && first + i < a.V ? x[first + i] : none_of<T>();
        uint4 q;
        memcpy(&q, e, 16);
        return q;
    }
    // Vectors j0, j0 + STEP, ... of this lane, those before `end` (j0 - lane is the warp's).
    template <int STEP> __device__ __forceinline__ void load(int j0, int end, uint4 (&q)[kLoad]) const {
        const int first = j0 - lane, last = first + STEP * (kLoad - 1) + 32;
        if (last <= end && id_of(first) >= 0 && id_of(last) <= a.V) {  // (all inside)
            const T* p = x + id_of(j0);
#pragma unroll
            for (int i = 0; i < kLoad; ++i) q[i] = ld_row(p + STEP * PV * i);
        } else {
            const uint4 none = make_uint4(Traits<T>::kNegInf, Traits<T>::kNegInf, Traits<T>::kNegInf,
                                          Traits<T>::kNegInf);
#pragma unroll
            for (int i = 0; i < kLoad; ++i) q[i] = j0 + STEP * i < end ? vec(j0 + STEP * i) : none;
        }
    }
    // The id of element 0 of vector j.
    __device__ __forceinline__ int id_of(int j) const { return j * PV - off; }
    __device__ __forceinline__ uint64_t mass_of(float v) const { return exp_fixed(v, m, sc, s.tab); }
    // By the logits' distance, to within 2^-39 of min_p: a mass has a unit's precision only.
    __device__ __forceinline__ bool has_min(float v) const {
        float lo;
        const float d = gap(v, m, lo);
        return (d - far) + (lo - far_lo) <= 0.f;  // (NaN where m - v is past a float's range)
    }
    __device__ __forceinline__ float approx(float v) const { return ex2((v - m) * c); }
    // f(vector, j) for this thread's vectors of the row, end(region) after a region's.
    template <typename F, typename E> __device__ __forceinline__ void each(F f, E end) const {
        for (int j0 = warp * depth; j0 < nvec; j0 += kWarps * depth) {
            const int stop = min(nvec, j0 + depth);
#pragma unroll 1
            for (int h = j0; h < stop; h += 32 * kLoad) {
                uint4 q[kLoad];
                load<32>(h + lane, stop, q);
#pragma unroll
                for (int i = 0; i < kLoad; ++i)
                    if (h + 32 * i < stop) f(q[i], h + 32 * i + lane);
            }
            end(j0 / depth);
        }
    }
    template <typename F> __device__ __forceinline__ void each(F f) const {
        each(f, [](int) {});
    }

    // ------------------------------------------------------------ the list
    // What a listing leaves beside the list: the exact mass and the number of the tokens
    // above, and the approximate mass of the rest.
    struct Found {
        uint64_t above, tail, slack;  // (how far the tail may be off)
        int n_above;
        bool below;  // whether there is a rest
    };
    // A sum of approximate masses.
    struct Sum {
        float hi = 0.f, lo = 0.f;
        __device__ __forceinline__ void add(float v) {
            const float t = hi + v;
            lo += v - (t - hi);
            hi = t;
        }
    };
    __device__ __forceinline__ void list(float v, int id) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.list[at] = (uint64_t)key_of(v) << 32 | (uint32_t)~id;
    }
    // The sum of a vector's masses relative to `ref`, off by 2^-17 of itself at most, where
    // exponents are 40 at most: ex2's 2^-22, and what v - ref, c and their product are
    // rounded by.  (An exponent in two floats takes three times the instructions: see
    // finer_tail.  One nucleus in twenty needs it.)
    __device__ __forceinline__ float approx_sum(const uint4& q, float ref) const {
        uint64_t p[PV / 2];
        vec_pairs<T>(q, p);
        const uint64_t m2 = f2(ref, ref), c2 = f2(c, c);
        uint64_t acc = f2_mass(p[0], m2, c2);
#pragma unroll
        for (int e = 1; e < PV / 2; ++e) acc = f2add(acc, f2_mass(p[e], m2, c2));
        float s0, s1;
        f2split(acc, s0, s1);
        return s0 + s1;
    }
    // One vector, its largest element `top`: its tokens from `lo` on are listed, the others'
    // masses relative to `ref` added up, and the largest of them kept.
    template <bool TAIL>
    __device__ __forceinline__ void list_vec(const uint4& q, float top, int j, float lo, float ref,
                                             Sum& sum, float& under) {
        if (top >= lo) {
            const uint4 in = mask_from<T>(q, lo), rest = cleared<T>(q, in);
            for (uint32_t h = bits_of<T>(in); h; h &= h - 1) {
                const int e = __ffs(h) - 1;
                list(element<T>(q, e), id_of(j) + e);
            }
            under = fmaxf(under, vec_max<T>(rest));
            if (TAIL) sum.add(approx_sum(rest, ref));
            return;
        }
        under = fmaxf(under, top);
        if (TAIL) sum.add(approx_sum(q, ref));
    }
    // How far an approximate sum, `bits` known, may be off the exact one: 2^-28 of the first
    // token for terms of large exponents, and what whole numbers are off, a unit for each
    // token.
    __device__ __forceinline__ uint64_t slack_of(uint64_t tail, int bits) const {
        return (tail >> bits) + (1ull << (62 - sc.shift) >> 28) + (uint64_t)a.V;
    }
    __device__ __forceinline__ uint64_t fixed_of(float v) const {
        return __float2ull_rn(v * ldexpf(1.f, 62 - sc.shift));
    }
    // Tokens from `hi` on are above, those from `lo` on are listed.  Left is the mass
    // above, by region too; of the rest it is approximate, or not summed at all.
    // (Tokens from `lo` on wait in a warp's queue until there are 32, so that all its lanes
    // are of use: a few in 100 tokens are above where a nucleus is wide.)
    template <bool TAIL> __device__ __forceinline__ Found collect(float hi, float lo) {
        if (tid == 0) s.count = 0;
        __syncthreads();
        Found f{0, 0, 0, 0, false};
        Sum sum;
        uint64_t above = 0;
        float under = -INFINITY;
        float* const value = reinterpret_cast<float*>(s.mass) + warp * kQueue;
        uint16_t* const place = reinterpret_cast<uint16_t*>(s.order) + warp * kQueue;
        int waiting = 0;
        // the last n that wait, of the region that begins at vector j0
        auto drain = [&](int n, int j0) {
            __syncwarp();
            waiting -= n;
            const bool on = lane < n;
            const float v = on ? value[waiting + lane] : 0.f;
            const int id = on ? id_of(j0) + place[waiting + lane] : 0;
            const bool over = on && v >= hi, in = on && !over;
            if (over) above += mass_of(v), ++f.n_above;
            const uint32_t w = __ballot_sync(0xffffffffu, in);
            if (w) {
                int at = 0;
                if (lane == 0) at = atomicAdd(&s.count, __popc(w));
                at = __shfl_sync(0xffffffffu, at, 0) + __popc(w & ((1u << lane) - 1));
                if (in && at < kList) s.list[at] = (uint64_t)key_of(v) << 32 | (uint32_t)~id;
            }
            __syncwarp();
        };
        for (int j0 = warp * depth; j0 < nvec; j0 += kWarps * depth) {
            const int stop = min(nvec, j0 + depth);
#pragma unroll 1
            for (int h = j0; h < stop; h += 32 * kLoad) {
                uint4 q4[kLoad];
                load<32>(h + lane, stop, q4);
#pragma unroll 1
                for (int i = 0; i < kLoad && h + 32 * i < stop; ++i) {
                    const uint4 q = i == 0 ? q4[0] : i == 1 ? q4[1] : i == 2 ? q4[2] : q4[3];
                    uint4 rest = q;
                    if (__any_sync(0xffffffffu, vec_max<T>(q) >= lo)) {
                        const uint4 in = mask_from<T>(q, lo);
                        const uint32_t b = bits_of<T>(in);
                        const int rel = (h - j0 + 32 * i + lane) * PV;
                        rest = cleared<T>(q, in);
                        float v[PV];
                        unpack<T>(q, v);
                        // where this lane's go: behind those of the lanes before, whose
                        // numbers (PV at most) are added bit by bit
                        const int n = __popc(b);
                        int at = waiting;
#pragma unroll
                        for (int i = 0; 1 << i <= PV; ++i) {
                            const uint32_t w = __ballot_sync(0xffffffffu, n >> i & 1);
                            at += __popc(w & ((1u << lane) - 1)) << i;
                            waiting += __popc(w) << i;
                        }
#pragma unroll
                        for (int e = 0; e < PV; ++e)
                            if (b >> e & 1) {
                                value[at] = v[e];
                                place[at++] = (uint16_t)(rel + e);
                            }
                        while (waiting >= 32) drain(32, j0);
                    }
                    under = fmaxf(under, vec_max<T>(rest));
                    if (TAIL) sum.add(approx_sum(rest, m));
                }
            }
            if (waiting) drain(waiting, j0);
            const uint64_t w = warp_sum_u64(above);
            if (lane == 0) s.region[j0 / depth] = w;
            f.above += above;
            above = 0;
        }
        if (TAIL) f.tail = fixed_of(sum.hi + sum.lo);
        f.below = __syncthreads_or(under > -INFINITY);
        f.above = block_sum(f.above);
        f.n_above = (int)block_sum((uint64_t)f.n_above);
        f.tail = TAIL ? block_sum(f.tail) : 0;
        f.slack = TAIL ? slack_of(f.tail, 17) : 0;
        return f;
    }
    // The approximate mass of what is below `lo` once more, off by 2^-20 of itself at most:
    // the exponent in two floats leaves ex2's 2^-22, the product's and the additions' 2^-24.
    // (It decides five of six nuclei that the first sum leaves open; the exact one, for the
    // sixth, takes three times as long.)
    __device__ __forceinline__ void finer_tail(float lo, Found& f) {
        Sum sum;
        each([&](const uint4& q, int) {
            float v[PV], t = 0.f;
            unpack<T>(cleared<T>(q, mask_from<T>(q, lo)), v);
#pragma unroll
            for (int e = 0; e < PV; ++e) {
                float d_lo;
                const float d = gap(v[e], m, d_lo), y = d * sc.c;
                const float y_lo = fmaf(d_lo, sc.c, fmaf(d, sc.c_lo, fmaf(d, sc.c, -y)));
                const float w = ex2(-y);
                t += y < 126.f ? fmaf(w, y_lo * -0.693147181f, w) : 0.f;
            }
            sum.add(t);
        });
        f.tail = block_sum(fixed_of(sum.hi + sum.lo));
        f.slack = slack_of(f.tail, 20);
    }
    // The exact one.
    __device__ __forceinline__ void exact_tail(float lo, Found& f) {
        f.tail = 0;
        each([&](const uint4& q, int) {
            const uint4 rest = cleared<T>(q, mask_from<T>(q, lo));
#pragma unroll 2
            for (int e = 0; e < PV; ++e) f.tail += mass_of(element<T>(rest, e));
        });
        f.tail = block_sum(f.tail);
        f.slack = 0;
    }
    __device__ __forceinline__ int bin_of(float v, float per) const {
        return (int)fminf((base - v) * per, (float)kBins);
    }

    // Sorts n <= NT Q entries (the array holds as many): Q a thread in its registers, a
    // comparison's other side in them too, or another lane's, or (32 Q and more entries
    // away) in shared memory.  A list of 2048: 24 us with all of them in shared memory.
    template <int Q, typename E, bool FALLING> __device__ __forceinline__ void sort(E* v, int n) {
        E e[Q];
#pragma unroll
        for (int i = 0; i < Q; ++i)
            e[i] = tid * Q + i < n ? v[tid * Q + i] : FALLING ? (E)0 : ~(E)0;
        int size = 2;
        while (size < n) size *= 2;
        const bool in = warp * 32 * Q < size;
#pragma unroll 1
        for (int k = 2; k <= size; k *= 2) {
            // entry i takes the larger or the smaller of itself and the one `j` away
            auto take = [&](int i, int j, E other) {
                const int p = tid * Q + i;
                const bool larger = (((p & k) == 0) == FALLING) == ((p & j) == 0);
                if ((e[i] > other) != larger) e[i] = other;
            };
            int j = k / 2;
#pragma unroll 1
            for (; j >= 32 * Q; j /= 2) {
                __syncthreads();
                if (in)
#pragma unroll
                    for (int i = 0; i < Q; ++i) v[i * NT + tid] = e[i];
                __syncthreads();
                if (in)
#pragma unroll
                    for (int i = 0; i < Q; ++i) take(i, j, v[i * NT + (tid ^ (j / Q))]);
            }
            if (in) {
#pragma unroll 1
                for (; j >= Q; j /= 2)
#pragma unroll
                    for (int i = 0; i < Q; ++i) take(i, j, __shfl_xor_sync(0xffffffffu, e[i], j / Q));
#pragma unroll
                for (int h = Q / 2; h >= 1; h /= 2)
                    if (h < k)
#pragma unroll
                        for (int i = 0; i < Q; ++i)
                            if (!(i & h)) {
                                const E a = e[i], b = e[i | h];
                                take(i, h, b);
                                take(i | h, h, a);
                            }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Q; ++i)
            if (tid * Q + i < n) v[tid * Q + i] = e[i];
        __syncthreads();
    }

    // Sorts the orders by id: of more than 32, or of a warp's list.
    template <int G, int Q> __device__ __forceinline__ void sort_ids(int n) {
        if constexpr (G > 32) {
            __syncthreads();
            sort<Q, uint32_t, false>(s.order, n);
        } else {
            __syncwarp();
            const uint32_t mine = lane < n ? s.order[lane] : ~0u;
            int rank = 0;
            for (int k = 0; k < n; ++k) rank += s.order[k] < mine;
            __syncwarp();
            if (lane < n) s.order[rank] = mine;
            __syncwarp();
        }
    }

    // Sorts the list by counting, for each entry, the larger ones: two threads an entry, n
    // at most NT / 2.  (A list of 256: 2 us less than by sort().)
    __device__ __forceinline__ void sort_by_rank(int n) {
        const int i = tid >> 1;
        const uint64_t mine = i < n ? s.list[i] : 0;
        int rank = 0;
        if (i < n)
            for (int k = tid & 1; k < n; k += 2) rank += s.list[k] > mine;
        rank += __shfl_xor_sync(0xffffffffu, rank, 1);
        __syncthreads();
        if (i < n && !(tid & 1)) s.list[rank] = mine;
        __syncthreads();
    }

    // From the list of n: every filter's place, the kept tokens and, where they are all
    // listed, the draw.  By G threads, Q entries each.  f: what is before and behind the
    // list; `floor`: no token behind it has min_p; `known`: the mass of the first top_k,
    // whose place is not looked for again.
    template <int G, int Q>
    __device__ __forceinline__ void decide(int n, const Found& f, bool floor, uint64_t known, int top_k,
                           float top_p, bool draw, float u) {
        if constexpr (Q > 1) sort<Q, uint64_t, true>(s.list, n);  // (else it is sorted)
        // masses and their prefix sums, Q entries a thread
        uint64_t e[Q], own = 0;
        int big = 0;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const int p = tid * Q + i;
            const float v = p < n ? of_key((uint32_t)(s.list[p] >> 32)) : -INFINITY;
            e[i] = p < n ? mass_of(v) : 0;
            if (p < n) s.mass[p] = e[i];
            own += e[i];
            big += by_min && p < n && has_min(v);
        }
        uint64_t listed;
        const uint64_t before = f.above + group_scan<G>(own, listed);
        listed += f.above;
        const int A = f.n_above + n, kNone = INT_MAX;
        const int big_n = (int)group_sum<G>((uint64_t)big);
        const int pos_k = known ? kNone : top_k > 0 && top_k <= A ? top_k : f.below ? kNone : A;
        const int pos_m = !by_min || (big_n == n && f.below && !floor) ? kNone : f.n_above + big_n;
        int kept = min(pos_k, pos_m), what = kDone;
        // (known: those behind the first top_k are not kept; here they are behind the place)
        if (pos_k <= f.n_above || (by_min && big_n == 0 && f.n_above > 0 && !floor)) {
            what = kSearch;  // a place is among those above
        } else if (top_p < 1.f) {
            uint64_t w0, w1;  // the mass that top_p is a share of, at least and at most
            if (known) {
                w0 = w1 = known;
            } else if (pos_k != kNone) {
                const int last = pos_k - f.n_above - 1;
                if (last / Q == tid) {
                    uint64_t w = before;
#pragma unroll
                    for (int i = 0; i < Q; ++i)
                        if (i <= last % Q) w += e[i];
                    s.value = w;
                }
                sync<G>();
                w0 = w1 = s.value;
                if (tid == 0) s.dec.all = w0, s.dec.listed = 0;
            } else {
                w0 = listed + (f.tail > f.slack ? f.tail - f.slack : 0);
                w1 = listed + f.tail + f.slack;
            }
            const uint64_t g0 = max(share_of(w0, top_p, true), (uint64_t)1);
            const uint64_t g1 = max(share_of(w1, top_p, true), (uint64_t)1);
            // how many prefix sums stay below either goal
            uint64_t cum = before;
            int n0 = 0, n1 = 0;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                cum += e[i];
                if (tid * Q + i < n) n0 += cum < g0, n1 += cum < g1;
            }
            const uint64_t both = group_sum<G>((uint64_t)n0 << 32 | (uint32_t)n1);
            const int p0 = min(kept, f.n_above + (int)(both >> 32) + 1);
            const int p1 = min(kept, f.n_above + (int)(uint32_t)both + 1);
            if (top_k > 0 && pos_k == kNone && !known) what = kSearch;
            else if (f.n_above > 0 && f.above >= g0) what = top_k > 0 && !known ? kAbove : kSearch;
            else if (p1 > A) what = kBracket;
            else if (p0 != p1) what = kExactTail;
            kept = p0;
        } else if (kept == kNone) {
            what = kSearch;
        }
        if (what == kDone) {
            const int here = kept - f.n_above;  // kept entries of the list
            uint64_t w = 0;
#pragma unroll
            for (int i = 0; i < Q; ++i)
                if (tid * Q + i < here) w += e[i];
            const uint64_t all = f.above + group_sum<G>(w);
            if (draw && f.n_above == 0) {
                // the kept tokens by id, and the first whose prefix sum passes the goal
                const uint64_t goal = share_of(all, u < 1.f ? u : 0.f, false);
                if (tid == 0) s.token = u >= 1.f ? here - 1 : 0;
                sync<G>();
                if (here <= 128 && u >= 0.f && u < 1.f) {
                    // each entry's mass before it, straight
                    for (int i = tid; i < here; i += G) {
                        const uint32_t id = ~(uint32_t)s.list[i];
                        uint64_t at = 0;
                        for (int k = 0; k < here; ++k)
                            if (~(uint32_t)s.list[k] < id) at += s.mass[k];
                        if (at <= goal && goal < at + s.mass[i]) s.order[0] = id << kPlaceBits, s.token = 0;
                    }
                } else {
                    for (int i = tid; i < here; i += G)
                        s.order[i] = ~(uint32_t)s.list[i] << kPlaceBits | (uint32_t)i;
                    sort_ids<G, Q>(here);
                    uint64_t o[Q], sum = 0, every;
#pragma unroll
                    for (int i = 0; i < Q; ++i) {
                        const int p = tid * Q + i;
                        o[i] = p < here ? s.mass[s.order[p] & (kList - 1)] : 0;
                        sum += o[i];
                    }
                    uint64_t at = group_scan<G>(sum, every);
                    if (u >= 0.f && u < 1.f && at <= goal && goal < at + sum) {
                        int hit = 0;
#pragma unroll
                        for (int i = 0; i < Q; ++i) {
                            at += o[i];
                            hit += at <= goal;
                        }
                        s.token = tid * Q + hit;
                    }
                }
                sync<G>();
            }
            if (tid == 0) {
                const uint64_t entry = here ? s.list[here - 1] : 0;
                s.dec.cut = here ? of_key((uint32_t)(entry >> 32)) : above_from;
                s.dec.limit = here ? (int)~(uint32_t)entry : INT_MAX;
                s.dec.kept = kept;
                s.dec.all = all;
                s.dec.token = draw && f.n_above == 0 ? (int)(s.order[s.token] >> kPlaceBits) : -1;
            }
            if (draw && f.n_above > 0)  // the list's part of the regions' masses
                for (int i = tid; i < here; i += G)
                    atomicAdd(reinterpret_cast<unsigned long long*>(
                                  &s.region[((int)~(uint32_t)s.list[i] + off) / PV / depth]),
                              (unsigned long long)s.mass[i]);
        } else if (tid == 0 && what == kBracket) {
            s.dec.all = listed + f.tail;
            s.dec.listed = f.n_above == 0 ? listed : 0;
        }
        if (tid == 0) s.dec.what = what;
    }
    // The same by as few threads as the list needs (what the others would do takes issue
    // slots from the SM's other block).
    __device__ __forceinline__ void decide_by(int n, const Found& f, bool floor, uint64_t known, int top_k,
                              float top_p, bool draw, float u) {
        __syncthreads();
        if (n <= NT / 2) sort_by_rank(n);
        else if (n <= NT) sort<1, uint64_t, true>(s.list, n);
        if (n <= 32) {
            if (warp == 0) decide<32, 1>(n, f, floor, known, top_k, top_p, draw, u);
        } else if (n <= NT) {
            decide<NT, 1>(n, f, floor, known, top_k, top_p, draw, u);
        } else if (n <= 2 * NT) {
            decide<NT, 2>(n, f, floor, known, top_k, top_p, draw, u);
        } else {
            decide<NT, kList / NT>(n, f, floor, known, top_k, top_p, draw, u);
        }
        __syncthreads();
    }

    // The first token alone: the largest entry of the list.
    __device__ __forceinline__ int first_alone() {
        uint64_t best = 0;
        for (int i = tid; i < s.count; i += NT) best = max(best, s.list[i]);
        const uint32_t key = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
        const uint32_t id =
            __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == key ? (uint32_t)best : 0u);
        __syncthreads();
        if (lane == 0) s.part[warp] = (uint64_t)key << 32 | id;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int i = 0; i < kWarps; ++i) best = max(best, s.part[i]);
            s.dec.cut = m;
            s.dec.limit = s.dec.token = (int)~(uint32_t)best;
            s.dec.kept = 1;
            s.dec.all = 1ull << (62 - sc.shift);
        }
        __syncthreads();
        return kDone;
    }

    // Leaves of a list of n, an entry a thread, the largest k and what equals the k-th.
    __device__ __forceinline__ int prune(int n, int k, Found& f) {
        const uint64_t mine = tid < n ? s.list[tid] : 0;
        const uint32_t key = (uint32_t)(mine >> 32);
        uint32_t t = 0;
        // (of bf16 the lower halves are alike)
        for (uint32_t bit = 1u << 31; bit >= (sizeof(T) == 2 ? 1u << 16 : 1u); bit >>= 1)
            if (__syncthreads_count(key >= (t | bit)) >= k) t |= bit;
        const bool in = key >= t && tid < n;
        const uint32_t w = __ballot_sync(0xffffffffu, in);
        if (lane == 0) s.part[warp] = __popc(w);
        __syncthreads();
        int at = __popc(w & ((1u << lane) - 1)), all = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            at += i < warp ? (int)s.part[i] : 0;
            all += (int)s.part[i];
        }
        if (in) s.list[at] = mine;
        f.below |= all < n;
        __syncthreads();
        return all;
    }
    // A logit that `want` entries of a full list reach.
    __device__ __forceinline__ float higher(int want) {
        uint32_t t = 0;
#pragma unroll 1
        for (uint32_t bit = 1u << 31; bit >= (sizeof(T) == 2 ? 1u << 16 : 1u); bit >>= 1) {
            int n = 0;
            for (int i = tid; i < kList; i += NT) n += (uint32_t)(s.list[i] >> 32) >= (t | bit);
            if ((int)block_sum((uint64_t)n) >= want) t |= bit;
        }
        return of_key(t | (sizeof(T) == 2 && !(t >> 31) ? 0xFFFFu : 0u));
    }
    // Whether a nucleus is certain to reach past the list.
    __device__ __forceinline__ bool past(int n, const Found& f, float top_p) {
        uint64_t w = 0;
#pragma unroll 1
        for (int i = tid; i < n; i += NT) w += mass_of(of_key((uint32_t)(s.list[i] >> 32)));
        w = block_sum(w);
        if (w >= share_of(w + (f.tail > f.slack ? f.tail - f.slack : 0), top_p, true)) return false;
        if (tid == 0) s.dec.all = w + f.tail, s.dec.listed = w;
        __syncthreads();
        return true;
    }
    // Decides by a list of the tokens from `lo` on, behind those from `hi` on, with the
    // rest's mass made exact where that is needed.  (f: of a list that is there; else it is
    // made.)
    __device__ __forceinline__ int settle(const Found* made, float hi, float lo, bool floor, uint64_t known,
                          int top_k, float top_p, bool draw, float u) {
        const bool tail = top_p < 1.f && top_k <= 0;
        __syncthreads();
        Found f = made ? *made : tail ? collect<true>(hi, lo) : collect<false>(hi, lo);
        int n = s.count;
        above_from = hi;
        if (n > kList || (n == 0 && !(floor && f.n_above > 0))) {
            if (tid == 0) s.dec.all = f.tail, s.dec.listed = f.above;
            __syncthreads();
            return kOverflow;
        }
        if (made && top_k > 0 && n > top_k && n > 64 && n <= NT) n = prune(n, top_k, f);
        if (made && tail && n > NT / 4 && !by_min && past(n, f, top_p)) return kBracket;
        for (int more = 0;; ++more) {
            if (more == 1) finer_tail(lo, f);
            else if (more == 2) exact_tail(lo, f);
            decide_by(n, f, floor, known, top_k, top_p, draw, u);
            if (s.dec.what != kExactTail) return s.dec.what;
        }
    }

    // ------------------------------------------------------------ the bracket
    // A histogram over bins of the logit from `base` down, each token in them weighing one
    // (COUNT) or its approximate mass in units.  Left are the bins that hold the place where
    // the weights pass the goal, which may be off by `slack`.  SAMPLE: of a quarter of the
    // row; the place is also where the weight from below, what is past the bins with it,
    // passes `tail`, and the better known of the two is taken.  (A nucleus of 0.95 that
    // is 12000 tokens of 128256: a bracket of 500 tokens from below, 7300 from above.)
    struct Aim {
        uint64_t goal, slack, tail;
    };
    template <bool COUNT, bool SAMPLE>
    __device__ __forceinline__ void histogram(float per, float unit, const Aim& aim) {
        // (every thread has read the bins that the last one left: which way row() goes on
        // hangs on them)
        __syncthreads();
        for (int i = tid; i < kBins; i += NT) s.order[i] = 0;
        if (tid == 0) s.dec.bin0 = 0, s.dec.bin1 = kBins - 1;
        __syncthreads();
        // (from a list's or bracket's edge down: those at it are before)
        const float edge = base < m ? base : INFINITY;
        Sum past;
        auto count = [&](const uint4& q, int) {
            if (bin_of(vec_max<T>(q), per) >= kBins) {
                if (SAMPLE) past.add(approx_sum(q, m));
                return;
            }
            float v[PV];
            unpack<T>(q, v);
#pragma unroll
            for (int e = 0; e < PV; ++e) {
                const int b = bin_of(v[e], per);
                if (b < kBins && v[e] < edge)
                    atomicAdd(&s.order[b], COUNT ? 1u : __float2uint_rn(approx(v[e]) * unit));
                else if (SAMPLE && b >= kBins)
                    past.add(approx(v[e]));
            }
        };
        if (SAMPLE) {
            for (int j0 = warp * depth; j0 < nvec; j0 += kWarps * depth)
                for (int j = j0 + lane; j < min(nvec, j0 + sampled()); j += 32) count(vec(j), 0);
        } else {
            each(count);
        }
        __syncthreads();
        constexpr int Q = kBins / NT;
        uint64_t w[Q], sum = 0, all, goal = aim.goal, slack = aim.slack;
#pragma unroll
        for (int i = 0; i < Q; ++i) sum += w[i] = s.order[tid * Q + i];
        uint64_t cum = block_scan(sum, all);
        if (SAMPLE) {
            // some deviations of the sampled weight up to the place, or from it on: the root
            // of the sum of its tokens' squares
            uint64_t squares = 0, every;
#pragma unroll
            for (int i = 0; i < Q; ++i)
                squares += w[i] * (uint64_t)(approx(base - ((float)(tid * Q + i) + 0.5f) / per) * unit);
            const uint64_t before = block_scan(squares, every);
            const uint64_t beyond = block_sum(__float2ull_rn((past.hi + past.lo) * unit));
            const uint64_t from = all + beyond > aim.tail ? all + beyond - aim.tail : 0;
            if (tid == 0) s.region[0] = every, s.region[1] = 0;
            __syncthreads();
            if (cum < goal && cum + sum >= goal) s.region[0] = before + squares;
            if (cum < from && cum + sum >= from) s.region[1] = before;
            __syncthreads();
            const uint64_t last = (uint64_t)(approx(base - (float)kBins / per) * unit);
            const uint64_t above = s.region[0], below = every - s.region[1] + beyond * last;
            if (below < above) goal = from;
            slack += (uint64_t)(2.5f * sqrtf((float)min(above, below)));
        }
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const uint64_t after = cum + w[i];
            if (cum + slack < goal && after + slack >= goal) s.dec.bin0 = tid * Q + i;
            if (cum < goal + slack && after >= goal + slack) s.dec.bin1 = tid * Q + i;
            cum = after;
        }
        if (tid == 0 && goal > all + slack) s.dec.bin0 = kBins;  // (past them all)
        __syncthreads();
    }
    // Vectors of a region that are a sample.
    __device__ __forceinline__ int sampled() const { return min(depth, 64); }
    // For a nucleus, of which `whole` is all: bins down to the least logit that it can
    // reach.  Returns bins per unit of the logit.
    __device__ __forceinline__ float bracket(float top_p, uint64_t whole) {
        // tokens whose logit leaves them less than (1 - top_p) / V of the mass are out
        const float z = (float)whole * ldexpf(1.f, sc.shift - 62);
        const float reach = T_ * (logf((float)a.V / ((1.f - top_p) * z)) + 0.01f);
        const float per = (float)kBins / reach;
        base = m;
        // in units of 2^-30 of the mass: half a unit a token, and 2^-15
        histogram<false, false>(per, 1073741824.f / z,
                                Aim{(uint64_t)(top_p * 1073741824.f), (uint64_t)a.V / 2 + (1 << 15) + 2, 0});
        return per;
    }
    // The same behind a list of the tokens from `lo` on, of mass `listed`, by a quarter of
    // the rest.  0 if there are none.
    __device__ __forceinline__ float bracket_rest(float top_p, uint64_t whole, uint64_t listed, float lo) {
        const float one = ldexpf(1.f, sc.shift - 62), z = (float)whole * one;
        const float rest = (float)(whole - listed) * one, need = top_p * z - (float)listed * one;
        const float reach = T_ * (logf((float)a.V / ((1.f - top_p) * z)) + 0.01f) - (m - lo);
        if (!(reach > 0.f) || !(need > 0.f) || !(need < rest)) return 0.f;
        const float per = (float)kBins / reach, unit = 1073741824.f / rest;
        base = lo;
        const int n = nvec / depth * sampled() + min(nvec % depth, sampled());
        const float part = unit * (float)n / (float)nvec;
        histogram<false, true>(per, unit, Aim{(uint64_t)(need * part), (uint64_t)a.V / 8 + 2,
                                              (uint64_t)((rest - need) * part)});
        return per;
    }

    // The same within logits of `hi` down to `lo`, with an exact mass `above` them and
    // `tail` behind.
    __device__ __forceinline__ float bracket_within(float top_p, uint64_t whole, uint64_t above,
                                                    uint64_t tail, float hi, float lo) {
        const float one = ldexpf(1.f, sc.shift - 62);
        const float here = (float)(whole - min(whole, above + tail)) * one;
        const float need = top_p * ((float)whole * one) - (float)above * one;
        const float per = ((float)kBins - 0.1f) / (hi - lo);
        if (!(here > 0.f) || !(per > 0.f) || !(per < INFINITY)) return 0.f;
        const float unit = 1073741824.f / here;
        base = hi;
        // (off: what `whole` may be, in these units, and half a unit a token)
        const uint64_t off = (uint64_t)((float)whole * one * 0x1p-16f * unit);
        histogram<false, false>(per, unit, Aim{need > 0.f ? (uint64_t)(need * unit) : 0,
                                               (uint64_t)a.V / 2 + (1 << 14) + off, 0});
        return per;
    }
    // The logits that the bracket's bins end at, and a step beyond.
    __device__ __forceinline__ void edges(float per, float& hi, float& lo) const {
        const float step = 0.01f / per + (fabsf(m) + fabsf(base)) * 1e-6f;
        const float top = base - (float)s.dec.bin0 / per + step;
        const float end = base - (float)(s.dec.bin1 + 1) / per - step;
        hi = s.dec.bin0 == 0 && base == m ? INFINITY : up_to<T>(top);
        lo = down_to<T>(end);
    }

    // ------------------------------------------------------------ the search
    // The tokens from a key on: how many, their mass, and the least key among them; and the
    // largest key below.
    struct From {
        int n;
        uint64_t mass;
        uint32_t least, under;
    };
    template <bool MASS> __device__ __forceinline__ From from_key(uint32_t k) {
        From f{0, 0, ~0u, 0};
        each([&](const uint4& q, int) {
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < PV; ++e) {
                const uint32_t y = key_of(element<T>(q, e));
                if (y >= k) {
                    in |= 1u << e;
                    f.least = min(f.least, y);
                } else {
                    f.under = max(f.under, y);
                }
            }
            f.n += __popc(in);
            if (MASS)
                for (; in; in &= in - 1) f.mass += mass_of(element<T>(q, __ffs(in) - 1));
        });
        f.n = (int)block_sum((uint64_t)f.n);
        if (MASS) f.mass = block_sum(f.mass);
        const uint64_t ends = (uint64_t)__reduce_min_sync(0xffffffffu, f.least) << 32 |
                              (uint32_t)~__reduce_max_sync(0xffffffffu, f.under);
        __syncthreads();
        if (lane == 0) s.part[warp] = ends;
        __syncthreads();
        f.least = ~0u;
        f.under = 0;
        for (int i = 0; i < kWarps; ++i) {
            f.least = min(f.least, (uint32_t)(s.part[i] >> 32));
            f.under = max(f.under, ~(uint32_t)s.part[i]);
        }
        return f;
    }
    __device__ __forceinline__ int count_from(uint32_t k) { return from_key<false>(k).n; }
    // The largest key in lo .. hi from which on the tokens are `goal`, in number or mass
    // (from lo on they are): bisection, each time to a key that is there.
    template <bool MASS>
    __device__ __forceinline__ uint32_t last_key(uint32_t lo, uint32_t hi, uint64_t goal) {
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo + 1) / 2;
            const From f = from_key<MASS>(mid);
            if ((MASS ? f.mass : (uint64_t)f.n) >= goal) lo = f.least;
            else hi = max(lo, f.under);
        }
        return lo;
    }
    // The place of the n-th token.
    struct Place {
        uint32_t key;
        int ties, n;  // of those at the key
    };
    __device__ __forceinline__ Place place(uint32_t top, int n) {
        const uint32_t k = last_key<false>(kKeyNone + 1, top, (uint64_t)n);
        return Place{k, n - count_from(k + 1), n};
    }
    // Every filter's place by bisection; leaves cut, limit and kept.
    __device__ __forceinline__ void search(uint32_t top, int top_k, float top_p) {
        const uint32_t bottom = kKeyNone + 1;
        const int live = count_from(bottom);
        Place at{bottom, live, live};
        if (top_k > 0 && top_k < live) at = place(top, top_k);
        else at.ties = live - count_from(bottom + 1);
        int n = at.n;
        if (top_p < 1.f) {
            const uint64_t all =
                from_key<true>(at.key + 1).mass + mass_of(of_key(at.key)) * (uint64_t)at.ties;
            const uint64_t goal = max(share_of(all, top_p, true), (uint64_t)1);
            const uint32_t lo = last_key<true>(at.key, top, goal);
            const From f = from_key<true>(lo + 1);
            const uint64_t one = max(mass_of(of_key(lo)), (uint64_t)1);
            n = (int)min((uint64_t)n, (uint64_t)f.n + (goal - f.mass + one - 1) / one);
        }
        if (by_min) {
            uint32_t lo = bottom, hi = top;
            while (lo < hi) {  // the lowest logit that has min_p
                const uint32_t mid = lo + (hi - lo) / 2;
                if (has_min(of_key(mid))) hi = mid;
                else lo = mid + 1;
            }
            n = min(n, count_from(lo));
        }
        if (n < at.n) at = place(top, n);
        if (tid == 0) {
            s.dec.cut = of_key(at.key);
            s.dec.kept = at.n;
            s.dec.limit = INT_MAX;
        }
        __syncthreads();
        if (at.ties < count_from(at.key) - (at.n - at.ties)) tie_limit(at.key, at.ties);
    }
    // The id of the ties-th token at the key.
    __device__ __forceinline__ void tie_limit(uint32_t key, int ties) {
        auto equal = [&](const uint4& q) {
            float v[PV];
            unpack<T>(q, v);
            int n = 0;
#pragma unroll
            for (int e = 0; e < PV; ++e) n += key_of(v[e]) == key;
            return n;
        };
        int n = 0;
        each([&](const uint4& q, int) { n += equal(q); },
             [&](int region) {
                 const uint64_t w = warp_sum_u64((uint64_t)n);
                 if (lane == 0) s.region[region] = w;
                 n = 0;
             });
        uint64_t goal = (uint64_t)ties - 1;
        const int j = pick_region(goal) * depth + tid;
        const bool there = tid < depth && j < nvec;
        const uint4 q = there ? vec(j) : uint4();
        const int mine = there ? equal(q) : 0;
        uint64_t all;
        uint64_t before = block_scan((uint64_t)mine, all);
        if (before <= goal && goal < before + mine) {
            float v[PV];
            unpack<T>(q, v);
#pragma unroll
            for (int e = 0; e < PV; ++e)
                if (key_of(v[e]) == key && before++ == goal) s.dec.limit = id_of(j) + e;
        }
        __syncthreads();
    }
    // The region whose sum, added to those before, passes the goal; less what is before.
    __device__ __forceinline__ int pick_region(uint64_t& goal) {
        const int n = (nvec + depth - 1) / depth;
        constexpr int Q = (kRegions + NT - 1) / NT;
        __syncthreads();
        if (tid == 0) s.token = n - 1, s.value = 0;
        uint64_t w[Q], sum = 0, all;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            w[i] = tid * Q + i < n ? s.region[tid * Q + i] : 0;
            sum += w[i];
        }
        uint64_t at = block_scan(sum, all);
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            if (at <= goal && goal < at + w[i]) s.token = tid * Q + i, s.value = at;
            at += w[i];
        }
        __syncthreads();
        goal -= s.value;
        return s.token;
    }

    // ------------------------------------------------------------ the draw
    __device__ __forceinline__ bool is_kept(float v, int id) const {
        return v > s.dec.cut || (v == s.dec.cut && id <= s.dec.limit);
    }
    // The kept tokens' number, and their masses by region.
    __device__ __forceinline__ void weigh(bool draw) {
        uint64_t w = 0, all = 0;
        int n = 0;
        each(
            [&](const uint4& q, int j) {
                float v[PV];
                unpack<T>(q, v);
#pragma unroll
                for (int e = 0; e < PV; ++e) n += is_kept(v[e], id_of(j) + e);
                if (!draw) return;
#pragma unroll
                for (int e = 0; e < PV; ++e)
                    if (is_kept(v[e], id_of(j) + e)) w += mass_of(v[e]);
            },
            [&](int region) {
                if (!draw) return;
                const uint64_t r = warp_sum_u64(w);
                if (lane == 0) s.region[region] = r;
                all += w;
                w = 0;
            });
        n = (int)block_sum((uint64_t)n);
        all = block_sum(all);
        if (tid == 0) s.dec.kept = n, s.dec.all = all;
        __syncthreads();
    }
    // The token of u, from the kept masses by region.
    __device__ __forceinline__ int find(float u) {
        if (!(u >= 0.f && u < 1.f)) {  // the last kept, or the first
            __syncthreads();
            if (tid == 0) s.token = u >= 1.f ? -1 : INT_MAX;
            __syncthreads();
            each([&](const uint4& q, int j) {
                float v[PV];
                unpack<T>(q, v);
#pragma unroll
                for (int e = 0; e < PV; ++e)
                    if (is_kept(v[e], id_of(j) + e)) {
                        if (u >= 1.f) atomicMax(&s.token, id_of(j) + e);
                        else atomicMin(&s.token, id_of(j) + e);
                    }
            });
            __syncthreads();
            return s.token;
        }
        uint64_t goal = share_of(s.dec.all, u, false);
        const int j = pick_region(goal) * depth + tid;
        const bool in = tid < depth && j < nvec;
        const uint4 q = in ? vec(j) : uint4();
        uint64_t w = 0, all;
        if (in)
#pragma unroll 1
            for (int e = 0; e < PV; ++e)
                if (is_kept(element<T>(q, e), id_of(j) + e)) w += mass_of(element<T>(q, e));
        uint64_t at = block_scan(w, all);
        if (in && at <= goal && goal < at + w)
#pragma unroll 1
            for (int e = 0; e < PV; ++e)
                if (is_kept(element<T>(q, e), id_of(j) + e)) {
                    const uint64_t after = at + mass_of(element<T>(q, e));
                    if (at <= goal && goal < after) s.token = id_of(j) + e;
                    at = after;
                }
        __syncthreads();
        return s.token;
    }

    // ------------------------------------------------------------ a row
    __device__ __forceinline__ void write_filtered(int64_t r, bool none) {
        T* o = static_cast<T*>(a.out.filtered) + r * a.V;
        each([&](const uint4& q, int j) {
            const int id = id_of(j);
            float v[PV];
            unpack<T>(q, v);
            T e[PV];
            memcpy(e, &q, 16);
#pragma unroll
            for (int i = 0; i < PV; ++i)
                if (none || !is_kept(v[i], id + i)) e[i] = none_of<T>();
            if (a.same_align && id >= 0 && id + PV <= a.V) {
                uint4 p;
                memcpy(&p, e, 16);
                *reinterpret_cast<uint4*>(o + id) = p;
            } else {
#pragma unroll
                for (int i = 0; i < PV; ++i)
                    if (id + i >= 0 && id + i < a.V) o[id + i] = e[i];
            }
        });
    }

    // Row r; the first thread has the next one's number, all get it back.
    __device__ __forceinline__ int row(int64_t r, int ticket, const T* logits) {
        const vsd_policy& p = a.policy;
        T_ = p.row_T ? p.row_T[r] : p.T;
        float top_p = p.row_top_p ? p.row_top_p[r] : p.top_p;
        float min_p = p.row_min_p ? p.row_min_p[r] : p.min_p;
        int top_k = p.row_top_k ? p.row_top_k[r] : p.top_k;
        const float u = a.u ? a.u[r] : 0.f;
        const bool ok = (T_ == 0.f || (T_ >= kMinT && T_ <= kMaxT)) && top_p == top_p && min_p == min_p;
        const bool draw = a.u != nullptr;
        if (T_ == 0.f) top_k = 1, top_p = 1.f, min_p = 0.f, T_ = 1.f;  // the first token alone
        if (top_p <= 0.f) top_k = 1, top_p = 1.f;
        sc = exp_scale(T_, a.shift);
        c = sc.c;
        by_min = min_p > 0.f;
        far = far_lo = 0.f;
        if (by_min && min_p < 1.f) {
            float lo;
            const float l = neg_log(min_p, s.tab, lo);
            far = T_ * l;
            far_lo = fmaf(T_, lo, fmaf(T_, l, -far));
        }
        const bool filters = top_k > 0 || top_p < 1.f || by_min;
        const bool tail = top_p < 1.f && top_k <= 0;
        // what rounding may make of the logit that min_p ends at
        auto rounding = [&](float top) { return (far + fabsf(top) + T_) * 1e-5f; };

        constexpr int kRound = kWarps * 32 * kLoad;
        // one pass: the maximum, the list and the rest's mass.  After the first round of
        // vectors a bound `lo` that `want` of the lanes' maxima reach, and a reference for
        // the masses: the maximum so far.
        // (for a long row's k a share of it and some more; were they too few, a histogram
        // finds the place)
        const int rounds = (nvec + kRound - 1) / kRound;
        const int want = top_k <= 0    ? max(kWant / rounds, 16)
                         : rounds == 1 ? top_k
                                       : min(top_k, 3 * min(top_k, 1 << 16) / (2 * rounds) + 24);
        float mx = -INFINITY, lo = lowest_of<T>(), ref = 0.f;
        float under = -INFINITY;
        bool floor = false;
        Found f{0, 0, 0, 0, false};
        Sum sum;
        if (tid == 0) s.count = 0;
        for (int j1 = 0; j1 < nvec; j1 += kRound) {
            const int j0 = j1 + tid;
            uint4 q[kLoad];
            load<NT>(j0, nvec, q);
            if (j1 == 0 || !filters) {
#pragma unroll
                for (int i = 0; i < kLoad; ++i) mx = max_nan(mx, vec_max_nan<T>(q[i]));
                if (!filters) continue;
                const uint32_t key = key_of(mx), high = key >> 16;
                const uint32_t w = __reduce_max_sync(0xffffffffu, key);
                if (lane == 0) s.part[warp] = w;
                uint32_t t = 0;
                if (top_k != 1)
                    for (uint32_t bit = 0x8000u; bit; bit >>= 1)
                        if (__syncthreads_count(high >= (t | bit)) >= want) t |= bit;
                __syncthreads();
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) top = max(top, (uint32_t)s.part[i]);
                // (a value of the type: the halved keys of negative bf16 end in ones)
                const uint32_t ones = sizeof(T) == 2 && !(t & 0x8000u) ? 0xFFFFu : 0u;
                const uint32_t lo_key = top_k == 1 ? top : t << 16 | ones;
                ref = of_key(top);
                lo = lo_key <= (kKeyNone | 0xFFFFu) ? lowest_of<T>() : of_key(lo_key);
                if (by_min && top_p >= 1.f) {
                    // no token below max + T ln(min_p) is kept, and the maximum may grow
                    const float bound = ref - far - rounding(ref);
                    floor = top_k <= 0 || bound > lo;
                    if (floor) lo = down_to<T>(bound);
                }
            }
#pragma unroll
            for (int i = 0; i < kLoad; ++i) {
                const float most = vec_max_nan<T>(q[i]);
                mx = max_nan(mx, most);
                if (tail) list_vec<true>(q[i], most, j0 + NT * i, lo, ref, sum, under);
                else list_vec<false>(q[i], most, j0 + NT * i, lo, ref, sum, under);
            }
        }
        if (tid == 0) s.next = ticket;
        const bool bad = __syncthreads_or(!(mx < INFINITY));
        const int next = s.next;
        if (next < a.R) bring(logits + (int64_t)next * a.V);  // (while this row is decided)
        const uint32_t w = __reduce_max_sync(0xffffffffu, key_of(mx));
        if (lane == 0) s.part[warp] = w;
        __syncthreads();
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) top = max(top, (uint32_t)s.part[i]);
        const bool dead = bad || top <= kKeyNone;
        if (dead || !ok) {
            if (tid == 0) {
                atomicOr(a.status, (dead ? VSD_STATUS_BAD_ROW : 0) | (ok ? 0 : VSD_STATUS_BAD_PARAM));
                if (a.out.tokens) a.out.tokens[r] = -1;
                if (a.out.logq_tok) a.out.logq_tok[r] = NAN;
                if (a.out.kept) a.out.kept[r] = 0;
            }
            if (a.out.filtered) write_filtered(r, true);
            return next;
        }
        m = of_key(top);
        if (tid == 0) s.dec.token = -1, s.dec.cut = -FLT_MAX, s.dec.limit = INT_MAX;
        bool sums = !filters;  // whether the kept tokens' masses are still to be summed
        if (filters) {
            bool made = true;
            uint64_t whole = 0, listed = 0;  // of a nucleus past the first list
            if (tail) {
                // (where the reference was too far below: once more, relative to m)
                const float t = (sum.hi + sum.lo) * ex2((ref - m) * c);
                f.tail = fixed_of(t);
                made = !__syncthreads_or(!(t < 2e6f) || !(sum.hi < 1e30f) || !(ref > -INFINITY));
                f.tail = block_sum(f.tail);
                f.slack = slack_of(f.tail, 17);
            }
            f.below = __syncthreads_or(under > -INFINITY);
            // A list from `low` on, behind what is from `high` on, until one decides.  First the
            // one at hand (kFirst); where k or min_p overflows it, or min_p may come before a
            // nucleus past it, one around their place (kNear); for a nucleus past it one around
            // its place by a sample, then by all of the row (kRest, kRow), and within one that
            // overflows a narrower one.
            enum { kFirst, kNear, kRest, kRow };
            float high = INFINITY, low = lo, per;
            uint64_t known = 0;
            int what, step = kFirst, tries = 0;
            for (;; made = false) {
                what = step == kFirst && top_k == 1 && s.count <= kList
                           ? first_alone()
                           : settle(made ? &f : nullptr, high, low, floor, known, top_k, top_p, draw,
                                    u);
                if (what == kDone) break;
                if (step == kFirst && what == kOverflow && tail) {
                    // (a bound that a quarter of the entries at hand reach)
                    const float raised = higher(kList / 4);
                    if (tries++ == 2 || !(raised > lo)) break;
                    low = lo = raised;
                    continue;
                }
                if (step == kFirst && (what == kBracket ? by_min
                                                        : what != kAbove && (floor || top_k > 0))) {
                    step = kNear;
                    whole = what == kBracket ? s.dec.all : 0;
                    listed = s.dec.listed;
                    high = up_to<T>(m - far + rounding(m));
                    low = down_to<T>(m - far - rounding(m));
                    floor = floor || what == kBracket;
                    if (floor) continue;
                    // the k-th token: among those at hand, or past them
                    per = ((float)kBins - 0.1f) / ((m - lo) * (what == kOverflow ? 1.f : 3.f));
                    if (!(per > 0.f && per < INFINITY)) break;
                    base = m;
                    histogram<true, false>(per, 0.f, Aim{(uint64_t)top_k, 0, 0});
                    if (s.dec.bin0 >= kBins) break;
                    edges(per, high, low);
                    continue;
                }
                if (step < kRest) {
                    if (what == kBracket || what == kAbove) whole = s.dec.all, listed = s.dec.listed;
                    if (!whole) break;
                    floor = false;
                    known = what == kAbove ? whole : 0;
                    step = kRest;
                    tries = 0;
                    per = listed && !known ? bracket_rest(top_p, whole, listed, lo) : 0.f;
                    if (per > 0.f && s.dec.bin0 < kBins) {
                        edges(per, high, low);
                        continue;
                    }
                } else if (what == kOverflow && s.count > kList && tries++ < 3) {
                    per = bracket_within(top_p, whole, s.dec.listed, s.dec.all, fminf(high, m), low);
                    if (per > 0.f && s.dec.bin0 < kBins) {
                        const float was_high = high, was_low = low;
                        edges(per, high, low);
                        high = fminf(high, was_high);
                        low = fmaxf(low, was_low);
                        continue;
                    }
                }
                if (step == kRow) break;
                step = kRow;
                tries = 0;
                per = bracket(top_p, whole);
                if (s.dec.bin0 >= kBins) break;
                edges(per, high, low);
            }
            if (what != kDone) {
                search(top, top_k, top_p);
                if (tid == 0) s.dec.token = -1;
                sums = true;
            }
        }
        __syncthreads();
        if (sums) weigh(draw);
        __syncthreads();
        if (draw) {
            const int id = s.dec.token >= 0 ? s.dec.token : find(u);
            if (tid == 0) {
                if (a.out.tokens) a.out.tokens[r] = id;
                if (a.out.logq_tok)
                    a.out.logq_tok[r] = log_share(float_of(x[id]), m, T_, s.dec.all, sc.shift, s.tab);
            }
        }
        if (tid == 0 && a.out.kept) a.out.kept[r] = s.dec.kept;
        if (a.out.filtered) write_filtered(r, false);
        return next;
    }
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 2)
    k_sample(const T* logits, const SampleArgs a) {
    using S = Sampler<T>;
    extern __shared__ __align__(128) unsigned char sample_smem[];
    typename S::Shared& s = *reinterpret_cast<typename S::Shared*>(sample_smem);
    S w(a, s);
    w.bring(logits + (int64_t)blockIdx.x * a.V);
    for (int j = threadIdx.x; j < kExpTab; j += kSampleThreads) s.tab[j] = exp_entry(kExpParts, j);
    // rows as blocks come to them: they take unlike times
    for (int64_t r = blockIdx.x; r < a.R;) {
        __syncthreads();
        w.open(logits + r * a.V);
        // (asked for here, looked at when the row has been read)
        int next = a.R;
        if (threadIdx.x == 0 && a.R > gridDim.x) next = (int)gridDim.x + atomicAdd(a.status + 1, 1);
        r = w.row(r, next, logits);
    }
}

}  // namespace

template <typename T>
cudaError_t sample(const void* logits, const SampleArgs& a, cudaStream_t st) {
    auto k = k_sample<T>;
    constexpr size_t smem = sizeof(typename Sampler<T>::Shared);
    const int blocks = blocks_per_sm((const void*)k, kSampleThreads, smem) * device_sm_count();
    if (blocks < 1) return cudaErrorInvalidConfiguration;
    k<<<std::min(blocks, a.R), kSampleThreads, smem, st>>>(static_cast<const T*>(logits), a);
    return cudaGetLastError();
}

}  // namespace vsd
