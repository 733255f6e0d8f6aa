// vsd_fixed.cuh -- exponentials as whole numbers: exp(-d / T) for d >= 0 in units
// of 2^-S, so that sums of them are exact and in any order the same, and decisions
// by them (which token a uniform number falls on, where a share of the mass is
// reached) are those of real arithmetic but near a border: a mass is within 2^-41 of
// itself and one unit (half of it by rounding, the rest by squares of the remainder's
// lower half, left out), so a sum of V within 2^-41 of itself and V units.
//
//   y = d log2(e) / T in two floats,  y = n + j / 2048 + r,  |r| <= 2^-12,
//   2^-y = 2^-n 2^-(j / 2048) (1 - z),  z = 1 - 2^-r = a - a^2/2 + a^3/6, a = r ln 2
//   (a in two floats; their cross term counts).
//
// 2^-(j / 2048) comes from a table of 2048 words (made of 32 + 64 constants), z is
// at most 2^-12.5 and known to some 2^-44.
#pragma once

#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

namespace vsd {

// 2^-(num / den) in units of 2^-62, 0 <= num < den, to the nearest: the exponential
// series in 2^-63.
constexpr uint64_t exp2_frac(int num, int den) {
    // x = (num / den) ln 2 in 2^-63
    const unsigned __int128 ln2 = 6393154322601327830ull;  // ln 2 in 2^-63
    const unsigned __int128 x = (ln2 * (unsigned)num + (unsigned)den / 2) / (unsigned)den;
    const unsigned __int128 one = (unsigned __int128)1 << 63;
    unsigned __int128 term = one, plus = one, minus = 0;
    for (int i = 1; i < 30; ++i) {
        term = ((term * x >> 63) + (unsigned)i / 2) / (unsigned)i;
        if (i & 1) minus += term;
        else plus += term;
    }
    return (uint64_t)((plus - minus + 1) >> 1);
}
struct ExpParts {
    uint64_t hi[32];  // 2^-(i / 32)
    uint64_t lo[64];  // 2^-(i / 2048)
};
constexpr ExpParts make_exp_parts() {
    ExpParts p{};
    for (int i = 0; i < 32; ++i) p.hi[i] = exp2_frac(i, 32);
    for (int i = 0; i < 64; ++i) p.lo[i] = exp2_frac(i, 2048);
    return p;
}

constexpr int kExpTab = 2048;

// 2^-(j / 2048) in units of 2^-62 from the parts.
__host__ __device__ __forceinline__ uint64_t exp_entry(const ExpParts& p, int j) {
    const uint64_t a = p.hi[j >> 6], b = p.lo[j & 63];
#ifdef __CUDA_ARCH__
    const uint64_t h = __umul64hi(a, b), l = a * b;
#else
    const unsigned __int128 w = (unsigned __int128)a * b;
    const uint64_t h = (uint64_t)(w >> 64), l = (uint64_t)w;
#endif
    return (h << 2 | l >> 62) + (l >> 61 & 1);
}

// log2(e) / T in two floats, and the units of the sums.
struct ExpScale {
    float c, c_lo;
    int shift;  // units of 2^-(62 - shift)
};
// The shift whose sums over V terms stay below 2^62 (at least 2^-50 to a unit: finer
// than the exponentials are known).
__host__ __device__ __forceinline__ int exp_shift(int V) {
    int s = 0;
    while (s < 30 && (1 << s) < V) ++s;
    return s < 12 ? 12 : s;
}
#ifdef __CUDA_ARCH__
#define VSD_ADD(a, b) __fadd_rn(a, b)
#define VSD_MUL(a, b) __fmul_rn(a, b)
#define VSD_FMA(a, b, c) __fmaf_rn(a, b, c)
#else
#define VSD_ADD(a, b) ((float)((a) + (b)))
#define VSD_MUL(a, b) ((float)((a) * (b)))
#define VSD_FMA(a, b, c) fmaf(a, b, c)
#endif

// n / T in two floats, n given in two.
__host__ __device__ __forceinline__ void over(float n, float n_lo, float T, float& hi, float& lo) {
    hi = n / T;
    lo = VSD_FMA(-hi, T, n);
    lo = VSD_ADD(lo, n_lo) / T;
}
__host__ __device__ __forceinline__ ExpScale exp_scale(float T, int shift) {
    ExpScale s;
    over(1.44269502162933349609375f, 1.92596299e-8f, T, s.c, s.c_lo);  // log2(e)
    s.shift = shift;
    return s;
}
// m - x in two floats.
__host__ __device__ __forceinline__ float gap(float x, float m, float& lo) {
    const float d = VSD_ADD(m, -x), b = VSD_ADD(d, -m);
    lo = VSD_ADD(VSD_ADD(m, -VSD_ADD(d, -b)), -VSD_ADD(x, b));
    return d;
}

// exp((x - m) / T) in units of 2^-(62 - shift), to the nearest; x <= m.
__host__ __device__ __forceinline__ uint64_t exp_fixed(float x, float m, const ExpScale& s,
                                                       const uint64_t* tab) {
    float e;
    const float d = gap(x, m, e);
    const float y = VSD_MUL(d, s.c);
    if (!(y < 63.f)) return 0;  // (and where m - x is past a float's range)
    const float yl = VSD_FMA(e, s.c, VSD_FMA(d, s.c_lo, VSD_FMA(d, s.c, -y)));
    // 6144 has its last bit at 2^-11
    const float t = VSD_ADD(y, 6144.f);
#ifdef __CUDA_ARCH__
    const int at = __float_as_int(t) - __float_as_int(6144.f);
#else
    const int at = (int)((t - 6144.f) * 2048.f);
#endif
    const float r = VSD_ADD(y, -VSD_ADD(t, -6144.f));
    const float kLn2 = 0.693147182464599609375f, kLn2Lo = -1.904654300e-9f;
    const float a = VSD_MUL(r, kLn2);
    float al = VSD_FMA(yl, kLn2, VSD_FMA(r, kLn2Lo, VSD_FMA(r, kLn2, -a)));
    al = VSD_FMA(a, VSD_FMA(a, VSD_FMA(a, 0.16666667f, -0.5f), -al), al);
    // z in units of 2^-43: |z| 2^43 < 2^31
#ifdef __CUDA_ARCH__
    const int z = __float2int_rn(VSD_MUL(a, 8796093022208.f)) +
                  __float2int_rn(VSD_MUL(al, 8796093022208.f));
#else
    const int z = (int)lrintf(VSD_MUL(a, 8796093022208.f)) +
                  (int)lrintf(VSD_MUL(al, 8796093022208.f));
#endif
    const uint64_t w = tab[at & (kExpTab - 1)];
    const int wh = (int)((w + 0x80000000ull) >> 32);
    const uint64_t v = w - (uint64_t)((int64_t)wh * z >> 11);
    const int sh = s.shift + (at >> 11);
    return sh < 64 ? (v + (1ull << (sh - 1))) >> sh : 0;
}

// -ln(p) in two floats, for 0 < p < 1, off by 2^-40 at most (2^-42 from p = 1/2 on): p = f 2^-k with 1/2 <= f < 1,
// ln(f) is the float l = logf(f) and what f exp(-l) is off 1.
__host__ __device__ __forceinline__ float neg_log(float p, const uint64_t* tab, float& lo) {
    int k;
    const float f = frexpf(p, &k), l = logf(f), n = (float)-k;
    const uint64_t near = exp_fixed(l, 0.f, exp_scale(1.f, 12), tab);  // exp(l) in 2^-50
    const float t = (float)((int64_t)(uint64_t)(f * 0x1p50f) - (int64_t)near) * 0x1p-50f / f;
    const float kLn2 = 0.693147182464599609375f, kLn2Lo = -1.904654300e-9f;
    const float a = VSD_MUL(n, kLn2);
    const float al = VSD_FMA(n, kLn2Lo, VSD_FMA(n, kLn2, -a));
    const float s = VSD_ADD(a, -l), b = VSD_ADD(s, -a);
    const float sl = VSD_ADD(VSD_ADD(a, -VSD_ADD(s, -b)), -VSD_ADD(l, b));
    lo = VSD_ADD(VSD_ADD(sl, al), -t);
    return s;
}

// ln(e / w) for e, w in such units, e = exp((x - m) / T) and w a sum of such with e
// among them: -(m - x) / T - ln(w), rounded once, of terms known to 2^-41 of each, and
// 2^-50 w for exp(-l) in its units.  ln(w) is the float l = logf(w) and what w exp(-l) is
// off 1.
__host__ __device__ __forceinline__ float log_share(float x, float m, float T, uint64_t w, int shift,
                                                    const uint64_t* tab) {
    float inv, inv_lo, e;
    over(1.f, 0.f, T, inv, inv_lo);
    const float d = gap(x, m, e), y = VSD_MUL(d, inv);
    if (!(y <= FLT_MAX)) return -INFINITY;  // (past a float's range)
    const float yl = VSD_FMA(e, inv, VSD_FMA(d, inv_lo, VSD_FMA(d, inv, -y)));
    const float one = ldexpf(1.f, shift - 62);
    const float l = logf((float)w * one);
    // w exp(-l), about 1
    const uint64_t back = exp_fixed(-l, 0.f, exp_scale(1.f, 12), tab);
#ifdef __CUDA_ARCH__
    const uint64_t hi = __umul64hi(w, back), lo = w * back;
#else
    const unsigned __int128 p = (unsigned __int128)w * back;
    const uint64_t hi = (uint64_t)(p >> 64), lo = (uint64_t)p;
#endif
    const uint64_t q = hi << (shift + 2) | lo >> (62 - shift);  // in units of 2^-50
    const float t = (float)((int64_t)(q - (1ull << 50))) * 0x1p-50f;
    const float s = VSD_ADD(y, l), b = VSD_ADD(s, -y);
    const float sl = VSD_ADD(VSD_ADD(y, -VSD_ADD(s, -b)), VSD_ADD(l, -b));
    return -VSD_ADD(s, VSD_ADD(VSD_ADD(sl, yl), t));
}

#undef VSD_ADD
#undef VSD_MUL
#undef VSD_FMA

}  // namespace vsd
