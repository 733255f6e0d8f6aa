"""CPU checks of the exponentials as whole numbers (csrc/vsd_fixed.cuh): the host's branch of
the functions, the same operations in the same order as the device's, against numpy's
long double."""
import ctypes as C
import subprocess

import numpy as np
import pytest

SOURCE = r"""
#include "vsd_fixed.cuh"
using namespace vsd;
static const ExpParts parts = make_exp_parts();
static uint64_t tab[kExpTab];
extern "C" {
void init() { for (int j = 0; j < kExpTab; ++j) tab[j] = exp_entry(parts, j); }
uint64_t entry(int j) { return tab[j]; }
int shift_of(int V) { return exp_shift(V); }
void masses(int n, const float* x, const float* m, const float* T, int shift, uint64_t* w) {
    for (int i = 0; i < n; ++i) w[i] = exp_fixed(x[i], m[i], exp_scale(T[i], shift), tab);
}
void shares(int n, const float* x, const float* m, const float* T, const uint64_t* w, int shift, float* r) {
    for (int i = 0; i < n; ++i) r[i] = log_share(x[i], m[i], T[i], w[i], shift, tab);
}
void logs(int n, const float* p, float* hi, float* lo) {
    for (int i = 0; i < n; ++i) hi[i] = neg_log(p[i], tab, lo[i]);
}
}
"""
L = np.longdouble
N = 400000

pytestmark = pytest.mark.skipif(np.finfo(L).nmant < 63, reason="long double is no longer than double here")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2602_05774_gb300 import build
    d = tmp_path_factory.mktemp("fixed")
    src, out = str(d / "fixed.cu"), str(d / "fixed.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([build.nvcc(), "-shared", "-Xcompiler", "-fPIC", "-O1", "-std=c++17", "-I" + build.CSRC, src, "-o",
                    out], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    lib = C.CDLL(out)
    lib.entry.restype = C.c_uint64
    lib.init()
    return lib


def ptr(a):
    return a.ctypes.data_as(C.c_void_p)


def rows(seed, temperatures, size, depth=43.0):
    """x <= m with (m - x) / T up to `depth` times ln 2."""
    g = np.random.default_rng(seed)
    T = np.exp2(g.uniform(*temperatures, N)).astype(np.float32)
    m = ((g.random(N) - 0.3) * size * np.maximum(T, 1e-30) ** (size == 10)).astype(np.float32)
    x = np.minimum((m - g.random(N) * depth * np.log(2) * T).astype(np.float32), m)
    return x, m, T


def test_table(lib):
    got = np.array([lib.entry(j) for j in range(2048)], dtype=np.uint64).astype(L)
    want = np.exp2(L(62) - np.arange(2048, dtype=L) / 2048)
    assert np.abs(got - want).max() <= 4


@pytest.mark.parametrize("shift", (12, 17, 20))
@pytest.mark.parametrize("temperatures,size", [((0, 0), 10), ((-2, 2), 10), ((-60, 60), 10), ((-3, 3), 100),
                                               ((-3, 3), 1e4)])
def test_masses_are_within_a_unit_and_2_to_the_minus_41(lib, shift, temperatures, size):
    x, m, T = rows(shift, temperatures, size)
    w = np.empty(N, dtype=np.uint64)
    lib.masses(N, ptr(x), ptr(m), ptr(T), shift, ptr(w))
    e = np.exp(-(m.astype(L) - x.astype(L)) / T.astype(L))
    unit = L(2) ** (shift - 62)
    assert (np.abs(w.astype(L) * unit - e) <= unit + e * L(2) ** -41).all()
    same = x == m
    assert (w[same] == 2 ** (62 - shift)).all()


def test_masses_fall_with_the_logit(lib):
    """A token never weighs less than one below it."""
    x = np.sort(np.random.default_rng(1).uniform(-30, 0, N).astype(np.float32))
    m, T = np.zeros(N, np.float32), np.ones(N, np.float32)
    w = np.empty(N, dtype=np.uint64)
    lib.masses(N, ptr(x), ptr(m), ptr(T), 17, ptr(w))
    fall = w[:-1].astype(np.int64) - w[1:].astype(np.int64)
    # (but for the rounding of neighbours, 2^-41 of either)
    assert (fall <= 2 + w[1:].astype(np.float64) * 2.0 ** -40).all()


def test_sums_stay_below_2_to_the_62(lib):
    for V in (1, 2, 4096, 4097, 128256, 1 << 20):
        s = lib.shift_of(V)
        assert s >= 12 and V * 2 ** (62 - s) <= 2 ** 62 and (s == 12 or V * 2 ** (62 - (s - 1)) > 2 ** 62)


@pytest.mark.parametrize("shift", (12, 17, 20))
def test_log_of_a_share(lib, shift):
    """One rounding of the result, and 2^-41 of what it is the difference of, and the 2^-51
    that exp(-ln(w)) is known to times w."""
    x, m, T = rows(5 + shift, (-3, 3), 10, 20.0)
    g = np.random.default_rng(shift)
    total = np.exp2(g.uniform(0, shift, N) * (g.random(N) < 0.8))
    w = np.maximum((total * 2.0 ** (62 - shift)).astype(np.uint64), 2 ** (62 - shift))
    got = np.empty(N, np.float32)
    lib.shares(N, ptr(x), ptr(m), ptr(T), ptr(w), shift, ptr(got))
    y = (m.astype(L) - x.astype(L)) / T.astype(L)
    share = w.astype(L) * L(2) ** (shift - 62)
    want = -y - np.log(share)
    half = np.exp2(np.floor(np.log2(np.maximum(np.abs(want), L(2) ** -126))) - 24)
    known = L(2) ** -41 * (1 + y + np.log(share)) + L(2) ** -50 * share
    assert (np.abs(got.astype(L) - want) <= half + known).all()


def test_negative_logs(lib):
    g = np.random.default_rng(3)
    bits = np.concatenate([g.integers(1, 0x3F800000, N), g.integers(0x3F000000, 0x3F800000, N), [1, 0x7FFFFF, 0x800000,
                                                                                             0x3F7FFFFF]])
    p = bits.astype(np.uint32).view(np.float32)
    hi, lo = np.empty(len(p), np.float32), np.empty(len(p), np.float32)
    lib.logs(len(p), ptr(p), ptr(hi), ptr(lo))
    off = np.abs(hi.astype(L) + lo.astype(L) + np.log(p.astype(L)))
    assert off.max() <= L(2) ** -40 and off[p >= 0.5].max() <= L(2) ** -42
