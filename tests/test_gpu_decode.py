"""GPU checks of drafting from an 8-bit head (vsd_quantize_fp8, vsd_lmhead_logits_fp8,
vsd_sample_filtered) against plain float64 implementations.

Tolerances:

* quantized matrices: the quotient by a power of two is exact and rounded once, so q
  and the scales are equal, bit for bit;
* logits of the 8-bit head: a block's products are exact (8 significant bits at most)
  and summed with at most one truncation of 2^-23 of the running sum a term, 128 terms;
  the blocks are joined in float32, two roundings of 2^-24 each and one for the product
  of the scales; then one rounding to bf16 (2^-8 of the value);
* tokens, counts and filtered rows: equal.  Exponentials are whole numbers with a relative
  error of 2^-41, rounded to units of 2^-(62 - s), s = max(12, ceil(log2 V)), so a sum of V
  of them is off by 2^-41 + V 2^-(63 - s) / (sum of e) of itself at most; float64's own sums
  by less.  A row that decides otherwise than the reference is an error unless the
  decision lies nearer to its border than four times that, and no more than one row in
  fifty of a call may;
* log probabilities: one rounding of the result (2^-24), of a difference of two terms
  that are known to 2^-40.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
U = 2.0 ** -24


@pytest.fixture(scope="module")
def vsd():
    from paper_2602_05774_gb300 import build, vsd as v
    build.build_library()
    v.load()
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    return v


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ------------------------------------------------------------------ quantizing
def plain_quantize(x, rows):
    """x on the CPU, float32: (q as float32, scale)."""
    R, H = x.shape
    q = torch.empty_like(x)
    s = torch.empty(-(-R // rows), -(-H // 128))
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            b = x[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128].double()
            a = float(b.abs().max())
            if not math.isfinite(a):
                scale = NAN
            elif a == 0:
                scale = 1.0
            else:
                scale = 2.0 ** -126
                while a / scale > 448:
                    scale *= 2
            s[i, j] = scale
            q[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128] = (b / scale).float().to(
                torch.float8_e4m3fn).float()
    return q, s


QSHAPES = [(1, 16), (1, 128), (3, 144), (127, 64), (128, 128), (129, 272), (300, 1040), (5, 4096)]


@pytest.mark.parametrize("rows", (1, 128))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shape", QSHAPES)
def test_quantize(vsd, shape, dtype, rows):
    g = gen(hash((shape, rows)) % 1000)
    x = torch.randn(*shape, generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-20, 20, (shape[0], 1), generator=g, device="cuda").float())
    x[0, :16] = torch.tensor([0.0, -0.0, 448.0, -448.0, 449.0, 1e-30, 2 ** -9, -(2 ** -10), 3.0,
                              17.0, 19.0, 0.3, -0.7, 1.0625, 1.1875, 240.0], device="cuda")
    if shape[0] > 2:
        x[2] = 0.0
    x = x.to(dtype)
    q, s = vsd.quantize_fp8(x, block_rows=rows)
    rq, rs = plain_quantize(x.float().cpu(), rows)
    assert torch.equal(s.cpu(), rs)
    assert torch.equal(q.float().cpu(), rq)
    assert torch.equal(torch.signbit(q.float().cpu()), torch.signbit(rq))


@pytest.mark.parametrize("rows", (1, 128))
def test_quantize_at_the_powers_border_and_the_ends(vsd, rows):
    """Blocks whose largest value is 448 2^k, just above it, or at a type's ends."""
    tops = [448.0 * 2.0 ** k * f for k in (-130, -100, -3, 0, 5, 100) for f in (1.0, 1 + 2 ** -23, 1 - 2 ** -24)]
    tops += [torch.finfo(torch.float32).max, 2.0 ** -149, 2.0 ** -126]
    n = len(tops)
    x = torch.zeros(rows, 128 * n, device="cuda")
    for i, t in enumerate(tops):
        x[-1, 128 * i] = t
        x[0, 128 * i + 1] = -t / 3
    q, s = vsd.quantize_fp8(x, block_rows=rows)
    rq, rs = plain_quantize(x.cpu(), rows)
    assert torch.equal(s.cpu(), rs) and torch.equal(q.float().cpu(), rq)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("rows", (1, 128))
def test_quantize_spreads_what_is_not_finite(vsd, rows, dtype):
    x = torch.randn(256, 256, generator=gen(3), device="cuda").to(dtype)
    clean = vsd.quantize_fp8(x, block_rows=rows)
    x[130, 5], x[7, 200] = NAN, -INF
    q, s = vsd.quantize_fp8(x, block_rows=rows)
    bad = torch.zeros_like(s, dtype=torch.bool)
    bad[130 // rows, 0] = bad[7 // rows, 1] = True
    assert torch.equal(torch.isnan(s), bad)
    wide = bad.repeat_interleave(rows, 0).repeat_interleave(128, 1)
    assert torch.equal(torch.isnan(q.float()), wide)
    assert torch.equal(q.float()[~wide], clean[0].float()[~wide])
    assert torch.equal(s[~bad], clean[1][~bad])


@pytest.mark.parametrize("shape,rows", [((70001, 144), 1), ((8388608 + 200, 16), 128), ((140000, 16400), 1)])
def test_quantize_many_rows(vsd, shape, rows):
    """More blocks than a grid's second dimension, and more than 2^31 elements."""
    x = torch.randn(shape[0], shape[1], generator=gen(5), device="cuda", dtype=torch.bfloat16)
    q, s = vsd.quantize_fp8(x, block_rows=rows)
    for lo in (0, shape[0] // 256 * 128, (shape[0] - 140) // 128 * 128):
        part = slice(lo, min(lo + 140, shape[0]))
        rq, rs = plain_quantize(x[part].float().cpu(), rows)
        n = rs.shape[0] - (1 if part.stop < shape[0] and rows > 1 else 0)  # (whole blocks)
        assert torch.equal(s[lo // rows:lo // rows + n].cpu(), rs[:n])
        assert torch.equal(q[part].float().cpu()[:n * rows], rq[:n * rows])


def test_quantize_into_given_tensors(vsd):
    x = torch.randn(129, 144, generator=gen(4), device="cuda")
    q0, s0 = vsd.quantize_fp8(x, block_rows=128)
    q = torch.zeros(129, 144, device="cuda").to(torch.float8_e4m3fn)
    s = torch.zeros(2, 2, device="cuda")
    q1, s1 = vsd.quantize_fp8(x, block_rows=128, q=q, scale=s)
    assert q1 is q and s1 is s and torch.equal(q.float(), q0.float()) and torch.equal(s, s0)


# ------------------------------------------------------------------ the head
def head_reference(h, hs, w, ws):
    """(float64 logits, bound of the error before the rounding to bf16) on the GPU."""
    R, H = h.shape
    V = w.shape[0]
    x = torch.zeros(R, V, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(x)
    nk = -(-H // 128)
    for j in range(nk):
        a = h[:, 128 * j:128 * (j + 1)].double()
        b = w[:, 128 * j:128 * (j + 1)].double()
        s = hs[:, j, None].double() * ws[:, j].double().repeat_interleave(128)[:V]
        x += s * (a @ b.T)
        mag += s.abs() * (a.abs() @ b.abs().T)
    return x, mag * (128 * 2.0 ** -23 + (2 * nk + 1) * U)


def check_head(vsd, h, hs, w, ws, out):
    x, err = head_reference(h, hs, w, ws)
    tol = err + 2.0 ** -8 * (x.abs() + err) + 2.0 ** -133
    off = (out.double() - x).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


def operands(R, V, H, seed, pow2=True):
    g = gen(seed)
    f = dict(generator=g, device="cuda")
    h = torch.randn(R, H, **f).to(torch.float8_e4m3fn)
    w = torch.randn(V, H, **f).to(torch.float8_e4m3fn)
    shape_h, shape_w = (R, -(-H // 128)), (-(-V // 128), -(-H // 128))
    if pow2:
        hs = torch.exp2(torch.randint(-6, 3, shape_h, **f).float())
        ws = torch.exp2(torch.randint(-6, 3, shape_w, **f).float())
    else:
        hs, ws = torch.rand(*shape_h, **f) + 0.01, torch.randn(*shape_w, **f)
    return h, hs, w, ws


HEADS = [(1, 1, 16), (1, 8, 128), (2, 127, 112), (7, 129, 144), (8, 500, 256), (16, 257, 400),
         (17, 1000, 128), (33, 640, 1040), (64, 300, 512), (65, 1023, 256), (100, 130, 2064),
         (127, 513, 384), (128, 512, 256), (129, 385, 272), (200, 1000, 640), (256, 256, 1024),
         (257, 2000, 384), (300, 32003, 64), (520, 777, 4096), (1000, 128, 160), (3, 128256, 96)]


@pytest.mark.parametrize("pow2", (True, False))
@pytest.mark.parametrize("R,V,H", HEADS)
def test_head(vsd, R, V, H, pow2):
    h, hs, w, ws = operands(R, V, H, R + V + H, pow2)
    wk = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    out = vsd.lmhead_logits_fp8(h, hs, w, ws, workspace=wk)
    assert out.shape == (R, V) and out.dtype == torch.bfloat16
    check_head(vsd, h, hs, w, ws, out)
    assert vsd.device_status(wk) == (0, 0)


@pytest.mark.parametrize("R,V,H", [(5, 300, 144), (128, 32000, 512), (129, 300, 144), (600, 3000, 528)])
def test_head_writes_its_rows_alone(vsd, R, V, H):
    """Logits at any 2-byte address; nothing before or behind them is written."""
    h, hs, w, ws = operands(R, V, H, 11)
    want = vsd.lmhead_logits_fp8(h, hs, w, ws)
    for shift in (0, 1, 3, 8):
        buf = torch.full((R * V + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        view = buf[shift:shift + R * V].view(R, V)
        got = vsd.lmhead_logits_fp8(h, hs, w, ws, out=view)
        assert got is view and torch.equal(got, want)
        assert bool((buf[:shift] == 7).all()) and bool((buf[shift + R * V:] == 7).all())


def test_head_is_the_same_for_a_row_alone_and_in_a_batch(vsd):
    """Few rows and many take different tiles; the sums are of the same blocks in the
    same order, so a row's logits agree to the bit."""
    h, hs, w, ws = operands(300, 1000, 640, 5, pow2=False)
    full = vsd.lmhead_logits_fp8(h, hs, w, ws)
    for lo, hi in ((0, 1), (3, 20), (100, 228)):
        part = vsd.lmhead_logits_fp8(h[lo:hi].contiguous(), hs[lo:hi].contiguous(), w, ws)
        assert torch.equal(part, full[lo:hi]), (lo, hi)


def test_head_spreads_nan(vsd):
    h, hs, w, ws = operands(140, 400, 256, 6)
    clean = vsd.lmhead_logits_fp8(h, hs, w, ws)
    hs[3, 1], ws[2, 0] = NAN, INF
    out = vsd.lmhead_logits_fp8(h, hs, w, ws)
    assert bool(torch.isnan(out[3]).all())
    assert not bool(torch.isfinite(out[:, 256:384]).any())
    keep = torch.ones(140, 400, dtype=torch.bool, device="cuda")
    keep[3], keep[:, 256:384] = False, False
    assert torch.equal(out[keep], clean[keep])


@pytest.mark.parametrize("R", (4, 300))
def test_head_offsets_past_32_bits(vsd, R):
    """A weight, or logits, of more than 2^31 elements."""
    V, H = (1 << 20, 2064) if R == 4 else (1 << 23 >> 3, 16)
    if R == 300:
        R = 2200  # 2.3e9 logits
    g = gen(8)
    h = torch.randn(R, H, generator=g, device="cuda").to(torch.float8_e4m3fn)
    w = torch.empty(V, H, dtype=torch.float8_e4m3fn, device="cuda")
    for at in range(0, V, 1 << 17):
        w[at:at + (1 << 17)] = torch.randn(min(1 << 17, V - at), H, generator=g, device="cuda").to(w.dtype)
    hs = torch.rand(R, -(-H // 128), generator=g, device="cuda")
    ws = torch.rand(V // 128, -(-H // 128), generator=g, device="cuda")
    out = vsd.lmhead_logits_fp8(h, hs, w, ws)
    for lo in (0, V // 2, V - 256):
        part = slice(lo, lo + 256)
        rows = slice(R - 4, R)
        check_head(vsd, h[rows], hs[rows], w[part], ws[lo // 128:lo // 128 + 2], out[rows, part])


# ------------------------------------------------------------------ sampling
def reference(x, T, k, p, mp):
    """Kept ids in their order, their e, and how near a decision was to its border
    (relative to what it was compared with).  x: float64 of the stored logits."""
    V = len(x)
    x = x + 0.0
    order = np.lexsort((np.arange(V), -x))
    order = order[x[order] > -np.inf]
    m = x[order[0]]
    if T == 0:
        return order[:1], np.ones(1), INF
    e = np.exp((x[order] - m) / T)
    n = len(order) if k <= 0 else min(k, len(order))
    near = INF
    cum = np.cumsum(e[:n])
    keep = n
    if p < 1:
        goal = max(p, 0.0) * cum[-1]
        by_p = 1 if p <= 0 else int(np.sum(cum < goal)) + 1
        at = cum - goal
        if p > 0:
            # (equal sums of equal terms are exact on both sides)
            gap = np.abs(at) / cum[-1]
            near = min(near, gap[gap > 0].min() if (gap > 0).any() else INF)
        keep = min(keep, by_p)
    if mp > 0:
        keep = min(keep, int(np.sum(e >= min(mp, 1.0))))
    return order[:keep], e[:keep], near


def draw(ids, e, u):
    """(token, its index among the kept, nearness) by inverse CDF in the ids' order."""
    at = np.argsort(ids)
    c = np.cumsum(e[at])
    if u >= 1:
        return ids[at[-1]], at[-1], INF
    if not u >= 0:
        return ids[at[0]], at[0], INF
    goal = u * c[-1]
    j = min(int(np.sum(c <= goal)), len(c) - 1)
    gap = np.abs(c - goal) / c[-1]
    return ids[at[j]], at[j], gap[gap > 0].min() if (gap > 0).any() else INF


def row_of(v, r):
    return v[r].item() if torch.is_tensor(v) else v


def f32(v):
    return float(np.float32(v))


def check_sample(x, u, out, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    R, V = x.shape
    xs = x.double().cpu().numpy()
    skipped = 0
    for r in range(R):
        t, p, mp = f32(row_of(T, r)), f32(row_of(top_p, r)), f32(row_of(min_p, r))
        ids, e, near = reference(xs[r], t, int(row_of(top_k, r)), p, mp)
        units = 2.0 ** -(62 - max(12, (V - 1).bit_length()))
        margin = 4 * (2.0 ** -41 + V * units / 2 / e.sum())
        if near < margin and out["kept"][r].item() != len(ids):
            skipped += 1
            continue
        assert out["kept"][r].item() == len(ids), (r, out["kept"][r].item(), len(ids))
        if "filtered" in out:
            want = torch.full((V,), -INF, dtype=x.dtype)
            sel = torch.as_tensor(ids.copy())
            want[sel] = x[r].cpu()[sel]
            assert torch.equal(out["filtered"][r].cpu(), want), r
        if u is not None:
            tok, at, near = draw(ids, e, float(u[r]))
            if near < margin and out["tokens"][r].item() != tok:
                skipped += 1
                continue
            assert out["tokens"][r].item() == tok, (r, out["tokens"][r].item(), tok)
            y = 0.0 if t == 0 else (xs[r][tok] - xs[r].max()) / t
            z = math.log(e.sum())
            lq = y - z
            tol = U * abs(lq) + 2.0 ** -38 * (1 + abs(y) + z) + 1e-45
            assert abs(out["logq_tok"][r].item() - lq) <= tol, (r, out["logq_tok"][r].item(), lq)
    assert skipped <= R // 50, skipped


def rows(R, V, dtype, seed, spread=2.0):
    g = gen(seed)
    f = dict(generator=g, device="cuda")
    x = spread * torch.randn(R, V, **f)
    x += 10 * torch.rand(R, 1, **f) * (torch.rand(R, V, **f) < 8.0 / V)
    return x.to(dtype), torch.rand(R, **f)


SETTINGS = [dict(), dict(T=0.0), dict(T=0.7), dict(top_k=1), dict(top_k=5, T=1.3), dict(top_k=300),
            dict(top_p=0.9), dict(top_p=0.5, T=2.5), dict(min_p=0.05), dict(min_p=1.0),
            dict(top_k=40, top_p=0.8, min_p=0.02, T=0.6), dict(top_k=3, top_p=0.9999), dict(top_p=1e-6),
            dict(top_p=0.0), dict(top_p=-1.0, min_p=-1.0, top_k=-3), dict(min_p=7.0),
            dict(top_k=1 << 30, top_p=2.0), dict(top_p=1 - 2.0 ** -24)]
SHAPES = [(3, 1), (4, 2), (5, 3), (7, 31), (6, 33), (9, 500), (5, 1000), (4, 1024), (3, 4099), (3, 32003),
          (2, 128256)]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shape", SHAPES)
def test_sample(vsd, shape, dtype):
    ws = torch.full((256,), 255, dtype=torch.uint8, device="cuda")
    for i, kw in enumerate(SETTINGS):
        x, u = rows(*shape, dtype, 31 * i + shape[1])
        out = vsd.sample_filtered(x, u, filtered=True, workspace=ws, **kw)
        check_sample(x, u, out, **kw)
        assert vsd.device_status(ws) == (0, 0)
        alone = vsd.sample_filtered(x, u, **kw)
        filt = vsd.filter_logits(x, **kw)
        for name in ("tokens", "logq_tok", "kept"):
            assert torch.equal(alone[name], out[name]), (kw, name)
        for name in ("filtered", "kept"):
            assert torch.equal(filt[name], out[name]), (kw, name)


@pytest.mark.parametrize("spread", (0.01, 0.5, 6.0, 30.0))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_flat_and_peaked_rows(vsd, dtype, spread):
    for i, kw in enumerate(SETTINGS):
        x, u = rows(6, 5000, dtype, 100 + i, spread)
        check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V,places", [(300, (1, 2, 40, 150, 299)), (5000, (3, 700, 2500, 4600)),
                                      (128256, (4, 600, 6000, 30000))])
def test_nuclei_that_end_at_a_border(vsd, V, places, dtype):
    """top_p is a prefix's share of the mass, rounded to float32: within 2^-25 of the
    border, where no approximate sum decides."""
    R = 3 * len(places)
    x, u = rows(R, V, dtype, 71)
    xs = x.double().cpu().numpy()
    share = []
    for r in range(R):
        cum = np.cumsum(reference(xs[r], 1.0, 0, 1.0, 0.0)[1])
        share.append(cum[places[r % len(places)] - 1] / cum[-1])
    top_p = torch.tensor(share, dtype=torch.float64).float().cuda()
    check_sample(x, u, vsd.sample_filtered(x, u, top_p=top_p, filtered=True), top_p=top_p)
    # and masked but for some: the rest has no mass
    x[:, 1::2] = -INF
    check_sample(x, u, vsd.sample_filtered(x, u, top_p=top_p, filtered=True), top_p=top_p)


@pytest.mark.parametrize("V", (700, 40000))
def test_settings_of_every_row(vsd, V):
    R = 48
    for dtype in (torch.float32, torch.bfloat16):
        x, u = rows(R, V, dtype, 9)
        g = gen(10)
        pick = lambda vals, dt: torch.tensor(vals, dtype=dt, device="cuda")[
            torch.randint(0, len(vals), (R,), generator=g, device="cuda")]
        kw = dict(T=pick((0.0, 0.5, 1.0, 1.7), torch.float32), top_k=pick((0, 1, 17, 600), torch.int32),
                  top_p=pick((1.0, 0.3, 0.95, 0.0), torch.float32), min_p=pick((0.0, 0.01, 0.3), torch.float32))
        out = vsd.sample_filtered(x, u, filtered=True, **kw)
        check_sample(x, u, out, **kw)
        # a row's results do not depend on the others
        for r in (0, 13, R - 1):
            one = {k: float(v[r]) if k != "top_k" else int(v[r]) for k, v in kw.items()}
            got = vsd.sample_filtered(x[r:r + 1].contiguous(), u[r:r + 1], filtered=True, **one)
            for name in out:
                assert torch.equal(got[name][0], out[name][r]), (r, name)


def test_equal_logits_go_by_id(vsd):
    """Rows of few values: the cut falls among equals, borders are met exactly."""
    for dtype in (torch.float32, torch.bfloat16):
        for V in (8, 64, 1000, 4096, 40000):
            x = torch.zeros(4, V, device="cuda")
            x[1, ::2] = -0.0
            x[2] = -3.5
            x[3, V // 2:] = 1.0
            x = x.to(dtype)
            u = torch.tensor([0.25, 0.5, 0.75, 0.0], device="cuda")
            for kw in (dict(), dict(top_k=max(1, V // 3)), dict(top_p=0.5), dict(top_p=0.25, T=0.5), dict(min_p=1.0),
                       dict(T=0.0), dict(top_k=V // 2, top_p=0.75)):
                check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


def test_masked_tokens_and_extreme_logits(vsd):
    big = torch.finfo(torch.float32).max
    low = torch.finfo(torch.bfloat16).min
    for dtype in (torch.float32, torch.bfloat16):
        top = torch.finfo(dtype).max
        x = torch.full((8, 3001), -INF, device="cuda")
        x[0, 1500] = 2.0                          # one token left
        x[1, [0, 3000]] = torch.tensor([1.0, 1.5], device="cuda")
        x[2] = low                                # a mask of the type's lowest value: all equal
        x[3] = low
        x[3, 7] = 0.0                             # ... under one live token
        x[4] = torch.linspace(-1, 1, 3001) * top  # differences past a float's range
        x[5] = -top
        x[5, 2999] = top
        x[6] = torch.arange(3001) * 1e-38         # near the smallest floats
        x[7, 100:200] = torch.randn(100, generator=gen(1), device="cuda")
        x = x.to(dtype)
        u = torch.full((8,), 0.6, device="cuda")
        for kw in (dict(), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.1), dict(T=0.0), dict(T=2.0 ** 64),
                   dict(T=2.0 ** -64), dict(top_k=2, top_p=0.5)):
            if "T" in kw and kw["T"] > 1:
                y = x[[0, 1, 2, 6, 7]]
            else:
                y = x
            check_sample(y, u[:len(y)], vsd.sample_filtered(y, u[:len(y)].contiguous(), filtered=True, **kw), **kw)
    assert big > 0


def test_uniforms_at_their_ends(vsd):
    x, _ = rows(1, 999, torch.float32, 2)
    x[0, 0], x[0, 998] = -INF, -INF
    x = x.expand(8, 999).contiguous()
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, 5.0, -1.0, NAN, 1e-30, -0.0], device="cuda")
    for kw in (dict(), dict(top_k=20), dict(top_p=0.7)):
        out = vsd.sample_filtered(x, u, filtered=True, **kw)
        check_sample(x, u, out, **kw)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_bad_rows_and_parameters(vsd, dtype):
    V = 1200
    x, u = rows(9, V, dtype, 21)
    x[1, 700], x[2, 3], x[3] = NAN, INF, -INF
    T = torch.ones(9, device="cuda")
    p, mp = torch.full((9,), 0.9, device="cuda"), torch.zeros(9, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    out = vsd.sample_filtered(x, u, top_p=0.9, filtered=True, workspace=ws)
    assert vsd.device_status(ws) == (6, vsd.STATUS_BAD_ROW)
    T[4], T[5], p[6], mp[7] = -1.0, 2.0 ** 65, NAN, NAN
    got = vsd.sample_filtered(x, u, T=T, top_p=p, min_p=mp, filtered=True, workspace=ws)
    assert vsd.device_status(ws) == (6, vsd.STATUS_BAD_ROW | vsd.STATUS_BAD_PARAM)
    for o, bad in ((out, (1, 2, 3)), (got, (1, 2, 3, 4, 5, 6, 7))):
        for r in range(9):
            if r in bad:
                assert o["tokens"][r] == -1 and o["kept"][r] == 0 and torch.isnan(o["logq_tok"][r])
                assert bool((o["filtered"][r] == -INF).all())
        good = [r for r in range(9) if r not in bad]
        check_sample(x[good], u[good], {k: v[good] for k, v in o.items()}, top_p=0.9)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (37, 1001, 33001))
def test_rows_at_any_alignment_and_in_place(vsd, dtype, V):
    R = 5
    x, u = rows(R, V, dtype, 5)
    kw = dict(top_k=30, top_p=0.95, T=0.9)
    want = vsd.sample_filtered(x, u, filtered=True, **kw)
    for shift in (0, 1, 3, 5, 7):
        buf = torch.full((R * V + 32,), 3.0, dtype=dtype, device="cuda")
        view = buf[shift:shift + R * V].view(R, V)
        view.copy_(x)
        for other in (0, 2):
            to = torch.full((R * V + 32,), 3.0, dtype=dtype, device="cuda")
            got = vsd.sample_filtered(view, u, filtered=to[other:other + R * V].view(R, V), **kw)
            for name in want:
                assert torch.equal(got[name], want[name]), (shift, name)
            assert bool((to[:other] == 3).all()) and bool((to[other + R * V:] == 3).all())
        got = vsd.sample_filtered(view, u, filtered=view, **kw)
        assert got["filtered"] is view
        for name in want:
            assert torch.equal(got[name], want[name]), (shift, name)
        assert bool((buf[:shift] == 3).all()) and bool((buf[shift + R * V:] == 3).all())


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (128257, 400003, 1 << 20))
def test_long_rows(vsd, V, dtype):
    """Rows past what a block, or a cluster, holds on chip."""
    for i, kw in enumerate((dict(), dict(top_k=100, top_p=0.9), dict(top_p=0.97), dict(min_p=0.01),
                            dict(top_k=V // 2, top_p=0.5))):
        x, u = rows(2, V, dtype, 70 + i)
        check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


def test_offsets_past_32_bits(vsd):
    R, V = 17000, 128256
    x = torch.empty(R, V, dtype=torch.bfloat16, device="cuda")
    g = gen(12)
    for at in range(0, R, 1000):
        x[at:at + 1000] = 2 * torch.randn(min(1000, R - at), V, generator=g, device="cuda")
    u = torch.rand(R, generator=g, device="cuda")
    out = vsd.sample_filtered(x, u, top_k=50, top_p=0.9)
    for lo in (0, 8400, 16800, R - 3):
        s = slice(lo, lo + 3)
        part = vsd.sample_filtered(x[s].contiguous(), u[s].contiguous(), top_k=50, top_p=0.9)
        for name in part:
            assert torch.equal(part[name], out[name][s]), (lo, name)
    check_sample(x[-3:], u[-3:], {k: v[-3:] for k, v in out.items()}, top_k=50, top_p=0.9)


def test_many_rows_agree_with_float64_on_the_gpu(vsd):
    """Every row of a large call, against float64 sums over the whole vocabulary."""
    R, V = 1024, 32000
    x, u = rows(R, V, torch.bfloat16, 77)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=64), dict(min_p=0.02)):
        out = vsd.sample_filtered(x, u, filtered=True, **kw)
        f = out["filtered"].double()
        e = torch.exp(f - x.double().max(1, keepdim=True).values)
        assert torch.equal((f > -INF).sum(1).int(), out["kept"])
        c = e.cumsum(1)
        t = out["tokens"].long()[:, None]
        goal = u.double()[:, None] * c[:, -1:]
        slack = c[:, -1:] * 2.0 ** -38
        assert bool((c.gather(1, t) > goal - slack).all())
        assert bool((c.gather(1, t) - e.gather(1, t) <= goal + slack).all())
        assert bool((f.gather(1, t) > -INF).all())


def test_frequencies_follow_the_kept_distribution(vsd):
    n = 40000
    x, _ = rows(1, 300, torch.float32, 8)
    u = torch.rand(n, generator=gen(9), device="cuda")
    out = vsd.sample_filtered(x.expand(n, 300).contiguous(), u, T=1.2, top_k=12, top_p=0.95)
    ids, e, _ = reference(x[0].double().cpu().numpy(), f32(1.2), 12, f32(0.95), 0.0)
    got = torch.bincount(out["tokens"].long().cpu(), minlength=300).numpy() / n
    want = np.zeros(300)
    want[ids] = e / e.sum()
    # 6 standard deviations of a count
    assert (np.abs(got - want) <= 6 * np.sqrt(want * (1 - want) / n) + 1e-12).all()


# ------------------------------------------------------------------ streams, graphs, together
def test_streams_and_graphs(vsd):
    x, u = rows(16, 5001, torch.bfloat16, 3)
    h, hs, w, ws8 = operands(9, 1000, 272, 2)
    kw = dict(top_k=40, top_p=0.9, T=0.8)
    want = vsd.sample_filtered(x, u, filtered=True, **kw)
    head = vsd.lmhead_logits_fp8(h, hs, w, ws8)
    q = vsd.quantize_fp8(x[:, :4992].contiguous())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = vsd.sample_filtered(x, u, filtered=True, **kw)
        got_head = vsd.lmhead_logits_fp8(h, hs, w, ws8)
    torch.cuda.current_stream().wait_stream(s)
    for n in want:
        assert torch.equal(want[n], got[n])
    assert torch.equal(head, got_head)
    wsa, wsb = (torch.empty(256, dtype=torch.uint8, device="cuda") for _ in range(2))
    xg, ug, cut = x.clone(), u.clone(), x[:, :4992].contiguous()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qg = vsd.quantize_fp8(cut)
        hg = vsd.lmhead_logits_fp8(h, hs, w, ws8, workspace=wsb)
        sg = vsd.sample_filtered(xg, ug, filtered=True, workspace=wsa, **kw)
    for seed in (3, 4):
        x2, u2 = rows(16, 5001, torch.bfloat16, seed)
        xg.copy_(x2)
        ug.copy_(u2)
        cut.copy_(x2[:, :4992])
        graph.replay()
        torch.cuda.synchronize()
        now = vsd.sample_filtered(x2, u2, filtered=True, **kw)
        for n in now:
            assert torch.equal(now[n], sg[n]), n
        assert torch.equal(hg, head)
        now = vsd.quantize_fp8(cut)
        assert torch.equal(now[0].float(), qg[0].float()) and torch.equal(now[1], qg[1])
        if seed == 3:
            assert torch.equal(q[0].float(), qg[0].float())
    assert vsd.device_status(wsa) == (0, 0) and vsd.device_status(wsb) == (0, 0)


def test_calls_at_once_on_two_streams(vsd):
    x, u = rows(64, 32000, torch.bfloat16, 14)
    h, hs, w, ws8 = operands(32, 32000, 512, 15)
    kw = dict(top_p=0.95)
    want, head = vsd.sample_filtered(x, u, **kw), vsd.lmhead_logits_fp8(h, hs, w, ws8)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append((vsd.sample_filtered(x, u, **kw), vsd.lmhead_logits_fp8(h, hs, w, ws8)))
    torch.cuda.synchronize()
    for a, b in got:
        assert all(torch.equal(a[n], want[n]) for n in want) and torch.equal(b, head)


def test_draft_from_an_8bit_head_then_verify(vsd, oracle):
    """A decoding step under a policy: hidden states and weight quantized, the draft's
    logits from them, tokens drawn from the filtered rows, both models' filtered rows
    verified; against the float64 oracle on the same filtered rows."""
    B, K, D, V, H, T = 3, 4, 3, 1000, 256, 0.8
    R = B * K * D
    g = gen(5)
    f = dict(generator=g, device="cuda")
    hidden = torch.randn(R, H, **f).to(torch.bfloat16)
    weight = 0.2 * torch.randn(V, H, **f)
    w8, wsc = vsd.quantize_fp8(weight, block_rows=128)
    h8, hsc = vsd.quantize_fp8(hidden)
    draft = vsd.lmhead_logits_fp8(h8, hsc, w8, wsc)
    check_head(vsd, h8, hsc, w8, wsc, draft)
    # the 8-bit head stands for the bf16 one: 3 bits after the point on both sides
    near = hidden.double() @ weight.double().T
    bound = (2.0 ** -4 * 2 + 2.0 ** -8) * (hidden.double().abs() @ weight.double().abs().T) * 1.2 + 0.05
    assert bool(((draft.double() - near).abs() <= bound).all())
    target = vsd.lmhead_logits(hidden, (weight + 0.05 * torch.randn(V, H, **f)).to(torch.bfloat16))
    u = torch.rand(3, R, **f)
    kw = dict(T=T, top_k=60, top_p=0.95)
    drawn = vsd.sample_filtered(draft, u[0], filtered=draft, **kw)
    vsd.filter_logits(target, out=target, **kw)
    got = vsd.verify_paths(draft, target, drawn["tokens"], u[1], u[2], K, D, T)
    # against the E-step's own sampling on the filtered rows, and the oracle's
    z = vsd.sample_paths(draft, u[0], K, D, T)
    assert torch.equal(z["tokens"], drawn["tokens"])
    assert bool(((z["logq_tok"] - drawn["logq_tok"]).abs() <= 2e-6 * (1 + drawn["logq_tok"].abs())).all())
    orc = oracle.linear(draft.float().cpu().numpy(), target.float().cpu().numpy(), T, u[0].cpu().numpy(),
                        u[1].cpu().numpy(), u[2].cpu().numpy(), K, D)
    assert np.array_equal(orc["tokens"].reshape(-1), drawn["tokens"].cpu().numpy())
    assert np.array_equal(orc["accept_len"].reshape(-1), got["accept_len"].cpu().numpy())
    assert np.array_equal(orc["corr_tokens"].reshape(-1), got["corr_tokens"].cpu().numpy())
    # the corrections come from the target's kept tokens too
    assert bool((target.gather(1, got["corr_tokens"].long()[:, None]) > -INF).all() |
                (draft.gather(1, got["corr_tokens"].long()[:, None]) > -INF).all())


def test_gradients_of_a_head_that_drafts_in_8_bits(vsd):
    """The E/M step on the 8-bit head's logits, then the head's backward: the products
    of the dense gradient with the bf16 master weight and hidden states."""
    B, K, D, V, H, T = 2, 4, 2, 512, 128, 1.0
    R = B * K * D
    g = gen(6)
    f = dict(generator=g, device="cuda")
    hidden = torch.randn(R, H, **f).to(torch.bfloat16)
    weight = (0.1 * torch.randn(V, H, **f)).to(torch.bfloat16)
    draft = vsd.lmhead_logits_fp8(*vsd.quantize_fp8(hidden), *vsd.quantize_fp8(weight, block_rows=128))
    target = (draft.float() + torch.randn(R, V, **f)).to(torch.bfloat16)
    u = torch.rand(3, R, **f)
    ws = vsd.new_workspace(vsd.layout(B, K, D, V), "cuda")
    dense = vsd.estep_mstep(draft, target, u[0], u[1], u[2], K, D, T)["grad"].double()
    vsd.estep_mstep(draft, target, u[0], u[1], u[2], K, D, T, workspace=ws, grad=False)
    got = vsd.lmhead_backward(hidden, weight, draft, K, D, T, ws)
    for name, want, mag in (("d_hidden", dense @ weight.double(), dense.abs() @ weight.double().abs()),
                            ("d_weight", dense.T @ hidden.double(), dense.abs().T @ hidden.double().abs())):
        n = V if name == "d_hidden" else R
        # exact products summed in float32, one truncation of 2^-23 a term
        assert bool(((got[name].double() - want).abs() <= n * 2.0 ** -23 * mag + 1e-30).all()), name


# ------------------------------------------------------------------ rows that leave the usual way
def gpu_reference(x, T=1.0, top_p=1.0, min_p=0.0):
    """Without top_k, in float64 on the GPU: per row the number kept, its nearest distance
    from a border (relative), and the filtered logits."""
    V = x.shape[1]
    xs, order = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True)
    e = torch.exp((xs - xs[:, :1]) / f32(T))
    c = e.cumsum(1)
    total = c[:, -1:]
    kept = (xs > -INF).sum(1, keepdim=True)
    near = torch.full_like(total, INF)
    if top_p < 1:
        gap = (c / total - f32(top_p)).abs()
        near = gap.amin(1, keepdim=True)
        kept = torch.minimum(kept, (c < f32(top_p) * total).sum(1, keepdim=True) + 1)
    if min_p > 0:
        near = torch.minimum(near, (e / min(f32(min_p), 1.0) - 1).abs().amin(1, keepdim=True))
        kept = torch.minimum(kept, (e >= min(f32(min_p), 1.0)).sum(1, keepdim=True))
    on = torch.zeros_like(x, dtype=torch.bool).scatter_(
        1, order, torch.arange(V, device=x.device) < kept)
    return kept[:, 0].int(), near[:, 0], torch.where(on, x, -INF)


def check_on_gpu(x, u, out, **kw):
    """Every row of a large call: kept tokens, filtered rows, and the draw by its prefix sums."""
    V = x.shape[1]
    kept, near, filtered = gpu_reference(x, **kw)
    margin = 4 * (2.0 ** -41 + V * 2.0 ** -(63 - max(12, (V - 1).bit_length())))
    sure = near > margin
    assert int((~sure).sum()) <= len(x) // 50
    assert torch.equal(out["kept"][sure], kept[sure])
    assert torch.equal(out["filtered"][sure], filtered[sure])
    f = out["filtered"].double()
    e = torch.exp((f - x.double().amax(1, keepdim=True)) / f32(kw.get("T", 1.0)))
    c = e.cumsum(1)
    t = out["tokens"].long()[:, None]
    goal, slack = u.double()[:, None] * c[:, -1:], c[:, -1:] * margin
    assert bool((f.gather(1, t) > -INF).all())
    assert bool((c.gather(1, t) > goal - slack).all())
    assert bool((c.gather(1, t) - e.gather(1, t) <= goal + slack).all())


def masked_by_id(R, V, dtype, seed, mask):
    """Rows of normal logits whose ids are masked by a rule."""
    x = torch.randn(R, V, generator=gen(seed), device="cuda")
    ids = torch.arange(V, device="cuda")
    if mask == "starts":       # the first quarter of each 2048 bf16, or 1024 float32
        off = ids % (2048 if dtype == torch.bfloat16 else 1024) < (512 if dtype == torch.bfloat16 else 256)
    elif mask == "ends":       # the other three quarters
        off = ids % (2048 if dtype == torch.bfloat16 else 1024) >= (512 if dtype == torch.bfloat16 else 256)
    elif mask == "bands":      # bands of allowed ids, elsewhere in every row
        n = V // 24
        at = torch.randint(0, n, (R, 1), generator=gen(seed + 1), device="cuda")
        off = (ids + at) // n % 4 != 0
    else:                      # heavy tokens at the regions' ends alone
        x += 6 * (ids % 2048 >= 1500)
        off = torch.zeros(V, dtype=torch.bool, device="cuda")
    return x.masked_fill(off, -INF).to(dtype), torch.rand(R, generator=gen(seed + 2), device="cuda")


@pytest.mark.parametrize("mask", ("starts", "ends", "bands", "heavy"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (40000, 128256))
def test_nuclei_whose_tokens_a_sample_of_the_row_misses(vsd, V, dtype, mask):
    """A nucleus past the list is looked for in a quarter of the row first, the first 512
    bf16 or 256 float32 of each four times as many; masks by id leave that quarter without
    mass, or without what the nucleus ends at, so that the whole row is asked."""
    x, u = masked_by_id(608, V, dtype, V, mask)
    for top_p in (0.5, 0.9, 0.95, 0.99):
        out = vsd.sample_filtered(x, u, top_p=top_p, filtered=True)
        check_on_gpu(x, u, out, top_p=top_p)
        for _ in range(5):
            again = vsd.sample_filtered(x, u, top_p=top_p, filtered=True)
            for n in out:
                assert torch.equal(again[n], out[n]), n


# ------------------------------------------------------------------ scales whose product leaves float32
@pytest.mark.parametrize("H", (128, 400))
@pytest.mark.parametrize("R", (3, 33, 100, 300))
def test_head_scales_whose_product_is_out_of_range(vsd, R, H):
    """hidden_scale . weight_scale past float32's range, or below its normal numbers, where
    the scaled sums are within it: by rows and by the weight's blocks, beside usual ones."""
    V = 700
    nk = -(-H // 128)
    h, _, w, _ = operands(R, V, H, 3 * R + H)
    g = gen(R)
    near1 = lambda *n: 1 + torch.rand(*n, generator=g, device="cuda")
    hs, ws = near1(R, nk), near1(6, nk)
    # blocks whose sums are 0 under scales of any size: a zero row, a zero block of the weight
    h[0] = 0
    w[128:256] = 0
    big, small = 2.0 ** 100, 2.0 ** -75
    hs[0] *= big
    ws[1] *= big
    # a row of 2^-75: times a block of 2^-68 (normal), 2^-73 (subnormal) and 2^-90 (nothing)
    hs[1] *= small
    ws[2] *= 2.0 ** -68
    ws[3] *= 2.0 ** -73
    ws[4] *= 2.0 ** -90
    # 2^-9 . 2^-9 under 2^127 . 2^8: 2^117
    h[2], hs[2] = 0, hs[2] * 0 + 1.5 * 2.0 ** 126
    h[2, 5] = 2.0 ** -9
    w[640:, 5] = 2.0 ** -9
    ws[5] *= 2.0 ** 8
    h[2, 6:] = 0
    w[0:128, 5] = 1.0
    ws[0] *= 2.0 ** -20
    out = vsd.lmhead_logits_fp8(h, hs, w, ws)
    x, err = head_reference(h, hs, w, ws)
    sure = x.abs() < 2.0 ** 127  # (the others are past bf16)
    assert bool(sure[:2].all()) and bool(sure[2, 640:].all()) and bool(sure[2, :256].all())
    assert float(x[2, 640:].abs().max()) > 2.0 ** 110 and float(x[1, 384:512].abs().max()) > 0
    tol = err + 2.0 ** -8 * (x.abs() + err) + 2.0 ** -133
    off = (out.double() - x).abs()
    assert bool((off <= tol)[sure].all())
    assert not bool(torch.isnan(out).any())
    # a row's logits hang on its own scales alone
    for r in range(3):
        part = vsd.lmhead_logits_fp8(h[r:r + 1].contiguous(), hs[r:r + 1].contiguous(), w, ws)
        assert torch.equal(part[0], out[r]), r
    if R > 3:
        plain = vsd.lmhead_logits_fp8(h[3:].contiguous(), hs[3:].contiguous(), w, ws)
        assert torch.equal(plain, out[3:])


@pytest.mark.parametrize("top_p24", (3, 9, 12, 17, 22, 30))
def test_a_nucleus_is_the_same_with_all_tokens_as_its_k(vsd, top_p24):
    """top_k = V leaves all tokens, as top_k = 0 does, by another way through the row.  The
    rest of this row, 2^20 tokens, weighs 1.49 units each: as whole numbers a third less."""
    V = 1 << 20
    x = torch.full((1, V), math.log(1.49) - 42 * math.log(2), device="cuda")
    x[0, 16:16 * 201:16] = -26 * math.log(2) - torch.arange(200, device="cuda") * 1e-4
    x[0, 5] = 0.0
    u = torch.tensor([0.3], device="cuda")
    p = 1 - top_p24 * 2.0 ** -24
    a = vsd.sample_filtered(x, u, top_p=p, filtered=True)
    b = vsd.sample_filtered(x, u, top_p=p, top_k=V, filtered=True)
    for n in a:
        assert torch.equal(a[n], b[n]), (n, a["kept"], b["kept"])
    # and by whole numbers
    e = np.exp(np.sort(x[0].double().cpu().numpy())[::-1])
    m = np.rint(e * 2.0 ** 42)
    goal, cum = p * m.sum(), np.cumsum(m)
    n = int((cum < goal).sum()) + 1
    if n <= 201:  # (else it ends among the small ones, whose number a unit decides)
        assert np.abs(cum - goal).min() > 2 * n  # (a unit for each of the n)
        assert int(a["kept"]) == n


TINY = (2.0 ** -149, 1e-38, 1e-30, 1e-20, 1e-15, 3e-13, 1e-12, 1e-9)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (700, 5000, 40000, 1 << 20))
def test_min_p_far_below_the_units_of_the_sums(vsd, V, dtype):
    """Which tokens reach min_p of the first one's probability, where their masses are a
    few units of the sums, or none: by the logits' distance."""
    for i, min_p in enumerate(TINY):
        g = gen(i)
        x = -120 * torch.rand(2, V, generator=g, device="cuda")
        x[1] = x[1] / 40 - 27.5  # many near 1e-12
        x[:, V // 3] = 0.0
        x[:, -1] = -INF
        x = (x * 1.25).to(dtype)
        u = torch.rand(2, generator=g, device="cuda")
        for kw in (dict(), dict(top_k=300), dict(top_p=0.999)):
            kw = dict(kw, min_p=min_p, T=1.25)
            out = vsd.sample_filtered(x, u, filtered=True, **kw)
            # (a log probability also has what the whole numbers of V masses are off, a unit
            # each of a sum of 1 at least: taken out for the comparison of the others)
            lq, units = out["logq_tok"].double().cpu(), V * 2.0 ** -(62 - max(12, (V - 1).bit_length()))
            for r in range(2):
                y = x[r].double().cpu().numpy() / 1.25
                on = out["filtered"][r].float().cpu().numpy() > -INF
                want = y[int(out["tokens"][r])] - y.max() - math.log(np.exp(y[on] - y.max()).sum())
                assert abs(float(lq[r]) - want) <= U * abs(want) + 2.0 ** -38 * (1 + abs(want)) + units
                out["logq_tok"][r] = want
            check_sample(x, u, out, **kw)


def test_min_p_next_to_a_logit(vsd):
    """min_p on either side of a token's probability, by steps of float32."""
    d = torch.tensor([0.0, 0.5, 3.0, 17.0, 29.0, 33.5, 60.0, 87.0], device="cuda")
    for T in (0.7, 1.0, 3.0):
        for m in (0.0, 11.25, -300.0):
            x = (m - T * d)[None].contiguous()
            e = np.exp((x[0].double().cpu().numpy() - float(x[0, 0])) / f32(T))
            for i in range(1, 8):
                p0 = np.float32(e[i])
                for p in (np.nextafter(p0, np.float32(0)), p0, np.nextafter(p0, np.float32(1))):
                    if abs(float(p) / e[i] - 1) < 2.0 ** -38:
                        continue
                    out = vsd.filter_logits(x, T=T, min_p=float(p))
                    assert int(out["kept"]) == int((e >= float(p)).sum()), (T, m, i, p)


def test_log_probability_past_a_floats_range(vsd):
    """The last kept token (u = 1) of a row whose logits lie further apart than floats go."""
    u = torch.ones(1, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        top = torch.finfo(dtype).max
        for x, T in (((top, -top), 1.0), ((0.9 * top, -0.3 * top), 1.0), ((0.0, -1e25), 2.0 ** -64),
                     ((0.0, -top), 0.5)):
            x = torch.tensor([x], device="cuda").to(dtype)
            for kw in (dict(), dict(top_k=2)):
                out = vsd.sample_filtered(x, u, T=T, **kw)
                assert int(out["tokens"]) == 1 and int(out["kept"]) == 2
                assert float(out["logq_tok"]) == -INF, (x, T, out["logq_tok"])
        x = torch.tensor([[0.0, -1e30]], device="cuda").to(dtype)
        out = vsd.sample_filtered(x, u, T=2.0)
        assert float(out["logq_tok"]) == float(x[0, 1]) / 2


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (20000, 128256))
def test_rows_that_begin_masked(vsd, V, dtype):
    """The first tokens, all that a block reads before it has a bound, are at -inf, or at
    the type's lowest value; a row may end so too."""
    x, u = rows(9, V, dtype, 17)
    low = torch.finfo(dtype).min
    lead = 16400
    x[:3, :lead] = -INF
    x[3:5, :lead] = low
    x[5, :V - 1] = -INF
    x[6, :] = low                    # equals at the lowest value
    x[6, ::3] = -INF
    x[7, :] = -INF                   # one token, at the lowest value
    x[7, V - 2] = low
    x[8, 7:] = -INF
    for kw in SETTINGS:
        check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (3, 100, 1023, 4001))
def test_rows_at_the_lowest_value_beside_masked_tokens(vsd, V, dtype):
    """min_p's bound below a maximum at the type's lowest value is -inf."""
    x = torch.full((4, V), torch.finfo(dtype).min, device="cuda", dtype=dtype)
    x[1, ::2] = -INF
    x[2, :-1] = -INF
    x[3, 1:] = -INF
    u = torch.tensor([0.0, 0.7, 1.0, 0.3], device="cuda")
    for kw in SETTINGS + [dict(min_p=1e-30), dict(min_p=0.5, top_k=3)]:
        check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


# ------------------------------------------------------------------ lengths between the others
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("V", (4097, 8192, 8193, 16384, 200003, 262144))
def test_rows_of_one_round_and_past_the_usual(vsd, V, dtype):
    for i, kw in enumerate((dict(top_p=0.95), dict(top_p=0.8, T=1.5), dict(top_k=200, top_p=0.9), dict(top_k=2000),
                            dict(top_p=0.9, min_p=1e-4), dict(T=0.0))):
        x, u = rows(4, V, dtype, 300 + i)
        check_sample(x, u, vsd.sample_filtered(x, u, filtered=True, **kw), **kw)


def filtered_pair(vsd, R, V, dtype, seed, **kw):
    """Draft and target rows that differ, both filtered in place by one policy."""
    g = gen(seed)
    q = 3 * torch.randn(R, V, generator=g, device="cuda")
    p = (q + 1.5 * torch.randn(R, V, generator=g, device="cuda")).to(dtype)
    q = q.to(dtype)
    vsd.filter_logits(q, out=q, **kw)
    vsd.filter_logits(p, out=p, **kw)
    return q, p


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("kw", (dict(top_k=8), dict(top_p=0.6), dict(min_p=0.1, top_k=30, top_p=0.9)))
def test_corrections_are_of_the_targets_kept_tokens(vsd, oracle, dtype, kw):
    B, K, D, V, T = 2, 3, 4, 600, 0.9
    R = B * K * D
    q, p = filtered_pair(vsd, R, V, dtype, 41, T=T, **kw)
    u = torch.rand(3, R, generator=gen(42), device="cuda")
    z = vsd.sample_paths(q, u[0], K, D, T)
    got = vsd.verify_paths(q, p, z["tokens"], u[1], u[2], K, D, T)
    orc = oracle.linear(q.float().cpu().numpy(), p.float().cpu().numpy(), T, u[0].cpu().numpy(), u[1].cpu().numpy(),
                        u[2].cpu().numpy(), K, D)
    assert np.array_equal(orc["accept_len"].reshape(-1), got["accept_len"].cpu().numpy())
    assert np.array_equal(orc["corr_tokens"].reshape(-1), got["corr_tokens"].cpu().numpy())
    # every path's first token that was not accepted is drawn from the target's rows
    corr = got["corr_tokens"].reshape(B * K, D).long()
    n = got["accept_len"].reshape(B * K).long()
    at = n.clamp(max=D - 1)[:, None]
    rejected = (n < D)
    assert bool(rejected.any())
    kept = p.reshape(B * K, D, V).gather(1, at[..., None].expand(-1, 1, V))[:, 0]
    assert bool((kept.gather(1, corr.gather(1, at))[rejected] > -INF).all())


def filtered_tree(vsd, B, N, depth, topk, V, seed, dtype, **kw):
    """A tree problem on the GPU whose rows are filtered; a node's token is its rank among
    the kept ones of its parent's draft row."""
    from paper_2602_05774_gb300 import inputs
    p = inputs.tree_problem(B, N, depth, topk, V, seed=seed)
    p = {k: v.cuda() if torch.is_tensor(v) else v for k, v in p.items()}
    for n in ("draft", "target"):
        p[n] = p[n].to(dtype)
        vsd.filter_logits(p[n], out=p[n], **kw)
    rows = (torch.arange(B, device="cuda").view(B, 1) * N + p["parent"].clamp(min=0).long()).view(-1)
    q = p["draft"].float()[rows]
    assert bool((q.gather(1, p["tokens"].long().view(-1, 1))[p["parent"].view(-1) >= 0] > -INF).all())
    return p


TREES = [(3, 12, 4, 3, 777), (2, 30, 6, 5, 4097), (4, 60, 8, 10, 1000)]


@pytest.mark.parametrize("rule", (0, 1))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("shape", TREES)
def test_filtered_rows_in_tree_verification(vsd, oracle, shape, dtype, rule):
    from tests.parity import compare_tree, compare_tree_sequential
    B, N = shape[:2]
    for T, kw in ((1.0, dict(top_k=24)), (0.8, dict(top_k=40, top_p=0.995, min_p=1e-4))):
        p = filtered_tree(vsd, *shape, 7, dtype, T=T, **dict(kw, top_p=1.0) if shape[3] > 3 else kw)
        got = vsd.verify_tree(p["draft"], p["target"], p["parent"], p["tokens"], p["u_accept"], p["u_correct"], T,
                              rule=rule)
        c = {k: v.float().cpu().numpy() if v.dtype != torch.int32 else v.cpu().numpy()
             for k, v in p.items() if torch.is_tensor(v)}
        orc = oracle.tree(c["draft"], c["target"], T, c["parent"], c["tokens"], c["u_accept"], c["u_correct"], rule=rule)
        (compare_tree_sequential if rule else compare_tree)(got, orc)
        # the bonus token and what replaces a rejected one are the target's
        bonus, rows = got["bonus"].long(), p["target"].view(B, N, -1)
        at = got["deepest"].long()
        assert bool((rows[torch.arange(B), at].gather(1, bonus[:, None]) > -INF).all())


def check_em(got, orc, n_rows, V):
    """The E/M step on filtered rows: a correction may be a token that the draft leaves out,
    of log q = -inf; the gradient has no log q in it."""
    from tests.parity import _grad_rows
    assert np.array_equal(got["corr_tokens"].cpu().numpy().ravel(), orc["corr_tokens"].ravel())
    for n, atol in (("logq_tok", 2e-5), ("logq_corr", 2e-5)):
        assert np.allclose(got[n].cpu().numpy().ravel(), orc[n].ravel(), rtol=1e-6, atol=atol), n
    a, b = got["grad"].float().cpu().numpy(), orc["grad"].reshape(n_rows, V)
    assert np.isfinite(b).all() and np.isfinite(a).all()
    _grad_rows("grad", a, b, "f32", float(np.abs(b).max()))
    return np.isinf(orc["logq_corr"])


@pytest.mark.parametrize("shape", TREES)
def test_filtered_rows_in_the_trees_em(vsd, oracle, shape):
    B, N = shape[:2]
    V = shape[4]
    p = filtered_tree(vsd, *shape, 9, torch.float32, T=0.8, top_k=24)
    got = vsd.tree_estep_mstep(p["draft"], p["target"], p["parent"], p["tokens"], p["u_accept"], p["u_correct"], 0.8,
                               prm=vsd.params(grad_dtype=torch.float32))
    c = {k: v.float().cpu().numpy() if v.dtype != torch.int32 else v.cpu().numpy()
         for k, v in p.items() if torch.is_tensor(v)}
    orc = oracle.tree_em(c["draft"], c["target"], 0.8, c["parent"], c["tokens"], c["u_accept"], c["u_correct"])
    check_em(got, orc, B * N, V)
    # the loss of a tree with such a correction that counts is infinite
    assert np.allclose(got["loss"].cpu().numpy(), orc["loss"], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("top_k", (24, 300))
def test_filtered_rows_in_the_em(vsd, oracle, top_k):
    B, K, D, V, T = 4, 3, 4, 600, 0.9
    R = B * K * D
    q, p = filtered_pair(vsd, R, V, torch.float32, 43, T=T, top_k=top_k)
    u = torch.rand(3, R, generator=gen(44), device="cuda")
    got = vsd.estep_mstep(q, p, u[0], u[1], u[2], K, D, T, prm=vsd.params(grad_dtype=torch.float32))
    orc = oracle.linear(q.cpu().numpy(), p.cpu().numpy(), T, u[0].cpu().numpy(), u[1].cpu().numpy(),
                        u[2].cpu().numpy(), K, D)
    assert check_em(got, orc, R, V).any() == (top_k == 24)
    # a log q of -inf counts as -2^20, so that the loss stays finite
    loss, want = got["loss"].cpu().numpy(), np.asarray(orc["loss"])
    off = np.isinf(want)
    assert off.any() == (top_k == 24) and (loss[off] > 1000).all() and np.isfinite(loss).all()
    assert np.allclose(loss[~off], want[~off], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("R", (5, 60, 128, 300))
def test_head_scales_out_of_range_in_some_tiles_alone(vsd, R):
    """A few of a thousand blocks of the weight, in any of a block of threads' tiles."""
    V, H = 128256, 272
    h, hs, w, ws = operands(R, V, H, 7 * R, pow2=False)
    want = vsd.lmhead_logits_fp8(h, hs, w, ws)
    odd = torch.randperm(V // 128, generator=gen(R), device="cuda")[:40]
    hs[R // 2] *= 2.0 ** -70
    ws[odd[:20], 1] *= 2.0 ** 126
    ws[odd[20:], 2] *= 2.0 ** -80
    out = vsd.lmhead_logits_fp8(h, hs, w, ws)
    x, err = head_reference(h, hs, w, ws)
    sure = x.abs() < 2.0 ** 127
    tol = err + 2.0 ** -8 * (x.abs() + err) + 2.0 ** -133
    assert bool((((out.double() - x).abs() <= tol) | ~sure).all())
    # what has usual scales keeps its bits
    on = torch.ones(R, V, dtype=torch.bool, device="cuda")
    on[R // 2] = False
    on.view(R, -1, 128)[:, odd] = False
    assert torch.equal(out[on], want[on])
