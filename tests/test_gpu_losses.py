"""GPU checks of the draft head's supervised losses (vsd_lmhead_cross_entropy,
vsd_lmhead_distill, vsd_topk_distill) against a plain float64 implementation.

The float64 side works from the exact bf16 / float32 inputs.  Tolerances:

* row losses and log-partitions: the logits are sums of H exact products in
  float32, off by at most H 2^-24 sum |h w| (one rounding per addition; the
  tensor cores' own order and truncation stay within it), a log-partition by
  no more than its logits are, plus 8 float32 ulps of the largest value that
  is rounded on the way (the row's log-partition and target logits over T)
  and the 2^-20 relative error of the exponentials in the sum;
* gradients of the logits: each element a (q - p): relative error of q from
  its exponent (the absolute error of its logit and log-partition, above) and
  of a few float32 steps, then one rounding to the gradient's type (bf16:
  2^-8 relative);
* d_hidden and d_weight: that error carried through |W| or |hidden|, plus the
  float32 summation bound n 2^-24 of the products' absolute sum, plus one bf16
  rounding of the result.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def vsd():
    from paper_2602_05774_gb300 import build, vsd as v
    build.build_library()
    v.load()
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    return v


def f64(t):
    return t.detach().double().cpu()


def plain(x, ids, p, counted, w, T):
    """Loss, row losses, log-partitions and d loss / d x of float64 logits x, for
    targets p on ids (one list per row, float64)."""
    y = x / T
    top = y.max(1).values
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    y = y - top[:, None]  # (all further terms relative to the row's maximum)
    ls = torch.log(torch.exp(y).sum(1))
    at = torch.gather(y, 1, ids)
    logp = torch.where(p > 0, torch.log(torch.where(p > 0, p, torch.ones_like(p))), 0.0)
    terms = torch.where(p > 0, p * (logp - at + ls[:, None]), torch.zeros_like(p))
    row = torch.where(counted, terms.sum(1), torch.zeros_like(ls))
    wr = torch.where(counted, w, torch.zeros_like(w))
    tot = wr.sum() if wr.sum() > 0 else torch.ones(())
    a = (wr / (tot * T))[:, None]
    g = torch.exp(y - ls[:, None])
    g.scatter_add_(1, ids, -p)
    g = torch.where(counted[:, None], a * g, torch.zeros_like(g))
    logz = top + ls
    loss = torch.where(wr > 0, wr * row, torch.zeros_like(row)).sum() / tot
    return dict(loss=loss, row_loss=row, logz=torch.where(counted, logz, 0.0), g=g, a=a)


def teacher_target(ids, t, T, V):
    """(ids, p, counted) in float64 from a teacher's list with negative ids and
    -inf logits."""
    ids = ids.cpu().long()
    t = f64(t)
    ok = (ids >= 0) & (ids < V)
    t = torch.where(ok, t, torch.full_like(t, -np.inf))
    m = t.max(1).values
    counted = torch.isfinite(m)
    e = torch.exp((t - torch.where(counted, m, torch.zeros_like(m))[:, None]) / T)
    z = torch.where(counted, e.sum(1), torch.ones_like(m))
    return torch.where(ok, ids, torch.zeros_like(ids)), e / z[:, None], counted


U = 2.0 ** -24


def logit_bound(h, w):
    """Per row: how far a float32 sum of the row's products may be off."""
    if w is None:
        return None
    return (h.shape[1] * U) * (h.abs() @ w.abs().T)


def check(got, ref, x, xerr, T, dtype, h=None, w=None, ids=None, p=None, scale=1.0):
    """got: the library's outputs; ref: plain()'s; xerr: bound of each logit's
    error (0 for logits in hand)."""
    y = x.abs().where(torch.isfinite(x), torch.zeros_like(x)) / T
    row_err = xerr.max(1).values / T
    # values that are rounded on the way to a row's loss and log-partition
    big = torch.maximum(y.max(1).values, ref["logz"].abs()).clamp(min=1.0)
    tol = 2 * row_err + 8 * 2 * U * big + 2.0 ** -20
    for name in ("row_loss", "logz"):
        a, b = f64(got[name]), ref[name]
        fin = torch.isfinite(b)
        assert torch.equal(torch.isnan(a), torch.isnan(b)), name
        assert torch.equal(a[~fin & ~torch.isnan(b)], b[~fin & ~torch.isnan(b)]), name
        err = (a - b).abs()[fin]
        assert (err <= tol[fin]).all(), (name, float((err - tol[fin]).max()), float(err.max()))
    if torch.isfinite(ref["loss"]):
        assert abs(float(got["loss"]) - float(ref["loss"])) <= float(tol.max()) + 2 * U * abs(
            float(ref["loss"]))
    # d loss / d x: q's relative error, then that of the coefficient and steps
    q_rel = 2 * (xerr / T + row_err[:, None]) + 16 * 2 * U * big[:, None] + 2.0 ** -20
    a = ref["a"] * abs(scale)
    q = (ref["g"] / ref["a"].where(ref["a"] > 0, torch.ones_like(ref["a"])))
    if ids is not None:
        q = q.scatter_add(1, ids, p)
    gerr = a * (q.abs() * q_rel + 8 * U)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    g = ref["g"] * scale
    gerr = gerr + half * (g.abs() + gerr) + 2.0 ** -126
    if "grad" in got:
        err = (f64(got["grad"]) - g).abs()
        assert (err <= gerr).all(), ("grad", float((err / gerr).max()))
    if h is not None and "d_hidden" in got:
        b = gerr @ w.abs() + (w.shape[0] * U) * (g.abs() @ w.abs())
        want = g @ w
        b = b + 2.0 ** -8 * (want.abs() + b) + 2.0 ** -126
        err = (f64(got["d_hidden"]) - want).abs()
        assert (err <= b).all(), ("d_hidden", float((err / b).max()))
    if h is not None and "d_weight" in got:
        b = gerr.T @ h.abs() + (h.shape[0] * U) * (g.abs().T @ h.abs())
        want = g.T @ h
        b = b + 2.0 ** -8 * (want.abs() + b) + 2.0 ** -126
        err = (f64(got["d_weight"]) - want).abs()
        assert (err <= b).all(), ("d_weight", float((err / b).max()))


def head(R, V, H, seed, gain=0.05):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(R, H, generator=g, device="cuda").to(torch.bfloat16)
    w = (gain * torch.randn(V, H, generator=g, device="cuda")).to(torch.bfloat16)
    return h, w, g


def teacher(R, V, K, g, dtype=torch.float32, dup=False):
    if dup:
        ids = torch.randint(0, V, (R, K), generator=g, device="cuda")
    else:
        ids = torch.rand(R, V, generator=g, device="cuda").topk(K, dim=1).indices
    t = 3.0 * torch.randn(R, K, generator=g, device="cuda")
    return ids.to(torch.int32), t.to(dtype)


XENT = [  # R, V, H, piece
    (1, 1, 8, 0), (1, 5, 8, 0), (3, 257, 64, 0), (32, 1024, 256, 0), (129, 1000, 72, 256),
    (257, 2049, 136, 512), (300, 777, 1032, 256), (513, 4096, 64, 1024), (64, 8191, 264, 0),
    (700, 1536, 512, 768), (100, 3000, 520, 0), (128, 700, 264, 0), (65, 33000, 40, 0),
    (17, 20011, 1000, 0)]


@pytest.mark.parametrize("R,V,H,piece", XENT)
@pytest.mark.parametrize("weighted", [False, True])
def test_cross_entropy(vsd, R, V, H, piece, weighted):
    h, w, g = head(R, V, H, 100 + R + V, gain=0.3 / H ** 0.5 + 0.02)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    if R > 2:
        labels[torch.randperm(R, generator=g, device="cuda")[: R // 3]] = -100
    rw = torch.rand(R, generator=g, device="cuda") if weighted else None
    got = vsd.lmhead_cross_entropy(h, w, labels, row_weight=rw, piece=piece)
    lab = labels.cpu().long()
    counted = lab != -100
    ids, p = lab.clamp(min=0)[:, None], counted.double()[:, None]
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, ids, p, counted, f64(rw) if weighted else torch.ones(R).double(), 1.0)
    check(got, ref, x, logit_bound(H64, W64), 1.0, torch.bfloat16, H64, W64, ids, p)


DISTILL = [  # R, V, H, K, T, teacher type, piece
    (1, 9, 8, 1, 1.0, torch.float32, 0), (5, 300, 64, 4, 2.0, torch.bfloat16, 0),
    (33, 1024, 256, 10, 0.7, torch.float32, 0), (200, 1537, 264, 64, 1.0, torch.bfloat16, 512),
    (260, 600, 128, 128, 2.0, torch.float32, 256), (130, 4100, 520, 33, 1.0, torch.float32, 1024)]


@pytest.mark.parametrize("R,V,H,K,T,tdt,piece", DISTILL)
def test_lmhead_distill(vsd, R, V, H, K, T, tdt, piece):
    h, w, g = head(R, V, H, 300 + R + V, gain=1.0 / H ** 0.5)
    ids, t = teacher(R, V, K, g, tdt)
    if R > 4:  # rows with shorter lists, one with none; what they lack holds NaN
        n = torch.randint(1, K + 1, (R, 1), generator=g, device="cuda")
        n[3] = 0
        lacks = torch.arange(K, device="cuda") >= n
        ids, t = ids.masked_fill(lacks, -1), t.masked_fill(lacks, NAN)
    rw = 1.05 ** (torch.arange(R, device="cuda") % 8).float()
    got = vsd.lmhead_distill(h, w, ids, t, T=T, row_weight=rw, grad_scale=T * T, piece=piece)
    i64, p, counted = teacher_target(ids, t, T, V)
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, i64, p, counted, f64(rw), T)
    check(got, ref, x, logit_bound(H64, W64), T, torch.bfloat16, H64, W64, i64, p, scale=T * T)


TOPK = [  # R, V, K, T, logits' type, teacher's type
    (1, 1, 1, 1.0, torch.float32, torch.float32), (2, 7, 3, 1.0, torch.bfloat16, torch.float32),
    (16, 1024, 10, 1.0, torch.float32, torch.float32), (9, 1031, 128, 0.7, torch.float32, torch.bfloat16),
    (7, 32003, 100, 2.0, torch.bfloat16, torch.bfloat16), (40, 32000, 32, 1.0, torch.bfloat16, torch.float32),
    (5, 128256, 10, 0.7, torch.bfloat16, torch.float32), (3, 128256, 64, 1.0, torch.float32, torch.float32),
    (2, 300008, 16, 1.0, torch.float32, torch.float32), (2, 1048576, 8, 1.0, torch.bfloat16, torch.bfloat16),
    (611, 520, 5, 1.0, torch.float32, torch.bfloat16)]


@pytest.mark.parametrize("R,V,K,T,dt,tdt", TOPK)
@pytest.mark.parametrize("inplace", [False, True])
def test_topk_distill(vsd, R, V, K, T, dt, tdt, inplace):
    g = torch.Generator(device="cuda").manual_seed(500 + R + V)
    x = (4.0 * torch.randn(R, V, generator=g, device="cuda")).to(dt)
    ids, t = teacher(R, V, K, g, tdt)
    rw = torch.rand(R, generator=g, device="cuda")
    x64 = f64(x)
    if R > 4:
        ids[2, K // 2:] = -1
        ids[4] = -1
        x[4] = NAN  # a row not counted may hold anything
    got = vsd.topk_distill(x, ids, t, T=T, row_weight=rw, grad_scale=T * T,
                           grad=x if inplace else True)
    i64, p, counted = teacher_target(ids, t, T, V)
    ref = plain(x64, i64, p, counted, f64(rw), T)
    check(got, ref, x64, torch.zeros_like(x64), T, dt, ids=i64, p=p, scale=T * T)
    if inplace:
        assert got["grad"].data_ptr() == x.data_ptr()


@pytest.mark.parametrize("R,V,dt", [(3000, 301, torch.float32), (2500, 1000, torch.bfloat16),
                                    (260, 100003, torch.bfloat16), (40, 500009, torch.float32)])
def test_topk_distill_many_rows(vsd, R, V, dt):
    """More rows than are resident at once (a cluster takes several in turn, the
    last ones in rounds), some not counted and full of NaN."""
    g = torch.Generator(device="cuda").manual_seed(R + V)
    K, T = 6, 1.5
    x = (3.0 * torch.randn(R, V, generator=g, device="cuda")).to(dt)
    ids = torch.randint(0, V, (R, K), generator=g, device="cuda").to(torch.int32)
    t = 3.0 * torch.randn(R, K, generator=g, device="cuda")
    x64 = f64(x)
    off = torch.randperm(R, generator=g, device="cuda")[: R // 4]
    ids[off] = -1
    x[off] = NAN
    got = vsd.topk_distill(x, ids, t, T=T)
    i64, p, counted = teacher_target(ids, t, T, V)
    ref = plain(x64, i64, p, counted, torch.ones(R).double(), T)
    check(got, ref, x64, torch.zeros(()).expand(R, 1).double(), T, dt, ids=i64, p=p)
    assert (got["grad"][off] == 0).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,skip,gskip", [(1000, 1, 1), (1003, 3, 3), (1000, 1, 0), (1003, 2, 5),
                                          (16, 1, 0), (2, 1, 1)])
def test_alignment(vsd, dt, V, skip, gskip):
    """Logits and gradients that start anywhere (contiguous views into larger
    tensors), on the same offset from a 16-byte boundary or not: the values of
    the aligned call, and nothing written outside."""
    R, K = 9, 2
    g = torch.Generator(device="cuda").manual_seed(V + skip)
    pool = torch.randn(R * V + 64, generator=g, device="cuda").to(dt)
    x = pool[skip:skip + R * V].view(R, V)
    ids, t = teacher(R, V, K, g)
    want = vsd.topk_distill(x.clone(), ids, t)
    gpool = torch.full((R * V + 64,), 7.0, device="cuda", dtype=dt)
    out = gpool[gskip:gskip + R * V].view(R, V)
    got = vsd.topk_distill(x, ids, t, grad=out)
    for name in ("row_loss", "logz", "grad"):
        a, b = got[name].float(), want[name].float()
        assert torch.allclose(a, b, rtol=2e-2 if dt == torch.bfloat16 and name == "grad" else 1e-5,
                              atol=1e-6), name
    assert (gpool[:gskip] == 7.0).all() and (gpool[gskip + R * V:] == 7.0).all()


def test_topk_offsets_past_32_bits(vsd):
    R, V, K = 20000, 128256, 4
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(R, V, dtype=torch.bfloat16, device="cuda")
    for r in range(0, R, 1000):
        x[r:r + 1000] = 3.0 * torch.randn(1000, V, generator=g, device="cuda")
    ids = torch.randint(0, V, (R, K), generator=g, device="cuda").to(torch.int32)
    t = torch.randn(R, K, generator=g, device="cuda")
    got = vsd.topk_distill(x, ids, t)
    rows = torch.tensor([0, 1, 16743, 16744, R - 2, R - 1], device="cuda")
    i64, p, counted = teacher_target(ids[rows], t[rows], 1.0, V)
    x64 = f64(x[rows])
    ref = plain(x64, i64, p, counted, torch.ones(len(rows)).double(), 1.0)
    # the mean is over all R rows
    for name in ("g", "a"):
        ref[name] = ref[name] * (len(rows) / R)
    ref["loss"] = torch.tensor(NAN)
    sub = dict(loss=got["loss"], row_loss=got["row_loss"][rows], logz=got["logz"][rows],
               grad=got["grad"][rows])
    check(sub, ref, x64, torch.zeros(()).expand(len(rows), 1).double(), 1.0, torch.bfloat16,
          ids=i64, p=p)


def test_lmhead_offsets_past_32_bits(vsd):
    """The largest vocabulary with a hidden size that takes the weight past 2^31
    elements; the last rows of its gradient against float64."""
    R, V, H = 5, 1 << 20, 2056
    g = torch.Generator(device="cuda").manual_seed(11)
    h = torch.randn(R, H, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    for v in range(0, V, 1 << 17):
        w[v:v + (1 << 17)] = 0.02 * torch.randn(1 << 17, H, generator=g, device="cuda")
    labels = torch.tensor([0, V - 1, 5, V - 300, 1044479], dtype=torch.int32, device="cuda")
    got = vsd.lmhead_cross_entropy(h, w, labels)
    x = torch.cat([(h.double() @ w[v:v + (1 << 17)].double().T).cpu() for v in range(0, V, 1 << 17)],
                  dim=1)
    lab = labels.cpu().long()[:, None]
    ref = plain(x, lab, torch.ones(R, 1).double(), torch.ones(R).bool(), torch.ones(R).double(), 1.0)
    H64 = f64(h)
    rows = slice(V - 400, V)
    tol = 2 * float((H * U) * (H64.abs() @ f64(w[rows]).abs().T).max()) + 2.0 ** -18
    assert ((f64(got["row_loss"]) - ref["row_loss"]).abs() <= tol).all()
    want = ref["g"][:, rows].T @ H64
    bound = 2.0 ** -7 * (ref["g"][:, rows].abs().T @ H64.abs()) + 2.0 ** -126
    assert ((f64(got["d_weight"][rows]) - want).abs() <= bound).all()


def test_gradients_against_differences(vsd):
    """Central differences of the library's own float32 loss along random
    directions (topk_distill on float32 logits): truncation of a third-order
    term, |d|^3 eps^2 / 6 with bounded third derivatives, and the loss's own
    rounding over 2 eps."""
    g = torch.Generator(device="cuda").manual_seed(9)
    R, V, K, T = 6, 500, 7, 1.3
    x = torch.randn(R, V, generator=g, device="cuda")
    ids, t = teacher(R, V, K, g)
    rw = torch.rand(R, generator=g, device="cuda") + 0.1
    grad = f64(vsd.topk_distill(x, ids, t, T=T, row_weight=rw)["grad"])
    eps = 2.0 ** -5
    for _ in range(6):
        d = torch.randint(0, 2, (R, V), generator=g, device="cuda").float() * 2 - 1
        up = vsd.topk_distill(x + eps * d, ids, t, T=T, row_weight=rw, grad=False)["loss"]
        dn = vsd.topk_distill(x - eps * d, ids, t, T=T, row_weight=rw, grad=False)["loss"]
        fd = (float(up) - float(dn)) / (2 * eps)
        an = float((grad * f64(d)).sum())
        # |d^3 lse| <= 2 (2 max|d| / T)^3 / 8; x +- eps d is rounded to 2^-24 |x|
        third = 2 * (2 / T) ** 3 / 8 * eps ** 2 / 6
        rounding = (2 ** -20 * 8 + 2 ** -22 * float(x.abs().max())) / eps
        assert abs(fd - an) <= third + rounding, (fd, an, third + rounding)


def test_duplicate_ids_add_and_mass_at_the_ends(vsd):
    """Equal ids add; -inf and lowest-value teacher logits carry no mass; a row
    of equal lowest values is uniform."""
    R, V, K, H = 6, 300, 8, 64
    h, w, g = head(R, V, H, 77, gain=0.1)
    ids, t = teacher(R, V, K, g, dup=True)
    ids[0] = 17                      # one token, eight times
    ids[1, :4] = ids[1, 4:]
    t[2, 1:] = -float("inf")
    t[3, 2] = torch.finfo(torch.float32).min
    t[4] = torch.finfo(torch.float32).min
    i64, p, counted = teacher_target(ids, t, 1.0, V)
    assert counted.all()
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    # p log p is taken entry by entry, as listed
    ref = plain(x, i64, p, counted, torch.ones(R).double(), 1.0)
    got = vsd.lmhead_distill(h, w, ids, t)
    check(got, ref, x, logit_bound(H64, W64), 1.0, torch.bfloat16, H64, W64, i64, p)
    xb = x.float().cuda()
    got = vsd.topk_distill(xb, ids, t)
    ref = plain(f64(xb), i64, p, counted, torch.ones(R).double(), 1.0)
    check(got, ref, f64(xb), torch.zeros_like(x), 1.0, torch.float32, ids=i64, p=p)


@pytest.mark.parametrize("piece", [0, 256])
def test_rows_not_counted_hold_anything(vsd, piece):
    """A row with an ignored label may hold NaN or infinities: the others'
    results do not change by a bit, and its own are zero."""
    R, V, H = 300, 900, 128
    h, w, g = head(R, V, H, 5)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    off = torch.randperm(R, generator=g, device="cuda")[:120]
    labels[off] = -100
    ws = torch.empty(vsd.lmhead_loss_workspace_bytes(R, V, H, 1, True, piece), dtype=torch.uint8,
                     device="cuda")
    a = vsd.lmhead_cross_entropy(h, w, labels, piece=piece, workspace=ws)
    h2 = h.clone()
    h2[off[:60]] = NAN
    h2[off[60:]] = float("inf")
    ws.fill_(0xFF)  # NaN in every workspace float
    b = vsd.lmhead_cross_entropy(h2, w, labels, piece=piece, workspace=ws)
    assert vsd.device_status(ws) == (0, 0)
    for name in a:
        assert torch.equal(a[name], b[name]), name
        assert torch.isfinite(a[name].float()).all(), name
    assert (b["row_loss"][off] == 0).all() and (b["d_hidden"][off] == 0).all()


@pytest.mark.parametrize("piece", [0, 256])
def test_no_row_counted(vsd, piece):
    h, w, g = head(40, 600, 64, 6)
    labels = torch.full((40,), 7, dtype=torch.int32, device="cuda")
    ws = torch.full((vsd.lmhead_loss_workspace_bytes(40, 600, 64, 1, True, piece),), 255,
                    dtype=torch.uint8, device="cuda")
    out = vsd.lmhead_cross_entropy(h * NAN, w, labels, ignore_index=7, piece=piece, workspace=ws)
    zero = vsd.lmhead_cross_entropy(h, w, labels, row_weight=torch.zeros(40, device="cuda"),
                                    piece=piece)
    ids = torch.full((40, 3), -1, dtype=torch.int32, device="cuda")
    t = torch.full((40, 3), NAN, device="cuda")
    x = torch.full((40, 600), NAN, device="cuda")
    top = vsd.topk_distill(x, ids, t)
    for o in (out, top):
        for name, v in o.items():
            assert (v == 0).all(), name
    assert float(zero["loss"]) == 0 and (zero["d_weight"] == 0).all()
    assert (zero["row_loss"] > 0).all()


def test_status_bits(vsd):
    """Bad labels, ids, weights and teacher logits: a status bit, and the row is
    not counted; a counted row of NaN sets the bit of a bad row."""
    R, V, H = 20, 300, 64
    h, w, g = head(R, V, H, 8)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    ws = torch.empty(vsd.lmhead_loss_workspace_bytes(R, V, H), dtype=torch.uint8, device="cuda")
    good = labels.clone()
    good[3] = -100
    want = vsd.lmhead_cross_entropy(h, w, good, workspace=ws)
    assert vsd.device_status(ws) == (0, 0)
    for bad in (V, -1, 2 ** 31 - 1, -2 ** 31):
        labels[3] = bad
        got = vsd.lmhead_cross_entropy(h, w, labels, workspace=ws)
        assert vsd.device_status(ws) == (6, vsd.STATUS_BAD_TOKEN)
        for name in want:
            assert torch.equal(got[name], want[name]), name
    rw = torch.ones(R, device="cuda")
    for bad in (-1.0, NAN, float("inf")):
        rw[3] = bad
        labels[3] = 5
        got = vsd.lmhead_cross_entropy(h, w, labels, row_weight=rw, workspace=ws)
        assert vsd.device_status(ws) == (6, vsd.STATUS_BAD_ROW)
        assert torch.equal(got["loss"], want["loss"])
    h[7, 5] = NAN
    got = vsd.lmhead_cross_entropy(h, w, good, workspace=ws)
    assert vsd.device_status(ws)[1] == vsd.STATUS_BAD_ROW
    assert torch.isnan(got["row_loss"][7]) and torch.isfinite(got["row_loss"][6])
    x = torch.randn(R, V, generator=g, device="cuda")
    ids, t = teacher(R, V, 4, g)
    wst = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    ids2, t2 = ids.clone(), t.clone()
    ids2[2, 1] = V
    got = vsd.topk_distill(x, ids2, t2, workspace=wst)
    assert vsd.device_status(wst) == (6, vsd.STATUS_BAD_TOKEN)
    ids2[2, 1] = -1
    want = vsd.topk_distill(x, ids2, t2, workspace=wst)
    assert vsd.device_status(wst) == (0, 0)
    assert torch.equal(got["grad"], want["grad"])
    t2[6, 0] = float("inf")
    got = vsd.topk_distill(x, ids, t2, workspace=wst)
    assert vsd.device_status(wst) == (6, vsd.STATUS_BAD_ROW)
    assert (got["grad"][6] == 0).all() and float(got["row_loss"][6]) == 0
    x[5] = -float("inf")
    got = vsd.topk_distill(x, ids, t, workspace=wst)
    assert vsd.device_status(wst)[1] == vsd.STATUS_BAD_ROW


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 1003])
def test_masked_vocabulary(vsd, dt, V):
    """-inf logits carry no mass and no gradient; one at a token the teacher
    wants makes the loss infinite and leaves the gradient finite; the type's
    lowest value is an ordinary logit."""
    R, K = 8, 5
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(R, V, generator=g, device="cuda").to(dt)
    ids, t = teacher(R, V, K, g)
    x[0, : V // 2] = -float("inf")
    ids[0] = torch.arange(V - K, V, device="cuda").to(torch.int32)
    x[1, :] = -float("inf")
    x[1, 11] = 2.0
    ids[1] = 11
    x[2] = torch.finfo(dt).min
    x[3, 1:] = torch.finfo(dt).min
    ids[3, 0] = 0
    t[3, 1:] = -float("inf")
    x[4, int(ids[4, 2])] = -float("inf")
    wst = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    got = vsd.topk_distill(x, ids, t, workspace=wst)
    assert vsd.device_status(wst) == (0, 0)
    x64 = f64(x)
    i64, p, counted = teacher_target(ids, t, 1.0, V)
    ref = plain(x64, i64, p, counted, torch.ones(R).double(), 1.0)
    assert float(got["row_loss"][4]) == float("inf") and float(got["loss"]) == float("inf")
    # rows 2 and 3 are at the type's lowest value, where a rounding of the
    # log-partition is of its size: their gradients are held exactly instead
    assert torch.allclose(f64(got["grad"][2]), ref["g"][2], rtol=2 ** -8, atol=0)
    assert float(got["row_loss"][3]) == 0.0
    keep = torch.tensor([0, 1, 4, 5, 6, 7])
    sub = {k: (v[keep.cuda()] if v.dim() and v.shape[0] == R else v) for k, v in got.items()}
    rs = {k: (v[keep] if v.dim() and v.shape[0] == R else v) for k, v in ref.items()}
    check(sub, rs, x64[keep], torch.zeros_like(x64[keep]), 1.0, dt, ids=i64[keep], p=p[keep])


def test_pieces_and_repeats_agree(vsd):
    """Any piece gives the same row losses within rounding; a repeated call gives
    the same bits, on another stream and a used workspace too."""
    R, V, H = 400, 3001, 264
    h, w, g = head(R, V, H, 21)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    base = vsd.lmhead_cross_entropy(h, w, labels)
    for piece in (256, 1024, 4096):
        a = vsd.lmhead_cross_entropy(h, w, labels, piece=piece)
        assert torch.allclose(a["row_loss"], base["row_loss"], rtol=1e-5, atol=1e-5)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            ws = torch.full((vsd.lmhead_loss_workspace_bytes(R, V, H, 1, True, piece),), 127,
                            dtype=torch.uint8, device="cuda")
            b = vsd.lmhead_cross_entropy(h, w, labels, piece=piece, workspace=ws)
        s.synchronize()
        for name in a:
            assert torch.equal(a[name], b[name]), (piece, name)


@pytest.mark.parametrize("R,V,H", [(70, 700, 128), (40, 60000, 264), (300, 30000, 72)])
def test_one_gradient_or_none(vsd, R, V, H):
    """One gradient alone (its sums may be cut into other parts than with both,
    so d_hidden agrees to a rounding), on a workspace of the size asked for."""
    h, w, g = head(R, V, H, 3)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    ws = torch.empty(vsd.lmhead_loss_workspace_bytes(R, V, H), dtype=torch.uint8, device="cuda")
    both = vsd.lmhead_cross_entropy(h, w, labels)
    dh = torch.empty_like(h)
    a = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=dh, d_weight=False, workspace=ws)
    b = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False, workspace=ws)
    n = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False, d_weight=False)
    assert a["d_hidden"] is dh and "d_weight" not in a
    scale = float(both["d_hidden"].float().abs().max())
    assert torch.allclose(dh.float(), both["d_hidden"].float(), rtol=2.0 ** -7, atol=1e-5 * scale)
    assert torch.equal(b["d_weight"], both["d_weight"]) and "d_hidden" not in b
    assert torch.equal(n["loss"], both["loss"]) and set(n) == {"loss", "row_loss", "logz"}


@pytest.mark.parametrize("R", [40, 700])
@pytest.mark.parametrize("exponent", [-140, -60, 100, 120])
def test_weights_by_a_factor(vsd, exponent, R):
    """Weights times a power of two, down to where only denormals hold them and up
    to where their sum passes a float: the same bits."""
    g = torch.Generator(device="cuda").manual_seed(R)
    w = torch.randint(1, 9, (R,), generator=g, device="cuda").float()
    far = w * 2.0 ** (exponent // 2) * 2.0 ** (exponent - exponent // 2)
    assert (far > 0).all() and torch.isfinite(far).all()
    x = torch.randn(R, 333, generator=g, device="cuda")
    ids = torch.randint(0, 333, (R, 5), generator=g, device="cuda").to(torch.int32)
    t = torch.randn(R, 5, generator=g, device="cuda")
    h = torch.randn(R, 64, generator=g, device="cuda").bfloat16()
    head_w = torch.randn(333, 64, generator=g, device="cuda").bfloat16()
    for call in (lambda rw: vsd.topk_distill(x, ids, t, row_weight=rw),
                 lambda rw: vsd.lmhead_distill(h, head_w, ids, t, row_weight=rw),
                 lambda rw: vsd.lmhead_cross_entropy(h, head_w, ids[:, 0].contiguous(),
                                                     row_weight=rw)):
        a, b = call(w), call(far)
        for name in a:
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("H", [64, 1024])
@pytest.mark.parametrize("grads", [False, True])
@pytest.mark.parametrize("piece", [0, 256])
def test_logits_at_the_lowest_value(vsd, H, grads, piece):
    """Tokens whose logits come to bfloat16's lowest value, whole tiles of them: as
    if the vocabulary did not have them."""
    R, V = 70, 700
    h, w, g = head(R, V, H, 21)
    h[:, 0] = 1
    w[:, 0] = 0
    labels = torch.randint(0, 128, (R,), generator=g, device="cuda").to(torch.int32)
    masked = torch.cat((w, w))
    masked[128:V] = 0
    masked[V:] = 0
    masked[128:, 0] = torch.finfo(torch.bfloat16).min
    got = vsd.lmhead_cross_entropy(h, masked, labels, d_hidden=grads, d_weight=grads, piece=piece)
    x = f64(h) @ f64(w[:128]).T
    lz = torch.logsumexp(x, 1)
    want = lz - x.gather(1, labels.long()[:, None].to(x.device))[:, 0]
    scale = (f64(h).abs() @ f64(w[:128]).abs().T).max(1).values
    # fp32 sums of H products, of 128 exponentials, and the logarithm's rounding
    bound = 2.0 ** -24 * (2 * H * scale + 300 + 8 * lz.abs())
    assert ((f64(got["row_loss"]) - want).abs() <= bound).all()
    assert torch.isfinite(got["loss"]).all() and torch.isfinite(got["logz"]).all()
    if grads:
        assert torch.isfinite(got["d_hidden"].float()).all()
        assert torch.isfinite(got["d_weight"].float()).all()
        assert (got["d_weight"][128:] == 0).all()


def test_hidden_states_of_paths(vsd):
    """Hidden states as [B, K, D, H]: rows in their order, the gradient in their
    shape; a graph that holds a call gives the call's bits."""
    h, w, g = head(2 * 3 * 8, 500, 64, 12)
    labels = torch.randint(0, 500, (48,), generator=g, device="cuda").to(torch.int32)
    flat = vsd.lmhead_cross_entropy(h, w, labels)
    got = vsd.lmhead_cross_entropy(h.view(2, 3, 8, 64), w, labels)
    assert got["d_hidden"].shape == (2, 3, 8, 64)
    assert torch.equal(got["d_hidden"].view(48, 64), flat["d_hidden"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = vsd.lmhead_cross_entropy(h, w, labels)
    h.add_(1.0)
    graph.replay()
    want = vsd.lmhead_cross_entropy(h, w, labels)
    for name in want:
        assert torch.equal(held[name], want[name]), name


def test_refusals(vsd):
    h, w, g = head(8, 100, 64, 1)
    labels = torch.zeros(8, dtype=torch.int32, device="cuda")
    ids, t = teacher(8, 100, 3, g)
    x = torch.zeros(8, 100, device="cuda")
    for bad in (lambda: vsd.lmhead_cross_entropy(h.float(), w, labels),
                lambda: vsd.lmhead_cross_entropy(h, w, labels.long()),
                lambda: vsd.lmhead_cross_entropy(h, w, labels[:7]),
                lambda: vsd.lmhead_cross_entropy(h, w[:, :32], labels),
                lambda: vsd.lmhead_cross_entropy(h, w, labels, d_hidden=h.float()),
                lambda: vsd.lmhead_cross_entropy(h, w, labels, d_weight=torch.empty_like(h)),
                lambda: vsd.lmhead_cross_entropy(h, w, labels, row_weight=labels),
                lambda: vsd.lmhead_cross_entropy(h, w.t().contiguous().t(), labels),
                lambda: vsd.lmhead_cross_entropy(h, w, labels.cpu()),
                lambda: vsd.lmhead_cross_entropy(h, w, labels, workspace=torch.empty(
                    256, dtype=torch.uint8, device="cuda")),
                lambda: vsd.lmhead_distill(h, w, ids, t[:, :2]),
                lambda: vsd.lmhead_distill(h, w, ids.long(), t),
                lambda: vsd.lmhead_distill(h, w, ids[:, :0], t[:, :0]),
                lambda: vsd.lmhead_distill(h[:, :60].contiguous(), w[:, :60].contiguous(), ids, t),
                lambda: vsd.topk_distill(x, ids[:4], t[:4]),
                lambda: vsd.topk_distill(x, ids, t, grad=x.bfloat16()),
                lambda: vsd.topk_distill(x[:0], ids[:0], t[:0])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        vsd.lmhead_distill(h, w, ids, t.half())
    with pytest.raises(TypeError):
        vsd.topk_distill(x.half(), ids, t)
    for T in (0.0, -1.0, NAN, float("inf"), 1e-39):
        with pytest.raises(vsd.VsdError) as e:
            vsd.topk_distill(x, ids, t, T=T)
        assert e.value.code == 1
        with pytest.raises(vsd.VsdError) as e:
            vsd.lmhead_distill(h, w, ids, t, T=T)
        assert e.value.code == 1
    with pytest.raises(vsd.VsdError) as e:
        vsd.lmhead_cross_entropy(h, w, labels, grad_scale=NAN)
    assert e.value.code == 1


@pytest.mark.parametrize("R,V,H,K,piece", [(130, 600, 200, 3, 256), (100, 700, 200, 3, 0),
                                           (65, 520, 72, 1, 0), (33, 3000, 456, 9, 1024)])
def test_lanes_that_differ(vsd, R, V, H, K, piece):
    """Warps whose lanes part ways between two reads of tensor memory: a list entry
    in one row of 32 alone, rows past the last, columns past the hidden size."""
    h, w, g = head(R, V, H, 700 + R, gain=1.0 / H ** 0.5)
    ids, t = teacher(R, V, K, g)
    r = torch.arange(R, device="cuda")[:, None]
    ids = torch.where(r % 32 == 5, ids, ids % 8)  # the others' entries: the first columns
    got = vsd.lmhead_distill(h, w, ids, t, piece=piece)
    i64, p, counted = teacher_target(ids, t, 1.0, V)
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, i64, p, counted, torch.ones(R).double(), 1.0)
    check(got, ref, x, logit_bound(H64, W64), 1.0, torch.bfloat16, H64, W64, i64, p)


@pytest.mark.parametrize("H", [64, 1024])
@pytest.mark.parametrize("grads,piece", [(False, 0), (True, 0), (True, 256)])
@pytest.mark.parametrize("T,K", [(1.0, 1), (0.7, 1), (0.7, 2)])
def test_exponents_by_difference(vsd, H, grads, piece, T, K):
    """Logits far from zero, exact (one product each): one or two tokens hold a
    row's mass, so its loss does not depend on how large they are.  The errors left
    are those of logf (an ulp), of one rounding of m / T in logz, and with two
    entries of their probabilities (expf and a division: 2^-20 in all)."""
    R, V = 200, 700
    g = torch.Generator(device="cuda").manual_seed(31)
    m = (100.0 + 4000.0 * torch.rand(H, generator=g, device="cuda") ** 2).bfloat16()
    pair = torch.rand(V, H, generator=g, device="cuda").topk(2, dim=0).indices  # two tokens a column
    two = torch.arange(H, device="cuda") % 2 == 1
    w = torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    w.scatter_(0, pair[:1], m[None])
    w.scatter_(0, pair[1:], torch.where(two, m, torch.zeros_like(m))[None])
    col = torch.arange(R, device="cuda") % H
    h = torch.zeros(R, H, dtype=torch.bfloat16, device="cuda")
    h[torch.arange(R, device="cuda"), col] = 1.0
    ids = pair[:, col].T.to(torch.int32)
    ids[:, 1].masked_fill_(~two[col], -1)
    ids = ids[:, :K].contiguous()
    t = torch.randn(R, K, generator=g, device="cuda")
    got = vsd.lmhead_distill(h, w, ids, t, T=T, d_hidden=grads, d_weight=grads, piece=piece)
    T = float(np.float32(T))  # (the temperature that the call takes)
    _, p, counted = teacher_target(ids, t, T, V)
    assert counted.all()
    two, m = two[col].cpu(), f64(m[col])
    ls = torch.where(two, np.log(2.0), 0.0).double()
    want = torch.where(p > 0, p * torch.log(p.clamp(min=1e-300)), 0.0).sum(1) + ls
    assert ((f64(got["row_loss"]) - want).abs() <= 2.0 ** -23 + (K - 1) * 2.0 ** -20).all()
    lz = m / T + ls
    assert ((f64(got["logz"]) - lz).abs() <= 2.0 ** -24 * lz + 2.0 ** -23).all()
    if grads:
        share = 1.0 / (R * T)
        dw, size = torch.zeros(2, V, H, dtype=torch.float64)
        for r in range(R):
            c = int(col[r])
            for k in range(2):
                q = 0.5 if two[r] else 1.0 - k
                term = share * (q - (float(p[r, k]) if k < K else 0.0))
                dw[int(pair[k, c]), c] += term
                size[int(pair[k, c]), c] += abs(term)
        # each term's rounding in G, the output's, and the probabilities' error
        err = (f64(got["d_weight"]) - dw).abs()
        bound = 2.0 ** -8 * (size + dw.abs()) + (K - 1) * 4 * share * 2.0 ** -20 + 1e-30
        assert (err <= bound).all()


@pytest.mark.parametrize("H", [64, 1024])
@pytest.mark.parametrize("grads,piece", [(False, 0), (True, 0), (True, 256)])
def test_rows_at_the_lowest_value(vsd, H, grads, piece):
    """Rows whose logits are all bfloat16's lowest value are uniform."""
    R, V = 70, 512
    h = torch.zeros(R, H, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1
    w = torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = torch.finfo(torch.bfloat16).min
    labels = (torch.arange(R, device="cuda") * 7 % V).to(torch.int32)
    ws = torch.empty(vsd.lmhead_loss_workspace_bytes(R, V, H, 1, grads, piece), dtype=torch.uint8,
                     device="cuda")
    got = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False, d_weight=grads, piece=piece,
                                   workspace=ws)
    assert vsd.device_status(ws) == (0, 0)
    assert (got["logz"] == torch.finfo(torch.bfloat16).min).all()  # log V is below its last bit
    # logf's ulp at 6.2 and the result's rounding
    assert ((f64(got["row_loss"]) - np.log(V)).abs() <= 2.0 ** -20).all()
    if grads:
        q = torch.full((V,), 1.0 / V, dtype=torch.float64)
        q -= torch.bincount(labels.cpu().long(), minlength=V) / R
        # G's entries, R of 1 / V and the label's, and the output: 2^-8 each
        label = torch.bincount(labels.cpu().long(), minlength=V) / R
        bound = 2.0 ** -8 * (2.0 / V + label + q.abs())
        assert ((f64(got["d_weight"])[:, 0] - q).abs() <= bound).all()


def test_d_weight_of_many_rows(vsd):
    """Eight million rows whose terms all have one sign: G is exact (q = 1/2), so
    what is left is the sum's error and the rounding to bfloat16.  An uncut part of
    the sum has 4096 steps, each truncated by an ulp at most."""
    R, V, H = 1 << 23, 2, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    h = (1.0 + torch.rand(R, H, generator=g, device="cuda")).bfloat16()
    w = torch.zeros(V, H, dtype=torch.bfloat16, device="cuda")
    labels = torch.zeros(R, dtype=torch.int32, device="cuda")
    got = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False)
    want = 0.5 * f64(h.double().mean(0))
    err = torch.maximum((f64(got["d_weight"][0]) + want).abs(),
                        (f64(got["d_weight"][1]) - want).abs()) / want
    assert (err <= 2.0 ** -8 + 4096 * 2.0 ** -23).all(), err


def test_gradient_at_a_long_hidden_size(vsd):
    """A hidden size whose sums take 32768 steps: the gradient's logits are as near
    as parts of 512 steps make them, each step truncated by an ulp at most."""
    R, V, H = 1, 512, 1 << 19
    g = torch.Generator(device="cuda").manual_seed(2)
    h = (1.0 + torch.rand(R, H, generator=g, device="cuda")).bfloat16()
    top = 12.0 + 4.0 * torch.rand(V, 1, generator=g, device="cuda")
    w = (top / (1.5 * H) * (0.5 + torch.rand(V, H, generator=g, device="cuda"))).bfloat16()
    labels = torch.zeros(R, dtype=torch.int32, device="cuda")
    got = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False, piece=256)
    x = torch.cat([h.double() @ w[v:v + 64].double().T for v in range(0, V, 64)], 1)[0]
    q = torch.softmax(x, 0)
    have = torch.cat([(got["d_weight"][v:v + 64].double() / h.double()).mean(1)
                      for v in range(0, V, 64)])
    rel = ((have - q) / q)[1:].cpu()  # (the label's q - 1 is rounded at 1)
    # G's rounding (the outputs' own averages out over H: 1e-4), and the parts of the
    # logits and of the log-partition
    assert (rel.abs() <= 2.0 ** -8 + 2 * 512 * 2.0 ** -23 * float(x.max()) + 1e-4).all()


@pytest.mark.parametrize("R,V,H,K,piece", [(300, 700, 16456, 5, 256), (66000, 300, 72, 1, 256),
                                           (40, 66000, 64, 3, 0)])
def test_sums_in_parts(vsd, R, V, H, K, piece):
    """Hidden sizes, rows and vocabularies at which sums are cut, or just are not."""
    h, w, g = head(R, V, H, 900 + R, gain=1.0 / H ** 0.5)
    ids = torch.randint(0, V, (R, K), generator=g, device="cuda").to(torch.int32)
    t = torch.randn(R, K, generator=g, device="cuda")
    ids[1::7] = -1
    got = vsd.lmhead_distill(h, w, ids, t, piece=piece)
    i64, p, counted = teacher_target(ids, t, 1.0, V)
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, i64, p, counted, torch.ones(R).double(), 1.0)
    check(got, ref, x, logit_bound(H64, W64), 1.0, torch.bfloat16, H64, W64, i64, p)


@pytest.mark.parametrize("R,V,H,dw", [(40, 65800, 38912, False), (100, 65800, 38912, False),
                                      (2048, 131072, 6144, True)])
def test_d_hidden_of_long_sums(vsd, R, V, H, dw):
    """d_hidden over more columns than an uncut sum has, in one part (many tiles), for
    turned tiles and others: some rows and columns against float64."""
    g = torch.Generator(device="cuda").manual_seed(R)
    h = torch.randn(R, H, generator=g, device="cuda").bfloat16()
    w = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    for v in range(0, V, 1 << 14):
        n = min(V, v + (1 << 14)) - v
        w[v:v + n] = 2.0 / H ** 0.5 * torch.randn(n, H, generator=g, device="cuda")
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    got = vsd.lmhead_cross_entropy(h, w, labels, d_weight=dw)
    rows = torch.arange(0, R, max(1, R // 13), device="cuda")
    cols = torch.arange(0, H, 97, device="cuda")
    x = torch.cat([(h[rows].double() @ w[v:v + 8192].double().T) for v in range(0, V, 8192)], 1)
    size = torch.cat([(h[rows].double().abs() @ w[v:v + 8192].double().abs().T).amax(1, keepdim=True)
                      for v in range(0, V, 8192)], 1).amax(1)
    lab = labels[rows].long()[:, None]
    G = torch.softmax(x, 1)
    assert ((torch.logsumexp(x, 1) - x.gather(1, lab)[:, 0] - got["row_loss"][rows].double()).abs()
            <= 2 * H * U * size + 2.0 ** -18).all()
    G.scatter_add_(1, lab, -torch.ones_like(lab, dtype=torch.float64))
    G /= R
    W64 = w[:, cols].double()
    want, mass = G @ W64, G.abs() @ W64.abs()
    # a logit's error in q, G's rounding, the cut sums' truncation (4096 steps a part),
    # the output's rounding
    bound = mass * (2 * H * U * size[:, None] + 2.0 ** -8 + 4096 * 2.0 ** -23) + 2.0 ** -8 * want.abs()
    assert ((got["d_hidden"][rows][:, cols].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("weighted", [False, True])
def test_mean_of_the_losses(vsd, weighted):
    """The mean of the rows' losses is taken in 64 bits and rounded once."""
    for seed in range(8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        R, V = 3001, 50
        x = 3.0 * torch.randn(R, V, generator=g, device="cuda")
        ids = torch.randint(0, V, (R, 2), generator=g, device="cuda").to(torch.int32)
        t = torch.randn(R, 2, generator=g, device="cuda")
        rw = torch.rand(R, generator=g, device="cuda") if weighted else None
        got = vsd.topk_distill(x, ids, t, row_weight=rw, grad=False)
        w64 = f64(rw) if weighted else torch.ones(R).double()
        want = float((w64 * f64(got["row_loss"])).sum() / w64.sum())
        assert abs(float(got["loss"]) - want) <= 2.0 ** -24 * (1 + 1e-6) * want, (seed, want)


@pytest.mark.parametrize("R,V,H,piece", [(40, 3000, 264, 0), (100, 700, 72, 0), (300, 2000, 136, 256),
                                         (300, 2000, 136, 0)])
def test_a_gradient_alone_in_its_tensors_place(vsd, R, V, H, piece):
    """One gradient alone may be written over the tensor it is the gradient of; with
    both that is refused, and so is any other overlap."""
    h, w, g = head(R, V, H, 40 + R)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    for skip in (False, True):
        if skip:
            labels[::3] = -100
        kw = dict(piece=piece)
        want_h = vsd.lmhead_cross_entropy(h, w, labels, d_weight=False, **kw)["d_hidden"]
        want_w = vsd.lmhead_cross_entropy(h, w, labels, d_hidden=False, **kw)["d_weight"]
        h2, w2 = h.clone(), w.clone()
        vsd.lmhead_cross_entropy(h2, w, labels, d_hidden=h2, d_weight=False, **kw)
        vsd.lmhead_cross_entropy(h, w2, labels, d_hidden=False, d_weight=w2, **kw)
        assert torch.equal(h2, want_h) and torch.equal(w2, want_w)
    x = torch.zeros(R * 50 + 8, device="cuda")
    ids, t = teacher(R, 50, 2, g)
    for bad in (lambda: vsd.lmhead_cross_entropy(h, w, labels, d_hidden=h),
                lambda: vsd.lmhead_cross_entropy(h, w, labels, d_weight=w),
                lambda: vsd.lmhead_cross_entropy(h, w[:R], labels, d_hidden=w[:R], d_weight=False),
                lambda: vsd.topk_distill(x[:R * 50].view(R, 50), ids, t,
                                         grad=x[8:].view(R, 50))):
        with pytest.raises(vsd.VsdError) as e:
            bad()
        assert e.value.code == 1


KEPT = [  # R, V, H, K: more than 128 rows whose logits are kept, in one part of K or several
    (129, 1000, 64, 1), (257, 3000, 264, 4), (300, 3000, 520, 1), (513, 1500, 1032, 33),
    (300, 33000, 40, 3), (1000, 2000, 136, 128)]


@pytest.mark.parametrize("R,V,H,K", KEPT)
@pytest.mark.parametrize("ignored", [False, True])
def test_kept_logits(vsd, R, V, H, K, ignored):
    """The library's choice for some hundred rows, with every row counted and not."""
    h, w, g = head(R, V, H, 1100 + R, gain=1.0 / H ** 0.5)
    ids, t = teacher(R, V, K, g)
    if ignored:
        ids[torch.randperm(R, generator=g, device="cuda")[: R // 3]] = -1
    rw = torch.rand(R, generator=g, device="cuda")
    got = vsd.lmhead_distill(h, w, ids, t, T=2.0, row_weight=rw)
    i64, p, counted = teacher_target(ids, t, 2.0, V)
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, i64, p, counted, f64(rw), 2.0)
    check(got, ref, x, logit_bound(H64, W64), 2.0, torch.bfloat16, H64, W64, i64, p)


def test_several_pieces_by_the_librarys_choice(vsd):
    """4096 rows whose G passes a piece: all gradients against float64."""
    R, V, H = 4096, 20000, 72
    h, w, g = head(R, V, H, 17, gain=0.1)
    labels = torch.randint(0, V, (R,), generator=g, device="cuda").to(torch.int32)
    labels[::5] = -100
    n = vsd.lmhead_loss_workspace_bytes
    assert n(R, V, H) < n(R, V, H, piece=V)  # (more than one piece)
    got = vsd.lmhead_cross_entropy(h, w, labels)
    counted = labels != -100
    H64, W64, lab = h.double(), w.double(), labels.clamp(min=0).long()[:, None]
    x = H64 @ W64.T
    size = (H64.abs() @ W64.abs().T).amax(1)
    G = torch.softmax(x, 1)
    row = torch.where(counted, torch.logsumexp(x, 1) - x.gather(1, lab)[:, 0], 0.0)
    tol = 2 * H * U * size + 16 * U * x.abs().amax(1) + 2.0 ** -20
    assert ((got["row_loss"].double() - row).abs() <= tol).all()
    G.scatter_add_(1, lab, -torch.ones_like(lab, dtype=torch.float64))
    G *= (counted / counted.sum())[:, None]
    # q's error by its logits', G's rounding, fp32 sums, the output's rounding
    rel = 2.0 ** -8 + 2 * float(tol.max())
    for name, a, b in (("d_hidden", G, W64), ("d_weight", G.T, H64)):
        want = a @ b
        bound = (rel + a.shape[1] * U) * (a.abs() @ b.abs()) + 2.0 ** -8 * want.abs()
        assert ((got[name].double() - want).abs() <= bound).all(), name


@pytest.mark.parametrize("R,V,H,K", [(40, 3000, 264, 5), (300, 1537, 1032, 64), (700, 5000, 72, 1)])
def test_distill_without_gradients(vsd, R, V, H, K):
    h, w, g = head(R, V, H, 1300 + R, gain=1.0 / H ** 0.5)
    ids, t = teacher(R, V, K, g, torch.bfloat16)
    ids[1::9] = -1
    rw = torch.rand(R, generator=g, device="cuda")
    got = vsd.lmhead_distill(h, w, ids, t, T=2.0, row_weight=rw, d_hidden=False, d_weight=False)
    assert set(got) == {"loss", "row_loss", "logz"}
    i64, p, counted = teacher_target(ids, t, 2.0, V)
    H64, W64 = f64(h), f64(w)
    x = H64 @ W64.T
    ref = plain(x, i64, p, counted, f64(rw), 2.0)
    check(got, ref, x, logit_bound(H64, W64), 2.0, torch.bfloat16, H64, W64, i64, p)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V,K", [(1, 1, 1), (9, 1031, 128), (700, 2000, 6), (40, 128256, 10)])
def test_topk_without_gradient(vsd, R, V, K, dt):
    g = torch.Generator(device="cuda").manual_seed(1500 + R)
    x = (4.0 * torch.randn(R, V, generator=g, device="cuda")).to(dt)
    ids, t = teacher(R, V, K, g)
    if R > 4:
        ids[3] = -1
        x[3] = NAN
    x64 = f64(x)
    got = vsd.topk_distill(x, ids, t, T=0.75, grad=False)
    assert set(got) == {"loss", "row_loss", "logz"}
    i64, p, counted = teacher_target(ids, t, 0.75, V)
    ref = plain(x64, i64, p, counted, torch.ones(R).double(), 0.75)
    check(got, ref, x64, torch.zeros(()).expand(R, 1).double(), 0.75, dt, ids=i64, p=p)
