"""CPU checks of the decoding side's C entry points (include/vsd_decode.h): exported
symbols, workspace sizes, and the host-side argument checks, which return before
anything is enqueued."""
import ctypes as C
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
host_only = pytest.mark.skipif(torch.cuda.is_available(),
                               reason="fake device pointers: host-only checks")
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def vsd():
    from paper_2602_05774_gb300 import build, vsd as v
    build.build_library()
    v.load()
    return v


def test_every_declared_symbol_is_exported(vsd):
    src = open(os.path.join(ROOT, "include", "vsd_decode.h")).read()
    names = set(re.findall(r"^\s*[\w\s\*]+?\b(vsd_\w+)\s*\(", src, re.M))
    assert names == set(vsd.DECODE_SYMBOLS)
    for n in names:
        assert hasattr(vsd.load(), n), n


def test_workspace_bytes(vsd):
    n = vsd.load().vsd_sample_filtered_workspace_bytes
    for bad in ((0, 10), (-1, 10), ((1 << 24) + 1, 10), (4, 0), (4, (1 << 20) + 1)):
        assert n(*bad) == 0, bad
    for good in ((1, 1), (4096, 128256), (1 << 24, 1 << 20)):
        assert n(*good) >= 256, good


P = 0x1000000  # never dereferenced: every call below fails its checks


@host_only
def test_quantize_refuses(vsd):
    lib = vsd.load()

    def call(x=P, dt=0, R=256, H=256, rows=1, q=2 * P, s=3 * P):
        return lib.vsd_quantize_fp8(x, dt, R, H, rows, q, s, None)

    for kw in (dict(x=None), dict(q=None), dict(s=None), dict(dt=2), dict(dt=-1), dict(R=0), dict(R=-4),
               dict(R=(1 << 24) + 1), dict(H=0), dict(H=8), dict(H=250), dict(H=(1 << 20) + 16), dict(rows=0),
               dict(rows=2), dict(rows=127), dict(rows=-1), dict(x=P + 4), dict(q=2 * P + 8), dict(s=3 * P + 2),
               dict(q=P), dict(q=P + 16), dict(q=P - 256 * 256 + 16), dict(s=P + 4), dict(s=2 * P + 256 * 256 - 4)):
        assert call(**kw) == 1, kw


@host_only
def test_head_refuses(vsd):
    lib = vsd.load()
    R, V, H = 40, 300, 256

    def call(h=P, hs=2 * P, w=3 * P, ws=4 * P, R=R, V=V, H=H, out=5 * P, wk=6 * P, n=256):
        return lib.vsd_lmhead_logits_fp8(h, hs, w, ws, R, V, H, out, wk, n, None)

    for kw in (dict(h=None), dict(hs=None), dict(w=None), dict(ws=None), dict(out=None), dict(R=0),
               dict(R=(1 << 24) + 1), dict(V=0), dict(V=-1), dict(V=(1 << 20) + 1), dict(H=0), dict(H=8), dict(H=24),
               dict(H=(1 << 20) + 16), dict(h=P + 8), dict(w=3 * P + 4), dict(out=5 * P + 1), dict(hs=2 * P + 2),
               dict(ws=4 * P + 1), dict(out=P), dict(out=P + R * H - 2), dict(out=3 * P + 2),
               dict(out=2 * P + 4 * R * 2 - 2), dict(out=4 * P - 2 * R * V + 2)):
        assert call(**kw) == 1, kw
    for kw in (dict(wk=None), dict(wk=6 * P + 4), dict(n=0), dict(n=255)):
        assert call(**kw) == 5, kw


@host_only
def test_sample_refuses(vsd):
    lib = vsd.load()
    R, V = 8, 1000
    rows = [0x100000 * i + 0x40000000 for i in range(1, 9)]
    T, K, TP, MP, UU, TOK, LQ, KEPT = rows

    def call(x=P, dt=0, R=R, V=V, T=1.0, k=0, p=1.0, mp=0.0, arrays=(None,) * 4, u=UU, out=(TOK, LQ, KEPT, None),
             ws=6 * P, n=1 << 20, null=()):
        pol = vsd.Policy(T, k, p, mp, *arrays)
        o = vsd.FilteredOutputs(*out)
        return lib.vsd_sample_filtered(x, dt, R, V, None if "policy" in null else C.byref(pol), u,
                                       None if "out" in null else C.byref(o), ws, n, None)

    for kw in (dict(x=None), dict(null=("policy",)), dict(null=("out",)), dict(dt=2), dict(R=0), dict(V=0),
               dict(R=(1 << 24) + 1), dict(V=(1 << 20) + 1), dict(x=P + 2), dict(dt=1, x=P + 1), dict(T=NAN),
               dict(T=-1.0), dict(T=INF), dict(T=2.0 ** -65), dict(T=2.0 ** 65), dict(T=1e-45), dict(p=NAN),
               dict(mp=NAN), dict(u=None), dict(u=UU + 2), dict(u=None, out=(TOK, None, KEPT, None)),
               dict(u=None, out=(None, LQ, KEPT, None)), dict(u=None, out=(None,) * 4),
               dict(out=(TOK + 1, LQ, KEPT, None)), dict(out=(TOK, LQ + 2, KEPT, None)),
               dict(out=(TOK, LQ, KEPT, P + 2)), dict(arrays=(T + 2, None, None, None)),
               # outputs over inputs or one another
               dict(out=(TOK, LQ, KEPT, P + 4)), dict(out=(TOK, LQ, KEPT, P - 4 * R * V + 4)),
               dict(out=(P, LQ, KEPT, None)), dict(out=(TOK, TOK, KEPT, None)), dict(out=(TOK, LQ, LQ + 28, None)),
               dict(out=(TOK, UU, KEPT, None)), dict(out=(TOK, LQ, T, None), arrays=(T, None, None, None)),
               dict(out=(K, LQ, KEPT, None), arrays=(None, K, None, None)),
               dict(out=(TOK, LQ, KEPT, TP - 64), arrays=(None, None, TP, None)),
               dict(out=(TOK, LQ, KEPT, KEPT - 128))):
        assert call(**kw) == 1, kw
    for kw in (dict(ws=None), dict(ws=6 * P + 16), dict(n=16)):
        assert call(**kw) == 5, kw


def test_binding_refuses_cpu_tensors(vsd):
    x = torch.zeros(4, 128)
    for bad in (lambda: vsd.quantize_fp8(x), lambda: vsd.sample_filtered(x, torch.zeros(4)),
                lambda: vsd.filter_logits(x)):
        with pytest.raises(ValueError):
            bad()


def _on_host(vsd, monkeypatch):
    """CPU tensors pass as CUDA ones; tensors on the meta device stand for those of
    another GPU; no call reaches the library."""
    monkeypatch.setattr(vsd, "_need_cuda", lambda *ts: None)

    def no_call(*a):
        raise AssertionError("the library was called")
    monkeypatch.setattr(vsd, "_loss_call", no_call)


def test_binding_refuses_other_devices_types_and_shapes(vsd, monkeypatch):
    _on_host(vsd, monkeypatch)
    f8 = torch.float8_e4m3fn
    x, u = torch.zeros(4, 256), torch.zeros(4)
    h, w = torch.zeros(4, 256, dtype=f8), torch.zeros(200, 256, dtype=f8)
    hs, ws = torch.zeros(4, 2), torch.zeros(2, 2)
    far = dict(device="meta")
    for bad in (lambda: vsd.quantize_fp8(x, q=torch.empty(4, 256, dtype=f8, **far)),
                lambda: vsd.quantize_fp8(x, scale=torch.empty(4, 2, **far)),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, torch.empty(2, 2, **far)),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, ws, out=torch.empty(4, 200, dtype=torch.bfloat16, **far)),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, ws, workspace=torch.empty(256, dtype=torch.uint8, **far)),
                lambda: vsd.sample_filtered(x, torch.empty(4, **far)),
                lambda: vsd.sample_filtered(x, u, T=torch.empty(4, **far)),
                lambda: vsd.sample_filtered(x, u, filtered=torch.empty(4, 256, **far)),
                lambda: vsd.sample_filtered(x, u, workspace=torch.empty(512, dtype=torch.uint8, **far))):
        with pytest.raises(ValueError, match="one device"):
            bad()
    for bad in (lambda: vsd.quantize_fp8(x[0]), lambda: vsd.quantize_fp8(x, block_rows=64),
                lambda: vsd.quantize_fp8(x, q=torch.zeros(4, 256)), lambda: vsd.quantize_fp8(x, q=w),
                lambda: vsd.quantize_fp8(x, scale=torch.zeros(4, 3)),
                lambda: vsd.quantize_fp8(x, block_rows=128, scale=torch.zeros(4, 2)),
                lambda: vsd.lmhead_logits_fp8(x, hs, w, ws), lambda: vsd.lmhead_logits_fp8(h, ws, w, ws),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, hs), lambda: vsd.lmhead_logits_fp8(h, hs.double(), w, ws),
                lambda: vsd.lmhead_logits_fp8(h, hs, w[:, :128], ws[:, :1]),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, ws, out=torch.zeros(4, 200)),
                lambda: vsd.lmhead_logits_fp8(h, hs, w, ws, out=torch.zeros(200, 4, dtype=torch.bfloat16)),
                lambda: vsd.sample_filtered(x, u[:3]), lambda: vsd.sample_filtered(x, u.double()),
                lambda: vsd.sample_filtered(x, u, T=torch.ones(4, dtype=torch.float64)),
                lambda: vsd.sample_filtered(x, u, T=torch.ones(3)), lambda: vsd.sample_filtered(x, u, T=torch.ones(())),
                lambda: vsd.sample_filtered(x, u, top_k=torch.ones(4)),
                lambda: vsd.sample_filtered(x, u, filtered=torch.zeros(4, 256, dtype=torch.bfloat16)),
                lambda: vsd.sample_filtered(x, u, workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: vsd.quantize_fp8(x.double()), lambda: vsd.sample_filtered(x.double(), u)):
        with pytest.raises(TypeError):
            bad()


def test_settings_reach_the_struct(vsd, monkeypatch):
    monkeypatch.setattr(vsd, "_need_cuda", lambda *ts: None)
    x = torch.zeros(3, 8)
    t, k = torch.ones(3), torch.ones(3, dtype=torch.int32)
    p = vsd._policy(3, x, t, k, 0.5, 0.25)
    assert (p.row_T, p.row_top_k, p.row_top_p, p.row_min_p) == (t.data_ptr(), k.data_ptr(), None, None)
    assert (p.top_p, p.min_p) == (0.5, 0.25)
    for given, held in ((-5, 0), (7, 7), (1 << 40, 2 ** 31 - 1)):  # (beyond 32 bits: off still)
        assert vsd._policy(3, x, 1.0, given, 1.0, 0.0).top_k == held


def test_settings_that_round_to_zero_are_refused(vsd, monkeypatch):
    """As float32 they would mean something else: greedy, or off."""
    monkeypatch.setattr(vsd, "_need_cuda", lambda *ts: None)
    x = torch.zeros(3, 8)
    for kw in (dict(T=1e-46), dict(min_p=1e-46), dict(min_p=1e-300)):
        with pytest.raises(ValueError, match="float32"):
            vsd._policy(3, x, **dict(dict(T=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw))
    p = vsd._policy(3, x, 0, 0, 1e-46, 2.0 ** -149)
    assert (p.T, p.top_p, p.min_p) == (0.0, 0.0, 2.0 ** -149)  # (top_p: the first token alone, either way)
