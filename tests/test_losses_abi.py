"""CPU checks of the supervised losses' C entry points: workspace sizes and the
host-side argument checks, which return before anything is enqueued."""
import ctypes as C

import pytest
import torch

host_only = pytest.mark.skipif(torch.cuda.is_available(),
                               reason="fake device pointers: host-only checks")


@pytest.fixture(scope="module")
def vsd():
    from paper_2602_05774_gb300 import build, vsd as v
    build.build_library()
    v.load()
    return v


def test_workspace_bytes(vsd):
    n = vsd.lmhead_loss_workspace_bytes
    for bad in ((0, 100, 64), (4, 0, 64), (4, 100, 0), (4, 100, 60), (4, (1 << 20) + 1, 64),
                ((1 << 24) + 1, 100, 64), (4, 100, 64, 0), (4, 100, 64, 129),
                (4, 100, 64, 1, True, -1)):
        assert n(*bad) == 0, bad
    # the logits are not kept: far less than R V of them, at any vocabulary
    R, H = 4096, 4096
    for V in (32000, 128256, 1 << 20):
        assert 0 < n(R, V, H) < 0.5 * 4 * R * V + (256 << 20), V
    assert n(R, 32000, H, grads=False) < n(R, 32000, H)
    assert n(R, 32000, H, piece=4096) < n(R, 32000, H, piece=16384)
    t = vsd.load().vsd_topk_distill_workspace_bytes
    for bad in ((0, 10, 1), (1, 0, 1), (1, (1 << 20) + 1, 1), (1, 10, 0), (1, 10, 129)):
        assert t(*bad) == 0, bad
    assert 0 < t(4096, 128256, 10) < (4 << 20)


@host_only
def test_argument_checks_before_any_launch(vsd):
    lib = vsd.load()
    p = 0x100000  # never dereferenced: every call below fails its checks
    big = 1 << 40
    o = vsd.LossOutputs(p, p, p, p, p, None)

    def xent(hidden=p, weight=p, R=4, V=100, H=64, labels=p, scale=1.0, piece=0, out=o, ws=p,
             n=big):
        return lib.vsd_lmhead_cross_entropy(hidden, weight, R, V, H, labels, -100, None, scale,
                                            piece, C.byref(out) if out else None, ws, n, None)

    def distill(ids=p, t=p, dt=0, K=4, T=1.0, H=64, out=o, ws=p, n=big):
        return lib.vsd_lmhead_distill(p, p, 4, 100, H, ids, t, dt, K, T, None, 1.0, 0,
                                      C.byref(out), ws, n, None)

    def topk(x=p, dt=0, R=4, V=100, ids=p, t=p, tdt=0, K=4, T=1.0, scale=1.0, out=o, ws=p, n=big):
        return lib.vsd_topk_distill(x, dt, R, V, ids, t, tdt, K, T, None, scale, C.byref(out), ws,
                                    n, None)

    nan, inf = float("nan"), float("inf")
    for kw in (dict(hidden=None), dict(weight=None), dict(labels=None), dict(out=None),
               dict(R=0), dict(V=0), dict(V=(1 << 20) + 1), dict(H=60), dict(H=0),
               dict(scale=nan), dict(scale=inf), dict(piece=-1), dict(hidden=p + 8),
               dict(weight=p + 2), dict(out=vsd.LossOutputs(None, p, p, p, p, None)),
               dict(out=vsd.LossOutputs(p, None, p, p, p, None)),
               dict(out=vsd.LossOutputs(p, p, None, p, p, None)),
               dict(out=vsd.LossOutputs(p, p, p, p + 8, p, None)),
               dict(out=vsd.LossOutputs(p, p, p, p, p + 8, None))):
        assert xent(**kw) == 1, kw
    for kw in (dict(ids=None), dict(t=None), dict(dt=2), dict(K=0), dict(K=129), dict(T=0.0),
               dict(T=-1.0), dict(T=nan), dict(T=inf), dict(T=1e-39), dict(H=4),
               dict(ids=p + 2), dict(t=p + 2)):
        assert distill(**kw) == 1, kw
    for kw in (dict(x=None), dict(x=p + 2), dict(ids=None), dict(t=None), dict(dt=2), dict(tdt=-1),
               dict(R=0),
               dict(V=0), dict(V=(1 << 20) + 1), dict(K=0), dict(K=129), dict(T=0.0), dict(T=nan),
               dict(scale=inf)):
        assert topk(**kw) == 1, kw
    for call in (xent, distill, topk):
        assert call(ws=None) == 5
        assert call(ws=p + 16) == 5
        assert call(n=16) == 5


def test_binding_refuses_cpu_tensors(vsd):
    h = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(100, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, 2, dtype=torch.int32)
    t = torch.zeros(4, 2)
    with pytest.raises(ValueError):
        vsd.lmhead_cross_entropy(h, w, i[:, 0].contiguous())
    with pytest.raises(ValueError):
        vsd.lmhead_distill(h, w, i, t)
    with pytest.raises(ValueError):
        vsd.topk_distill(torch.zeros(4, 100), i, t)


def _on_host(vsd, monkeypatch):
    """CPU tensors pass as CUDA ones; tensors on the meta device stand for those of
    another GPU; no call reaches the library."""
    monkeypatch.setattr(vsd, "_need_cuda", lambda *ts: None)

    def no_call(*a):
        raise AssertionError("the library was called")
    monkeypatch.setattr(vsd, "_loss_call", no_call)


def test_gradients_on_another_device_are_refused(vsd, monkeypatch):
    _on_host(vsd, monkeypatch)
    h = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(100, 64, dtype=torch.bfloat16)
    x = torch.zeros(4, 100)
    i = torch.zeros(4, 2, dtype=torch.int32)
    t = torch.zeros(4, 2)
    far = dict(dtype=torch.bfloat16, device="meta")
    for bad in (lambda: vsd.lmhead_cross_entropy(h, w, i[:, 0], d_hidden=torch.empty(4, 64, **far)),
                lambda: vsd.lmhead_cross_entropy(h, w, i[:, 0], d_weight=torch.empty(100, 64, **far)),
                lambda: vsd.lmhead_distill(h, w, i, t, d_hidden=torch.empty(4, 64, **far)),
                lambda: vsd.lmhead_distill(h, w, i, t, d_weight=torch.empty(100, 64, **far)),
                lambda: vsd.topk_distill(x, i, t, grad=torch.empty(4, 100, device="meta"))):
        with pytest.raises(ValueError, match="one device"):
            bad()


def test_losses_launch_on_their_tensors_device(vsd, monkeypatch):
    """The device of the tensors is the current one when the library is called."""
    now = [0]

    class On:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, now[0] = now[0], self.device.index

        def __exit__(self, *a):
            now[0] = self.before

    class Lib:
        def entry(self, *args):
            calls.append((now[0], args))
            return 0

    calls = []
    monkeypatch.setattr(vsd, "_lib", lambda: Lib())
    monkeypatch.setattr(vsd, "_stream", lambda i: "stream of %d" % i)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", On)
    vsd._loss_call("entry", torch.device("cuda", 1), 7)
    vsd._loss_call("entry", torch.device("cuda", 0), 8)
    assert calls == [(1, (7, "stream of 1")), (0, (8, "stream of 0"))] and now == [0]


@host_only
def test_overlapping_gradients_are_refused(vsd):
    lib = vsd.load()
    h, w, x, y, z = (0x1000000 * i for i in range(1, 6))  # never dereferenced
    R, V, H, big = 4, 100, 64, 1 << 40
    hb, wb = 2 * R * H, 2 * V * H

    def code(dh, dw):
        o = vsd.LossOutputs(z, z, z, dh, dw, None)
        a = lib.vsd_lmhead_cross_entropy(h, w, R, V, H, z, -100, None, 1.0, 0, C.byref(o), z, big,
                                         None)
        b = lib.vsd_lmhead_distill(h, w, R, V, H, z, z, 0, 4, 1.0, None, 1.0, 0, C.byref(o), z, big,
                                   None)
        return a, b

    for dh, dw in ((h, x), (x, w), (h, w), (w, None), (None, h), (x, x), (x, x + hb - 16),
                   (x + wb - 16, x), (h + 16, None), (None, w + 16), (None, w - wb + 16),
                   (w + wb - 16, None)):
        assert code(dh, dw) == (1, 1), (hex(dh or 0), hex(dw or 0))
    for dt, size in ((0, 4), (1, 2)):
        n = R * V * size
        for grad in (x + size, x - size, x + n - size, x - n + size):
            o = vsd.LossOutputs(z, z, z, None, None, grad)
            assert lib.vsd_topk_distill(x, dt, R, V, z, z, 0, 4, 1.0, None, 1.0, C.byref(o), z, big,
                                        None) == 1
