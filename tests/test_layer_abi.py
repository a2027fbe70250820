"""Host-only checks of the entry points around the attention (include/slim_layer.h):
sizes, and refusals before anything is enqueued.  No call here reaches a CUDA launch;
the pointers are never dereferenced."""
import ctypes
import os
import re

import pytest
import torch

import layer_common as ref
from paper_2012_11346_gb300 import slim

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x10000
F32, BF16, I32, I64 = 0, 1, 0, 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(slim._LIB_PATH):
        from paper_2012_11346_gb300 import build
        build.build()
    return slim.library()


def test_every_declared_symbol_is_bound(lib):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                               "slim_layer.h")).read()
    names = set(re.findall(r"^slim_status (slim_\w+)\(", header, re.M))
    assert names
    for n in names:
        assert n in slim.SIGNATURES and getattr(lib, n)


# ---------------------------------------------------------------- norms of queries and keys
def strides(*s):
    return (ctypes.c_longlong * 3)(*s)


def freqs(*f):
    return (ctypes.c_double * max(1, len(f)))(*f)


def qk_fwd(lib, q=FAKE, qs=None, k=FAKE, ks=None, wq=FAKE, wk=FAKE, pos=FAKE, pt=I64, freq=freqs(1.0, 0.1), rotary=4,
           inter=0, B=2, Hq=2, Hk=2, L=3, d=8, dt=F32, eps=1e-6, scale=1.0, qo=FAKE, qos=None, ko=FAKE, kos=None):
    return lib.slim_qk_norm_fwd(q, qs, k, ks, wq, wk, pos, pt, freq, rotary, inter, B, Hq, Hk, L, d, dt, eps, scale,
                                qo, qos, ko, kos, None)


def qk_bwd(lib, q=FAKE, qs=None, k=FAKE, ks=None, wq=FAKE, wk=FAKE, pos=FAKE, pt=I64, freq=freqs(1.0, 0.1), rotary=4,
           inter=0, B=2, Hq=2, Hk=2, L=3, d=8, dt=F32, eps=1e-6, scale=1.0, qo=FAKE, qos=None, ko=FAKE, kos=None,
           dq=FAKE, dqs=None, dk=FAKE, dks=None, dwq=FAKE, dwk=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.slim_qk_norm_bwd(q, qs, k, ks, wq, wk, pos, pt, freq, rotary, inter, B, Hq, Hk, L, d, dt, eps, scale,
                                qo, qos, ko, kos, dq, dqs, dk, dks, dwq, dwk, ws, nbytes, None)


BIG = 1 << 40
QK_BAD = [
    dict(B=-1), dict(L=-1), dict(B=1 << 16, L=1 << 15), dict(Hq=0), dict(Hk=-1), dict(Hq=4097), dict(Hk=4097),
    dict(d=0), dict(d=257), dict(dt=2), dict(rotary=-2), dict(rotary=3), dict(rotary=10), dict(inter=2), dict(inter=-1),
    dict(freq=None), dict(pt=2), dict(freq=freqs(1.0, float("nan"))), dict(freq=freqs(float("inf"), 1.0)),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=FAKE + 2), dict(k=FAKE + 1),
    dict(qo=FAKE + 2), dict(dt=BF16, ko=FAKE + 1), dict(wq=FAKE + 2), dict(wk=FAKE + 1), dict(pos=FAKE + 4),
    dict(pt=I32, pos=FAKE + 2), dict(qs=strides(-1, 24, 8)), dict(ks=strides(48, 24, BIG + 1)),
    dict(qs=strides(BIG, BIG, BIG), B=1 << 22, L=1, Hq=1), dict(B=1 << 15, L=1 << 15, Hq=4096)]


@pytest.mark.parametrize("kw", QK_BAD)
def test_qk_rejects(lib, kw):
    assert qk_fwd(lib, **kw) == INVALID
    assert qk_bwd(lib, **kw) == INVALID


# written tensors whose elements share places
@pytest.mark.parametrize("s", [(48, 24, 0), (48, 24, 7), (0, 24, 8), (48, 0, 8), (24, 24, 8), (47, 24, 8), (48, 8, 8),
                               (8, 16, 16)])
def test_qk_rejects_shared_places(lib, s):
    assert qk_fwd(lib, qos=strides(*s)) == INVALID
    assert qk_fwd(lib, kos=strides(*s)) == INVALID
    assert qk_bwd(lib, dqs=strides(*s)) == INVALID
    assert qk_bwd(lib, dks=strides(*s)) == INVALID


def test_qk_rejects_more(lib):
    for bad in (None, FAKE + 2):
        assert qk_bwd(lib, dq=bad) == INVALID
        assert qk_bwd(lib, dk=bad) == INVALID
    assert qk_bwd(lib, dwq=FAKE + 2) == INVALID and qk_bwd(lib, dwk=FAKE + 1) == INVALID
    need = slim.qk_norm_workspace_size(2, 2, 2, 3, 8)
    assert qk_bwd(lib, nbytes=need - 1) == WORKSPACE and qk_bwd(lib, ws=None) == WORKSPACE
    assert qk_bwd(lib, ws=FAKE + 16) == INVALID
    assert lib.slim_qk_norm_bwd_workspace_size(2, 2, 2, 3, 8, None) == INVALID
    n = ctypes.c_size_t()
    assert lib.slim_qk_norm_bwd_workspace_size(2, 0, 2, 3, 8, ctypes.byref(n)) == INVALID
    # a fixed number of blocks, whatever the length
    assert slim.qk_norm_workspace_size(1, 1, 1, 1, 8) == slim.qk_norm_workspace_size(8, 8, 8, 1 << 20, 8)


def test_qk_without_rows_enqueues_nothing(lib):
    for kw in (dict(B=0), dict(L=0)):
        assert qk_fwd(lib, q=None, k=None, qo=None, ko=None, **kw) == OK
        assert qk_bwd(lib, q=None, k=None, qo=None, ko=None, dq=None, dk=None, dwq=None, dwk=None, ws=None, nbytes=0,
                      **kw) == OK


def test_qk_binding(monkeypatch):
    q = torch.zeros(1, 2, 3, 8)
    with pytest.raises(RuntimeError, match="CUDA"):
        slim.qk_norm_forward(q, q)
    monkeypatch.setattr(slim, "_device_of", lambda *t: 0)
    bad = [
        (ValueError, lambda: slim.qk_norm_forward(q[0], q)),
        (ValueError, lambda: slim.qk_norm_forward(q, q.bfloat16())),
        (ValueError, lambda: slim.qk_norm_forward(q, q[:, :, :2])),
        (TypeError, lambda: slim.qk_norm_forward(q.half(), None)),
        (ValueError, lambda: slim.qk_norm_forward(q, q, torch.ones(7))),
        (ValueError, lambda: slim.qk_norm_forward(q, q, torch.ones(8).bfloat16())),
        (ValueError, lambda: slim.qk_norm_forward(q, q, positions=torch.zeros(3, dtype=torch.long))),
        (TypeError, lambda: slim.qk_norm_forward(q, q, positions=torch.zeros(1, 3))),
        (ValueError, lambda: slim.qk_norm_forward(q, q, inv_freq=[1.0] * 5)),
        (RuntimeError, lambda: slim.qk_norm_forward(q.transpose(2, 3).contiguous().transpose(2, 3), q)),
        (ValueError, lambda: slim.qk_norm_forward(q.expand(1 << 32, 2, 3, 8), None)),
        (ValueError, lambda: slim.qk_norm_backward(q, q, None, None, q, None)),
        (ValueError, lambda: slim.qk_norm_backward(q, q, None, None, q, q[:, :1])),
        (ValueError, lambda: slim.qk_norm_backward(q, None, None, None, q, q)),
        (ValueError, lambda: slim.rotary_frequencies(3)),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()


# ---------------------------------------------------------------- the formulas themselves
def test_qk_formula_against_differences():
    """The gradient that the kernels compute, r (g - n mean(g n)) after turning back,
    against central differences of the definition."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(1, 2, 3, 6, generator=g, dtype=torch.float64)
    w = 1 + 0.3 * torch.randn(6, generator=g, dtype=torch.float64)
    up = torch.randn(1, 2, 3, 6, generator=g, dtype=torch.float64)
    freq = [1.0, 0.1]

    def f(a, b):
        return (ref.qk64(a, b, None, freq, False, 1e-6, 0.7) * up).sum()

    back = ref.angles64(None, freq, 1, 3, "cpu")
    dz = up.clone()
    i, k = ref.pairs_of(6, 2, False)
    dz[..., i], dz[..., k] = up[..., i] * back.cos() + up[..., k] * back.sin(), up[..., k] * back.cos() - up[..., i] * back.sin()
    dz = 0.7 * dz
    r = 1 / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    n = x * r
    dx = r * (dz * w - n * (dz * w * n).mean(-1, keepdim=True))
    dw = (dz * n).sum((0, 1, 2))
    h = 1e-6
    for t, grad, call in ((x, dx, lambda e: f(x + e, w)), (w, dw, lambda e: f(x, w + e))):
        for j in range(t.numel()):
            e = torch.zeros_like(t).view(-1)
            e[j] = h
            e = e.view_as(t)
            assert abs((call(e) - call(-e)) / (2 * h) - grad.reshape(-1)[j]) < 1e-7


# ---------------------------------------------------------------- gated recurrence
def scan_fwd(lib, gate=FAKE, gp=8, x=FAKE, xp=8, h0=FAKE, B=2, L=100, D=8, dt=F32, kind=0, h=FAKE, last=FAKE, kept=FAKE, ws=FAKE,
             nbytes=1 << 60):
    return lib.slim_gated_scan_fwd(gate, gp, x, xp, h0, B, L, D, dt, kind, h, last, kept, ws, nbytes, None)


def scan_bwd(lib, gate=FAKE, gp=8, x=FAKE, xp=8, kept=FAKE, h=FAKE, last=FAKE, B=2, L=100, D=8, dt=F32, kind=0, dg=FAKE,
             dgp=8, dx=FAKE, dxp=8, h0=FAKE, ws=FAKE, nbytes=1 << 60):
    return lib.slim_gated_scan_bwd(gate, gp, x, xp, kept, h, last, B, L, D, dt, kind, dg, dgp, dx, dxp, h0, ws, nbytes, None)


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(L=-1), dict(L=(1 << 30) + 1), dict(D=0), dict(D=(1 << 30) + 1), dict(dt=2),
    dict(kind=3), dict(kind=-1), dict(gate=None), dict(x=None), dict(h=None), dict(gate=FAKE + 2), dict(x=FAKE + 1),
    dict(h=FAKE + 2), dict(dt=BF16, h=FAKE + 1), dict(gp=-1), dict(xp=-8), dict(gp=BIG + 1), dict(h0=FAKE + 2),
    dict(last=FAKE + 1), dict(kept=FAKE + 2), dict(B=60000, L=1 << 30, D=1 << 10),
    dict(B=60000, L=1, D=1 << 25), dict(L=1 << 30, D=1, gp=1 << 35)])
def test_scan_rejects(lib, kw):
    assert scan_fwd(lib, **kw) == INVALID
    assert scan_bwd(lib, **kw) == INVALID


def test_scan_rejects_more(lib):
    for kw in (dict(dg=None), dict(dx=None), dict(dg=FAKE + 2), dict(dx=FAKE + 1), dict(dgp=7), dict(dxp=0), dict(kept=None)):
        assert scan_bwd(lib, **kw) == INVALID


def test_scan_workspace(lib):
    """None for short and few sequences; else it is asked for, aligned, and its size does
    not depend on what the channels' alignment is."""
    def size(B, L, D, dt=F32):
        n = ctypes.c_size_t(7)
        assert lib.slim_gated_scan_workspace_size(B, L, D, dt, ctypes.byref(n)) == 0
        return n.value

    assert size(2, 100, 8) == size(0, 1 << 20, 8) == size(1 << 20, 8, 512) == size(1 << 20, 64, 512) == 0
    assert size(1, 512, 8) == 0 and size(2, 3000, 8) > 0 and size(1 << 10, 200, 512) > 0
    for kw in (dict(B=-1), dict(D=0), dict(L=-1), dict(dt=2)):
        n = ctypes.c_size_t(7)
        a = {**dict(B=1, L=5000, D=8, dt=F32), **kw}
        assert lib.slim_gated_scan_workspace_size(a["B"], a["L"], a["D"], a["dt"], ctypes.byref(n)) == INVALID
    assert lib.slim_gated_scan_workspace_size(1, 5000, 8, F32, None) == INVALID
    need = size(2, 5000, 8)
    for call in (scan_fwd, scan_bwd):
        assert call(lib, L=5000, ws=None) == call(lib, L=5000, nbytes=need - 1) == WORKSPACE
        assert call(lib, L=5000, ws=FAKE + 128) == INVALID


def test_scan_constant_is_the_headers():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                               "slim_layer.h")).read()
    assert int(re.search(r"#define SLIM_SCAN_CHUNK (\d+)", header).group(1)) == slim.SCAN_CHUNK


def test_scan_binding(monkeypatch):
    x = torch.zeros(2, 70, 8)
    with pytest.raises(RuntimeError, match="CUDA"):
        slim.gated_scan_forward(x, x)
    monkeypatch.setattr(slim, "_device_of", lambda *t: 0)
    monkeypatch.setattr(slim, "_at", lambda dev, stream: slim._HERE)
    monkeypatch.setattr(slim, "library", lambda: (_ for _ in ()).throw(AssertionError("reached")))
    h0, kept = torch.zeros(2, 8), torch.zeros(2, 2, 8)
    bad = [
        (ValueError, lambda: slim.gated_scan_forward(x[0], x[0])),
        (ValueError, lambda: slim.gated_scan_forward(x, x[:, :3])),
        (TypeError, lambda: slim.gated_scan_forward(x, x.bfloat16())),
        (TypeError, lambda: slim.gated_scan_forward(x.half(), x.half())),
        (ValueError, lambda: slim.gated_scan_forward(x, x, "tanh")),
        (ValueError, lambda: slim.gated_scan_forward(x, x, h0=h0[:1])),
        (ValueError, lambda: slim.gated_scan_forward(x, x, h0=h0.bfloat16())),
        (ValueError, lambda: slim.gated_scan_forward(x, x, last=h0.double())),
        (ValueError, lambda: slim.gated_scan_forward(*[x[:1, :1].expand(1, 1 << 32, 8)] * 2)),
        (ValueError, lambda: slim.gated_scan_backward(x, x, None, x)),
        (ValueError, lambda: slim.gated_scan_backward(x, x, kept[:, :1], x)),
        (ValueError, lambda: slim.gated_scan_backward(x, x, kept, x[:, :3])),
        (ValueError, lambda: slim.gated_scan_backward(x, x, kept, x.bfloat16())),
        (ValueError, lambda: slim.gated_scan_backward(x, x, kept, x, dx=x.bfloat16())),
        (ValueError, lambda: slim.gated_scan_backward(x, x, kept, x, dlast=h0[:1])),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    for t in (x.transpose(1, 2).contiguous().transpose(1, 2), torch.zeros(4, 70, 8)[::2][:, :35]):
        with pytest.raises(RuntimeError):
            slim._pitch(t.shape, t.stride(), "t")
    for t, want in ((torch.zeros(2, 70, 24)[..., 8:16], 24), (torch.zeros(5, 3, 8)[:, :1], 24), (torch.zeros(1, 1, 8), 8)):
        assert slim._pitch(t.shape, t.stride(), "t") == want


def test_scan_formula_against_differences():
    """Autograd on the recurrence, which the kernels are held to, against central differences."""
    g = torch.Generator().manual_seed(0)
    gate, x = (torch.randn(1, 4, 3, generator=g, dtype=torch.float64).requires_grad_() for _ in range(2))
    h0 = torch.randn(1, 3, generator=g, dtype=torch.float64).requires_grad_()
    for kind in slim.GATES:
        assert torch.autograd.gradcheck(lambda a, b, c: ref.scan64(a, b, kind, c), (gate, x, h0))


# ---------------------------------------------------------------- gated feed-forward
def ff_fwd(lib, x=FAKE, w=FAKE, N=20, D=8, F=16, dt=F32, act=0, h=FAKE, z=None, ws=FAKE, nbytes=1 << 60):
    return lib.slim_gated_ff_fwd(x, w, N, D, F, dt, act, h, z, ws, nbytes, None)


def ff_bwd(lib, x=FAKE, w=FAKE, h=FAKE, N=20, D=8, F=16, dt=F32, act=0, z=None, dx=FAKE, dw=FAKE, ws=FAKE,
           nbytes=1 << 60):
    return lib.slim_gated_ff_bwd(x, w, h, N, D, F, dt, act, z, dx, dw, ws, nbytes, None)


@pytest.mark.parametrize("kw", [
    dict(N=-1), dict(N=(1 << 31) - 512), dict(D=0), dict(D=(1 << 30) + 1), dict(F=0), dict(F=(1 << 29) + 1), dict(dt=2),
    dict(act=-1), dict(act=5), dict(N=1 << 20, F=1 << 26), dict(N=1 << 20, D=(1 << 20) + 1), dict(F=1 << 20, D=1 << 20),
    dict(x=None), dict(w=None), dict(h=None), dict(x=FAKE + 8), dict(w=FAKE + 8), dict(h=FAKE + 4), dict(ws=FAKE + 16),
    dict(N=3, ws=FAKE + 16), dict(N=3, x=FAKE + 2), dict(z=FAKE + 16), dict(dt=BF16, z=FAKE), dict(N=8, z=FAKE)])
def test_ff_rejects(lib, kw):
    assert ff_fwd(lib, **kw) == INVALID
    assert ff_bwd(lib, **kw) == INVALID


def test_ff_rejects_more(lib):
    for bad in (None, FAKE + 8):
        assert ff_bwd(lib, dx=bad) == INVALID and ff_bwd(lib, dw=bad) == INVALID
    for N in (3, 20):
        for back, call in ((False, ff_fwd), (True, ff_bwd)):
            need = slim.gated_ff_workspace_size(N, 8, 16, torch.float32, back)
            if N == 3 and not back:
                assert need == 0
                continue
            assert call(lib, N=N, nbytes=need - 1) == WORKSPACE and call(lib, N=N, ws=None) == WORKSPACE
    n = ctypes.c_size_t()
    assert lib.slim_gated_ff_workspace_size(20, 8, 16, F32, 0, None) == INVALID
    assert lib.slim_gated_ff_workspace_size(20, 8, 16, F32, 2, ctypes.byref(n)) == INVALID
    size = lambda N, F, back: slim.gated_ff_workspace_size(N, 512, F, torch.bfloat16, back)
    # bf16 rows that need no staging: nothing forward, dz backward
    assert size(32768, 2048, False) <= 256
    assert 2 * 2 * 32768 * 2048 <= size(32768, 2048, True) <= 2 * 2 * 32768 * 2048 + (1 << 26)
    assert ff_fwd(lib, N=0, x=None, h=None, ws=None, nbytes=0) == OK


def test_ff_binding(monkeypatch):
    x, w = torch.zeros(4, 8), torch.zeros(12, 8)
    with pytest.raises(RuntimeError, match="CUDA"):
        slim.gated_ff_forward(x, w)
    monkeypatch.setattr(slim, "_device_of", lambda *t: 0)
    monkeypatch.setattr(slim, "_require_cuda", lambda *t: None)
    monkeypatch.setattr(slim, "_at", lambda dev, stream: slim._HERE)
    monkeypatch.setattr(slim, "library", lambda: (_ for _ in ()).throw(AssertionError("reached")))
    bad = [
        (TypeError, lambda: slim.gated_ff_forward(x, w.bfloat16())),
        (TypeError, lambda: slim.gated_ff_forward(x.half(), w.half())),
        (ValueError, lambda: slim.gated_ff_forward(x, w[:11])),
        (ValueError, lambda: slim.gated_ff_forward(x, w[:, :7])),
        (ValueError, lambda: slim.gated_ff_forward(x, w[0])),
        (ValueError, lambda: slim.gated_ff_forward(x, w, "tanh")),
        (ValueError, lambda: slim.gated_ff_forward(x, w, out=torch.zeros(4, 7))),
        (ValueError, lambda: slim.gated_ff_forward(x, w, out=torch.zeros(4, 6).bfloat16())),
        (ValueError, lambda: slim.gated_ff_forward(x, torch.zeros(1, 8).expand(1 << 33, 8))),
        (ValueError, lambda: slim.gated_ff_backward(x, w, torch.zeros(4, 12))),
        (ValueError, lambda: slim.gated_ff_backward(x, w, torch.zeros(4, 6).bfloat16())),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()


@pytest.mark.parametrize("act", list(ref.ACTS))
def test_ff_formula_against_differences(act):
    g = torch.Generator().manual_seed(0)
    x = torch.randn(3, 4, generator=g, dtype=torch.float64).requires_grad_()
    w = torch.randn(6, 4, generator=g, dtype=torch.float64).requires_grad_()
    assert torch.autograd.gradcheck(lambda a, b: ref.ff64(a, b, act), (x, w))
