"""What the differentiable calls around the attention hand to the library's entry points:
host-only, with stand-ins in the entry points' place."""
import array
import os
import types

import pytest
import torch

from paper_2012_11346_gb300 import slim


@pytest.fixture
def qk_calls(monkeypatch):
    """What each direction of qk_norm was called with."""
    calls = []

    def forward(q, k, *weights, **how):
        calls.append(dict(how, inv_freq=list(how["inv_freq"] or ())))
        return q.clone(), None if k is None else k.clone()

    def backward(q, k, q_weight, k_weight, dq_out, dk_out, **how):
        calls.append(dict(how, inv_freq=list(how["inv_freq"] or ())))
        return dq_out, dk_out, None, None

    monkeypatch.setattr(slim, "qk_norm_forward", forward)
    monkeypatch.setattr(slim, "qk_norm_backward", backward)
    return calls


@pytest.mark.parametrize("form", [iter, list, torch.tensor, lambda f: array.array("d", f)])
def test_both_directions_turn_alike(qk_calls, form):
    """Frequencies that can be read once, or that change between the directions."""
    q = torch.randn(1, 2, 3, 8, requires_grad=True)
    freq = form([1.0, 0.5])
    out, _ = slim.qk_norm(q, None, inv_freq=freq)
    if hasattr(freq, "__setitem__"):
        freq[0] = 7.0
    out.sum().backward()
    assert [c["inv_freq"] for c in qk_calls] == [[1.0, 0.5]] * 2


def test_an_eps_past_the_range_is_refused():
    if not os.path.exists(slim._LIB_PATH):
        from paper_2012_11346_gb300 import build
        build.build()
    one = array.array("d", [1.0]).buffer_info()[0]
    for eps, status in ((1e38, 0), (1.1e38, 1), (3e38, 1)):  # no rows: nothing is enqueued
        assert slim.library().slim_qk_norm_fwd(None, None, None, None, None, None, None, 0, one, 2, 0, 0, 1, 1, 3, 4, 0,
                                               eps, 1.0, None, None, None, None, None) == status


@pytest.fixture
def kept(monkeypatch):
    """What each forward was asked to keep."""
    asked = []

    def ff(x, w, act="silu", keep=False):
        asked.append(keep)
        h = x.new_zeros(*x.shape[:-1], w.shape[0] // 2)
        return (h, None) if keep else h

    def scan(gate, x, kind="sigmoid", h0=None, keep=False):
        asked.append(keep)
        out = (x.clone(), x[:, -1].float().clone())
        return (*out, torch.zeros(1)) if keep else out

    monkeypatch.setattr(slim, "gated_ff_forward", ff)
    monkeypatch.setattr(slim, "gated_scan_forward", scan)
    return asked


@pytest.mark.parametrize("recorded", [False, True])
@pytest.mark.parametrize("needed", [False, True])
def test_nothing_is_kept_for_a_gradient_that_is_not_wanted(kept, recorded, needed):
    """Neither under no_grad with parameters that require gradients nor without any."""
    x, w, gate = torch.randn(4, 8), torch.randn(12, 8), torch.randn(1, 4, 8)
    w.requires_grad_(needed)
    gate.requires_grad_(needed)
    with torch.set_grad_enabled(recorded):
        h = slim.gated_ff(x, w)
        states, last = slim.gated_scan(gate, x[None])
    assert kept == [recorded and needed] * 2
    assert h.requires_grad == states.requires_grad == last.requires_grad == (recorded and needed)


def test_the_functions_themselves_keep_unless_told(kept):
    x, w = torch.randn(4, 8), torch.randn(12, 8, requires_grad=True)
    slim.GatedFeedForward.apply(x, w, "silu")
    slim.GatedScan.apply(x[None], x[None].clone().requires_grad_(), "log", None)
    assert kept == [True, True]


def test_positions_of_one_row_for_all(qk_calls):
    q = torch.randn(2, 2, 3, 8, requires_grad=True)
    slim.qk_norm(q, None, positions=torch.arange(3).expand(2, 3))[0].sum().backward()
    for call in qk_calls:
        assert call["positions"].is_contiguous() and call["positions"].tolist() == [[0, 1, 2]] * 2
    assert len(qk_calls) == 2


def test_a_stream_of_another_device_is_refused():
    with pytest.raises(ValueError):
        slim._at(0, types.SimpleNamespace(device_index=1))


class Elsewhere(torch.Tensor):
    """A tensor that gives itself out as one of a GPU."""

    @staticmethod
    def on(t, index):
        t = t.as_subclass(Elsewhere)
        t.index = index
        return t

    is_cuda = True

    def get_device(self):
        return self.index


def test_a_workspace_of_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(slim, "library", lambda: (_ for _ in ()).throw(AssertionError("reached")))
    here = lambda *shape: Elsewhere.on(torch.zeros(*shape), 0)
    x, w, h, q = here(4, 8), here(12, 8), here(4, 6), here(1, 2, 3, 8)
    ws = Elsewhere.on(torch.zeros(1 << 20, dtype=torch.uint8), 1)
    for call in (lambda: slim.gated_ff_forward(x, w, workspace=ws), lambda: slim.gated_ff_backward(x, w, h, workspace=ws),
                 lambda: slim.qk_norm_backward(q, None, None, None, q, None, workspace=ws)):
        with pytest.raises(ValueError, match="different devices"):
            call()


def test_an_output_over_an_input_is_refused(monkeypatch):
    """Its tiles are written while others still read the rows."""
    monkeypatch.setattr(slim, "_device_of", lambda *t: 0)
    monkeypatch.setattr(slim, "_require_cuda", lambda *t: None)
    monkeypatch.setattr(slim, "_at", lambda dev, stream: slim._HERE)
    monkeypatch.setattr(slim, "library", lambda: (_ for _ in ()).throw(AssertionError("reached")))
    rows, w = torch.zeros(10, 8), torch.zeros(16, 8)
    for out in (rows[:4], rows[2:6], rows[3:7], w[:4], w[12:]):
        with pytest.raises(ValueError, match="share memory"):
            slim.gated_ff_forward(rows[:4], w, out=out)
    assert slim._apart(rows[:4], rows[4:]) and slim._apart(rows[4:], rows[:4])


def test_modes_see_what_is_allocated(monkeypatch):
    from torch.utils._python_dispatch import TorchDispatchMode

    class Watching(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    made = []
    monkeypatch.setattr(torch, "empty_strided", lambda *a, **kw: made.append("dispatched"))
    monkeypatch.setattr(slim, "_undispatched", lambda *a: made.append("undispatched"), raising=False)
    slim._allocate((2,), (1,), torch.float32)
    with Watching():
        slim._allocate((2,), (1,), torch.float32)
    assert made[1] == "dispatched" and made[0] == ("dispatched" if slim._modes() else "undispatched")


def test_the_diagnostic_wait_refuses():
    """Sizes without a wait, and what the forward refuses."""
    call, ok = slim.library().slim_diag_gated_scan_wait, 0x10000
    for L, D in ((8, 8), (2048, 8), (-1, 8), (5000, 0)):
        assert call(ok, ok, L, D, ok, ok, 1 << 40, None) == 1
    for a in ((None, ok, ok), (ok, None, ok), (ok, ok, None), (ok + 2, ok, ok)):
        assert call(a[0], a[1], 5000, 8, a[2], ok, 1 << 40, None) == 1
    assert call(ok, ok, 5000, 8, ok, None, 0, None) == 3
