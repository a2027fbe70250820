"""A wait that gave up stays known until it has been reported, whichever call of
the language model's ends uses the workspace next.  The wait runs out on a
barrier that nothing arrives at (about a second); nothing faults."""
import ctypes

import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

TIMEOUT = 5


def fail_on(ws):
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert slim.library().slim_diag_wait_timeout(ws.data_ptr(), stream) == 0
    torch.cuda.synchronize()


def loss_inputs(dev, N, dt=torch.float32):
    g = torch.Generator().manual_seed(N)
    x, w = torch.randn(N, 64, generator=g), torch.randn(100, 64, generator=g)
    return x.to(dt).to(dev), w.to(dt).to(dev), torch.arange(N, device=dev) % 100


def embed_grad(dev, ws):
    ids = torch.arange(50, device=dev) % 7
    slim.embed_backward(ids, torch.ones(50, 16, device=dev), 7, workspace=ws)


def clip(dev, ws):
    slim.clip_grad_norm([torch.ones(50, device=dev)], 1.0, workspace=ws)


@pytest.mark.parametrize("call", [embed_grad, clip])
def test_a_call_without_waits_between_loses_nothing(cuda_device, call):
    """It clears the error word; the blocking check still reports the failure, once."""
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=cuda_device)
    fail_on(ws)
    call(cuda_device, ws)
    with pytest.raises(slim.SlimError) as e:
        slim.check_device_error(ws)
    assert e.value.status == TIMEOUT
    slim.check_device_error(ws)
    call(cuda_device, ws)
    slim.check_device_error(ws)


@pytest.mark.parametrize("N", [1, 3, 300])
@pytest.mark.parametrize("backward", [False, True])
def test_the_next_loss_call_reports_it(cuda_device, N, backward):
    """Whether it has few rows or many: it launches nothing and returns the error,
    and the call after it runs."""
    x, w, t = loss_inputs(cuda_device, N)
    ref = slim.vocab_loss_forward(x, w, t)
    one = torch.ones(1, device=cuda_device)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=cuda_device)

    def call():
        if backward:
            return slim.vocab_loss_backward(x, w, t, ref[1], one, workspace=ws)
        return slim.vocab_loss_forward(x, w, t, workspace=ws)

    fail_on(ws)
    before = slim.launch_count()
    with pytest.raises(slim.SlimError) as e:
        call()
    assert e.value.status == TIMEOUT and slim.launch_count() == before
    out = call()
    slim.check_device_error(ws)
    want = slim.vocab_loss_backward(x, w, t, ref[1], one) if backward else ref
    assert all(torch.equal(a, b) for a, b in zip(out, want))
