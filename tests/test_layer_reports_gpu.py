"""What the recurrence reports of its waits, whatever its workspace held before."""
import ctypes

import pytest
import torch

from layer_common import F32
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


def stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("L", [1025, 1500, 2048, 5000])
def test_no_failure_that_never_was(cuda_device, L):
    """A call that asks for a workspace leaves its error word clear, also where only the other
    direction waits (fp32, 1025 to 2048 steps of one sequence: the forward is a cluster)."""
    gate, x = torch.zeros(2, 1, L, 64, device=cuda_device)
    need = slim.gated_scan_workspace_size(1, L, 64, F32)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device=cuda_device)
    _, _, kept = slim.gated_scan_forward(gate, x, "log", keep=True, workspace=ws)
    slim.check_device_error(ws)
    ws.fill_(255)
    slim.gated_scan_backward(gate, x, kept, x, "log", workspace=ws)
    slim.check_device_error(ws)
    # and none is reported twice
    assert slim.library().slim_diag_wait_timeout(ws.data_ptr(), stream()) == 0
    torch.cuda.synchronize()
    with pytest.raises(slim.SlimError):
        slim.gated_scan_forward(gate, x, "log", workspace=ws)
    slim.gated_scan_forward(gate, x, "log", workspace=ws)
    slim.check_device_error(ws)


@pytest.mark.parametrize("L,D", [(2100, 36), (20000, 512)])
def test_a_look_back_that_gives_up(cuda_device, L, D):
    """The first tile's state is never there: all blocks come to their end, the next call
    launches nothing and says so, and the one after it runs."""
    gate, x = torch.zeros(2, 1, L, D, device=cuda_device)
    gate -= 0.5
    x += 1.0
    want = slim.gated_scan_forward(gate, x, "log")
    ws = torch.full((slim.gated_scan_workspace_size(1, L, D, F32),), 255, dtype=torch.uint8, device=cuda_device)
    h = torch.full((L, D), 7.0, device=cuda_device)
    args = (gate.data_ptr(), x.data_ptr(), L, D, h.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    assert slim.library().slim_diag_gated_scan_wait(*args) == 0
    torch.cuda.synchronize()
    assert (h[:128] == 7.0).all()  # the tile that nobody ran
    before = slim.launch_count()
    with pytest.raises(slim.SlimError) as e:
        slim.gated_scan_forward(gate, x, "log", workspace=ws)
    assert e.value.status == 5 and slim.launch_count() == before
    got = slim.gated_scan_forward(gate, x, "log", workspace=ws)
    slim.check_device_error(ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
