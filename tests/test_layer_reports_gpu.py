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
