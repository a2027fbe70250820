"""A workspace that the caller gives has to be device memory in one piece, as
every other tensor: the library cannot tell, and its kernels would write to what
they are given."""
import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ws", [torch.empty(1 << 20, dtype=torch.uint8),
                                lambda dev: torch.empty(1 << 21, dtype=torch.uint8, device=dev)[::2]])
def test_workspaces_elsewhere_are_refused(cuda_device, ws):
    ws = ws(cuda_device) if callable(ws) else ws
    g = torch.Generator().manual_seed(1)
    one = torch.ones(1, device=cuda_device)
    before = slim.launch_count()
    with pytest.raises(RuntimeError):
        slim.clip_grad_norm([torch.ones(50, device=cuda_device)], 1.0, workspace=ws)
    with pytest.raises(RuntimeError):
        slim.embed_backward(torch.arange(5, device=cuda_device), torch.ones(5, 16, device=cuda_device), 7,
                            workspace=ws)
    for N in (3, 40):
        x, w = (torch.randn(n, 64, generator=g).to(cuda_device) for n in (N, 100))
        t = torch.arange(N, device=cuda_device)
        with pytest.raises(RuntimeError):
            slim.vocab_loss_forward(x, w, t, workspace=ws)
        with pytest.raises(RuntimeError):
            slim.vocab_loss_backward(x, w, t, torch.zeros(N, device=cuda_device), one, workspace=ws)
    assert slim.launch_count() == before
