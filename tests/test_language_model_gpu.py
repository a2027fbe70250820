"""The example model: its step's gradients against autograd on the plain
formulas, and a short training run."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "language_model.py")


@pytest.fixture(scope="module")
def lm():
    spec = importlib.util.spec_from_file_location("language_model", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def plain_loss(table, omegas, ids, targets, heads, scale):
    """The model in 64 bits, quadratic attention (FAVOR+ features, inclusive mask)."""
    B, L = ids.shape
    D = table.shape[1]
    d = D // heads
    ok = (ids >= 0)[..., None]
    x = (table[ids.clamp(min=0)] * scale * ok).view(B, L, heads, d).transpose(1, 2)
    for om in omegas:
        u = d ** -0.25 * x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        phi = (u @ om.T - u.pow(2).sum(-1, keepdim=True) / 2).exp() / math.sqrt(om.shape[0])
        A = (phi @ phi.transpose(-1, -2)).tril()
        x = x + (A @ u) / A.sum(-1, keepdim=True)
    rows = x.transpose(1, 2).reshape(B * L, D)
    return torch.nn.functional.cross_entropy(rows @ table.T, targets.reshape(-1), ignore_index=-100)


def test_step_against_autograd(cuda_device, lm):
    """fp32: the clipped update of both parameters is the one of the plain
    formulas (the stack's fp32 path is held to 1e-5 per gradient; the two layers
    and the loss add theirs: 5e-5)."""
    model = lm.LanguageModel(300, heads=2, d=32, features=64, layers=2, C=32, dtype="f32", seed=3)
    gen = torch.Generator(device="cuda").manual_seed(7)
    follow = torch.randperm(300, generator=gen, device="cuda")
    ids, targets = lm.batch(gen, follow, 2, 100)
    table = model.table.double().requires_grad_()
    omegas = model.omegas.double().requires_grad_()
    loss64 = plain_loss(table, omegas, ids, targets, 2, model.scale)
    gt, go = torch.autograd.grad(loss64, (table, omegas))
    norm64 = torch.sqrt(gt.pow(2).sum() + go.pow(2).sum())
    lr, max_norm = 0.5, 0.25 * norm64.item()
    loss, norm = model.step(ids, targets, lr, max_norm)
    assert abs(loss.item() - loss64.item()) <= 1e-5 * abs(loss64.item())
    assert abs(norm.item() - norm64.item()) <= 5e-5 * norm64.item()
    for new, old, g in ((model.table, table, gt), (model.omegas, omegas, go)):
        move = (new.double() - old.detach()) / -lr
        # the new master is rounded to fp32: 2^-24 of it
        room = 5e-5 * 0.25 * norm64 + 2.0 ** -24 * old.detach().norm() / lr
        assert (move - 0.25 * g).norm() <= room


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_learns(cuda_device, lm, dtype):
    before = slim.launch_count()
    losses = lm.train(steps=25, vocab=300, B=4, L=256, dtype=dtype, log=None)
    assert slim.launch_count() > before
    assert all(math.isfinite(x) for x in losses)
    assert losses[-1] < losses[0] - 0.5
