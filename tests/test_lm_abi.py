"""Host-only checks of the language-model entry points (include/slim_lm.h):
sizes, and refusals before anything is enqueued.  No call here reaches a CUDA
launch; the pointers are never dereferenced."""
import ctypes

import pytest
import torch

from paper_2012_11346_gb300 import slim

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x10000
F32, BF16, I32, I64 = 0, 1, 0, 1


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(slim._LIB_PATH):
        from paper_2012_11346_gb300 import build
        build.build()
    return slim.library()


# ---------------------------------------------------------------- embedding
def embed_fwd(lib, ids=FAKE, it=I64, table=FAKE, N=4, D=8, V=16, dt=F32, out=FAKE):
    return lib.slim_embed_fwd(ids, it, table, N, D, V, dt, 1.0, out, None)


def embed_bwd(lib, ids=FAKE, it=I64, dout=FAKE, N=4, D=8, V=16, dt=F32, acc=0, dtable=FAKE,
              ws=FAKE, nbytes=1 << 40):
    return lib.slim_embed_bwd(ids, it, dout, N, D, V, dt, 1.0, acc, dtable, ws, nbytes, None)


@pytest.mark.parametrize("kw", [dict(N=-1), dict(N=1 << 31), dict(D=0), dict(V=0), dict(dt=2),
                                dict(it=2), dict(ids=None), dict(ids=FAKE + 4),
                                dict(it=I32, ids=FAKE + 2)])
def test_embed_rejects(lib, kw):
    assert embed_fwd(lib, **kw) == INVALID
    assert embed_bwd(lib, **kw) == INVALID


def test_embed_rejects_tensors(lib):
    for bad in (None, FAKE + 8):
        assert embed_fwd(lib, table=bad) == INVALID
        assert embed_fwd(lib, out=bad) == INVALID
        assert embed_bwd(lib, dout=bad) == INVALID
        assert embed_bwd(lib, dtable=bad) == INVALID
    assert embed_bwd(lib, acc=2) == INVALID


def test_embed_workspace(lib):
    need = slim.embed_workspace_size(1000, 64, 300, torch.float32)
    assert embed_bwd(lib, N=1000, D=64, V=300, nbytes=need - 1) == WORKSPACE
    assert embed_bwd(lib, N=1000, D=64, V=300, ws=None) == WORKSPACE
    assert embed_bwd(lib, N=1000, D=64, V=300, ws=FAKE + 16, nbytes=need) == INVALID
    assert lib.slim_embed_bwd_workspace_size(4, 8, 16, F32, None) == INVALID
    # grows with the tokens, not with the table (beyond the sort's second buffer)
    a = slim.embed_workspace_size(100000, 64, 300, torch.float32)
    b = slim.embed_workspace_size(100000, 64, 60000, torch.float32)
    assert a == b


def test_embed_no_tokens_enqueues_nothing(lib):
    assert embed_fwd(lib, N=0, ids=None, out=None) == OK
    assert embed_bwd(lib, N=0, ids=None, dout=None, acc=1, ws=None, nbytes=0) == OK


# ---------------------------------------------------------------- vocabulary loss
def loss_fwd(lib, x=FAKE, w=FAKE, t=FAKE, it=I64, N=4, D=8, V=16, dt=F32, loss=FAKE, lse=FAKE,
             total=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.slim_vocab_loss_fwd(x, w, t, it, N, D, V, dt, -100, loss, lse, total, ws, nbytes, None)


def loss_bwd(lib, x=FAKE, w=FAKE, t=FAKE, it=I64, lse=FAKE, dloss=FAKE, stride=1, count=None, N=4,
             D=8, V=16, dt=F32, piece=256, dx=FAKE, dw=FAKE, ws=FAKE, nbytes=1 << 40):
    return lib.slim_vocab_loss_bwd(x, w, t, it, lse, dloss, stride, count, N, D, V, dt, piece, -100,
                                   dx, dw, ws, nbytes, None)


@pytest.mark.parametrize("kw", [dict(N=-1), dict(N=1 << 31), dict(D=0), dict(V=0), dict(V=1 << 30 | 1),
                                dict(dt=2), dict(it=2), dict(x=None), dict(w=None), dict(t=None),
                                dict(lse=None), dict(x=FAKE + 8), dict(w=FAKE + 8),
                                dict(t=FAKE + 4), dict(it=I32, t=FAKE + 2), dict(lse=FAKE + 2),
                                dict(ws=FAKE + 16)])
def test_loss_rejects(lib, kw):
    assert loss_fwd(lib, **kw) == INVALID
    assert loss_bwd(lib, **kw) == INVALID


def test_loss_rejects_more(lib):
    for bad in (None, FAKE + 2):
        assert loss_fwd(lib, loss=bad) == INVALID
        assert loss_fwd(lib, total=bad) == INVALID
        assert loss_bwd(lib, dloss=bad) == INVALID
    assert loss_bwd(lib, dx=None) == INVALID and loss_bwd(lib, dw=FAKE + 8) == INVALID
    assert loss_bwd(lib, stride=2) == INVALID and loss_bwd(lib, piece=0) == INVALID
    assert loss_bwd(lib, count=FAKE + 1) == INVALID


def test_loss_workspace(lib):
    for bwd, call in ((False, loss_fwd), (True, loss_bwd)):
        need = slim.vocab_loss_workspace_size(4, 8, 16, torch.float32, bwd, piece=256)
        assert call(lib, nbytes=need - 1) == WORKSPACE
        assert call(lib, ws=None) == WORKSPACE
    assert lib.slim_vocab_loss_workspace_size(4, 8, 16, F32, 256, 1, None) == INVALID
    assert lib.slim_vocab_loss_workspace_size(4, 8, 16, F32, 0, 1, ctypes.byref(ctypes.c_size_t())) == INVALID
    # bf16 rows that need no staging: the forward keeps O(N), the backward N x piece
    N, D, bf = 32768, 512, torch.bfloat16
    size = lambda V, bwd, piece=8192: slim.vocab_loss_workspace_size(N, D, V, bf, bwd, piece)
    assert size(65536, False) < 128 * N and size(16384, False) <= size(65536, False) * 1.1
    assert size(65536, True) == size(32768, True)
    assert size(65536, True, 16384) - size(65536, True) == 2 * N * 8192


# ---------------------------------------------------------------- clipping
def clip(lib, n=2, src=(FAKE, FAKE), dst=(FAKE, FAKE), numel=(8, 8), dts=(F32, BF16), max_norm=1.0,
         norm=FAKE, ws=FAKE, nbytes=1 << 40):
    p = ctypes.c_void_p * len(src)
    return lib.slim_clip_grads(p(*src), p(*dst), (ctypes.c_longlong * len(numel))(*numel),
                               (ctypes.c_int * len(dts))(*dts), n, max_norm, norm, ws, nbytes,
                               None)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(max_norm=0.0), dict(max_norm=-1.0),
                                dict(max_norm=float("nan")), dict(norm=None),
                                dict(norm=FAKE + 2), dict(dts=(F32, 2)), dict(numel=(8, -1)),
                                dict(src=(FAKE, None)), dict(dst=(None, FAKE)),
                                dict(src=(FAKE + 2, FAKE)), dict(dst=(FAKE, FAKE + 1)),
                                dict(numel=(1 << 41, 8)), dict(ws=FAKE + 8)])
def test_clip_rejects(lib, kw):
    assert clip(lib, **kw) == INVALID


def test_clip_workspace(lib):
    need = slim.clip_workspace_size(2)
    assert clip(lib, nbytes=need - 1) == WORKSPACE
    assert clip(lib, ws=None) == WORKSPACE
    assert lib.slim_clip_workspace_size(2, None) == INVALID
    assert lib.slim_clip_grads(None, None, None, None, 1, 1.0, FAKE, FAKE, 1 << 40, None) == INVALID


# ---------------------------------------------------------------- the binding
def test_binding_refuses_cpu_tensors():
    with pytest.raises(RuntimeError):
        slim.embed_forward(torch.zeros(3, dtype=torch.long), torch.zeros(4, 8))
    with pytest.raises(RuntimeError):
        slim.embed_backward(torch.zeros(3, dtype=torch.long), torch.zeros(3, 8), 4)
    with pytest.raises(RuntimeError):
        slim.clip_grad_norm([torch.zeros(3)], 1.0)
    with pytest.raises(RuntimeError):
        slim.vocab_loss_forward(torch.zeros(3, 8), torch.zeros(4, 8), torch.zeros(3, dtype=torch.long))
    with pytest.raises(ValueError):
        slim.clip_grad_norm([], 1.0)
