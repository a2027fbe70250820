"""Sizes that the language model's ends refuse because their index arithmetic, or
the C types of their arguments, end there.  Host only: nothing here reaches a
launch, and the pointers are never dereferenced."""
import ctypes
import os

import pytest
import torch

from paper_2012_11346_gb300 import slim

OK, INVALID = 0, 1
FAKE = 0x10000
F32, BF16, I64 = 0, 1, 1
WIDEST = 1 << 30


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(slim._LIB_PATH):
        from paper_2012_11346_gb300 import build
        build.build()
    return slim.library()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [WIDEST + 1, (1 << 31) - 1024, (1 << 31) - 1])
def test_embedding_width(lib, D, dt):
    """Column indices of a row are 32-bit, and step past its end by a block's worth."""
    n = ctypes.c_size_t()
    assert lib.slim_embed_fwd(FAKE, I64, FAKE, 1, D, 1, dt, 1.0, FAKE, None) == INVALID
    assert lib.slim_embed_bwd(FAKE, I64, FAKE, 1, D, 1, dt, 1.0, 0, FAKE, FAKE, 1 << 50, None) == INVALID
    assert lib.slim_embed_bwd_workspace_size(1, D, 1, dt, ctypes.byref(n)) == INVALID
    assert lib.slim_embed_bwd_workspace_size(1, WIDEST, 1, dt, ctypes.byref(n)) == OK


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [WIDEST + 1, (1 << 31) - 64, (1 << 31) - 1])
def test_loss_width(lib, D, dt):
    """Rounded up to whole stages, the features have to stay in 32 bits."""
    n = ctypes.c_size_t()
    assert lib.slim_vocab_loss_fwd(FAKE, FAKE, FAKE, I64, 9, D, 1, dt, -100, FAKE, FAKE, FAKE, FAKE, 1 << 60,
                                   None) == INVALID
    assert lib.slim_vocab_loss_bwd(FAKE, FAKE, FAKE, I64, FAKE, FAKE, 0, None, 9, D, 1, dt, 256, -100, FAKE,
                                   FAKE, FAKE, 1 << 60, None) == INVALID
    for backward in (0, 1):
        size = lambda d: lib.slim_vocab_loss_workspace_size(9, d, 1, dt, 256, backward, ctypes.byref(n))
        assert size(D) == INVALID and size(WIDEST) == OK


class NoLibrary:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was reached")


BIG = (1 << 32) + 5  # 5 as a C int


@pytest.mark.parametrize("call", [
    lambda e, i: slim.embed_workspace_size(4, 8, BIG, torch.float32),
    lambda e, i: slim.embed_workspace_size(4, BIG, 8, torch.float32),
    lambda e, i: slim.embed_forward(i, e),
    lambda e, i: slim.embed_backward(i, torch.zeros(3, 1), BIG, dtable=e),
    lambda e, i: slim.vocab_loss_workspace_size(4, 8, BIG, torch.float32, False),
    lambda e, i: slim.vocab_loss_workspace_size(4, BIG, 8, torch.float32, True, 256),
    lambda e, i: slim.vocab_loss_forward(torch.zeros(3, 1), e, i),
    lambda e, i: slim.vocab_loss_backward(torch.zeros(3, 1), e, i, torch.zeros(3), torch.zeros(1)),
    lambda e, i: slim.clip_workspace_size(BIG),
])
def test_sizes_past_c_ints_are_refused(monkeypatch, call):
    """They would reach the library as their low 32 bits: a table of 2^32 + 5 rows
    as one of 5, with every other id as padding."""
    monkeypatch.setattr(slim, "library", NoLibrary)
    monkeypatch.setattr(slim, "_require_cuda", lambda *t: None)
    with pytest.raises(ValueError):
        call(torch.zeros(1, 1).expand(BIG, 1), torch.zeros(3, dtype=torch.long))


def test_a_piece_of_any_size_is_the_whole_vocabulary(lib):
    size = lambda piece: slim.vocab_loss_workspace_size(100, 64, 3000, torch.bfloat16, True, piece)
    assert size((1 << 32) + 256) == size(1 << 20) == size(3000) > size(256)
