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
