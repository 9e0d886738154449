"""Tokens and labels are read as int32 in order: tensors of another type, or whose elements are not
in order, are refused in Python before anything is enqueued (these calls need no device)."""
import numpy as np
import pytest
import torch

from paper_1704_04560_amd import mtx
from paper_1704_04560_amd import workloads as wl

F = mtx.MTX_F32
TOK = torch.arange(12, dtype=torch.int32).view(3, 4)
BAD = {"int64": TOK.long(), "int16": TOK.short(), "float32": TOK.float(), "columns": TOK[:, :-1],
       "transposed": TOK.t(), "every second": TOK.view(-1)[::2], "numpy int64": TOK.numpy().astype(np.int64),
       "numpy columns": TOK.numpy()[:, 1:]}


@pytest.mark.parametrize("name", list(BAD))
def test_tokens_and_labels(name):
    bad, a = BAD[name], 1 << 33
    labels = TOK.view(-1)
    for call in (
            lambda: mtx.mtx_embed_forward(a, F, 16, 8, bad, 12, -1, 1.0, 2 * a, F, 8, stream=0),
            lambda: mtx.mtx_embed_backward(bad, 12, 1, a, F, 8, 16, 8, -1, 1.0, 2 * a, 128, False, None,
                                           stream=0),
            lambda: mtx.mtx_train_step_tokens(None, bad, labels, 0.1, 0.0, stream=0),
            lambda: mtx.mtx_train_step_tokens(None, labels, bad, 0.1, 0.0, stream=0),
            lambda: mtx.mtx_train_step(None, a, bad, 0.1, 0.0, stream=0)):
        with pytest.raises(ValueError):
            call()


def test_int32_in_order_passes():
    """The library's own checks come next: a NULL model."""
    for ids in (TOK, TOK[1:], TOK.view(-1), TOK.numpy(), 1 << 33, None, TOK[:, :1][:1]):
        with pytest.raises(mtx.MtxError):
            mtx.mtx_train_step_tokens(None, ids, ids, 0.1, 0.0, stream=0)
    x, y = wl.make_batch(wl.MLP, 4, seed=1)
    assert y.dtype == np.int32
    with pytest.raises(mtx.MtxError):
        mtx.mtx_train_step(None, 1 << 33, y, 0.1, 0.0, stream=0)
