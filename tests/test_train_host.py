"""Host side of the training operators: the binding's own refusals (no GPU is touched: every call below
fails before the library is called), and the plans of the products' splits and pieces."""
import ctypes

import pytest
import torch

from paper_2608_05448_amd import dblast as D

BF = torch.bfloat16


def _head(dtype=BF, B=2, K=3, R=2, d=16, V=40):
    return (torch.zeros((B, K, R, d), dtype=dtype), torch.zeros((V, d), dtype=dtype),
            torch.zeros((B, K), dtype=torch.int32))


def test_head_nll_refuses_what_is_no_gpu_tensor_or_of_another_type_or_shape():
    h, w, x = _head()
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_head_nll(h, w, x)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        D.dbl_head_nll(h.half(), w.half(), x)
    with pytest.raises(ValueError, match=r"\[B, K, R, d\]"):
        D.dbl_head_nll(h[0], w, x)
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_head_nll_backward(h, w, x, None, None, None)


def test_expander_backward_refuses_other_shapes():
    h, dout = torch.zeros((2, 3, 32), dtype=BF), torch.zeros((2, 3, 4, 32), dtype=BF)
    with pytest.raises(ValueError, match="GPU tensor"):
        D.dbl_expand_branches_backward(h, torch.zeros((128, 32), dtype=BF), dout)
    with pytest.raises(ValueError, match=r"\[B, K, d\]"):
        D.dbl_expand_branches_backward(h[0], torch.zeros((128, 32), dtype=BF), dout)


def test_gradient_lists_are_checked():
    with pytest.raises(ValueError, match="GPU tensors"):
        D.dbl_grad_norm([torch.ones(3)])
    with pytest.raises(ValueError, match="empty"):
        D.dbl_grad_norm([])
    with pytest.raises(TypeError):
        D.dbl_grad_norm([1.0, 2.0])
    assert D.dbl_clip_grads([], None, 1.0) == []


def test_workspaces_grow_with_the_pieces_not_with_the_vocabulary():
    """The backward pass holds at most about 1 GiB of the logits' gradient, however many rows there are
    (as long as a piece has more than 8192 ids), beside its copies of the rows and its sums of dh."""
    d, V = 64, 151936
    for rows in (256, 2048, 8192, 32768):
        n = D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, rows, 1, 1, d, V)
        copies = rows * (2 * 4 * d + 16 + 4)
        assert n <= (1 << 30) + 4096 * 4 * rows + copies + 600 * rows * d * 4, rows
        # loss alone: 4 bytes for every 32 ids of a row at most
        f = D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL, rows, 1, 1, d, V)
        assert f <= rows * (V // 8 + 8 + 4 * d + 64) + 2048
    # a small vocabulary is not padded to a piece
    rows, small = 1 << 20, 200
    n = D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, rows, 1, 1, d, small)
    assert n <= rows * (256 * 4 + 2 * 4 * d + 16 + 4) + rows * d * 4 + 64 * small * d * 4 + 4096
    assert D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, 0, 1, 1, d, V) >= 0
    assert D.dbl_workspace_bytes(15, 1, 1, 1, 8, 8) == ctypes.c_size_t(-1).value
    assert D.dbl_workspace_bytes(20, 1, 1, 1, 8, 8) == ctypes.c_size_t(-1).value
