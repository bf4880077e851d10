"""Workspaces of the training operators, on the host: what dbl_workspace_bytes answers for them, part by
part, and what the binding takes as a workspace."""
import ctypes

import pytest
import torch

from paper_2608_05448_amd import dblast as D

SIZE_MAX = ctypes.c_size_t(-1).value


def _up(n, to):
    return -(-n // to) * to


def _piece(rows, V, elem):
    """Ids that the gradient takes at a time, as the header has it: about 1 GiB of the logits' gradient, at
    least 8192 ids, in equal pieces of a multiple of 4096 (256 for one)."""
    cap = max(8192, (1 << 30) // (elem * rows) // 4096 * 4096)
    pieces = -(-V // cap)
    return _up(-(-V // pieces), 4096 if pieces > 1 else 256)


# rows, d, V, copies of dh in fp32, sums of dw in parts (of a piece's ids)
PARTS = [
    (8, 64, 256, 8, 0),              # fp32 parts of 32 terms; one part for the weight
    (60, 2560, 151936, 38, 0),       # fp32: 768 workgroups over 20 tiles; bf16: 256 over 10 (25 parts)
    (256, 64, 151936, 256, 0),       # 128 x 128 tiles: 512 workgroups over 2
    (2048, 64, 151936, 32, 0),
    (8192, 64, 151936, 8, 0),
    (32768, 64, 151936, 2, 4),       # pieces of 8192 ids: their weights in 4 parts (fp32)
    (2048, 4096, 151936, 2, 0),      # 128 tiles of 256 x 256 on 256 CUs: two parts
    (8192, 4096, 151936, 1, 0),
    (65536, 4096, 151936, 1, 0),
]


@pytest.mark.parametrize("case", PARTS, ids=str)
def test_gradient_workspace_part_by_part(case):
    rows, d, V, dh, dw = case
    grad = max(rows * _piece(rows, V, e) * e for e in (2, 4))
    ids = min(V, _piece(rows, V, 4))
    parts = [4, 4 * rows, 16 * rows, 4 * rows * d, 4 * rows * d, grad, 4 * rows * d * dh, 4 * ids * d * dw]
    want = sum(_up(n, 256) for n in parts)
    assert D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, rows, 1, 1, d, V) == want, \
        (D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL_BACKWARD, rows, 1, 1, d, V) - want) / (4 * rows * d)


@pytest.mark.parametrize("rows", [1, 60, 2048, 65536])
def test_loss_workspace_part_by_part(rows):
    d, V = 4096, 151936
    parts = [4, 4 * rows, 16 * rows, 4 * rows * d, 4 * rows * (V // 32), 4 * rows]
    assert D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL, rows, 1, 1, d, V) == sum(_up(n, 256) for n in parts)


def test_norm_workspace_is_sized_for_what_the_call_takes():
    """dbl_grad_norm takes up to 2^20 tensors: more have no workspace (the product of a count near 2^62 and
    the partial sums of a launch does not fit 64 bits either)."""
    size = lambda n: D.dbl_workspace_bytes(D.DBL_OP_GRAD_NORM, n, 1, 1, 1, 1)
    assert size(0) == 0
    assert size(1) == size(180) == 1024 * 8 and size(181) == 2 * 1024 * 8
    assert size(1 << 20) == -(-(1 << 20) // 180) * 1024 * 8
    for n in ((1 << 20) + 1, 1 << 40, 3 * 10 ** 18, (1 << 61) + 12345):
        assert size(n) == SIZE_MAX, n


def test_a_workspace_that_is_not_memory_in_one_piece_is_refused():
    """The kernels write the whole size from the tensor's first byte on: a view that repeats or skips elements
    has the number of elements, but not the memory."""
    shape = D.Shape(1, 4, 2, 64, 256)
    n = D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL, 1, 4, 2, 64, 256)
    dev = torch.device("cuda", 0)
    for ws in (torch.empty(1, dtype=torch.uint8).expand(n), torch.empty(2 * n, dtype=torch.uint8)[::2],
               torch.empty((64, n), dtype=torch.uint8).t()):
        with pytest.raises(ValueError, match="contiguous"):
            D._workspace(D.DBL_OP_HEAD_NLL, shape, dev, ws)
    with pytest.raises(ValueError, match="GPU tensor"):
        D._workspace(D.DBL_OP_HEAD_NLL, shape, dev, torch.empty(n, dtype=torch.uint8))
    with pytest.raises(ValueError, match=f"needs {n} bytes"):
        D._workspace(D.DBL_OP_HEAD_NLL, shape, dev, torch.empty(n - 1, dtype=torch.uint8))
    with pytest.raises(TypeError, match="torch.Tensor"):
        D._workspace(D.DBL_OP_HEAD_NLL, shape, dev, bytearray(n))


def test_a_shape_without_a_workspace_is_left_to_the_call_to_refuse():
    """No memory is asked for: the call's own check of the shape comes before that of the workspace, and says
    what is wrong."""
    shape = D.Shape(1, 1, 65, 8, 16)  # R <= 64
    assert D.dbl_workspace_bytes(D.DBL_OP_HEAD_NLL, 1, 1, 65, 8, 16) == SIZE_MAX
    assert D._workspace(D.DBL_OP_HEAD_NLL, shape, torch.device("cpu")) == (None, 0)
    lib = D.load()
    at = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(8)]
    none = ctypes.c_void_p(None)
    assert lib.dbl_head_nll(shape, D.DBL_BF16, *at[:5], none, 0, none) == D.DBL_ESHAPE
    assert lib.dbl_head_nll_backward(shape, D.DBL_BF16, *at[:8], none, 0, none) == D.DBL_ESHAPE
    many = D.Shape(1 << 24, 1, 1, 8, 16)
    assert D._workspace(D.DBL_OP_HEAD_NLL, many, torch.device("cpu")) == (None, 0)
    assert lib.dbl_head_nll(many, D.DBL_BF16, *at[:5], none, 0, none) == D.DBL_ESHAPE
    assert D._workspace(D.DBL_OP_EXPAND_BACKWARD, many, torch.device("cpu")) == (None, 0)
