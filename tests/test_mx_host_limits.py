"""Host side of the serving operators at the ends of their arguments' ranges. No GPU is touched."""
import pytest
import torch

from paper_2608_05448_amd import dblast as D


def test_row_length_of_every_64_bit_number():
    """0 where there is no row, also where the next multiple of 128 does not fit 64 bits."""
    row = D.load().dbl_mx_row
    top = (1 << 63) - 1
    assert row(top - 127) == top - 127 and row(top - 128) == top - 127
    for d in (top, top - 1, top - 126):
        assert row(d) == 0, d


@pytest.mark.parametrize("call", [
    lambda: D.dbl_mx_dequantize([1], None, 100),
    lambda: D.dbl_mx_matmul([1], None, None, None),
    lambda: D.dbl_mx_matmul(torch.zeros((1, 64), dtype=torch.uint8).numpy(), None, None, None),
    lambda: D.dbl_mx_head_logprobs(None, None, None, None),
    lambda: D.dbl_add_rmsnorm_mx(None, None, None),
])
def test_what_is_no_tensor_is_a_type_error(call):
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        call()
