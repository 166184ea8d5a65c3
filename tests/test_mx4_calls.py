"""Microscaled 4-bit operators: calls at the edge of what their documentation allows, and refusals of those beyond it."""
import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import mx4_oracle as mx
from test_mx4 import Problem, as_f64, counts_to_offsets, edge_values, grouped_reference, off_by_at_most, to_gpu


def test_the_row_form_needs_its_exponents(lutq):
    """Without them the arguments are those of the packed form, of which the caller has not spoken."""
    import torch
    x, p = torch.zeros((16, 128), dtype=torch.float16), torch.zeros(lutq.lutq_mx4_packed_bytes(16, 128), dtype=torch.uint8)
    for call in (lambda: lutq.lutq_mx4_quantize(x, p, None), lambda: lutq.lutq_mx4_dequant(p, None, x)):
        with pytest.raises(TypeError, match="exponents"):
            call()


@pytest.mark.gpu
def test_the_row_form_needs_its_exponents_on_the_device(lutq):
    import torch
    x = torch.ones((16, 128), dtype=torch.float16, device="cuda")
    p = torch.full((lutq.lutq_mx4_packed_bytes(16, 128),), 0xA5, dtype=torch.uint8, device="cuda")
    for call in (lambda: lutq.lutq_mx4_quantize(x, p, None), lambda: lutq.lutq_mx4_dequant(p, None, x)):
        with pytest.raises(TypeError, match="exponents"):
            call()
    torch.cuda.synchronize()
    assert (p == 0xA5).all().item() and (x == 1.0).all().item()
