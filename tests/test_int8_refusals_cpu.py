"""Refusals of the 8-bit layer, the norm and the rows' quantization that need no GPU."""
import pytest
import torch

from paper_2505_18663_b200 import binding as B


def test_host_tensors_are_refused_as_such():
    x, c, s = torch.zeros(4, 16, dtype=torch.float16), torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    y = torch.zeros(4, 4, dtype=torch.float16)
    for call in (lambda: B.dvdq_rms_norm(x, None, None, 1e-6, None, x), lambda: B.dvdq_quantize_rows(x, c, s), lambda: B.dvdq_linear_int8(c, s, c, s, None, None, 0, y),
                 lambda: B.dvdq_rms_norm_backward(x, x, s, None, None, x, None)):
        with pytest.raises(TypeError, match="must be a CUDA tensor"):
            call()
