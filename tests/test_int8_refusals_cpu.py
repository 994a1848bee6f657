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


def test_outputs_whose_rows_lie_over_one_another_are_refused():
    """Before any CUDA call; where the pitches are fine, what is refused next is an address off its alignment, or a missing workspace."""
    lib = B.load()
    one, two, odd = 256, 512, 514   # never dereferenced

    def norm(N, S, Ch, outer, row):
        return lib.dvdq_rms_norm(B.RMS_NORM_ARGS.pack(one, 0, 0, 0, 0, 0, 0, 0, 0, two, outer, row, 0, 0, 0, N, S, Ch, 0, 0, odd, B.F32, B.F32, 1e-6), None)

    def back(N, S, Ch, outer, row):
        return lib.dvdq_rms_norm_backward(B.RMS_NORM_BACKWARD_ARGS.pack(one, 0, 0, one, 0, 0, 0, 0, 0, two, outer, row, N, S, Ch, 0, one, one, 0, 0, B.F32, B.F32), None)

    for shape in ((2, 3, 8, 8, 8), (2, 3, 8, 16, 8), (2, 3, 8, 23, 8), (3, 2, 8, 8, 20), (4, 4, 8, 12, 18), (2, 2, 8, 15, 8), (1000, 1000, 8, 8, 7999)):
        assert norm(*shape) == back(*shape) == B.ERR_SHAPE, shape
    for shape in ((2, 3, 8, 24, 8), (3, 2, 8, 8, 24), (2, 2, 8, 24, 16), (1, 3, 8, 0, 8), (3, 1, 8, 8, 0), (1000, 1000, 8, 8, 8000), (2, 2, 8, 1 << 62, 1 << 61)):
        assert norm(*shape) == B.ERR_ALIGN and back(*shape) == B.ERR_NULL, shape
