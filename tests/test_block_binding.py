"""What the binding of dropout, norms and ends of blocks refuses before the
library sees it (no GPU: matrices that only say where they would be)."""

import pytest

from paper_2106_10207_amd import dedloc as D

torch = pytest.importorskip("torch")


class Matrix:
    """A matrix of a device that this machine need not have; its address is never followed."""

    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self.device_index = shape, dtype, device
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def stride(self):
        return (self.shape[-1], 1)[-len(self.shape):]

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 1 << 20


@pytest.fixture(autouse=True)
def first_device(monkeypatch):
    monkeypatch.setattr(D, "_current_device", lambda: lambda: 0)


@pytest.mark.parametrize("gate_rows", [1 << 32, (1 << 32) + 4, -1])
def test_group_sizes_are_numbers_of_32_bits(gate_rows):
    """2^32 rows to a gate would reach the library as none: the 16-bit gate of a group read as an fp32 vector, past its end."""
    h, gate = Matrix(4, 8, dtype=torch.bfloat16), Matrix(1, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="gate_rows.*32 bits"):
        D.ResidualCall(h, h, sum=h, gate=gate, gate_rows=gate_rows)
    with pytest.raises(ValueError, match="gate_rows.*32 bits"):
        D.ResidualGradCall(None, None, None, h, None, h, h, gate=gate, gate_rows=gate_rows)
    with pytest.raises(ValueError, match="gate_rows.*32 bits"):
        D.make_residual_workspace(4, 8, gate_rows, device="cpu")


@pytest.mark.parametrize("width", [1 << 32, (1 << 32) + 8])
def test_widths_are_numbers_of_32_bits(width):
    """2^32 + 8 columns would reach the library as 8."""
    x = Matrix(1, width)
    for call in (lambda: D.dedloc_dropout(x, D.dropout_cfg(0.1), out=x),
                 lambda: D.dedloc_norm(x, D.norm_cfg(D.DEDLOC_NORM_RMS), out=x, keep_stats=False),
                 lambda: D.dedloc_norm_grad(x, x, Matrix(1, 1, 2), D.norm_cfg(D.DEDLOC_NORM_RMS), dx=x),
                 lambda: D.ResidualCall(x, x, sum=x),
                 lambda: D.ResidualGradCall(None, None, None, x, None, x, x),
                 lambda: D.make_residual_workspace(4, width, device="cpu")):
        with pytest.raises(ValueError, match="width.*32 bits"):
            call()
