"""Norms and ends of blocks where the answer is known exactly: one gate for
all rows, norms left out, rows of equal entries, sums of whole numbers."""

import pytest

from paper_2106_10207_amd import dedloc as D
from . import block_ref as R
from .test_gpu_block import BF16, DEV, EPS, F16, F32, KINDS, PAIRS, gen, make_norm, rows, vector

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# ------------------------------------------------------- one gate for all rows

@pytest.mark.parametrize("n,width", [(1, 40), (2000, 40), (1500, 700), (300, 2500)])
def test_a_group_longer_than_all_rows(n, width):
    """Any gate_rows of at least the rows is one group: the same bits as for exactly the rows, up to the largest number there is."""
    g = gen(n)
    h, f, dsum, dout = (rows(n, width, BF16, g)[0] for _ in range(4))
    post, pre = make_norm("rms", width, g)[0], make_norm("layer", width, g)[0]
    gate = rows(1, width, BF16, g)[0].contiguous()

    def run(gate_rows):
        common = dict(alpha=1.0, beta=0.5, post=post, pre=pre, gate=gate, gate_rows=gate_rows, drop=D.dropout_cfg(0.1, 3))
        total, out, stats = D.dedloc_residual(h, f, **common)
        sums, dgate = torch.zeros(4, width, device=DEV), torch.full((1, width), 7.0, device=DEV)
        dh, df = D.dedloc_residual_grad(total, f, stats, dsum, dout, dgate=dgate, dpre=(sums[0], sums[1]), dpost=(sums[2], sums[3]), **common)
        return total, out, stats, dh, df, sums, dgate

    want = run(n)
    for gate_rows in (n + 1, (1 << 31) + 5, (1 << 32) - n, (1 << 32) - 1):
        assert all(torch.equal(a, b) for a, b in zip(run(gate_rows), want)), gate_rows
