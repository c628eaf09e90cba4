"""The tolerance of the tight tests of dedloc_orthogonalize and
dedloc_muon_step: an emulation of the arithmetic stays well inside it on their
inputs, and one with a product left out does not pass (no GPU needed)."""

import numpy as np
import pytest

from tests import ns_planes as N


@pytest.mark.parametrize("shape", N.SHAPES)
def test_emulation_is_inside_and_a_lost_product_is_not(shape):
    u = N.noise(*shape, seed=shape[0] + 7 * shape[1])
    want = N.formula(u)
    blocked = shape in N.LISTS["blocks"]
    inside = N.relative(N.emulated(u, blocked), want)
    lost = [N.relative(N.emulated(u, blocked, d), want) for d in (("hi lo",), ("lo hi",), ("hi lo", "lo hi"))]
    print(shape, f"{inside:.2g}, without a product", *(f"{v:.2g}" for v in lost))
    assert inside <= N.TIGHT / 2
    assert min(lost) >= 10 * N.TIGHT


@pytest.mark.parametrize("shape", [s for s in N.SHAPES if min(s) * max(s) > 10000])
@pytest.mark.parametrize("name", ["float16", "bfloat16"])
def test_share_of_16_bit_roundings(shape, name):
    """How many entries of a 16-bit result are not the rounding of the 64-bit value: the emulation's, and with a product left out."""
    torch = pytest.importorskip("torch")
    dtype = getattr(torch, name)
    u = torch.from_numpy(N.noise(*shape, seed=1)).to(dtype).double().numpy()
    blocked = shape in N.LISTS["blocks"]
    right = torch.from_numpy(N.formula(u)).to(dtype)
    share = [float((torch.from_numpy(np.ascontiguousarray(N.emulated(u, blocked, d))).to(dtype) != right).float().mean())
             for d in ((), ("hi lo",), ("lo hi",))]
    print(shape, name, share)
    assert share[0] <= N.MISROUNDED[name] / 4 and min(share[1:]) >= 2 * N.MISROUNDED[name]
