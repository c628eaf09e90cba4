"""What dropout, the norms and the ends of a block refuse, on the host, before
anything reaches the GPU (no GPU needed: the addresses are never followed), their
workspace, and the generator of the tests' own reference."""

import ctypes

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D
from . import block_ref as R

A = 1 << 20  # an aligned address
OK, ARG, ALIGN, WS = D.DEDLOC_OK, D.DEDLOC_ERR_INVALID_ARG, D.DEDLOC_ERR_ALIGN, D.DEDLOC_ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


def drop(p=0.1, step_at=None):
    return D.dedloc_dropout_cfg(p, 1, 2, 3, 4, step_at)


def norm(kind=1, eps=1e-6, gain=A, bias=A):
    return D.dedloc_norm_cfg(kind, eps, gain, bias)


NONE = norm(0, 0.0, None, None)


def test_reference_generator():
    """The three known answers that the generator's authors publish with it."""
    full = 0xFFFFFFFF
    for ctr, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((full,) * 4, (full,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(w) for w in R.philox(*ctr, *key)) == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_reference_mask(p):
    """The share that is kept, to 5 standard deviations, and sums that keep their mean."""
    n = 512 * 1000
    keep, factor = R.kept(512, 1000, p, seed=12345678901234567, site=3, step=9)
    rate = round(p * 65536) / 65536
    assert abs(keep.mean() - (1 - rate)) <= 5 * (rate * (1 - rate) / n) ** 0.5
    assert float(factor) == np.float32(1 / (1 - rate))
    again, _ = R.kept(100, 1000, p, seed=12345678901234567, site=3, step=9, row0=300)
    assert np.array_equal(again, keep[300:400])


def test_dropout_refusals():
    lib = D.load()

    def call(cfg=None, rows=4, width=8, dtype=0, x=A, ldx=8, out=A, ldo=8):
        return lib.dedloc_dropout(drop() if cfg is None else cfg, rows, width, dtype, x, ldx, out, ldo, None)

    assert lib.dedloc_dropout(None, 4, 8, 0, A, 8, A, 8, None) == ARG
    assert call(rows=0, x=None, out=None) == OK and call(width=0, x=None, out=None) == OK
    for p in (-0.1, 1.0001, NAN, INF):
        assert call(drop(p)) == ARG and call(drop(p), rows=0) == ARG
    assert call(dtype=3) == ARG and call(dtype=-1) == ARG
    assert call(rows=(1 << 30) + 1) == ARG and call(width=(1 << 20) + 1, ldx=1 << 21, ldo=1 << 21) == ARG
    assert call(x=None) == ARG and call(out=None) == ARG and call(ldx=7) == ARG and call(ldo=7) == ARG
    assert call(x=A + 2) == ALIGN and call(out=A + 1, dtype=2) == ALIGN and call(drop(step_at=A + 4)) == ALIGN


def test_norm_refusals():
    lib = D.load()

    def call(cfg=None, rows=4, width=8, td=0, od=0, x=A, ldx=8, out=A, ldo=8, stats=A):
        return lib.dedloc_norm(norm() if cfg is None else cfg, rows, width, td, od, x, ldx, out, ldo, stats, None)

    def back(cfg=None, rows=4, width=8, td=0, od=0, dout=A, ldd=8, x=A, ldx=8, stats=A, add=None, lda=8, dx=A, ldo=8, dgain=A,
             dbias=A, ws=A, wsb=1 << 30):
        return lib.dedloc_norm_grad(norm() if cfg is None else cfg, rows, width, td, od, dout, ldd, x, ldx, stats, add, lda, dx,
                                    ldo, dgain, dbias, 1.0, ws, wsb, None)

    assert lib.dedloc_norm(None, 4, 8, 0, 0, A, 8, A, 8, A, None) == ARG
    assert call(rows=0, x=None, out=None) == OK and call(width=0) == OK
    assert back(rows=0, dout=None, x=None, dx=None, ws=None) == OK and back(width=0, ws=None) == OK
    for f in (call, back):
        assert f(NONE) == ARG and f(norm(3)) == ARG and f(norm(-1)) == ARG
        for eps in (0.0, -1.0, NAN, INF, 1e-31):
            assert f(norm(eps=eps)) == ARG
        assert f(norm(gain=A + 2)) == ALIGN and f(norm(bias=A + 1)) == ALIGN
        assert f(rows=(1 << 30) + 1) == ARG and f(width=16385, ldx=20000, ldo=20000) == ARG
        assert f(td=3) == ARG and f(od=7) == ARG and f(td=1, od=2) == ARG and f(td=1, od=0) == ARG
        assert f(x=None) == ARG and f(ldx=7) == ARG and f(ldo=7) == ARG and f(x=A + 2) == ALIGN and f(stats=A + 4) == ALIGN
    assert call(out=None) == ARG and call(out=A + 1, od=1) == ALIGN
    assert back(dout=None) == ARG and back(dx=None) == ARG and back(stats=None) == ARG and back(ldd=7) == ARG
    assert back(add=A, lda=7) == ARG and back(add=A + 2) == ALIGN and back(dout=A + 1, od=2) == ALIGN
    assert back(norm(gain=None)) == ARG and back(norm(bias=None)) == ARG  # gradients of what is not there
    assert back(dgain=A + 2) == ALIGN and back(dbias=A + 1) == ALIGN
    need = lib.dedloc_residual_workspace_bytes(4, 8, 0)
    assert need > 0 and back(wsb=need - 1) == WS and back(ws=None) == WS and back(ws=A + 128) == ALIGN


def test_residual_refusals():
    lib = D.load()

    def cfg(post=NONE, pre=None, gate=None, ldg=8, gate_rows=0, d=None):
        return D.dedloc_residual_cfg(1.0, 1.0, post, norm() if pre is None else pre, gate, ldg, gate_rows, drop(0.0) if d is None else d)

    def call(c=None, rows=4, width=8, sd=0, bd=0, h=A, ldh=8, f=A, ldf=8, sum=A, lds=8, out=A, ldo=8, stats=A):
        return lib.dedloc_residual(cfg() if c is None else c, rows, width, sd, bd, h, ldh, f, ldf, sum, lds, out, ldo, stats, None)

    full = dict(sum=A, f=A, dsum=A, dout=A, dh=A, df=A, stats=A, ld_sum=8, ld_f=8, ld_dsum=8, ld_dout=8, ld_dh=8, ld_df=8)

    def back(c=None, rows=4, width=8, sd=0, bd=0, ws=A, wsb=1 << 30, **over):
        g = D.dedloc_residual_grads(**{**full, **over})
        return lib.dedloc_residual_grad(cfg() if c is None else c, rows, width, sd, bd, ctypes.byref(g), 1.0, ws, wsb, None)

    assert lib.dedloc_residual(None, 4, 8, 0, 0, A, 8, A, 8, A, 8, A, 8, A, None) == ARG
    assert lib.dedloc_residual_grad(cfg(), 4, 8, 0, 0, None, 1.0, A, 1 << 30, None) == ARG
    assert call(rows=0, h=None, f=None, sum=None, out=None) == OK and call(width=0) == OK and back(rows=0, dh=None) == OK
    for f in (call, back):
        assert f(cfg(post=norm(5))) == ARG and f(cfg(pre=norm(eps=0.0))) == ARG and f(cfg(d=drop(2.0))) == ARG
        assert f(cfg(gate_rows=2)) == ARG and f(cfg(gate=A, gate_rows=2, ldg=7)) == ARG
        assert f(cfg(gate=A + 2)) == ALIGN and f(cfg(gate=A + 1, gate_rows=2), sd=1, bd=1) == ALIGN
        assert f(cfg(d=drop(step_at=A + 2))) == ALIGN
        assert f(rows=(1 << 30) + 1) == ARG and f(width=16385) == ARG
        assert f(sd=3) == ARG and f(bd=3) == ARG and f(sd=1) == ARG and f(sd=2, bd=1) == ARG
        assert f(stats=A + 4) == ALIGN
        assert f(sum=A + 2) == ALIGN and f(f=None, c=cfg(post=norm())) == ARG
    assert call(h=None) == ARG and call(f=None) == ARG and call(out=None) == ARG
    assert call(cfg(pre=NONE)) == ARG            # out without a norm to give it
    assert call(cfg(pre=NONE), out=None, sum=None) == ARG
    assert call(ldh=7) == ARG and call(ldf=7) == ARG and call(lds=7) == ARG and call(ldo=7) == ARG
    assert back(dh=None) == ARG and back(df=None) == ARG and back(dout=None) == ARG and back(sum=None) == ARG and back(stats=None) == ARG
    assert back(cfg(pre=NONE)) == ARG            # dout without a norm
    assert back(cfg(pre=NONE), dout=None, dsum=None) == ARG
    for name in ("sum", "f", "dsum", "dout", "dh", "df"):
        c = cfg(post=norm())
        assert back(c, **{"ld_" + name: 7}) == ARG and back(c, **{name: A + 1}) == ALIGN
    assert back(dgate=A) == ARG and back(dpost_gain=A) == ARG and back(dpost_bias=A) == ARG
    assert back(cfg(pre=norm(gain=None)), dpre_gain=A) == ARG and back(cfg(pre=norm(bias=None)), dpre_bias=A) == ARG
    assert back(cfg(gate=A, gate_rows=2), dgate=A, ld_dgate=7) == ARG
    assert back(dpre_gain=A + 1) == ALIGN and back(cfg(gate=A), dgate=A + 2) == ALIGN
    assert back(cfg(gate=A), dgate=A, f=None) == ARG
    need, gated = (lib.dedloc_residual_workspace_bytes(4, 8, k) for k in (0, 2))
    assert 0 < need < gated
    assert back(dpre_gain=A, wsb=need - 1) == WS and back(dpre_gain=A, ws=None) == WS and back(dpre_gain=A, ws=A + 8) == ALIGN
    assert back(cfg(gate=A, gate_rows=2), dgate=A, ld_dgate=8, wsb=gated - 1) == WS


def test_workspace_never_falls():
    need = D.load().dedloc_residual_workspace_bytes
    assert need((1 << 30) + 1, 8, 0) == 0 and need(4, 16385, 0) == 0 and need(0, 0, 0) > 0
    rows = sorted({n for e in (1, 4, 16, 128, 1000, 4096, 16384, 1 << 17, 1 << 20, 1 << 30) for n in (e - 1, e, e + 1, e + 3) if 1 <= n <= 1 << 30})
    widths = sorted({w for e in (1, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384) for w in (e - 1, e, e + 1) if 1 <= w <= 16384})
    for gate_rows in (0, 5):
        sizes = np.array([[need(n, w, gate_rows) for w in widths] for n in rows], dtype=object)
        assert (sizes > 0).all()
        assert (sizes[1:] >= sizes[:-1]).all() and (sizes[:, 1:] >= sizes[:, :-1]).all()
    assert need(1 << 30, 16384, 1) < 1 << 30


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 6)
    with pytest.raises(ValueError, match="device tensor"):
        D.dedloc_dropout(x, D.dropout_cfg(0.1))
    with pytest.raises(ValueError, match="device tensor"):
        D.norm_cfg(D.DEDLOC_NORM_LAYER, torch.ones(6))
    with pytest.raises(ValueError, match="device tensor"):
        D.dedloc_norm(x, D.norm_cfg(D.DEDLOC_NORM_RMS))
    cfg = D.norm_cfg(D.DEDLOC_NORM_LAYER)
    cfg._width = 7  # as norm_cfg leaves it, had it been given vectors of 7
    with pytest.raises(ValueError, match="7 elements"):
        D._check_norm(cfg, 6, "norm")
    with pytest.raises(ValueError, match="one int64"):
        D.dropout_cfg(0.1, step_at=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="device tensor"):
        D.dedloc_residual(x, x)
    with pytest.raises(ValueError, match="sum or dsum"):
        D.dedloc_residual_grad(None, None, None, None, x)
