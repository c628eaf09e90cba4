"""What the orthogonalised update, the Muon step and the embedding's entry
points refuse, on the host, before anything reaches the GPU (no GPU needed:
the addresses are never followed)."""

import ctypes

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D

A = 1 << 20  # an aligned address
OK, ARG, ALIGN, WS = D.DEDLOC_OK, D.DEDLOC_ERR_INVALID_ARG, D.DEDLOC_ERR_ALIGN, D.DEDLOC_ERR_WORKSPACE


def mats(*ms):
    return (D.dedloc_matrix * len(ms))(*[D.dedloc_matrix(*m) for m in ms])


def test_orthogonalize_refusals():
    lib = D.load()
    good = (A, A, 20, 24, 10, 20)

    def call(m=(good,), n=None, dtype=0, cfg=D.ortho_cfg(), ws=A, wsb=1 << 30):
        arr = mats(*m) if m else None
        return lib.dedloc_orthogonalize(arr, len(m) if n is None else n, dtype, ctypes.byref(cfg) if cfg else None, ws,
                                        wsb, None)

    empty = (None, None, 0, 0, 0, 20)
    assert call([empty]) == OK  # nothing to do: nothing is enqueued
    assert call([empty, (None, None, 0, 0, 7, 0)]) == OK
    assert call((), n=1) == ARG
    assert call(n=0) == ARG
    assert call(cfg=None) == ARG
    assert call(dtype=3) == ARG and call(dtype=-1) == ARG
    assert call(cfg=D.ortho_cfg(steps=0)) == ARG
    assert call(cfg=D.ortho_cfg(steps=65)) == ARG
    assert call([empty, (None, A, 20, 20, 10, 20)]) == ARG
    assert call([(A, None, 20, 20, 10, 20)]) == ARG
    assert call([(A, A, 19, 20, 10, 20)]) == ARG
    assert call([(A, A, 20, 19, 10, 20)]) == ARG
    assert call([(A + 2, A, 20, 20, 10, 20)]) == ALIGN
    assert call([(A + 1, A, 20, 20, 10, 20)], dtype=2) == ALIGN
    assert call([(A, A, 40000, 40000, 32769, 40000)]) == ARG
    assert call([(A, A, (1 << 26) + 1, (1 << 26) + 1, 1, (1 << 26) + 1)]) == ARG
    need = lib.dedloc_orthogonalize_workspace_bytes(mats(good), 1)
    assert need > 0
    assert call(wsb=need - 1) == WS and call(ws=None) == WS
    assert call(ws=A + 128) == ALIGN


def test_orthogonalize_workspace():
    lib = D.load()
    one = lib.dedloc_orthogonalize_workspace_bytes(mats((A, A, 300, 300, 200, 300)), 1)
    # X, two transposes and two squares at 4 bytes an element, both sides padded; room for the sums of cut products
    assert 4 * (3 * 200 * 300 + 2 * 200 * 200) <= one <= 8 * (3 * 256 * 320 + 2 * 256 * 256) + (4 << 20)
    # blocks of steps take four squares more
    wide = lib.dedloc_orthogonalize_workspace_bytes(mats((A, A, 4096, 4096, 1024, 4096)), 1)
    assert 4 * (3 * 1024 * 4096 + 6 * 1024 * 1024) <= wide <= 8 * (3 * 1024 * 4096 + 6 * 1024 * 1024)
    many = mats(*[(A, A, 300, 300, 200, 300)] * 200)
    # worked on in batches: 200 take no more than some of them
    assert one < lib.dedloc_orthogonalize_workspace_bytes(many, 200) < 100 * one
    assert lib.dedloc_orthogonalize_workspace_bytes(mats((A, A, 40000, 40000, 40000, 40000)), 1) == 0
    assert "exceeds" in lib.dedloc_last_error().decode()
    assert lib.dedloc_orthogonalize_workspace_bytes(None, 1) == 0
    assert lib.dedloc_orthogonalize_workspace_bytes(mats((None, None, 0, 0, 0, 0)), 1) > 0


def test_muon_refusals():
    lib = D.load()

    def call(off=(0, 200, 208), rows=(10, 1), cols=(20, 8), flags=(3, 3), P=None, x=A, m=A, grad=A, scales=None, codec=0,
             block=1024, cfg=D.muon_cfg(), ws=A, wsb=1 << 30, n=None):
        off = np.array(off, np.uint64)
        r, c = np.array(rows, np.uint32), np.array(cols, np.uint32)
        f = np.array(flags, np.uint8) if flags is not None else None
        return lib.dedloc_muon_step(x, m, grad, scales, codec, block, int(off[-1]) if P is None else P, off.ctypes.data,
                                    r.ctypes.data, c.ctypes.data, None if f is None else f.ctypes.data,
                                    len(r) if n is None else n, ctypes.byref(cfg) if cfg else None, ws, wsb, None)

    # tensors that are not matrices: nothing is enqueued
    assert call(rows=(0, 0), cols=(20, 0)) == OK
    assert call(off=(0, 0), rows=(0,), cols=(0,), flags=(3,), x=None, m=None, grad=None) == OK
    assert call(cfg=None) == ARG
    assert call(cfg=D.muon_cfg(ortho=D.ortho_cfg(steps=0))) == ARG
    assert call(codec=7) == ARG and call(codec=2, scales=None) == ARG and call(codec=2, scales=A, block=512) == ARG
    assert call(codec=2, scales=A + 2) == ARG
    assert call(flags=None) == ARG and call(n=0) == ARG
    assert call(P=209) == ARG
    assert call(off=(0, 204, 212)) == ALIGN
    assert call(off=(0, 208, 200)) == ARG
    assert call(rows=(11, 1)) == ARG          # 220 elements in a tensor of 200
    assert call(cols=(19, 8)) == ARG          # 190 of 200: more than 7 left over
    assert call(x=None) == ARG and call(m=None) == ARG and call(grad=None) == ARG
    assert call(x=A + 4) == ALIGN and call(m=A + 8) == ALIGN and call(grad=A + 2) == ALIGN
    assert call(rows=(1, 1), cols=((1 << 26) + 8, 8), off=(0, (1 << 26) + 8, (1 << 26) + 16)) == ARG
    r, c = np.array([10, 1], np.uint32), np.array([20, 8], np.uint32)
    need = lib.dedloc_muon_workspace_bytes(r.ctypes.data, c.ctypes.data, 2)
    assert need > 0 and call(wsb=need - 1) == WS and call(ws=None) == WS and call(ws=A + 64) == ALIGN
    assert lib.dedloc_muon_workspace_bytes(None, c.ctypes.data, 2) == 0


def test_embed_refusals():
    lib = D.load()

    def call(table=A, td=0, vocab=10, width=8, ldt=8, ids=A, idb=8, n=4, out=A, od=0, ldo=8):
        return lib.dedloc_embed(table, td, vocab, width, ldt, ids, idb, n, 1.0, out, od, ldo, None)

    def back(grad=A, vocab=10, width=8, ldg=8, ids=A, idb=8, n=4, dy=A, dd=0, ldd=8, ws=A, wsb=1 << 30):
        return lib.dedloc_embed_grad(grad, vocab, width, ldg, ids, idb, n, dy, dd, ldd, 1.0, 1.0, ws, wsb, None)

    assert call(n=0, table=None, ids=None, out=None) == OK and call(width=0) == OK
    assert back(n=0, grad=None, ids=None, dy=None, ws=None) == OK and back(vocab=0, grad=None) == OK
    assert call(td=3) == ARG and call(od=-1) == ARG and back(dd=9) == ARG
    assert call(idb=2) == ARG and back(idb=16) == ARG
    for f in (call, back):
        assert f(n=(1 << 30) + 1) == ARG and f(vocab=(1 << 30) + 1) == ARG and f(width=(1 << 20) + 1) == ARG
        assert f(ids=None) == ARG and f(ids=A + 4) == ALIGN and f(ids=A + 2, idb=4) == ALIGN
    assert call(table=None) == ARG and call(out=None) == ARG and back(grad=None) == ARG and back(dy=None) == ARG
    assert call(ldt=7) == ARG and call(ldo=7) == ARG and back(ldg=7) == ARG and back(ldd=7) == ARG
    assert call(table=A + 2) == ALIGN and call(td=1, table=A + 1) == ALIGN and call(out=A + 2) == ALIGN
    assert back(grad=A + 2) == ALIGN and back(dd=2, dy=A + 1) == ALIGN
    need = lib.dedloc_embed_workspace_bytes(4, 10, 8)
    assert need > 0 and back(wsb=need - 1) == WS and back(ws=None) == WS and back(ws=A + 16) == ALIGN
    assert lib.dedloc_embed_workspace_bytes((1 << 30) + 1, 10, 8) == 0


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    g = torch.zeros(4, 6)
    with pytest.raises(ValueError, match="device tensor"):
        D.dedloc_orthogonalize([g], [g])
    with pytest.raises(ValueError, match="device tensor"):
        D.dedloc_embed(g, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="int32 or int64"):
        D.dedloc_embed(g, torch.zeros(2))
    with pytest.raises(ValueError, match="at least one"):
        D.OrthogonalizeCall([], [])


def test_embed_workspace_never_falls():
    """A workspace holds every call of fewer ids or narrower rows: over the sizes where the sort's chunks, and the
    chunks of the sums (products of 2^20, 2^23 and 2^25), change."""
    need = D.load().dedloc_embed_workspace_bytes
    steps = lambda at: range(max(0, at - 3), at + 4)  # noqa: E731
    for width in (1, 2, 7, 128, 333, 1024, 1 << 20):
        ends = [1, 4, 8, 1024, 2048, 4352, 16384, 1 << 20, 1 << 21, 1 << 29] + [(1 << k) // width for k in (20, 23, 25, 30)]
        ns = sorted({n for e in ends for n in steps(e) if n <= 1 << 30})
        sizes = [need(n, 1000, width) for n in ns]
        assert all(sizes) and sizes == sorted(sizes), width
    for n in (1, 5, 1000, 8191, 8192, 8193, 65537, 1 << 25):
        ends = [1, 8, 1 << 20] + [(1 << k) // n for k in (20, 23, 25)]
        widths = sorted({w for e in ends for w in steps(e) if w <= 1 << 20})
        sizes = [need(n, 1000, w) for w in widths]
        assert all(sizes) and sizes == sorted(sizes), n
    # and it holds the parts: two per chunk of 4 positions at least where there are few
    assert need(8191, 30000, 128) >= 2 * 8 * 8191 + 2048 * 2 * 128 * 4
