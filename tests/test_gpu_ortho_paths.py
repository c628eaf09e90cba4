"""dedloc_orthogonalize and dedloc_muon_step on each way that a call works on
its matrices, near enough to the definition in 64 bits that one lost product
of two fp16 planes shows (test_ortho_tolerance.py has the tolerance's reason),
and calls of more matrices than one table holds."""

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D
from tests import ns_planes as N

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def inputs(shapes, dtype, pad=0):
    """Matrices of noise, rows `pad` elements longer than the matrix; the gaps hold NaN."""
    out = []
    for k, (r, c) in enumerate(shapes):
        buf = torch.full((r, c + pad), float("nan"), dtype=dtype, device=DEV)
        out.append(buf[:, :c])
        out[-1].copy_(torch.from_numpy(N.noise(r, c, seed=r + 7 * c + k)))
    return out


def near(out, g):
    """fp32: the relative error.  16 bits: how many entries are not the rounding of the 64-bit value, and by more than
    one place (a step of 2^-10 or 2^-7 of an entry at most, and what TIGHT leaves of the small ones)."""
    want = N.formula(g.double().cpu().numpy())
    if out.dtype is torch.float32:
        got = N.relative(out.double().cpu().numpy(), want)
        print(tuple(out.shape), f"error {got:.2g}")
        assert got <= N.TIGHT, (tuple(out.shape), got)
        return
    right = torch.from_numpy(want).to(out.dtype).to(DEV)
    share = float((out != right).float().mean())
    step = 2.0 ** (-10 if out.dtype is torch.float16 else -7)
    # 60 times the entries' mean size: the tail of errors that are at most TIGHT of it in the mean
    room = step * right.double().abs() + 60 * N.TIGHT * float(right.double().square().mean().sqrt())
    print(tuple(out.shape), out.dtype, f"{share:.2g} not the rounding")
    allowed = N.MISROUNDED[str(out.dtype)[6:]]
    assert share <= max(allowed, 3.0 / out.numel()), (tuple(out.shape), share)
    assert bool(((out.double() - right.double()).abs() <= room).all())


def launches(call):
    """How many launches of each kernel a call takes."""
    torch.cuda.synchronize()
    D.dedloc_profile_begin(1 << 12)
    call()
    return {k: n for k, (_, n) in D.dedloc_profile_end().items()}


def check_path(path, n, join=False):
    if path == "narrow":
        assert n.get("ns_narrow") == 6 and "ns_product" not in n, n
    else:
        assert n.get("ns_product") == (17 if path == "blocks" else 15) and "ns_narrow" not in n, n
    assert not join or n.get("ns_join", 0) > 0, n


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("path", N.LISTS)
def test_orthogonalize(path, dtype):
    g = inputs(N.LISTS[path], dtype, pad=3)
    out = [torch.empty_like(v) for v in g]
    check_path(path, launches(D.OrthogonalizeCall(g, out)), join=path == "cut")
    for o, v in zip(out, g):
        near(o, v)


def message(flat, wire):
    """(what the step takes, scales, codec, its values) of a gradient."""
    if wire == "f32":
        return flat, None, D.DEDLOC_CODEC_F32, flat
    codec = D.CODECS[wire]
    codes, scales = D.dedloc_encode(flat, codec)
    return codes, scales, codec, D.dedloc_decode(codes, scales, flat.numel(), codec)


def muon(shapes, wire, nesterov, flags, lr, decay, rms, x0):
    """One step from a momentum of noise; x' against the definition, from the momentum that the step leaves."""
    off = np.cumsum([0] + [-(-r * c // 8) * 8 for r, c in shapes])
    P = int(off[-1])
    flat, m0 = torch.zeros(P, device=DEV), torch.zeros(P, device=DEV)
    for k, ((r, c), o) in enumerate(zip(shapes, off)):
        flat[o:o + r * c] = torch.from_numpy(N.noise(r, c, seed=2 * k).reshape(-1))
        m0[o:o + r * c] = torch.from_numpy(N.noise(r, c, seed=2 * k + 1).reshape(-1))
    grad, scales, codec, values = message(flat, wire)
    x = torch.randn(P, generator=torch.Generator(device=DEV).manual_seed(P), device=DEV) * x0
    before, m = x.double().cpu().numpy(), m0.clone()
    cfg = D.muon_cfg(lr=lr, momentum=0.9, weight_decay=decay, rms=rms, nesterov=nesterov)
    call = D.MuonCall(x, m, grad, off, shapes, flags, cfg, codec, scales)
    n = launches(call)
    mu, lr, decay, rms = (float(np.float32(v)) for v in (0.9, lr, decay, rms))
    x, m, g = (v.double().cpu().numpy() for v in (x, m, values))
    assert np.abs(m - (mu * m0.double().cpu().numpy() + g)).max() <= 2.0 ** -24 * np.abs(m).max() * 2
    for (r, c), o, f in zip(shapes, off, flags):
        p = slice(o, o + r * c)
        u = (mu * m[p] + g[p] if nesterov else m[p]).reshape(r, c)
        rate = lr * (rms * np.sqrt(max(r, c)) if f & 2 else 1.0)
        step = rate * N.formula(u).reshape(-1)
        want = (1 - lr * decay if f & 1 else 1.0) * before[p] - step
        # two roundings of x', of its factor 1 - lr lambda and of the rate
        room = N.TIGHT * np.linalg.norm(step) + 2.0 ** -22 * np.linalg.norm(np.abs(before[p]) + np.abs(step))
        got = np.linalg.norm(x[p] - want)
        print((r, c), f"error {got / np.linalg.norm(step):.2g} of the step")
        assert got <= room, ((r, c), got, room)
    for (r, c), o, e in zip(shapes, off, off[1:]):  # between the tensors
        assert np.array_equal(x[o + r * c:e], before[o + r * c:e]) and not m[o + r * c:e].any()
    return n


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("wire", ["f32", "fp16", "i8"])
@pytest.mark.parametrize("path", N.LISTS)
def test_muon_update_alone(path, wire, nesterov):
    """x = 0, no decay, a rate of 1: x' is the update."""
    shapes = N.LISTS[path]
    check_path(path, muon(shapes, wire, nesterov, [0] * len(shapes), 1.0, 0.0, 0.2, 0.0), join=path == "cut")


@pytest.mark.parametrize("first", [0, 1])
@pytest.mark.parametrize("wire", ["f32", "i8"])
@pytest.mark.parametrize("path", N.LISTS)
def test_muon_step_of_parameters(path, wire, first):
    """Decay and the adapted rate by turns: the flag's bit lies beside a narrow matrix' turns (up to 4, of 64 x 4096)."""
    shapes = N.LISTS[path]
    flags = [(3, 1, 2, 0)[(k + first) % 4] for k in range(len(shapes))]
    check_path(path, muon(shapes, wire, True, flags, 0.05, 0.3, 0.2, 0.02))


def many(kind):
    """More products than the 72 that a table holds."""
    rng = np.random.default_rng(3)
    side = lambda lo, hi: int(rng.integers(lo, hi))  # noqa: E731
    if kind == "narrow":
        return [(side(1, 129), side(1, 400)) for _ in range(160)]
    if kind == "products":
        return [(side(129, 200), side(129, 260)) for _ in range(80)]
    # two products each of the matrices in blocks: the table is full in the middle of them
    return [(side(1, 129), side(1, 300)) if k % 3 == 0 else (300, 1100 + k) if k % 2 else (1190 - k, 310) for k in range(60)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["narrow", "products", "blocks"])
def test_orthogonalize_more_than_a_table_holds(kind, dtype):
    """Batch after batch on the same workspace, whose contents are arbitrary; into other matrices with gaps, and in place."""
    shapes = many(kind)
    g = inputs(shapes, dtype, pad=5)
    bufs = [torch.full((r, c + 2), 7.0, dtype=dtype, device=DEV) for r, c in shapes]
    out = [b[:, :c] for b, (_, c) in zip(bufs, shapes)]
    call = D.OrthogonalizeCall(g, out)
    call.ws.fill_(255)
    n = launches(call)
    batches = {"narrow": 3, "products": 2, "blocks": 2}[kind]
    assert n["ns_sum"] == n["ns_prepare"] == batches, n
    for o, v, b in zip(out, g, bufs):
        near(o, v)
        assert bool((b[:, -2:] == 7.0).all())
    D.OrthogonalizeCall(g)()
    for o, v in zip(out, g):
        assert torch.equal(o, v)


@pytest.mark.parametrize("kind", ["narrow", "products", "blocks"])
def test_muon_more_than_a_table_holds(kind):
    shapes = many(kind)
    n = muon(shapes, "fp16", True, [(3, 0, 1)[k % 3] for k in range(len(shapes))], 0.05, 0.3, 0.2, 0.02)
    assert n["muon_sum"] == n["ns_prepare"] == {"narrow": 3, "products": 2, "blocks": 2}[kind], n
