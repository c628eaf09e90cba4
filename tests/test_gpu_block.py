"""dedloc_dropout, dedloc_norm, dedloc_residual and their gradients against
their definitions in 64 bits (tests/block_ref.py, which also derives the bounds):
sizes from one element to rows of 16384, types, strides, gates, masks, infinities and NaN,
streams and graphs."""

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D
from . import block_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
PAIRS = [(F32, F32), (F32, F16), (F32, BF16), (F16, F16), (BF16, BF16)]
KINDS = {"layer": D.DEDLOC_NORM_LAYER, "rms": D.DEDLOC_NORM_RMS}
EPS = {"layer": 1e-12, "rms": 1e-6}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows(n, width, dtype, g, pad=0, offset=0, std=1.0, mean=0.0, fill=float("nan")):
    """n rows of width, `pad` apart, `offset` elements into a buffer whose gaps hold `fill`; (rows, buffer)."""
    buf = torch.full((n * (width + pad) + offset + 1,), fill, dtype=dtype, device=DEV)
    v = buf[offset:offset + n * (width + pad)].view(n, width + pad)[:, :width]
    v.copy_(torch.randn(n, width, generator=g, device=DEV) * std + mean)
    return v, buf


def gaps_hold(v, buf, fill):
    """Whether nothing but v's elements of its buffer was written."""
    mark = torch.zeros_like(buf, dtype=torch.bool)
    mark.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(True)
    return bool((buf[~mark] == fill).all())


def vector(width, g, mean, std=0.3):
    return torch.randn(width, generator=g, device=DEV) * std + mean


def make_norm(kind, width, g, gain=True, bias=True):
    """(the call's cfg, the reference's)"""
    if kind is None:
        return None, None
    a, b = vector(width, g, 1.0) if gain else None, vector(width, g, 0.0) if bias else None
    return D.norm_cfg(KINDS[kind], a, b, EPS[kind]), R.N(kind, EPS[kind], a, b)


def check(got, want, bound, dtype, what):
    """|got - want| within bound and got's rounding to dtype."""
    got = got.detach().double().cpu()
    bad = (got - want).abs() > bound + R.half_step(want, dtype) * 1.01
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got - want).abs() / (bound + R.half_step(want, dtype))).max()))


# ------------------------------------------------------------------- dropout

def dropped(x, p, **cfg):
    """By the reference, bit for bit: one fp32 product, one rounding."""
    keep, factor = R.kept(x.shape[0], x.shape[1], p, **cfg)
    y = x.float().cpu() * torch.tensor(factor)
    return torch.where(torch.from_numpy(keep), y, 0.0).to(x.dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,width,pad,offset,p", [(1, 1, 0, 0, 0.5), (3, 7, 0, 1, 0.5), (1, 8, 0, 0, 0.9), (65, 9, 3, 1, 0.1),
                                                  (257, 64, 0, 0, 0.1), (31, 333, 5, 3, 0.25), (5, 16383, 1, 0, 0.3),
                                                  (2, 16385, 1, 1, 0.3), (3, 40001, 0, 0, 0.7), (1000, 128, 0, 0, 1e-4), (37, 2049, 0, 0, 0.2), (19, 4098, 1, 0, 0.2), (1, 1, 0, 0, 0.25)])
def test_dropout(dtype, n, width, pad, offset, p):
    g = gen(n + width)
    x, _ = rows(n, width, dtype, g, pad, offset)
    out, buf = rows(n, width, dtype, g, pad + 1, offset, fill=7.0)
    cfg = dict(seed=0xFEDCBA9876543210 + n, site=n, step=width)
    D.dedloc_dropout(x, D.dropout_cfg(p, **cfg), out=out)
    assert torch.equal(out.cpu(), dropped(x, p, **cfg)) and gaps_hold(out, buf, 7.0)
    D.dedloc_dropout(x, D.dropout_cfg(p, **cfg), out=x)  # in place
    assert torch.equal(x, out)


def test_dropout_ends():
    x, _ = rows(50, 70, F32, gen(1))
    x[3, 5], x[4, 6], x[5] = float("inf"), float("nan"), float("-inf")
    assert torch.equal(D.dedloc_dropout(x, D.dropout_cfg(0.0, 1)).nan_to_num(9), x.nan_to_num(9))
    assert bool((D.dedloc_dropout(x, D.dropout_cfg(1.0, 1)) == 0).all())
    assert bool((D.dedloc_dropout(x, D.dropout_cfg(1e-6, 1)).nan_to_num(9) == x.nan_to_num(9)).all())  # less than half of 2^-16: none
    y = D.dedloc_dropout(x, D.dropout_cfg(0.999999, 1)).cpu()  # at most 65535 of 65536
    assert torch.equal(y.nan_to_num(9), dropped(x, 0.999999, seed=1).nan_to_num(9))
    y = D.dedloc_dropout(x, D.dropout_cfg(0.5, 2)).cpu()
    keep, _ = R.kept(50, 70, 0.5, seed=2)
    assert torch.equal(torch.isfinite(y), torch.isfinite(x.cpu()) | torch.from_numpy(~keep))
    for n, w in ((0, 8), (3, 0)):
        e = torch.empty(n, w, device=DEV)
        assert D.dedloc_dropout(e, D.dropout_cfg(0.5)).shape == (n, w)


def test_dropout_of_parts():
    """Rows of a larger matrix, named by row0; sites, steps and seeds that wrap."""
    x, _ = rows(300, 100, BF16, gen(2))
    cfg = dict(seed=(1 << 64) - 1, site=(1 << 32) - 1, step=(1 << 32) - 2)
    whole = D.dedloc_dropout(x, D.dropout_cfg(0.3, **cfg))
    assert torch.equal(whole.cpu(), dropped(x, 0.3, **cfg))
    part = D.dedloc_dropout(x[100:250], D.dropout_cfg(0.3, row0=100, **cfg))
    assert torch.equal(part, whole[100:250])
    at = torch.tensor([7 + (1 << 40)], device=DEV)  # only the low half counts
    got = D.dedloc_dropout(x, D.dropout_cfg(0.3, step_at=at, **cfg))
    assert torch.equal(got.cpu(), dropped(x, 0.3, **{**cfg, "step": 5}))


def test_dropout_many_rows():
    """Rows of three columns, and masks that have nothing in common."""
    n = 3_000_001
    x = torch.ones(n, 3, device=DEV, dtype=F16)
    y = D.dedloc_dropout(x, D.dropout_cfg(0.5, 3)).cpu()
    assert torch.equal(y[-1000:], dropped(x[-1000:], 0.5, seed=3, row0=n - 1000))
    assert torch.equal(y[:1000], dropped(x[:1000], 0.5, seed=3))
    z = D.dedloc_dropout(x, D.dropout_cfg(0.5, 3, site=1)).cpu()
    both = float(((y != 0) & (z != 0)).float().mean())
    assert abs(both - 0.25) < 5 * (0.1875 / (3 * n)) ** 0.5


# --------------------------------------------------------------------- norms

SIZES = [(1, 1, 0, 0), (3, 7, 0, 1), (9, 64, 0, 0), (33, 65, 1, 0), (50, 128, 0, 0), (17, 200, 3, 1), (9, 256, 0, 0), (70, 333, 5, 3),
         (5, 512, 0, 0), (6, 513, 1, 0), (7, 1024, 0, 0), (3, 1500, 0, 2), (5, 2048, 0, 0), (3, 4001, 0, 1), (2, 8192, 0, 0),
         (3, 8193, 0, 0), (2, 16384, 0, 0), (1, 16000, 7, 1),
         (5, 768, 0, 0), (3, 2560, 0, 0), (2, 6144, 0, 0), (2, 12000, 0, 0)]


@pytest.mark.parametrize("n,width,pad,offset", SIZES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("types", PAIRS)
def test_norm_and_gradient(types, kind, n, width, pad, offset):
    stream, branch = types
    g = gen(n * width)
    x, _ = rows(n, width, stream, g, pad, offset, 1.5, 0.4)
    out, buf = rows(n, width, branch, g, pad + 1, offset, fill=7.0)
    cfg, ref = make_norm(kind, width, g, gain=n != 9, bias=n % 2 == 1)
    got, stats = D.dedloc_norm(x, cfg, out=out)
    want, bound, mean, rstd, dm, dr = R.norm(R.f64(x), ref)
    assert got is out and stats.shape == (1, n, 2) and gaps_hold(out, buf, 7.0)
    check(out, want, bound, branch, "out")
    check(stats[0, :, :1], mean, dm, F32, "mean")
    check(stats[0, :, 1:], rstd, dr, F32, "rstd")
    # the gradient takes the statistics as they are
    dout, _ = rows(n, width, branch, g, pad, offset, 0.1)
    add = rows(n, width, stream, g, pad + 2, offset, 0.1)[0] if n % 3 else None
    dx, buf = rows(n, width, stream, g, pad + 1, offset, fill=7.0)
    dgain, dbias = (vector(width, g, 0.0, 1.0) if v is not None else None for v in (ref.gain, ref.bias))
    before = [R.f64(v) for v in (dgain, dbias)]
    ws = D.make_residual_workspace(n, width)
    ws.fill_(255)
    D.dedloc_norm_grad(dout, x, stats, cfg, dgain, dbias, 12.0, add, dx, ws)
    st = R.f64(stats[0])
    d, e, *sums = R.norm_back(R.f64(dout), torch.zeros(n, width, dtype=torch.float64), R.f64(x), st[:, :1], st[:, 1:], ref)
    if add is not None:
        d = d + R.f64(add)
    check(dx, d, e + R.U * d.abs(), stream, "dx")
    assert gaps_hold(dx, buf, 7.0)
    for k, acc in enumerate((dgain, dbias)):
        if acc is not None:
            check(acc, *R.columns(before[k], 12.0, *sums[2 * k:2 * k + 2]), F32, "dgain dbias".split()[k])


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("n,width", [(4000, 8), (5001, 64), (3001, 100), (9000, 256), (4097, 333), (9001, 512), (5000, 1000),
                                     (2500, 2000), (1500, 4096), (700, 8000), (300, 16384)])
def test_norm_grad_of_many_rows(kind, n, width):
    """Rows enough for every workgroup to take several."""
    g = gen(n)
    x, dout = (rows(n, width, BF16, g)[0] for _ in range(2))
    cfg, ref = make_norm(kind, width, g)
    _, stats = D.dedloc_norm(x, cfg)
    dgain, dbias = torch.zeros(2, width, device=DEV)
    dx = D.dedloc_norm_grad(dout, x, stats, cfg, dgain, dbias, 3.0)
    st = R.f64(stats[0])
    d, e, *sums = R.norm_back(R.f64(dout), torch.zeros(n, width, dtype=torch.float64), R.f64(x), st[:, :1], st[:, 1:], ref)
    check(dx, d, e, BF16, "dx")
    check(dgain, *R.columns(None, 3.0, *sums[:2]), F32, "dgain")
    check(dbias, *R.columns(None, 3.0, *sums[2:]), F32, "dbias")
    again = torch.zeros(2, width, device=DEV)
    dx2 = D.dedloc_norm_grad(dout, x, stats, cfg, again[0], again[1], 3.0)
    assert torch.equal(dx2, dx) and torch.equal(again[0], dgain) and torch.equal(again[1], dbias)  # equal calls, equal bits


@pytest.mark.parametrize("width", [5, 64, 100, 300, 1000, 4000, 9000])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_of_odd_rows(kind, width):
    """Zeros, equal entries, entries near the ends of fp32, infinities and NaN: each row by itself."""
    x = torch.randn(9, width, generator=gen(3), device=DEV)
    x[1], x[2], x[3] = 0.0, 2.5, x[3] * 1e30
    x[4] = torch.where(x[4] > 0, 1e37, -1e37)
    x[5] = x[5] * 1e-30
    x[6, width // 2], x[7, 0] = float("inf"), float("nan")
    cfg, ref = make_norm(kind, width, gen(4))
    out, stats = D.dedloc_norm(x, cfg)
    fine = [0, 1, 2, 3, 4, 5, 8]
    want, bound, mean, rstd, dm, dr = R.norm(R.f64(x[fine]), ref)
    check(out[fine], want, bound, F32, "out")
    check(stats[0, fine, 1:], rstd, dr, F32, "rstd")
    assert bool(torch.isnan(out[7]).all()) and bool(torch.isnan(out[6, width // 2]))
    one = D.dedloc_norm(x[:1].contiguous(), cfg, keep_stats=False)
    assert one[1] is None and torch.equal(one[0], out[:1])  # a row does not depend on the others


def test_norm_in_place_and_empty():
    x, _ = rows(20, 300, BF16, gen(5))
    cfg, _ = make_norm("layer", 300, gen(6))
    want, stats = D.dedloc_norm(x, cfg)
    y = x.clone()
    D.dedloc_norm(y, cfg, out=y)
    assert torch.equal(y, want)
    dout, _ = rows(20, 300, BF16, gen(7))
    dx = D.dedloc_norm_grad(dout, x, stats, cfg, add=x)
    a, b = dout.clone(), x.clone()
    D.dedloc_norm_grad(a, x, stats, cfg, add=x, dx=a)
    D.dedloc_norm_grad(dout, x, stats, cfg, add=b, dx=b)
    assert torch.equal(a, dx) and torch.equal(b, dx)
    acc = torch.ones(300, device=DEV)
    e = torch.empty(0, 300, device=DEV, dtype=BF16)
    assert D.dedloc_norm(e, cfg)[0].shape == (0, 300)
    D.dedloc_norm_grad(e, e, torch.empty(1, 0, 2, device=DEV), cfg, acc, None)
    assert bool((acc == 1).all())


# ------------------------------------------------------------- ends of a block

def block(n, width, stream, branch, post, pre, gate, p, seed, pad=0, offset=0, gate_rows=0, both=True, alpha=1.25, beta=0.75, gain=True,
          bias=True):
    """One forward and backward call against the reference."""
    g = gen(seed)
    h, _ = rows(n, width, stream, g, pad, offset, 1.5, 0.3)
    f, _ = rows(n, width, branch, g, pad + 3, offset, 0.5)
    (post_c, post_r), (pre_c, pre_r) = make_norm(post, width, g, gain, bias), make_norm(pre, width, g, gain, bias)
    gate_t = None
    if gate == "channel":
        gate_t = vector(width, g, 0.5)
    elif gate == "group":
        gate_t = rows(-(-n // gate_rows), width, branch, g, pad, offset, 0.3, 0.7)[0]
    draw = dict(seed=seed * 77 + 5, site=3, step=n)
    drop = D.dropout_cfg(p, **draw) if p is not None else None
    mask = R.kept(n, width, p, **draw) if p is not None else None
    total, sbuf = rows(n, width, stream, g, pad + 1, offset, fill=7.0)
    out, obuf = rows(n, width, branch, g, pad + 2, offset, fill=7.0)
    if pre is None:
        out = None
    common = dict(alpha=alpha, beta=beta, post=post_c, pre=pre_c, gate=gate_t, gate_rows=gate_rows, drop=drop)
    stats = torch.full((2, n, 2), 7.0, device=DEV)
    D.dedloc_residual(h, f, sum=total, out=out, stats=stats, **common)
    h6, f6 = R.f64(h), R.f64(f)
    want, bound, st = R.residual_sum(h6, f6, alpha, beta, post_r, gate_t, gate_rows, mask)
    check(total, want, bound, stream, "sum")
    assert gaps_hold(total, sbuf, 7.0)
    if post:
        check(stats[1, :, :1], st[0], st[2], F32, "post mean")
        check(stats[1, :, 1:], st[1], st[3], F32, "post rstd")
    else:
        assert bool((stats[1] == 7).all())
    if pre:
        want, bound, mean, rstd, dm, dr = R.norm(R.f64(total), pre_r)
        check(out, want, bound, branch, "out")
        check(stats[0, :, :1], mean, dm, F32, "pre mean")
        check(stats[0, :, 1:], rstd, dr, F32, "pre rstd")
        assert gaps_hold(out, obuf, 7.0)
        # for its output alone
        alone = D.dedloc_residual(h, f, keep=False, **common)
        assert alone[0] is None and alone[2] is None and torch.equal(alone[1], out)
    else:
        assert bool((stats[0] == 7).all())

    dsum = rows(n, width, stream, g, pad + 2, offset, 0.1)[0] if both or pre is None else None
    dout = rows(n, width, branch, g, pad, offset, 0.1)[0] if pre else None
    dh, hbuf = rows(n, width, stream, g, pad + 1, offset, fill=7.0)
    df, fbuf = rows(n, width, branch, g, pad + 2, offset, fill=7.0)
    accs = {k: vector(width, g, 0.0, 1.0) if use else None
            for k, use in (("dpre_gain", pre and gain), ("dpre_bias", pre and bias), ("dpost_gain", post and gain), ("dpost_bias", post and bias))}
    dgate = dbuf = None
    if gate == "channel":
        dgate = vector(width, g, 0.0, 1.0)
    elif gate == "group":
        dgate, dbuf = rows(gate_t.shape[0], width, F32, g, pad + 1, fill=7.0)
    before = {k: R.f64(v) for k, v in list(accs.items()) + [("dgate", dgate)]}
    ws = D.make_residual_workspace(n, width, gate_rows)
    ws.fill_(255)
    args = dict(common, dgate=dgate, dpre=(accs["dpre_gain"], accs["dpre_bias"]), dpost=(accs["dpost_gain"], accs["dpost_bias"]),
                batch_samples=12.0, ws=ws)
    D.dedloc_residual_grad(total, f, stats, dsum, dout, dh=dh, df=df, **args)
    ref = R.residual_grad(R.f64(total), f6, R.f64(stats), R.f64(dsum), R.f64(dout), alpha, beta, post_r, pre_r, gate_t, gate_rows, mask)
    check(dh, *ref["dh"], stream, "dh")
    check(df, *ref["df"], branch, "df")
    assert gaps_hold(dh, hbuf, 7.0) and gaps_hold(df, fbuf, 7.0)
    for k, acc in accs.items():
        if acc is not None:
            check(acc, *R.columns(before[k], 12.0, *ref[k]), F32, k)
    if gate == "channel":
        check(dgate, *R.columns(before["dgate"], 12.0, *ref["dgate"]), F32, "dgate")
    elif gate == "group":
        for k in range(gate_t.shape[0]):
            part = [t[k * gate_rows:(k + 1) * gate_rows] for t in ref["dgate"]]
            check(dgate[k], *R.columns(None, 1.0, *part), F32, f"dgate {k}")
        assert gaps_hold(dgate, dbuf, 7.0)
    # equal calls, equal bits; and in place
    dh2, df2 = dsum.clone() if dsum is not None else torch.empty_like(dh), f.clone()
    if gate == "group":
        first = dgate.clone()
    D.dedloc_residual_grad(total, df2, stats, dh2 if dsum is not None else None, dout, dh=dh2, df=df2, **args)
    assert torch.equal(dh2, dh) and torch.equal(df2, df)
    if gate == "group":
        assert torch.equal(first, dgate)
    h2, f2 = h.clone(), f.clone()
    D.dedloc_residual(h2, f2, sum=h2, out=f2 if pre else None, stats=torch.empty_like(stats), **common)
    assert torch.equal(h2, total) and (not pre or torch.equal(f2, out))


NORMS = [(None, "layer"), (None, "rms"), ("layer", "layer"), ("rms", "rms"), ("layer", None), (None, None), ("rms", "layer")]


@pytest.mark.parametrize("gate", [None, "channel", "group"])
@pytest.mark.parametrize("post,pre", NORMS)
@pytest.mark.parametrize("n,width,pad,offset", [(1, 1, 0, 0), (13, 64, 0, 0), (29, 100, 3, 1), (37, 333, 5, 3), (11, 1000, 0, 0), (6, 4100, 0, 0)])
def test_residual(n, width, pad, offset, post, pre, gate):
    k = NORMS.index((post, pre)) + n
    stream, branch = PAIRS[k % 5]
    block(n, width, stream, branch, post, pre, gate, [None, 0.1, 0.5][k % 3], seed=n, pad=pad, offset=offset, gate_rows=max(1, n // 3) if gate == "group" else 0,
          both=k % 2 == 0)


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("n,width,pad,offset", SIZES)
def test_residual_of_every_width(types, n, width, pad, offset):
    block(n, width, *types, "layer", "layer", "channel", 0.2, seed=n + width, pad=pad, offset=offset, both=n % 2 == 0)


@pytest.mark.parametrize("gate_rows", [1, 2, 7, 64, 501, 5000])
@pytest.mark.parametrize("n,width", [(1500, 40), (1001, 128), (700, 257), (2000, 700), (600, 2500)])
def test_residual_gates_of_groups(n, width, gate_rows):
    """Groups shorter and longer than a team's rows, that its range cuts or holds."""
    block(n, width, BF16, BF16, "rms", "layer", "group", 0.1, seed=n, gate_rows=gate_rows)


@pytest.mark.parametrize("gain,bias", [(False, False), (True, False), (False, True)])
def test_residual_without_vectors(gain, bias):
    block(70, 300, F32, BF16, "layer", "rms", "channel", 0.3, seed=9, gain=gain, bias=bias)
    block(70, 100, F16, F16, "rms", "layer", "group", None, seed=9, gate_rows=9, gain=gain, bias=bias)


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("n,width", [(1, 1), (20, 5), (33, 100), (21, 300), (17, 333), (9, 768), (7, 1000), (5, 2500), (3, 6100), (2, 12001)])
def test_residual_of_bare_norms(types, n, width):
    """Norms without a gain and no gate: nothing makes what the threads behind the row's end hold zero but themselves."""
    for post, pre in (("layer", "layer"), ("layer", "rms"), ("rms", "layer")):
        block(n, width, *types, post, pre, None, 0.2, seed=n, gain=False, bias=False)
        block(n, width, *types, post, pre, None, None, seed=n, gain=False, bias=True)


@pytest.mark.parametrize("gate", ["channel", "group", None])
@pytest.mark.parametrize("post,pre", [("layer", "rms"), (None, "layer"), ("rms", None), (None, None)])
def test_gradients_that_are_not_wanted(post, pre, gate):
    """Any of the vectors' gradients left out leaves the others as they are (other sums and shapes of the rows: a few roundings of sums
    of at most 300 terms, 600 U of the largest value), and untouched what is not named."""
    n, width, g = 300, 520, gen(51)
    total, f, dsum, dout = (rows(n, width, F32, g)[0] for _ in range(4))
    (post_c, post_r), (pre_c, pre_r) = make_norm(post, width, g), make_norm(pre, width, g)
    gate_t = vector(width, g, 0.5) if gate == "channel" else rows(6, width, F32, g)[0].contiguous() if gate else None
    st = torch.zeros(2, n, 2, device=DEV)
    for k, (x, r) in enumerate(((total, pre_r), (f, post_r))):
        if r is not None:
            st[k] = torch.cat(R.stats(R.f64(x), r)[:2], 1).float()
    common = dict(alpha=1.0, beta=0.5, post=post_c, pre=pre_c, gate=gate_t, gate_rows=50 if gate == "group" else 0, drop=D.dropout_cfg(0.2, 8))
    names = (["dgate"] if gate else []) + (["pre gain", "pre bias"] if pre else []) + (["post gain", "post bias"] if post else [])

    def run(wanted):
        accs = {k: torch.zeros_like(gate_t) if k == "dgate" else torch.zeros(width, device=DEV) for k in wanted}
        get = accs.get
        dh, df = D.dedloc_residual_grad(total if pre else None, f, st, dsum, dout if pre else None, dgate=get("dgate"),
                                        dpre=(get("pre gain"), get("pre bias")), dpost=(get("post gain"), get("post bias")), **common)
        return dict(accs, dh=dh, df=df)

    every = run(names)
    for wanted in [[]] + [[k] for k in names] + [[k for k in names if k != out] for out in names]:
        got = run(wanted)
        for k, v in got.items():
            assert float((v - every[k]).abs().max()) <= 600 * R.U * float(every[k].abs().max()), (wanted, k)
        assert all(float(got[k].abs().max()) > 0 for k in wanted)


def test_residual_ends_of_p():
    block(20, 100, F32, F32, None, "layer", None, 1.0, seed=1)
    block(20, 100, F32, F32, None, "layer", None, 0.0, seed=1)


def test_dropped_infinities_stay_out():
    """An infinity or NaN of the branch passes only where it is kept, forward and backward."""
    n, width = 40, 200
    g = gen(8)
    h, f = (rows(n, width, F32, g)[0] for _ in range(2))
    keep, _ = R.kept(n, width, 0.5, seed=1)
    f[torch.from_numpy(~keep).to(DEV)] = float("inf")
    total, out, stats = D.dedloc_residual(h, f, pre=D.norm_cfg(D.DEDLOC_NORM_LAYER), drop=D.dropout_cfg(0.5, 1))
    assert bool(torch.isfinite(total).all()) and bool(torch.isfinite(out).all())
    d, _ = rows(n, width, F32, g)
    d[torch.from_numpy(~keep).to(DEV)] = float("nan")
    dh, df = D.dedloc_residual_grad(None, None, None, d, None, drop=D.dropout_cfg(0.5, 1))
    assert torch.equal(torch.isnan(dh).cpu(), torch.from_numpy(~keep)) and bool(torch.isfinite(df).all())


@pytest.mark.parametrize("post,pre,gate", [("layer", "layer", "channel"), ("rms", "rms", "group"), (None, "layer", None)])
def test_gradients_against_differences(post, pre, gate):
    """Central differences of the reference's forward form in 64 bits along random directions, of step 1e-5: off by at most 1e-8 of
    the terms' magnitudes (1e-10 of the third derivative, 1e-11 of rounding), beside the call's own fp32."""
    n, width, gate_rows, p = 12, 40, 5, 0.3
    g = gen(11)
    h, f, dsum, dout = (rows(n, width, F32, g)[0] for _ in range(4))
    (post_c, post_r), (pre_c, pre_r) = make_norm(post, width, g), make_norm(pre, width, g)
    gate_t = vector(width, g, 0.5) if gate == "channel" else rows(3, width, F32, g)[0].contiguous() if gate else None
    rows_of = gate_rows if gate == "group" else 0
    common = dict(alpha=1.25, beta=0.75, post=post_c, pre=pre_c, gate=gate_t, gate_rows=rows_of, drop=D.dropout_cfg(p, 4))
    total, out, stats = D.dedloc_residual(h, f, **common)
    grads = {k: torch.zeros(width, device=DEV) for k in ("pg", "pb", "qg", "qb")}
    dgate = torch.zeros_like(gate_t) if gate else None
    dh, df = D.dedloc_residual_grad(total, f, stats, dsum, dout, dgate=dgate, dpre=(grads["pg"], grads["pb"]),
                                    dpost=(grads["qg"], grads["qb"]) if post else None, **common)
    mask = R.kept(n, width, p, seed=4)
    leaves = dict(h=R.f64(h), f=R.f64(f), pg=R.f64(pre_r.gain), pb=R.f64(pre_r.bias))
    got = dict(h=dh, f=df, pg=grads["pg"], pb=grads["pb"])
    if post:
        leaves.update(qg=R.f64(post_r.gain), qb=R.f64(post_r.bias))
        got.update(qg=grads["qg"], qb=grads["qb"])
    if gate:
        leaves["gate"] = R.f64(gate_t)
        got["gate"] = dgate

    def loss(v):
        q = R.N(post, EPS[post], v["qg"], v["qb"]) if post else None
        s, _, _ = R.residual_sum(v["h"], v["f"], 1.25, 0.75, q, v.get("gate"), rows_of, mask)
        y = R.norm(s, R.N(pre, EPS[pre], v["pg"], v["pb"]))[0]
        return float((s * R.f64(dsum)).sum() + (y * R.f64(dout)).sum())

    for name in leaves:
        d = torch.randn(leaves[name].shape, dtype=torch.float64, generator=torch.Generator().manual_seed(5))
        step = 1e-5
        slope = (loss({**leaves, name: leaves[name] + step * d}) - loss({**leaves, name: leaves[name] - step * d})) / (2 * step)
        mine = float((R.f64(got[name]) * d).sum())
        size = float((R.f64(got[name]).abs() * d.abs()).sum())
        assert abs(mine - slope) <= (1e-7 + 200 * R.U) * (size + float(R.f64(dout).abs().sum()) / width), name


@pytest.mark.parametrize("width", [512, 1000, 4096, 5120])
@pytest.mark.parametrize("post,pre,gate", [("layer", "rms", "channel"), (None, "layer", None), ("rms", "layer", "group")])
@pytest.mark.parametrize("types", PAIRS)
def test_large_calls_are_their_parts(types, post, pre, gate, width):
    """A call that reads past the caches (96 MiB and more) gives the bits of calls on a few rows; the sums over its rows are those
    of the definition with dout = dsum = 1, in 64 bits of the rows' own values."""
    stream, branch = types
    n, g = (100 << 20) // (2 * width) // 64 * 64 + 24, gen(width)
    h, f = (rows(n, width, t, g)[0] for t in types)
    (post_c, post_r), (pre_c, pre_r) = make_norm(post, width, g), make_norm(pre, width, g)
    gate_rows = 64 if gate == "group" else 0
    gate_t = vector(width, g, 0.5) if gate == "channel" else rows(-(-n // 64), width, branch, g)[0].contiguous() if gate else None
    common = lambda a: dict(alpha=1.0, beta=0.5, post=post_c, pre=pre_c, gate_rows=gate_rows, drop=D.dropout_cfg(0.1, 3, row0=a),  # noqa: E731
                            gate=gate_t[a // 64:a // 64 + 2] if gate_rows and a else gate_t)
    total, out, stats = D.dedloc_residual(h, f, **common(0))
    ones = torch.ones(n, width, dtype=branch, device=DEV)
    dpre = torch.zeros(2, width, device=DEV)
    dh, df = D.dedloc_residual_grad(total, f, stats, None, ones, dpre=(dpre[0], dpre[1]), **common(0))
    for a in (n // 2 // 64 * 64, n - 88):  # at a group of rows
        b = min(a + 88, n)
        t, o, st = D.dedloc_residual(h[a:b], f[a:b], **common(a))
        assert torch.equal(t, total[a:b]) and torch.equal(o, out[a:b]) and torch.equal(st[0], stats[0, a:b])
        x, y = D.dedloc_residual_grad(t, f[a:b], st, None, ones[a:b], **common(a))
        assert torch.equal(x, dh[a:b]) and torch.equal(y, df[a:b])
    assert bool((dpre[1] == n).all())
    xhat = (total.double() - stats[0, :, :1].double()) * stats[0, :, 1:].double()
    want, size = xhat.sum(0).cpu(), xhat.abs().sum(0).cpu()
    check(dpre[0], want, (n + 6) * R.U * size, F32, "dgain")


def test_offsets_past_32_bits():
    """Matrices of more than 2^32 elements, in place: their last rows against the definitions, and the sums over all rows."""
    n, width = 66000, 65600
    x = torch.ones(n, width, dtype=BF16, device=DEV)
    D.dedloc_dropout(x, D.dropout_cfg(0.25, 9), out=x)
    assert torch.equal(x[-3:].cpu(), dropped(torch.ones(3, width, dtype=BF16, device=DEV), 0.25, seed=9, row0=n - 3))
    del x
    n, width = 270000, 16000
    part, _ = rows(9, width, BF16, gen(41))
    x = part.repeat(n // 9, 1)
    cfg, ref = make_norm("layer", width, gen(42))
    drop = D.dropout_cfg(0.25, 9)
    total, _, stats = D.dedloc_residual(x, x, pre=cfg, drop=drop, out=torch.empty_like(x))
    keep = R.kept(9, width, 0.25, seed=9, row0=n - 9)
    want, bound, _ = R.residual_sum(R.f64(part), R.f64(part), 1.0, 1.0, None, None, 0, keep)
    check(total[-9:], want, bound, BF16, "sum")
    dgain, dbias = torch.zeros(2, width, device=DEV)
    # every nine rows' gradient of the bias is the same: whole numbers, exact in any order below 2^24
    ones = torch.ones(n, width, dtype=BF16, device=DEV)
    dh, df = D.dedloc_residual_grad(total, None, stats, None, ones, pre=cfg, drop=drop, dpre=(dgain, dbias), dh=ones, df=x)
    assert bool((dbias == n).all()) and dh is ones
    d, e, *_ = R.norm_back(torch.ones(9, width, dtype=torch.float64), torch.zeros(9, width, dtype=torch.float64), R.f64(total[-9:]),
                           R.f64(stats[0, -9:, :1]), R.f64(stats[0, -9:, 1:]), ref)
    check(dh[-9:], d, e, BF16, "dh")
    kept, factor = torch.from_numpy(keep[0]), float(keep[1])
    check(df[-9:], torch.where(kept, d * factor, 0.0), torch.where(kept, e * factor + R.U * (d * factor).abs(), 0.0), BF16, "df")


# --------------------------------------------------------- streams and graphs

def test_captured_calls_draw_anew():
    """A training step's pass, captured: the graph advances the step, every replay draws that step's mask, with eager
    work and synchronisations between the replays."""
    n, width = 300, 500
    g = gen(21)
    h, f, dsum, dout = (rows(n, width, BF16, g)[0] for _ in range(4))
    post, pre = make_norm("rms", width, g)[0], make_norm("layer", width, g)[0]
    gate = vector(width, g, 0.5)
    at = torch.zeros(1, dtype=torch.int64, device=DEV)
    total, out = torch.empty(n, width, dtype=BF16, device=DEV), torch.empty(n, width, dtype=BF16, device=DEV)
    dh, df, x = torch.empty_like(total), torch.empty_like(total), torch.empty_like(total)
    stats, acc = torch.empty(2, n, 2, device=DEV), torch.zeros(4, width, device=DEV)

    def calls(step, step_at, acc, total, out, dh, df, x, stats):
        drop = D.dropout_cfg(0.2, 6, step=step, step_at=step_at)
        block = dict(alpha=1.0, beta=0.5, post=post, pre=pre, gate=gate, drop=drop)
        fwd = D.ResidualCall(h, f, total, out, stats, **block)
        back = D.ResidualGradCall(total, f, stats, dsum, dout, dh, df, dgate=acc[0], dpre=(acc[1], acc[2]), dpost=(acc[3], None),
                                  batch_samples=2.0, **block)
        return lambda: (D.dedloc_dropout(h, drop, out=x), fwd(), back())

    eager = [t.clone() for t in (total, out, dh, df, x)] + [stats.clone()]
    run = calls(0, at, acc, total, out, dh, df, x, stats)
    run()
    torch.cuda.synchronize()
    acc.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
        at.add_(1)
    acc.zero_()
    at.zero_()
    sums = torch.zeros_like(acc)
    for step in range(5):
        graph.replay()
        torch.cuda.synchronize()
        calls(step, None, sums, *eager)()
        torch.cuda.synchronize()
        for got, want in zip((total, out, dh, df, x, stats, acc), (*eager, sums)):
            assert torch.equal(got, want), step
    assert int(at) == 5


def test_two_graphs_of_one_call_keep_their_workspaces():
    n, width = 4000, 256
    g = gen(22)
    x, dout = (rows(n, width, BF16, g)[0] for _ in range(2))
    cfg, _ = make_norm("layer", width, g)
    _, stats = D.dedloc_norm(x, cfg)
    dh, df = torch.empty_like(x), torch.empty_like(x)
    gain, bias = torch.zeros(2, width, device=DEV)
    call = D.ResidualGradCall(x, None, stats, None, dout, dh, df, pre=cfg, dpre=(gain, bias))
    call()
    want = gain.clone()
    graphs, at = [], []
    torch.cuda.synchronize()
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
        at.append(call._ws.captured.data_ptr())
    assert len({call.ws.data_ptr(), *at}) == 3
    gain.zero_()
    graphs.pop(0)
    torch.cuda.empty_cache()
    others = [torch.zeros(1 << 22, dtype=torch.uint8, device=DEV) for _ in range(8)]
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(gain, want) and all(int(o.max()) == 0 for o in others)


def dropout_call(stream):
    x, _ = rows(2000, 333, F32, gen(31))
    return x, lambda: D.dedloc_dropout(x, D.dropout_cfg(0.3, 1), stream=stream)


def norm_call(stream):
    x, _ = rows(2000, 333, F32, gen(32))
    cfg, _ = make_norm("layer", 333, gen(33))
    return (x, cfg), lambda: D.dedloc_norm(x, cfg, stream=stream)[0]


def norm_grad_call(stream):
    x, dout = (rows(2000, 333, F32, gen(34 + k))[0] for k in range(2))
    cfg, _ = make_norm("layer", 333, gen(33))
    _, stats = D.dedloc_norm(x, cfg)
    acc = torch.zeros(333, device=DEV)
    return (x, dout, cfg), lambda: (D.dedloc_norm_grad(dout, x, stats, cfg, acc, stream=stream), acc)[1]


def residual_grad_call(stream):
    x, dout = (rows(2000, 333, F32, gen(36 + k))[0] for k in range(2))
    cfg, _ = make_norm("rms", 333, gen(33))
    total, _, stats = D.dedloc_residual(x, dout, pre=cfg)
    acc = torch.zeros(333, device=DEV)
    return (x, dout, cfg, total), lambda: (D.dedloc_residual_grad(total, None, stats, None, dout, pre=cfg, dpre=(acc, None), stream=stream), acc)[1]


@pytest.mark.parametrize("make", [dropout_call, norm_call, norm_grad_call, residual_grad_call])
def test_waiting_call_keeps_its_memory(make):
    _, call = make(None)
    want = call().clone()
    side = torch.cuda.Stream()
    keep, call = make(side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)  # some 20 milliseconds
    got = call()
    others = [torch.zeros(1 << k, dtype=torch.uint8, device=DEV) for k in range(10, 25) for _ in range(3)]
    torch.cuda.current_stream().synchronize()  # the call still waits here
    side.synchronize()
    assert torch.equal(got, want) and all(int(o.max()) == 0 for o in others)
