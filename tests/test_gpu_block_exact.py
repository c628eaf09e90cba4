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


# ------------------------------------------------------------ norms left out

@pytest.mark.parametrize("gate", [None, "channel", "group"])
@pytest.mark.parametrize("left_out", ["post", "pre"])
def test_what_a_norm_left_out_points_to_is_not_there(left_out, gate):
    """A kind of DEDLOC_NORM_NONE leaves a norm out, whatever else its struct holds: the same bits as with NULL vectors, forward and backward."""
    n, width, g = 300, 520, gen(61)
    h, f, dsum, dout = (rows(n, width, BF16, g)[0] for _ in range(4))
    gate_t = vector(width, g, 0.5) if gate == "channel" else rows(6, width, BF16, g)[0].contiguous() if gate else None
    gain, bias = vector(width, g, 3.0), vector(width, g, -2.0)
    other = make_norm("layer", width, g)[0]
    post, pre = (None, other) if left_out == "post" else (other, None)
    common = dict(alpha=1.0, beta=0.5, post=post, pre=pre, gate=gate_t, gate_rows=50 if gate == "group" else 0, drop=D.dropout_cfg(0.2, 8))

    def run(vectors):
        total, out, stats = torch.empty_like(h), torch.empty_like(h) if pre else None, torch.zeros(2, n, 2, device=DEV)
        dh, df, acc = torch.empty_like(h), torch.empty_like(h), torch.zeros(2, width, device=DEV)
        dgate = torch.zeros_like(gate_t, dtype=F32) if gate else None
        calls = [D.ResidualCall(h, f, total, out, stats, **common),
                 D.ResidualGradCall(total, f, stats, dsum, dout if pre else None, dh, df, dgate=dgate,
                                    **{"dpre" if pre else "dpost": (acc[0], acc[1])}, **common)]
        for call in calls:
            norm = getattr(call.cfg, left_out)
            assert norm.kind == D.DEDLOC_NORM_NONE
            if vectors:
                norm.gain, norm.bias, norm.eps = gain.data_ptr(), bias.data_ptr(), 1e-6
            call()
        return [t for t in (total, out, stats, dh, df, acc, dgate) if t is not None]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))


def test_calls_without_a_norm_by_its_kind():
    """A norm_cfg of DEDLOC_NORM_NONE through the binding is no norm."""
    g = gen(62)
    h, f, dsum = (rows(20, 96, F32, g)[0] for _ in range(3))
    none = D.norm_cfg(D.DEDLOC_NORM_NONE)
    total, out, stats = D.dedloc_residual(h, f, post=none, pre=none)
    assert out is None and stats is None and torch.equal(total, D.dedloc_residual(h, f)[0])
    got = D.dedloc_residual_grad(None, None, None, dsum, None, post=none, pre=none)
    assert all(torch.equal(a, b) for a, b in zip(got, D.dedloc_residual_grad(None, None, None, dsum, None)))


# ------------------------------------------------------ rows of equal entries

@pytest.mark.parametrize("width", [1, 4, 8, 16, 32])
def test_equal_entries_whose_mean_times_rstd_overflows(width):
    """Rows of 2^117, eps 1e-12: the mean is exact, 1e6 times it is none of fp32.  What the threads behind the row's end
    hold stays zero all the same, forward and backward, for the norm before the sum and the one behind it."""
    n, big = 5, 2.0 ** 117
    g = gen(width)
    cfg, _ = make_norm("layer", width, g)
    gain, bias = (v for v in cfg._keep)
    x = torch.full((n, width), big, device=DEV)
    out, stats = D.dedloc_norm(x, cfg)
    assert bool((out == bias).all()) and bool((stats[0, :, 0] == big).all())
    dout, _ = rows(n, width, F32, g)
    acc = torch.zeros(2, width, device=DEV)
    stats[0, :, 1] = 1e6
    dx = D.dedloc_norm_grad(dout, x, stats, cfg, acc[0], acc[1])
    gy = R.f64(dout) * R.f64(gain)
    want = 1e6 * (gy - gy.mean(1, keepdim=True))  # xhat = 0
    assert float((R.f64(dx) - want).abs().max()) <= (R.K + 8) * R.U * float(want.abs().max() + 1e6 * gy.abs().max())
    assert bool((acc[0] == 0).all())
    # the branch's norm, then the sum's
    h, _ = rows(n, width, F32, g)
    total, out, st = D.dedloc_residual(h, x, post=cfg, pre=cfg)
    assert torch.equal(total, h + bias)
    assert bool(torch.isfinite(out).all()) and bool((st[1, :, 0] == big).all())
    st[1, :, 1] = 1e6
    dh, df = D.dedloc_residual_grad(total, x, st, dout, dout, post=cfg, pre=cfg)
    assert bool(torch.isfinite(dh).all()) and bool(torch.isfinite(df).all())


@pytest.mark.parametrize("width", [4, 32, 64, 512, 1024, 8192])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_entries_whose_squares_leave_fp32(dtype, width):
    """Rows of 2^126 have no squares in fp32 and no variance: eps alone makes their deviation, as for smaller entries."""
    x = torch.full((3, width), 2.0 ** 126, device=DEV, dtype=dtype)
    x[1] = -x[1]
    bias = vector(width, gen(1), 0.0)
    out, stats = D.dedloc_norm(x, D.norm_cfg(KINDS["layer"], None, bias, 1e-12))
    assert bool((stats[0, :, 0] == x[:, 0].float()).all())
    want = 1 / float(torch.tensor(1e-12)) ** 0.5
    assert float((stats[0, :, 1].double() - want).abs().max()) <= 4 * R.U * want
    assert torch.equal(out, bias.to(dtype).expand_as(out))


WIDTHS = [1, 5, 32, 48, 100, 300, 333, 520, 768, 1000, 2000, 2560, 4001, 5120, 9000, 12000, 16384]


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("width", WIDTHS)
def test_equal_entries_give_the_bias(types, width):
    """(x - mean) is zero: the mean is the entry, the deviation sqrt(eps), the output the bias, each to its last bit but for rstd's
    (four roundings)."""
    stream, branch = types
    values = [1000.0, 15.9375, -3.140625, 2.5, 3 * 2.0 ** -20, 0.0]
    values += [] if stream is F16 else [3e37, -1e35, 2.0 ** 126, 1e-30]
    values += [1000.1, 1e4 / 3, 1e9 / 7] if stream is F32 else []
    x = torch.tensor(values, device=DEV)[:, None].expand(-1, width).to(stream).contiguous()
    for eps in (1e-12, 1e-5):
        g = gen(width)
        gain, bias = vector(width, g, 1.0), vector(width, g, 0.0)
        out, stats = D.dedloc_norm(x, D.norm_cfg(KINDS["layer"], gain, bias, eps), out_dtype=branch)
        assert torch.equal(stats[0, :, 0], x[:, 0].float())
        want = 1 / float(torch.tensor(eps)) ** 0.5
        assert float((stats[0, :, 1].double() - want).abs().max()) <= 4 * R.U * want
        assert torch.equal(out, bias.to(branch).expand_as(out))


def centred_stats(x, eps):
    """(mean, rstd, bound of the mean, relative bound of rstd) where the sum of what entries differ from a first mean puts that right.

    The first mean is off by at most a = (K + 2) U mean |x|.  The differences from it are exact to U, their mean is off by
    (K + 4) U mean |d| with |d| <= |x - mean| + a; the corrected mean is rounded once.  What squares about the first mean exceed the
    variance by is taken off from the same sums, so they are off by the roundings of sums of d^2 <= 2 (x - mean)^2 + 2 a^2: K + 8 of
    the squares and 4 of what is taken off; waves that differ in their means count theirs once more: twice 2 (K + 12)."""
    mean = x.mean(1, keepdim=True)
    spread, a = (x - mean).abs().mean(1, keepdim=True), (R.K + 2) * R.U * x.abs().mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    dvar = 4 * (R.K + 12) * R.U * (var + a ** 2)
    dm = R.U * mean.abs() + (R.K + 6) * R.U * (spread + a)
    return mean, 1 / (var + eps).sqrt(), R.SLACK * dm, R.SLACK * (dvar / (var + eps) / 2 + 4 * R.U)


@pytest.mark.parametrize("width", WIDTHS[2:])
def test_rows_far_from_zero(width):
    """Rows whose mean is up to 2^22 deviations: the mean is the rounded one, the deviation that about the true mean."""
    g = gen(width)
    base = torch.tensor([1000.0, -777.7, 3e4, 16777.215, 0.0, 4e6], device=DEV)[:, None]
    x = base.repeat(20, 1) + torch.randn(120, width, generator=g, device=DEV) * torch.tensor([0.01, 1.0], device=DEV).repeat(60)[:, None]
    gain, bias = vector(width, g, 1.0), vector(width, g, 0.0)
    out, stats = D.dedloc_norm(x, D.norm_cfg(KINDS["layer"], gain, bias, 1e-12))
    eps = float(torch.tensor(1e-12))
    mean, rstd, dm, dr = centred_stats(R.f64(x), eps)
    got, got_r = R.f64(stats[0, :, :1]), R.f64(stats[0, :, 1:])
    assert bool(((got - mean).abs() <= dm).all()), float(((got - mean).abs() / dm).max())
    assert bool(((got_r - rstd).abs() <= dr * rstd).all()), float(((got_r / rstd - 1).abs() / dr).max())
    y = (R.f64(x) - mean) * rstd * R.f64(gain) + R.f64(bias)
    c = (R.f64(x) - mean).abs() * rstd
    bound = R.SLACK * (R.f64(gain).abs() * (dm * rstd + c * (dr + 3 * R.U)) + 2 * R.U * y.abs())
    assert bool(((R.f64(out) - y).abs() <= bound).all())


# ------------------------------------------------------ sums of whole numbers

def whole(n, width, dtype, g, most=2):
    return torch.randint(-most, most + 1, (n, width), generator=g, device=DEV).to(dtype)


def unit_stats(norms, n):
    """(mean 0, rstd 1): the gradient takes the statistics that it is given, so every product is a whole number."""
    st = torch.zeros(norms, n, 2, device=DEV)
    st[..., 1] = 1
    return st


def same(got, want, what):
    assert float(want.abs().max()) < 2 ** 24, what  # exact in fp32 in any order
    assert torch.equal(got.double(), want), (what, int((got.double() != want).sum()))


MANY = [(9001, 512), (9000, 64), (4097, 333), (2500, 2560), (1500, 5120), (2000, 3000), (1400, 6144), (300, 16384), ((100 << 20) // 2048 + 3, 1024),
        ((100 << 20) // 5120 + 3, 2560)]


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("n,width", MANY)
def test_sums_of_a_norm_count_every_row_once(types, n, width):
    g = gen(n)
    stream, branch = types
    x, dout = whole(n, width, stream, g), whole(n, width, branch, g)
    for kind in ("layer", "rms"):
        acc = torch.ones(2, width, device=DEV)
        cfg = D.norm_cfg(KINDS[kind], torch.ones(width, device=DEV), torch.zeros(width, device=DEV), EPS[kind])
        D.dedloc_norm_grad(dout, x, unit_stats(1, n), cfg, acc[0], acc[1], 4.0)
        same(acc[0], 1 + 4 * (dout.double() * x.double()).sum(0), "dgain")
        same(acc[1], 1 + 4 * dout.double().sum(0), "dbias")


@pytest.mark.parametrize("gate", [None, "channel", 1, 7, 512, 1 << 20])
@pytest.mark.parametrize("types", [(F32, BF16), (F32, F32), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("n,width", MANY)
def test_sums_of_a_block_count_every_row_once(types, n, width, gate):
    """Without a pre norm the sum's gradient is dsum itself: dw = 2 dsum, fhat = f, gates, gains and biases whole."""
    g = gen(n + width)
    stream, branch = types
    f, dsum = whole(n, width, branch, g), whole(n, width, stream, g)
    gain, bias = (whole(1, width, F32, g)[0] for _ in range(2))
    gate_rows = gate if isinstance(gate, int) else 0
    q = whole(1, width, F32, g)[0] if gate == "channel" else whole(-(-n // gate_rows), width, branch, g) if gate_rows else None
    acc = torch.zeros(2, width, device=DEV)
    dgate = torch.zeros(q.shape, device=DEV) if gate else None
    dh, df = D.dedloc_residual_grad(None, f, unit_stats(2, n), dsum, None, beta=2.0, post=D.norm_cfg(KINDS["rms"], gain, bias, 1e-6), gate=q,
                                    gate_rows=gate_rows, dgate=dgate, dpost=(acc[0], acc[1]))
    assert torch.equal(dh, dsum)
    dw, f = 2 * dsum.double(), f.double()
    each = 1.0 if q is None else q.double().repeat_interleave(gate_rows, 0)[:n] if gate_rows else q.double()
    same(acc[0], (dw * each * f).sum(0), "dgain")
    same(acc[1], (dw * each).sum(0), "dbias")
    if gate is None:
        return
    terms = dw * (gain.double() * f + bias.double())
    if gate_rows:
        want = torch.zeros(q.shape, dtype=torch.float64, device=DEV).index_add_(0, torch.arange(n, device=DEV) // gate_rows, terms)
    else:
        want = terms.sum(0)
    same(dgate, want, "dgate")
