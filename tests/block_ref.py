"""dropout, norms and the ends of a block by their definitions in 64 bits, on
the CPU, with bounds of what fp32 arithmetic may be off.

U = 2^-24 is half a step of fp32.  A row's sum of n terms runs through at most 16 terms
of a thread, 6 levels over lanes and 16 waves, and one product makes it a mean: K = 40 roundings, so it is off by at
most K U sum |terms|, plus what the terms are off.  Each value comes with its
bound, carried through the formulas to first order with a factor of 1.01 for the rest."""

import numpy as np
import torch

U = 2.0 ** -24
K = 40
SLACK = 1.01
M32 = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 of arrays of 32-bit words (as uint64): four arrays."""
    c0, c1, c2, c3 = (np.asarray(c, np.uint64) & M32 for c in (c0, c1, c2, c3))
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & M32, (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & M32
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def kept(rows, width, p, seed=0, site=0, step=0, row0=0):
    """(bool [rows, width], the factor as fp32)"""
    p = float(np.float32(p))
    T = 65536 if p == 1 else min(int(np.rint(p * 65536)), 65535)
    n = -(-width // 8)
    with np.errstate(over="ignore"):
        words = philox(np.arange(n)[None, :] + np.zeros((rows, 1)), (row0 + np.arange(rows, dtype=np.uint64))[:, None] + np.zeros((1, n), np.uint64),
                       np.full((rows, n), site), np.full((rows, n), step & 0xFFFFFFFF), seed & 0xFFFFFFFF, seed >> 32)
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2).reshape(rows, n * 8)[:, :width]
    return halves >= T, np.float32(65536.0 / (65536 - T)) if T < 65536 else np.float32(0)


def f64(t):
    return None if t is None else t.detach().double().cpu()


def half_step(t, dtype):
    """Of rounding values t to dtype: half a step of a normal number, or of the smallest."""
    fi = torch.finfo(dtype)
    return torch.maximum(t.abs() * (fi.eps / 2), torch.tensor(fi.tiny * fi.eps / 2, dtype=torch.float64))


class N:
    """A norm: kind "layer" or "rms", eps, gain and bias or None (fp32 tensors)."""

    def __init__(self, kind, eps, gain=None, bias=None):
        self.kind, self.eps, self.gain, self.bias = kind, float(np.float32(eps)), gain, bias

    def g(self, width):
        return f64(self.gain) if self.gain is not None else torch.ones(width, dtype=torch.float64)

    def b(self, width):
        return f64(self.bias) if self.bias is not None else torch.zeros(width, dtype=torch.float64)


def stats(x, n):
    """(mean, rstd, bound of mean, relative bound of rstd)"""
    D = x.shape[1]
    zero = torch.zeros(x.shape[0], 1, dtype=torch.float64)
    mean = x.mean(1, keepdim=True) if n.kind == "layer" else zero
    dm = (K + 2) * U * x.abs().mean(1, keepdim=True) if n.kind == "layer" else zero
    var = (x - mean).square().mean(1, keepdim=True)
    # squares about a mean that is off by dm add its square; each wave's own mean, rounded, adds twice that at most
    dvar = (K + 8) * U * var + 4 * dm ** 2
    rstd = 1 / (var + n.eps).sqrt()
    return mean, rstd, dm, dvar / (var + n.eps) / 2 + 4 * U


def norm(x, n):
    """(y, bound, mean, rstd, their bounds)"""
    D = x.shape[1]
    mean, rstd, dm, dr = stats(x, n)
    g, b = n.g(D).abs(), n.b(D)
    c = (x - mean).abs() * rstd
    y = (x - mean) * rstd * n.g(D) + b
    return y, SLACK * (g * (dm * rstd + c * (dr + 3 * U)) + U * y.abs()), mean, rstd, dm, dr * rstd


def norm_back(dy, edy, x, mean, rstd, n):
    """From dy with its bound and statistics taken as they are: (dx, bound, dgain terms, bound, dbias terms, bound)."""
    D = x.shape[1]
    xhat = (x - mean) * rstd
    ex = 2 * U * xhat.abs()
    g = dy * n.g(D)
    eg = edy * n.g(D).abs() + U * g.abs()
    mgx, emgx = (g * xhat).mean(1, keepdim=True), ((K + 2) * U * (g * xhat).abs() + eg * xhat.abs() + g.abs() * ex).mean(1, keepdim=True)
    mg, emg = torch.zeros_like(mgx), torch.zeros_like(mgx)
    if n.kind == "layer":
        mg, emg = g.mean(1, keepdim=True), ((K + 2) * U * g.abs() + eg).mean(1, keepdim=True)
    inner = g - mg - xhat * mgx
    # the means are multiplied by rstd first: one rounding each, then xhat's fused product with the other, then the sum
    e = eg + emg + ex * mgx.abs() + xhat.abs() * emgx + U * (2 * mg.abs() + 3 * (xhat * mgx).abs() + 2 * (g - mg).abs() + inner.abs())
    dx = rstd * inner
    return dx, SLACK * (rstd * e + U * dx.abs()), dy * xhat, SLACK * (edy * xhat.abs() + dy.abs() * ex), dy, edy


def columns(acc, samples, terms, bound, size=None):
    """fma(samples, sum of terms over rows, acc) and its bound: any order of an fp32 sum.  size: of the terms as they
    are summed, where that is not their own."""
    total = terms.sum(0)
    e = bound.sum(0) + (terms.shape[0] + 4) * U * (terms.abs() if size is None else size).sum(0)
    out = (0 if acc is None else f64(acc)) + samples * total
    return out, SLACK * (samples * (e + U * total.abs()) + U * out.abs())


def gate_of(gate, gate_rows, rows):
    if gate is None:
        return torch.ones((), dtype=torch.float64)
    return f64(gate)[torch.arange(rows) // gate_rows] if gate_rows else f64(gate)


def residual_sum(h, f, alpha, beta, post, gate, gate_rows, mask):
    """(sum before its rounding, bound, post's mean, rstd and bounds); mask: (kept, factor) or None."""
    rows, _ = h.shape
    ev, st = torch.zeros_like(f), None
    v = f
    if post is not None:
        v, ev, *st = norm(f, post)
    if gate is not None:
        q = gate_of(gate, gate_rows, rows)
        # a norm's gain and bias may be multiplied by the gate first: one rounding each
        bias = post.b(f.shape[1]) if post is not None else 0.0
        size = (v - bias).abs() + abs(bias)
        v, ev = v * q, ev * q.abs() + U * size * q.abs()
        ev = ev + U * v.abs()
    if mask is not None:
        keep, factor = torch.from_numpy(mask[0]), float(mask[1])
        v, ev = torch.where(keep, v * factor, 0.0), torch.where(keep, ev * factor, 0.0)
        ev = ev + U * v.abs()
    a, b = float(np.float32(alpha)), float(np.float32(beta))
    s = a * h + b * v
    return s, SLACK * (abs(b) * ev + U * ((a * h).abs() + s.abs())), st


def residual_grad(x, f, st, dsum, dout, alpha, beta, post, pre, gate, gate_rows, mask):
    """A dict of (value, bound): dh, df, and (terms, bound of each) of the parameters' sums: dpre_gain and the rest.
    st: (mean, rstd) of pre, then of post, [2, rows, 2]."""
    like = dsum if dsum is not None else x
    rows, width = like.shape
    out = {}
    d = dsum if dsum is not None else torch.zeros_like(like)
    ed = torch.zeros_like(d)
    if pre is not None:
        dx, e, *sums = norm_back(dout, torch.zeros_like(dout), x, st[0, :, :1], st[0, :, 1:], pre)
        out["dpre_gain"], out["dpre_bias"] = sums[:2], sums[2:]
        d = d + dx
        ed = e + U * d.abs()
    a, b = float(np.float32(alpha)), float(np.float32(beta))
    out["dh"] = a * d, SLACK * (abs(a) * ed + U * (a * d).abs())
    dw, ew = b * d, abs(b) * ed + U * (b * d).abs()
    if mask is not None:
        keep, factor = torch.from_numpy(mask[0]), float(mask[1])
        dw, ew = torch.where(keep, dw * factor, 0.0), torch.where(keep, ew * factor, 0.0)
        ew = ew + U * dw.abs()
    q = gate_of(gate, gate_rows, rows)
    dv, ev = dw * q, ew * q.abs()
    ev = ev + (U * dv.abs() if gate is not None else 0)
    if post is not None:
        fhat = (f - st[1, :, :1]) * st[1, :, 1:]
        v = fhat * post.g(width) + post.b(width)
        evv = U * (4 * (fhat * post.g(width)).abs() + v.abs())
        df, e, *sums = norm_back(dv, ev, f, st[1, :, :1], st[1, :, 1:], post)
        out["df"], out["dpost_gain"], out["dpost_bias"] = (df, e), sums[:2], sums[2:]
    else:
        v, evv = f, torch.zeros_like(like)
        out["df"] = dv, ev
    if gate is not None and v is not None:
        # a learned gate's is taken from the norm's sums: gain sum(dw fhat) + bias sum(dw)
        mag = (fhat * post.g(width)).abs() + post.b(width).abs() if post is not None else v.abs()
        out["dgate"] = dw * v, SLACK * (ew * mag + dw.abs() * evv + 2 * U * dw.abs() * mag), dw.abs() * mag
    return out
