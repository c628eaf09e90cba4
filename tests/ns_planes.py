"""The Newton-Schulz steps in 64 bits, and an emulation of the arithmetic that
the kernels take them in: every factor in two fp16 planes, X times 2^12 and
the symmetric matrices times 2^8, a product as hi hi' + hi lo' + lo hi' (and
lo lo' for a shorter side up to 64) summed in fp32.  Tests of the kernels and
of their tolerance share the inputs here."""

import numpy as np

ABC = (3.4445, -4.7750, 2.0315)
EPS = 1e-7

# Lists of matrices by how a call works on them.
LISTS = {
    "narrow": [(64, 147), (33, 31), (128, 128), (100, 1000), (5, 300), (64, 4096), (300, 70)],
    "products": [(200, 300), (300, 130), (147, 64)],
    "blocks": [(300, 1100), (1100, 300), (520, 1700)],
    "cut": [(130, 3000)],
}
SHAPES = sorted({s for shapes in LISTS.values() for s in shapes})

# Of a result's 2-norm.  The emulation is at most half of it off over these inputs; one plane of one factor left out is
# ten times as far off at least (test_ortho_tolerance.py).
TIGHT = 1e-5
# Of a 16-bit result's entries, those that are not the rounding of the 64-bit value: the emulation's are at most a quarter of
# this, twice it at least with a product left out.
MISROUNDED = {"float16": 0.08, "bfloat16": 0.02}


def noise(rows, cols, seed):
    """Independent entries: singular values within a factor of a hundred of one another, mostly of three."""
    return np.random.default_rng(seed).standard_normal((rows, cols)) * 1e-3


def formula(u, steps=5):
    x = np.asarray(u, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.sqrt(np.sum(x * x)) + EPS)
    a, b, c = ABC
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.T if tall else x


def _planes(v):
    v = np.asarray(v, np.float32)
    hi = v.astype(np.float16)
    lo = (v - hi.astype(np.float32)).astype(np.float16)
    return hi.astype(np.float32), lo.astype(np.float32)


def emulated(u, blocks=False, drop=()):
    """The kernels' arithmetic on u.  drop: products left out, of "hi lo", "lo hi" (the left factor's plane first)."""
    X = np.asarray(u, np.float64)
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    X = (X * (4096.0 / (np.sqrt(np.sum(X * X)) + EPS))).astype(np.float32)
    a, b, c = ABC
    s = X.shape[0]

    def times(left, right, scale):  # left right^T
        (lh, ll), (rh, rl) = _planes(left), _planes(right)
        out = lh @ rh.T
        if "hi lo" not in drop:
            out = out + lh @ rl.T
        if "lo hi" not in drop:
            out = out + ll @ rh.T
        if s <= 64 and not drop:
            out = out + ll @ rl.T
        return (out * np.float32(scale)).astype(np.float32)

    def kept(v):  # what is stored of it
        hi, lo = _planes(v)
        return hi + lo

    def polynomial(A):
        A2 = times(A, A, 1 / 256.0).astype(np.float64)
        return (b * kept(A).astype(np.float64) + c * A2 + a * 256.0 * np.eye(s)).astype(np.float32)

    for n in ((3, 2) if blocks else (1,) * 5):
        A = times(X, X, 256.0 / 4096.0 ** 2)
        Q = M = polynomial(A)
        for _ in range(n - 1):
            A = times(times(M, M, 1 / 256.0), A, 1 / 256.0)
            M = polynomial(A)
            Q = times(M, Q, 1 / 256.0)
        X = times(Q, np.ascontiguousarray(X.T), 1 / 256.0)
    out = X.astype(np.float64) / 4096.0
    return out.T if tall else out


def relative(got, want):
    return float(np.linalg.norm(np.asarray(got, np.float64) - want) / np.linalg.norm(want))
