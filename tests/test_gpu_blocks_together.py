"""Dropout, norms and the ends of blocks as a peer's step uses them: a small
model from tokens to its loss, its gradients in the flat accumulator beside the
table's and the matrices', then the averaging and the optimizers' steps."""

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D
from . import block_ref as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
VOCAB, WIDTH, HIDDEN, BLOCKS, P, SEED, STEP = 60, 48, 96, 2, 0.1, 77, 3
SCALE = WIDTH ** 0.5


class Flat:
    """Named parts of one flat fp32 vector, each at a multiple of 8: the matrices first, then the table and the vectors."""

    def __init__(self):
        self.parts, self.matrices, at = {}, [], 0
        names = [(f"{w}{b}", (HIDDEN, WIDTH) if w == "up" else (WIDTH, HIDDEN)) for b in range(BLOCKS) for w in ("up", "down")]
        names += [("table", (VOCAB, WIDTH)), ("emb gain", (WIDTH,)), ("emb bias", (WIDTH,))]
        names += [(f"{v}{b}", (WIDTH,)) for b in range(BLOCKS) for v in ("post gain", "post bias", "pre gain", "pre bias", "gate")]
        for name, shape in names:
            self.parts[name] = (at, shape)
            at += -(-int(np.prod(shape)) // 8) * 8
        self.split = self.parts["table"][0]
        self.size = at

    def view(self, flat, name):
        at, shape = self.parts[name]
        return flat[at:at + int(np.prod(shape))].view(shape)


def start(flat):
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(flat.size, generator=g, device=DEV) * 0.2
    for name in flat.parts:
        if "gain" in name or "gate" in name:
            flat.view(x, name).add_(1.0)
    return x


def cfgs(flat, x, b):
    v = lambda n: flat.view(x, n)  # noqa: E731
    post = D.norm_cfg(D.DEDLOC_NORM_RMS, v(f"post gain{b}"), v(f"post bias{b}"), 1e-6)
    pre = D.norm_cfg(D.DEDLOC_NORM_LAYER, v(f"pre gain{b}"), v(f"pre bias{b}"), 1e-6)
    return dict(alpha=1.0, beta=0.5, post=post, pre=pre, gate=v(f"gate{b}"), drop=D.dropout_cfg(P, SEED, site=1 + b, step=STEP))


def library_step(flat, x, acc, ids, target):
    """Forward and backward, the layers between in plain torch; adds len(ids) times the mean loss's gradients into acc."""
    n = len(ids)
    v, a = (lambda t: lambda name: flat.view(t, name))(x), (lambda t: lambda name: flat.view(t, name))(acc)
    emb_norm = D.norm_cfg(D.DEDLOC_NORM_LAYER, v("emb gain"), v("emb bias"), 1e-6)
    drop = D.dropout_cfg(P, SEED, site=0, step=STEP)
    rows = D.dedloc_embed(v("table"), ids, SCALE)
    h = D.dedloc_dropout(rows, drop)
    inputs, st = D.dedloc_norm(h, emb_norm)
    keep = [(h, inputs, st)]
    for b in range(BLOCKS):
        up = torch.tanh(inputs @ v(f"up{b}").t())
        f = up @ v(f"down{b}").t()
        total, out, stats = D.dedloc_residual(h, f, **cfgs(flat, x, b))
        keep.append((inputs, up, f, total, stats))
        h, inputs = total, out
    logits = (inputs @ v("table").t()).requires_grad_()
    loss = torch.nn.functional.cross_entropy(logits, target)
    (dlogits,) = torch.autograd.grad(loss, logits)
    D.dedloc_accumulate(a("table").reshape(-1), (dlogits.t() @ inputs).reshape(-1), n)
    dout, dsum = dlogits @ v("table"), None
    for b in reversed(range(BLOCKS)):
        inputs, up, f, total, stats = keep[1 + b]
        dsum, df = D.dedloc_residual_grad(total, f, stats, dsum, dout, dgate=a(f"gate{b}"),
                                          dpre=(a(f"pre gain{b}"), a(f"pre bias{b}")),
                                          dpost=(a(f"post gain{b}"), a(f"post bias{b}")), batch_samples=n, **cfgs(flat, x, b))
        D.dedloc_accumulate(a(f"down{b}").reshape(-1), (df.t() @ up).reshape(-1), n)
        dup = (df @ v(f"down{b}")) * (1 - up * up)
        D.dedloc_accumulate(a(f"up{b}").reshape(-1), (dup.t() @ inputs).reshape(-1), n)
        dout = dup @ v(f"up{b}")
    h, inputs, st = keep[0]
    dh = D.dedloc_norm_grad(dout, h, st, emb_norm, a("emb gain"), a("emb bias"), n, add=dsum)
    D.dedloc_embed_grad(a("table"), ids, D.dedloc_dropout(dh, drop), SCALE, n)
    return float(loss.detach())


def reference_step(flat, x, ids, target):
    """The same by autograd in 64 bits on the CPU: (loss, gradients)."""
    x = x.double().cpu().requires_grad_()
    v = lambda name: flat.view(x, name)  # noqa: E731
    ids, target, n = ids.cpu(), target.cpu(), len(ids)

    def drop(t, site):
        keep, factor = R.kept(n, WIDTH, P, seed=SEED, site=site, step=STEP)
        return torch.where(torch.from_numpy(keep), t * float(factor), 0.0)

    def norm(t, rms, gain, bias):
        c = t if rms else t - t.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + float(np.float32(1e-6))).sqrt() * gain + bias

    rows = torch.where((ids >= 0)[:, None], v("table")[ids.clamp(min=0)] * float(np.float32(SCALE)), 0.0)
    h = drop(rows, 0)
    inputs = norm(h, False, v("emb gain"), v("emb bias"))
    for b in range(BLOCKS):
        f = torch.tanh(inputs @ v(f"up{b}").t()) @ v(f"down{b}").t()
        h = h + 0.5 * drop(v(f"gate{b}") * norm(f, True, v(f"post gain{b}"), v(f"post bias{b}")), 1 + b)
        inputs = norm(h, False, v(f"pre gain{b}"), v(f"pre bias{b}"))
    loss = torch.nn.functional.cross_entropy(inputs @ v("table").t(), target)
    return float(loss.detach()), torch.autograd.grad(loss, x)[0]


def batch(seed, n=200):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, VOCAB, (n,), generator=g, device=DEV)
    ids[::17] = -1
    return ids, torch.randint(0, VOCAB, (n,), generator=g, device=DEV)


def test_gradients_are_autograds():
    """fp32 sums of at most 200 terms through some 20 operations: 4000 * 2^-24 of each part's largest gradient."""
    flat = Flat()
    x = start(flat)
    acc, want = torch.zeros_like(x), 0
    for k in range(2):
        loss = library_step(flat, x, acc, *batch(k))
        ref, grad = reference_step(flat, x, *batch(k))
        assert abs(loss - ref) <= 4000 * R.U * abs(ref)
        want = want + 200 * grad
    for name in flat.parts:
        a, w = flat.view(acc, name).double().cpu(), flat.view(want, name)
        assert float((a - w).abs().max()) <= 4000 * R.U * float(w.abs().max()), name


def test_a_round_of_two_peers():
    """The accumulators become messages, their average the update: LAMB over the whole vector moves every part."""
    flat = Flat()
    x = start(flat)
    before = x.clone()
    messages, counts = [], []
    for peer in range(2):
        acc = torch.zeros_like(x)
        for k in range(peer + 1):
            library_step(flat, x, acc, *batch(10 * peer + k))
        counts.append(200 * (peer + 1))
        messages.append(D.dedloc_finalize(acc, counts[-1], D.DEDLOC_CODEC_FP16)[0])
        assert bool((acc == 0).all())
    mean, _ = D.dedloc_reduce_shard(messages, counts, flat.size, D.DEDLOC_CODEC_FP16)
    m, v = torch.zeros_like(x), torch.zeros_like(x)
    offsets = [at for at, _ in flat.parts.values()] + [flat.size]
    D.dedloc_lamb_step(x, m, v, mean, offsets, [3] * len(flat.parts), D.lamb_cfg(lr=0.01, step=1), D.DEDLOC_CODEC_FP16)
    for name in flat.parts:
        moved = (flat.view(x, name) - flat.view(before, name)).abs()
        assert bool(torch.isfinite(moved).all()) and float(moved.max()) > 0, name
