"""What stands between the matrix products of a language model's training
step, timed operator by operator.

Five of them, through the public Python binding over libdedloc:

  dropout        from a counter-based generator, the mask never stored; its
                 gradient is the same call;
  norm           layer and root-mean-square norms of rows, with their statistics;
  norm_grad      the norm's gradient; the gain's and the bias' are added into a
                 peer's fp32 accumulator;
  residual       the end of a block and the start of the next in one pass: the
                 branch's norm, its gate, dropout, the scaled residual sum and
                 the norm of that sum;
  residual_grad  the gradients of that pass.

The definitions.  A mask comes from Philox4x32-10 (Salmon, Moraes, Dror and
Shaw 2011) with the key (seed's low, high word) and the counter (column / 8, row0 +
row, site, step): the four words are eight halves, the low half of a word
first, one for each of eight columns.  With T = p rounded to 65536ths a half below T
drops its element, and what is kept is multiplied by 65536 / (65536 - T).

  N(x) = (x - mean) * rstd * gain + bias     (mean = 0 for the rms norm)
  sum  = alpha * h + beta * dropout(gate * post(f)), rounded to its type
  out  = pre(sum)

With `own` false, run() computes the same in elementary torch operations in
32 bits.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "fp16": 2, "bf16": 2}
EPS = {"layer": 1e-12, "rms": 1e-6}
SAMPLES = 16.0  # of the micro-batch: its weight in the accumulator
SITE = 5        # which dropout of the model this is
STEP = 1234     # of the training


# ------------------------------------------------------------------ the cases

def case_of(kind, rows, width, stream="f32", branch=None, post="none", pre="none", gate="none", gate_rows=0, p=0.0,
            alpha=1.0, beta=1.0, pad=0, stepped=False, both=True, bias=True, **name):
    """stream: the type of h and the sum; branch: of f and the norm's output.  stepped: the step is read from the
    device, as a captured training step does.  both: whether the sum has a gradient of its own."""
    return dict(name, kind=kind, rows=rows, width=width, stream=stream, branch=branch or stream, post=post, pre=pre,
                gate=gate, gate_rows=gate_rows, p=p, alpha=alpha, beta=beta, pad=pad, stepped=stepped, both=both, bias=bias)


def listed():
    return [
        # ALBERT's embeddings of one micro-batch, 16 sequences of 512 tokens by 128: launches count
        case_of("dropout", 8192, 128, "f32", p=0.1, name="dropout embeddings f32"),
        # attention probabilities of ALBERT-large: 16 sequences, 16 heads, 512 by 512; the step read from the device
        case_of("dropout", 131072, 512, "bf16", p=0.1, stepped=True, name="dropout attention bf16"),
        # one token in service: the smallest call
        case_of("norm", 1, 2048, "bf16", pre="rms", bias=False, name="norm token bf16"),
        # the embeddings' norm over one micro-batch
        case_of("norm", 8192, 128, "f32", pre="layer", name="norm embeddings f32"),
        # its gradient
        case_of("norm_grad", 8192, 128, "f32", pre="layer", both=False, name="norm_grad embeddings f32"),
        # norms of queries per head: many short rows
        case_of("norm_grad", 262144, 64, "bf16", pre="rms", both=False, bias=False, name="norm_grad heads bf16"),
        # a few tokens in service through a block of ALBERT-xlarge's width
        case_of("residual", 8, 2048, "bf16", pre="rms", bias=False, name="residual tokens bf16"),
        # LayerNorm(h + dropout(f)) of ALBERT-large, one micro-batch in fp16
        case_of("residual", 8192, 1024, "fp16", pre="layer", p=0.1, name="residual albert_large fp16"),
        # norms on both sides of the block, a learned gate, an fp32 residual stream with bf16 branches: the largest
        case_of("residual", 65536, 2048, "f32", "bf16", post="rms", pre="rms", gate="channel", p=0.1, alpha=1.0, beta=0.5,
                bias=False, name="residual sandwich f32 bf16"),
        # the gradient of ALBERT-large's
        case_of("residual_grad", 8192, 1024, "fp16", pre="layer", p=0.1, both=False, name="residual_grad albert_large fp16"),
        # odd sizes, rows at a stride, a gate per group of rows whose last one is short
        case_of("residual_grad", 1001, 333, "bf16", post="layer", pre="layer", gate="group", gate_rows=143, p=0.25, alpha=1.25,
                beta=0.75, pad=7, stepped=True, name="residual_grad ragged bf16"),
        # everything at once at ALBERT-xlarge's width
        case_of("residual_grad", 65536, 2048, "bf16", post="layer", pre="layer", gate="channel", p=0.1, alpha=1.0, beta=0.5,
                name="residual_grad sandwich bf16"),
    ]


def draw(rng):
    """One more case of the listed ones' ranges."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["dropout", "norm", "norm_grad", "residual", "residual_grad"])
    width = log(16, 8192)
    if rng.random() < 0.5:
        width = max(64, width // 64 * 64)
    rows = min(log(1, 262144), (1 << 26) // width)
    stream = rng.choice(["f32", "fp16", "bf16"])
    branch = rng.choice(["f32", "fp16", "bf16"]) if stream == "f32" and kind != "dropout" else stream
    more = dict(pad=rng.choice([0, 0, 8, 7]), stepped=rng.random() < 0.5, bias=rng.random() < 0.5)
    if kind == "dropout":
        return case_of(kind, rows, width, stream, p=rng.choice([0.1, 0.5, rng.random()]), **more)
    if kind in ("norm", "norm_grad"):
        return case_of(kind, rows, width, stream, branch, pre=rng.choice(["layer", "rms"]), both=rng.random() < 0.5, **more)
    gate = rng.choice(["none", "channel", "group"])
    post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("layer", "layer"), ("rms", "rms"), ("layer", "none"), ("none", "none")])
    return case_of(kind, rows, width, stream, branch, post=post, pre=pre, gate=gate,
                   gate_rows=log(1, rows) if gate == "group" else 0, p=rng.choice([0.0, 0.1, 0.3]),
                   alpha=rng.choice([1.0, 0.8125]), beta=rng.choice([1.0, 0.25]), both=pre == "none" or rng.random() < 0.5, **more)


def groups_of(case):
    return -(-case["rows"] // case["gate_rows"]) if case["gate"] == "group" else 1


def work(case):
    """Each input read once, each output written once; accumulators are read and written."""
    kind, n, es, eb = case["kind"], case["rows"] * case["width"], SIZE[case["stream"]], SIZE[case["branch"]]
    stats = 8 * case["rows"] * ((case["pre"] != "none") + (case["post"] != "none"))
    per = 1 + (case["bias"])  # vectors of a norm
    vectors = 4 * case["width"] * per * ((case["pre"] != "none") + (case["post"] != "none"))
    gate = {"none": 0, "channel": 4 * case["width"], "group": eb * case["width"] * groups_of(case)}[case["gate"]]
    if kind == "dropout":
        return dict(bytes=2 * n * es, flops=n)
    if kind == "norm":
        return dict(bytes=n * (es + eb) + stats + vectors, flops=5 * n)
    if kind == "norm_grad":
        return dict(bytes=n * (2 * es + eb + es * case["both"]) + stats + 3 * vectors, flops=10 * n)
    has_pre, reads_f = case["pre"] != "none", case["post"] != "none" or case["gate"] != "none"
    if kind == "residual":
        return dict(bytes=n * (2 * es + eb + eb * has_pre) + stats + vectors + gate, flops=14 * n)
    dgate = {"none": 0, "channel": 2 * gate, "group": 4 * case["width"] * groups_of(case)}[case["gate"]]
    return dict(bytes=n * (es * case["both"] + (eb + es) * has_pre + eb * reads_f + es + eb) + stats + 3 * vectors + gate + dgate,
                flops=25 * n)


# ------------------------------------------------------------ inputs of a case

def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def strided(rows, width, pad, dtype):
    """A rows x width view into a buffer whose rows are `pad` elements longer."""
    return torch.empty(rows, width + pad, dtype=dtype, device="cuda")[:, :width]


def prepare(case, seed):
    g, kind, rows, width = generator(seed), case["kind"], case["rows"], case["width"]
    stream, branch = TYPES[case["stream"]], TYPES[case["branch"]]

    def normal(dtype, std, mean=0.0, channels=False):
        out = strided(rows, width, case["pad"], dtype)
        out.normal_(mean, std, generator=g)
        if channels:  # a few channels of a hidden state are much larger than the others
            loud = torch.rand(width, generator=g, device="cuda") < 0.01
            out.mul_(torch.where(loud, 12.0, 1.0).to(dtype))
        return out

    def vector(mean, std):
        return torch.randn(width, generator=g, device="cuda") * std + mean

    def norm(which):
        if case[which] == "none":
            return None
        return dict(kind=case[which], eps=EPS[case[which]], gain=vector(1.0, 0.2), bias=vector(0.0, 0.1) if case["bias"] else None)

    def accumulators(n):
        """After earlier micro-batches."""
        return None if n is None else {k: vector(0.0, 1.0) for k in ("gain", "bias") if n[k] is not None}

    s = dict(kind=kind, case=case, post=norm("post"), pre=norm("pre"))
    s["seed"] = (seed * 0x9E3779B97F4A7C15 + 1) % (1 << 64)
    s["step_at"] = torch.tensor([STEP - 1000], dtype=torch.int64, device="cuda") if case["stepped"] else None
    s["step"] = 1000 if case["stepped"] else STEP
    s["gate"] = s["dgate"] = None
    if case["gate"] == "channel":
        s["gate"] = vector(0.5, 0.2)
    elif case["gate"] == "group":
        s["gate"] = (torch.randn(groups_of(case), width, generator=g, device="cuda") * 0.3 + 0.7).to(branch)
    if kind == "dropout":
        s["x"], s["out"] = normal(stream, 1.0), strided(rows, width, case["pad"], stream)
    elif kind == "norm":
        s["x"], s["out"] = normal(stream, 1.5, 0.3, True), strided(rows, width, case["pad"], branch)
        s["stats"] = torch.empty(1, rows, 2, device="cuda")
    elif kind == "residual":
        s["h"], s["f"] = normal(stream, 1.5, 0.3, True), normal(branch, 0.5)
        s["sum"] = strided(rows, width, case["pad"], stream)
        s["out"] = strided(rows, width, case["pad"], branch) if s["pre"] else None
        s["stats"] = torch.empty(2, rows, 2, device="cuda")
    else:
        s["sum"] = normal(stream, 1.5, 0.3, True)
        s["dsum"] = normal(stream, 1e-3) if case["both"] else None
        s["dout"] = normal(branch, 1e-3) if s["pre"] else None
        s["dh"] = strided(rows, width, case["pad"], stream)
        s["f"] = s["df"] = None
        if kind == "residual_grad":
            s["f"], s["df"] = normal(branch, 0.5), strided(rows, width, case["pad"], branch)
        # what the forward pass kept: (mean, 1 / standard deviation) of every row, of the sum and of the branch
        s["stats"] = torch.zeros(2 if kind == "residual_grad" else 1, rows, 2, device="cuda")
        for k, (x, n) in enumerate(((s["sum"], s["pre"]), (s["f"], s["post"]))):
            if n:
                x = x.double()
                if n["kind"] == "layer":
                    s["stats"][k, :, 0] = x.mean(1)
                    x = x - x.mean(1, keepdim=True)
                s["stats"][k, :, 1] = 1 / (x.square().mean(1) + n["eps"]).sqrt()
        s["dpre"], s["dpost"] = accumulators(s["pre"]), accumulators(s["post"])
        if case["gate"] == "channel":
            s["dgate"] = vector(0.0, 1.0)
        elif case["gate"] == "group":
            s["dgate"] = torch.empty(groups_of(case), width, device="cuda")
    if own:
        handles(s)
    return s


def handles(s):
    """What a user's program makes of the framework before its first step."""
    from paper_2106_10207_amd import dedloc as D
    case, kinds = s["case"], {"layer": D.DEDLOC_NORM_LAYER, "rms": D.DEDLOC_NORM_RMS}

    def norm(n):
        return None if n is None else D.norm_cfg(kinds[n["kind"]], n["gain"], n["bias"], n["eps"])

    pre, post = norm(s["pre"]), norm(s["post"])
    drop = D.dropout_cfg(case["p"], s["seed"], site=SITE, step=s["step"], step_at=s["step_at"])
    if s["kind"] == "dropout":
        s["drop"] = drop
        return
    if s["kind"] in ("norm", "norm_grad"):
        s["norm"] = pre
        if s["kind"] == "norm_grad":
            s["ws"] = D.make_residual_workspace(case["rows"], case["width"])
        return
    block = dict(alpha=case["alpha"], beta=case["beta"], post=post, pre=pre, gate=s["gate"], gate_rows=case["gate_rows"],
                 drop=drop if case["p"] else None)
    if s["kind"] == "residual":
        s["call"] = D.ResidualCall(s["h"], s["f"], s["sum"], s["out"], s["stats"], **block)
    else:
        pair = lambda acc: None if acc is None else (acc["gain"], acc.get("bias"))  # noqa: E731
        s["call"] = D.ResidualGradCall(s["sum"], s["f"], s["stats"], s["dsum"], s["dout"], s["dh"], s["df"], dgate=s["dgate"],
                                       dpost=pair(s["dpost"]), dpre=pair(s["dpre"]), batch_samples=SAMPLES, **block)


# -------------------------------------------------------------- the plain forms

LOW = 0xFFFFFFFF


def plain_kept(s):
    """(kept elements, their factor); 64-bit products wrap, their halves are what the generator needs."""
    case = s["case"]
    rows, width, p = case["rows"], case["width"], case["p"]
    T = 65536 if p == 1 else min(int(round(p * 65536)), 65535)
    groups = -(-width // 8)
    step = s["step"] + (s["step_at"] if s["step_at"] is not None else 0)
    zero = torch.zeros(rows, groups, dtype=torch.int64, device="cuda")
    c0 = zero + torch.arange(groups, device="cuda")
    c1 = zero + torch.arange(rows, device="cuda")[:, None]
    c2, c3 = zero + SITE, zero + step
    k0, k1 = s["seed"] & LOW, s["seed"] >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & LOW) ^ c1 ^ k0, b & LOW, (a >> 32 & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    halves = torch.stack([h for c in (c0, c1, c2, c3) for h in (c & 0xFFFF, c >> 16)], dim=2)
    return halves.view(rows, groups * 8)[:, :width] >= T, 65536 / (65536 - T) if T < 65536 else 0.0


def plain_dropout(x, s):
    """fp32 x with the case's mask."""
    if s["case"]["p"] == 0:
        return x
    kept, factor = plain_kept(s)
    return torch.where(kept, x * factor, 0.0)


def plain_stats(x, n):
    mean = x.mean(1, keepdim=True) if n["kind"] == "layer" else torch.zeros_like(x[:, :1])
    return mean, 1 / ((x - mean).square().mean(1, keepdim=True) + n["eps"]).sqrt()


def plain_apply(x, mean, rstd, n):
    y = (x - mean) * rstd * n["gain"]
    return y if n["bias"] is None else y + n["bias"]


def plain_norm_grad(dy, x, mean, rstd, n, acc):
    """dx; acc's vectors take theirs."""
    xhat = (x - mean) * rstd
    acc["gain"].add_((dy * xhat).sum(0), alpha=SAMPLES)
    if "bias" in acc:
        acc["bias"].add_(dy.sum(0), alpha=SAMPLES)
    g = dy * n["gain"]
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if n["kind"] == "layer":
        dx -= g.mean(1, keepdim=True)
    return dx * rstd


def plain_gate(s):
    gate, case = s["gate"], s["case"]
    if case["gate"] == "none":
        return 1.0
    if case["gate"] == "channel":
        return gate
    return gate.float().repeat_interleave(case["gate_rows"], 0)[:case["rows"]]


def plain_residual(s):
    case, f, stats = s["case"], s["f"].float(), s["stats"]
    stats.zero_()
    if s["post"]:
        mean, rstd = plain_stats(f, s["post"])
        stats[1] = torch.cat([mean, rstd], 1)
        f = plain_apply(f, mean, rstd, s["post"])
    s["sum"].copy_(case["alpha"] * s["h"].float() + case["beta"] * plain_dropout(plain_gate(s) * f, s))
    if s["pre"]:
        x = s["sum"].float()
        mean, rstd = plain_stats(x, s["pre"])
        stats[0] = torch.cat([mean, rstd], 1)
        s["out"].copy_(plain_apply(x, mean, rstd, s["pre"]))
    return kept_outputs(s)


def plain_grad(s):
    case, d = s["case"], 0.0
    if s["dsum"] is not None:
        d = s["dsum"].float()
    if s["pre"]:
        d = d + plain_norm_grad(s["dout"].float(), s["sum"].float(), s["stats"][0, :, :1], s["stats"][0, :, 1:], s["pre"], s["dpre"])
    s["dh"].copy_(case["alpha"] * d)
    if s["kind"] == "residual_grad":
        dw = case["beta"] * plain_dropout(d, s)
        f, post = s["f"].float(), s["post"]
        if post:
            mean, rstd = s["stats"][1, :, :1], s["stats"][1, :, 1:]
        if case["gate"] != "none":
            dgate = dw * (plain_apply(f, mean, rstd, post) if post else f)
            if case["gate"] == "channel":
                s["dgate"].add_(dgate.sum(0), alpha=SAMPLES)
            else:
                short = groups_of(case) * case["gate_rows"] - case["rows"]  # of the last group
                dgate = torch.nn.functional.pad(dgate, (0, 0, 0, short))
                s["dgate"].copy_(dgate.view(groups_of(case), case["gate_rows"], case["width"]).sum(1))
        dv = plain_gate(s) * dw
        s["df"].copy_(plain_norm_grad(dv, f, mean, rstd, post, s["dpost"]) if post else dv)
    return grad_outputs(s)


def kept_outputs(s):
    """What a forward pass leaves; a norm that is not there leaves no statistics."""
    out = dict(sum=s["sum"])
    if s["pre"]:
        out.update(out=s["out"], pre=s["stats"][0])
    if s["post"]:
        out["post"] = s["stats"][1]
    return out


def grad_outputs(s):
    out = dict(dh=s["dh"])
    if s["kind"] == "residual_grad":
        out["df"] = s["df"]
    for which in ("dpre", "dpost"):
        for k, v in (s[which] or {}).items():
            out[which + " " + k] = v
    if s["dgate"] is not None:
        out["dgate"] = s["dgate"]
    return out


def run(s):
    kind = s["kind"]
    if not own:
        if kind == "dropout":
            return s["out"].copy_(plain_dropout(s["x"].float(), s))
        if kind == "norm":
            x = s["x"].float()
            mean, rstd = plain_stats(x, s["pre"])
            s["stats"][0] = torch.cat([mean, rstd], 1)
            return dict(out=s["out"].copy_(plain_apply(x, mean, rstd, s["pre"])), pre=s["stats"][0])
        return plain_residual(s) if kind == "residual" else plain_grad(s)
    from paper_2106_10207_amd import dedloc as D
    if kind == "dropout":
        return D.dedloc_dropout(s["x"], s["drop"], out=s["out"])
    if kind == "norm":
        D.dedloc_norm(s["x"], s["norm"], out=s["out"], stats=s["stats"])
        return dict(out=s["out"], pre=s["stats"][0])
    if kind == "norm_grad":
        D.dedloc_norm_grad(s["dout"], s["sum"], s["stats"], s["norm"], add=s["dsum"], dx=s["dh"], dgain=s["dpre"]["gain"],
                           dbias=s["dpre"].get("bias"), batch_samples=SAMPLES, ws=s["ws"])
        return grad_outputs(s)
    s["call"]()
    return kept_outputs(s) if kind == "residual" else grad_outputs(s)


# ------------------------------------------------------- the definitions, in 64 bits

def exact_factor(s):
    """0 where dropped, else the factor, as doubles: the generator's products from 16-bit pieces, rows of counters."""
    case = s["case"]
    if case["p"] == 0:
        return torch.ones((), dtype=torch.float64, device="cuda")
    T = 65536 if case["p"] == 1 else min(int(math.floor(case["p"] * 65536 + 0.5)), 65535)
    count = (case["width"] + 7) // 8
    where = torch.arange(case["rows"] * count, device="cuda")
    ctr = [where % count, where // count, torch.full_like(where, SITE), torch.full_like(where, STEP)]
    key = [s["seed"] % (1 << 32), s["seed"] // (1 << 32)]

    def halves(x, m):
        """(high word, low word) of the product of x and the constant m."""
        x1, x0, m1, m0 = x // 65536, x % 65536, m // 65536, m % 65536
        low, mid1, mid2 = x0 * m0, x1 * m0, x0 * m1
        carry = low // 65536 + mid1 % 65536 + mid2 % 65536
        return x1 * m1 + mid1 // 65536 + mid2 // 65536 + carry // 65536, (carry % 65536) * 65536 + low % 65536

    for r in range(10):
        (h0, l0), (h1, l1) = halves(ctr[0], 0xD2511F53), halves(ctr[2], 0xCD9E8D57)
        ctr = [torch.bitwise_xor(torch.bitwise_xor(h1, ctr[1]), (key[0] + r * 0x9E3779B9) % (1 << 32)), l1,
               torch.bitwise_xor(torch.bitwise_xor(h0, ctr[3]), (key[1] + r * 0xBB67AE85) % (1 << 32)), l0]
    out = torch.empty(case["rows"], count * 8, dtype=torch.float64, device="cuda")
    for j in range(8):
        r16 = (ctr[j // 2] // (65536 if j % 2 else 1)) % 65536
        out[:, j::8] = torch.where(r16 < T, 0.0, 65536 / max(65536 - T, 1)).view(case["rows"], count)
    return out[:, :case["width"]]


def exact(case, seed):
    if case["rows"] * case["width"] > 1 << 27:
        return None
    s, kind = prepare(case, seed), case["kind"]
    factor = exact_factor(s)

    def norm(x, n):
        """(y, statistics) as functions of x that autograd can follow."""
        mean = x.sum(1, keepdim=True) / case["width"] * (n["kind"] == "layer")
        var = ((x - mean) ** 2).sum(1, keepdim=True) / case["width"]
        rstd = (var + n["eps"]) ** -0.5
        y = (x - mean) * rstd * n["gain64"]
        return y + n["bias64"], torch.cat([mean, rstd], 1)

    for n in (s["pre"], s["post"]):
        if n:
            n["gain64"] = n["gain"].double().requires_grad_()
            n["bias64"] = (n["bias"].double() if n["bias"] is not None else torch.zeros_like(n["gain"]).double()).requires_grad_()
    if kind == "dropout":
        return torch.where(factor == 0, 0.0, s["x"].double() * factor)
    with torch.no_grad():
        if kind == "norm":
            y, stats = norm(s["x"].double(), s["pre"])
            return dict(out=y, pre=stats)
        gate = s["gate"].double() if s["gate"] is not None else None
        per = torch.arange(case["rows"], device="cuda") // max(case["gate_rows"], 1)
        if kind == "residual":
            out, v = {}, s["f"].double()
            if s["post"]:
                v, post = norm(v, s["post"])
            if gate is not None:
                v = v * (gate[per] if case["gate"] == "group" else gate)
            out["sum"] = case["alpha"] * s["h"].double() + case["beta"] * (v * factor)
            if s["pre"]:
                out["out"], out["pre"] = norm(out["sum"].to(s["sum"].dtype).double(), s["pre"])
            if s["post"]:
                out["post"] = post
            return out
    # gradients: autograd's of the definition
    out, x = {}, s["sum"].double().requires_grad_()
    total = s["dsum"].double() if s["dsum"] is not None else 0.0
    if s["pre"]:
        y, _ = norm(x, s["pre"])
        dx, dgain, dbias = torch.autograd.grad(y, [x, s["pre"]["gain64"], s["pre"]["bias64"]], s["dout"].double())
        del y
        total = total + dx
        out["dpre gain"] = s["dpre"]["gain"].double() + SAMPLES * dgain
        if "bias" in s["dpre"]:
            out["dpre bias"] = s["dpre"]["bias"].double() + SAMPLES * dbias
    out["dh"] = case["alpha"] * total
    if kind == "residual_grad":
        f, leaves = s["f"].double().requires_grad_(), []
        v = f
        if s["post"]:
            v, _ = norm(f, s["post"])
            leaves += [s["post"]["gain64"], s["post"]["bias64"]]
        if gate is not None:
            leaves.append(gate.requires_grad_())
            v = v * (gate[per] if case["gate"] == "group" else gate)
        v = v * factor * case["beta"]
        df, *grads = torch.autograd.grad(v, [f] + leaves, total)
        out["df"] = df
        if s["post"]:
            out["dpost gain"] = s["dpost"]["gain"].double() + SAMPLES * grads[0]
            if "bias" in s["dpost"]:
                out["dpost bias"] = s["dpost"]["bias"].double() + SAMPLES * grads[1]
        if gate is not None:
            out["dgate"] = grads[-1] if case["gate"] == "group" else s["dgate"].double() + SAMPLES * grads[-1]
    return {k: out[k].detach() for k in grad_outputs(s)}
