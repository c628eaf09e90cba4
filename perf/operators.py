"""The operators of a language model's training step that are timed one by one.

Four of them, through the public Python binding over libdedloc:

  orthogonalize  updates orthogonalised by Newton-Schulz products, several
                 matrices in a call;
  muon           the optimizer step built on it, on the flat vector of the
                 model's matrices, from an averaged gradient as the round
                 leaves it (fp32, or an fp16 or int8 message);
  embed          rows of an embedding table looked up and scaled;
  embed_grad     the gradient of that lookup, added into a peer's fp32
                 accumulator.

With `own` false, run() computes the same in elementary torch operations in
32 bits.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 1024  # elements to a scale of an int8 message
NS = dict(a=3.4445, b=-4.7750, c=2.0315, eps=1e-7, steps=5)
MUON = dict(lr=1e-3, momentum=0.95, weight_decay=0.01, rms=0.2)
TYPES = {"f32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # ALBERT's embedding projection alone: the smallest matrix of the model, launches count
        dict(name="orthogonalize projection bf16", kind="orthogonalize", shapes="128x1024", type="bf16", pad=0),
        # the tiny workload's eight tensors as matrices
        dict(name="orthogonalize tiny f32", kind="orthogonalize", shapes="8*256x512", type="f32", pad=0),
        # every matrix of ALBERT-large in one call
        dict(name="orthogonalize albert_large f32", kind="orthogonalize",
             shapes="1024x128,4*1024x1024,4096x1024,1024x4096,1024x1024", type="f32", pad=0),
        # odd and ragged matrices, tall and wide, rows at a stride (views into larger buffers)
        dict(name="orthogonalize ragged bf16", kind="orthogonalize",
             shapes="1000x2048,64x147,513x1025,1x3001,2x128,4097x301", type="bf16", pad=13),
        # the optimizer step of ALBERT-large on an fp16 message
        dict(name="muon albert_large fp16", kind="muon",
             shapes="1024x128,4*1024x1024,4096x1024,1024x4096,1024x1024", wire="fp16", nesterov=True),
        # ResNet-50's convolutions as matrices (output channels by the rest), fp32 gradient
        dict(name="muon resnet50 f32", kind="muon",
             shapes="64x147,64x64,3*64x576,4*256x64,2*64x256,128x256,4*128x1152,4*512x128,3*128x512,512x256,"
                    "256x512,6*256x2304,6*1024x256,5*256x1024,1024x512,512x1024,3*512x4608,3*2048x512,2*512x2048,"
                    "2048x1024,1000x2048", wire="f32", nesterov=True),
        # the largest: ALBERT-xlarge (hidden size 2048) on an int8 message
        dict(name="muon albert_xlarge i8", kind="muon",
             shapes="2048x128,4*2048x2048,8192x2048,2048x8192,2048x2048", wire="i8", nesterov=False),
        # a short sequence through ALBERT's table: latency
        dict(name="embed short f32", kind="embed", tokens=128, vocab=30000, width=128, table="f32", out="f32",
             index=64, masked=0.0, pad=0),
        # a large batch of long sequences
        dict(name="embed long bf16", kind="embed", tokens=131072, vocab=30000, width=2048, table="bf16", out="bf16",
             index=64, masked=0.05, pad=0),
        # one micro-batch of ALBERT-large: 16 sequences of 512 tokens, embedding size 128
        dict(name="embed_grad albert f32", kind="embed_grad", tokens=8192, vocab=30000, width=128, dy="f32",
             index=64, masked=0.0, pad=0),
        # odd sizes, rows at a stride, a quarter of the positions masked, 32-bit ids
        dict(name="embed_grad ragged fp16", kind="embed_grad", tokens=10007, vocab=50021, width=333, dy="fp16",
             index=32, masked=0.25, pad=7),
        # a large batch at a hidden size's width
        dict(name="embed_grad long bf16", kind="embed_grad", tokens=131072, vocab=30000, width=1024, dy="bf16",
             index=64, masked=0.05, pad=0),
    ]


def draw(rng):
    """One more case of the listed ones' ranges."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["orthogonalize", "muon", "embed", "embed_grad"])
    if kind in ("orthogonalize", "muon"):
        left, shapes = 8e11, []  # products; the largest listed case has 8.6e11
        for _ in range(log(1, 12)):
            rows, cols, many = log(1, 4096), log(16, 8192), rng.choice([1, 1, 1, log(1, 8)])
            if rng.random() < 0.5:  # multiples of 64, as models have them
                rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
            need = many * flops_of(rows, cols)
            if need <= left:
                left -= need
                shapes.append("%d*%dx%d" % ((many,) + ((rows, cols) if rng.random() < 0.5 else (cols, rows))))
        shapes = ",".join(shapes or ["256x512"])
        if kind == "muon":
            return dict(kind=kind, shapes=shapes, wire=rng.choice(["f32", "fp16", "i8"]), nesterov=rng.random() < 0.5)
        return dict(kind=kind, shapes=shapes, type=rng.choice(["f32", "bf16", "fp16"]), pad=rng.choice([0, 0, 8, 13]))
    width = log(16, 2048)
    if rng.random() < 0.5:
        width = max(64, width // 64 * 64)
    tokens = min(log(1, 131072), (1 << 28 if kind == "embed" else 1 << 27) // width)
    case = dict(kind=kind, tokens=tokens, vocab=log(1000, 262144), width=width, index=rng.choice([32, 64]),
                masked=rng.choice([0.0, 0.05, 0.3]), pad=rng.choice([0, 0, 8, 7]))
    if kind == "embed":
        case.update(table=rng.choice(["f32", "bf16", "fp16"]), out=rng.choice(["f32", "bf16", "fp16"]))
    else:
        case.update(dy=rng.choice(["f32", "bf16", "fp16"]))
    return case


def shapes_of(case):
    out = []
    for s in case["shapes"].split(","):
        many, _, one = s.rpartition("*")
        rows, cols = (int(v) for v in one.split("x"))
        out += [(rows, cols)] * int(many or 1)
    return out


def flops_of(rows, cols):
    """One matrix: a symmetric product of the short side over the long one, its square, and one full product."""
    s, l = min(rows, cols), max(rows, cols)
    return NS["steps"] * (3 * s * s * l + s ** 3)


def work(case):
    kind = case["kind"]
    if kind in ("orthogonalize", "muon"):
        n = sum(r * c for r, c in shapes_of(case))
        flops = sum(flops_of(r, c) for r, c in shapes_of(case))
        if kind == "orthogonalize":
            return dict(bytes=2 * n * (4 if case["type"] == "f32" else 2), flops=flops)
        wire = {"f32": 4.0, "fp16": 2.0, "i8": 1.0 + 4.0 / BLOCK}[case["wire"]]
        return dict(bytes=n * (16 + wire), flops=flops)
    n, width = case["tokens"], case["width"]
    kept = n * (1 - case["masked"])
    rows = sum_distinct(kept, case["vocab"])
    size = {"f32": 4, "fp16": 2, "bf16": 2}
    ids = n * case["index"] // 8
    if kind == "embed":
        return dict(bytes=int(rows * width * size[case["table"]] + n * width * size[case["out"]] + ids),
                    flops=n * width)
    return dict(bytes=int(kept * width * size[case["dy"]] + rows * width * 8 + ids), flops=int(kept * width))


def sum_distinct(n, vocab):
    """Distinct tokens expected among n whose rank is drawn log-uniformly over the vocabulary."""
    k = np.arange(vocab, dtype=np.float64)
    p = np.log((k + 2) / (k + 1)) / math.log(vocab + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-p))))


# ------------------------------------------------------------ inputs of a case

def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def gradient(rows, cols, g):
    """A matrix's mean gradient: strong directions, a sixteenth of the rank, over the noise of the samples."""
    r = max(1, min(rows, cols) // 16)
    u = torch.randn(rows, r, generator=g, device="cuda") * torch.logspace(0, -2, r, device="cuda")
    v = torch.randn(r, cols, generator=g, device="cuda")
    return (u @ v).mul_(1e-3).add_(torch.randn(rows, cols, generator=g, device="cuda"), alpha=1e-3)


def message(x, wire):
    """(codes, scales) of an averaged gradient as the wire formats define them."""
    if wire == "f32":
        return x, None
    if wire == "fp16":
        return x.half().view(torch.int16), None
    n = x.numel()
    pad = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    s = pad.abs().amax(1) / 127.0
    q = (pad / torch.where(s > 0, s, 1.0)[:, None]).round_().clamp_(-127, 127).to(torch.int8)
    return q.view(-1)[:n].clone(), s


def layout_of(case):
    """The flat vector of the case's matrices: [(offset, rows, cols)] and its length.  A matrix starts at a multiple
    of 8 elements, as the framework's tensor tables have it."""
    out, at = [], 0
    for r, c in shapes_of(case):
        out.append((at, r, c))
        at += -(-r * c // 8) * 8
    return out, at


def strided(rows, cols, pad, dtype):
    """A rows x cols view into a buffer whose rows are `pad` elements longer."""
    return torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def tokens_of(case, g):
    """Token ids with natural frequencies (rank drawn log-uniformly), spread over the table; -1 where masked."""
    n, V = case["tokens"], case["vocab"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    ids = rank * 7919 % V
    if case["masked"]:
        ids[torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
    return ids.int() if case["index"] == 32 else ids


def prepare(case, seed):
    kind, g = case["kind"], generator(seed)
    s = dict(kind=kind, case=case)
    if kind == "orthogonalize":
        dtype, shapes = TYPES[case["type"]], shapes_of(case)
        s["g"] = [strided(r, c, case["pad"], dtype).copy_(gradient(r, c, g)) for r, c in shapes]
        s["out"] = [strided(r, c, case["pad"], dtype) for r, c in shapes]
        if own:
            from paper_2106_10207_amd import dedloc as D
            s["call"] = D.OrthogonalizeCall(s["g"], s["out"], D.ortho_cfg(**NS))
    elif kind == "muon":
        s["layout"], P = layout_of(case)
        grad = torch.zeros(P, device="cuda")
        s["x"], s["m"] = torch.zeros(P, device="cuda"), torch.zeros(P, device="cuda")
        for at, r, c in s["layout"]:
            grad[at:at + r * c] = gradient(r, c, g).view(-1)
            s["m"][at:at + r * c] = gradient(r, c, g).view(-1)
            s["x"][at:at + r * c].normal_(std=0.02, generator=g)
        s["grad"], s["scales"] = message(grad, case["wire"])
        if own:
            from paper_2106_10207_amd import dedloc as D
            codec = {"f32": D.DEDLOC_CODEC_F32, "fp16": D.DEDLOC_CODEC_FP16, "i8": D.DEDLOC_CODEC_I8}[case["wire"]]
            cfg = D.muon_cfg(nesterov=case["nesterov"], ortho=D.ortho_cfg(**NS), **MUON)
            s["call"] = D.MuonCall(s["x"], s["m"], s["grad"], [at for at, _, _ in s["layout"]] + [P],
                                   [(r, c) for _, r, c in s["layout"]], [3] * len(s["layout"]), cfg, codec, s["scales"])
    else:
        n, width, pad = case["tokens"], case["width"], case["pad"]
        s["ids"] = tokens_of(case, g)
        s["scale"] = math.sqrt(width)
        if kind == "embed":
            s["table"] = strided(case["vocab"], width, pad, TYPES[case["table"]])
            s["table"].normal_(std=0.02, generator=g)
            s["out"] = strided(n, width, pad, TYPES[case["out"]])
        else:
            s["dy"] = strided(n, width, pad, TYPES[case["dy"]])
            s["dy"].normal_(std=1e-3, generator=g)
            s["samples"] = 16.0  # samples of the micro-batch: its weight in the accumulator
            # the accumulator after earlier micro-batches
            s["acc"] = torch.randn(case["vocab"], width, generator=g, device="cuda").mul_(1e-2)
            if own:
                from paper_2106_10207_amd import dedloc as D
                s["ws"] = D.make_embed_workspace(n, case["vocab"], width)
    return s


# -------------------------------------------------------------- the plain forms

def plain_orthogonalize(g):
    """Newton-Schulz steps towards the nearest matrix with orthogonal rows or columns, in 32 bits."""
    x = g.float()
    if x.shape[0] > x.shape[1]:
        x = x.t()
    x = x / (x.square().sum().sqrt() + NS["eps"])
    for _ in range(NS["steps"]):
        gram = x @ x.t()
        x = NS["a"] * x + (NS["b"] * gram + NS["c"] * (gram @ gram)) @ x
    return x.t() if g.shape[0] > g.shape[1] else x


def plain_decode(codes, scales, wire):
    if wire == "f32":
        return codes
    if wire == "fp16":
        return codes.view(torch.float16).float()
    n = codes.numel()
    return (torch.nn.functional.pad(codes.float(), (0, -n % BLOCK)).view(-1, BLOCK) * scales[:, None]).view(-1)[:n]


def plain_muon(s):
    x, m = s["x"], s["m"]
    grad = plain_decode(s["grad"], s["scales"], s["case"]["wire"])
    for at, r, c in s["layout"]:
        part = slice(at, at + r * c)
        m[part] = MUON["momentum"] * m[part] + grad[part]
        u = MUON["momentum"] * m[part] + grad[part] if s["case"]["nesterov"] else m[part]
        rate = MUON["lr"] * MUON["rms"] * math.sqrt(max(r, c))
        x[part] = (1 - MUON["lr"] * MUON["weight_decay"]) * x[part] - rate * plain_orthogonalize(u.view(r, c)).reshape(-1)
    return dict(x=x, m=m)


def plain_embed(s):
    table, ids = s["table"], s["ids"].long()
    named = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(named, ids, 0)].float() * s["scale"]
    s["out"].copy_(torch.where(named[:, None], rows, 0.0))
    return s["out"]


def plain_embed_grad(s):
    acc, ids = s["acc"], s["ids"].long()
    named = (ids >= 0) & (ids < acc.shape[0])
    total = torch.zeros_like(acc).index_add_(0, torch.where(named, ids, 0), s["dy"].float() * named[:, None])
    acc.add_(total, alpha=s["scale"] * s["samples"])
    return acc


def run(s):
    kind = s["kind"]
    if not own:
        if kind == "orthogonalize":
            for g, out in zip(s["g"], s["out"]):
                out.copy_(plain_orthogonalize(g))
            return s["out"]
        return {"muon": plain_muon, "embed": plain_embed, "embed_grad": plain_embed_grad}[kind](s)
    from paper_2106_10207_amd import dedloc as D
    if kind == "orthogonalize":
        s["call"]()
        return s["out"]
    if kind == "muon":
        s["call"]()
        return dict(x=s["x"], m=s["m"])
    if kind == "embed":
        return D.dedloc_embed(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    return D.dedloc_embed_grad(s["acc"], s["ids"], s["dy"], scale=s["scale"], batch_samples=s["samples"], ws=s["ws"])


# ------------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("orthogonalize", "muon"):
        def polar(u):
            """The same polynomial of the singular values, applied from the left by Horner's rule."""
            u = u.double()
            u = u / (torch.linalg.vector_norm(u) + NS["eps"])
            for _ in range(NS["steps"]):
                left = u.shape[0] <= u.shape[1]
                gram = u @ u.mT if left else u.mT @ u
                one = torch.eye(gram.shape[0], dtype=torch.float64, device=gram.device)
                poly = NS["a"] * one + gram @ (NS["b"] * one + NS["c"] * gram)
                u = poly @ u if left else u @ poly
            return u

        if kind == "orthogonalize":
            return [polar(g) for g in s["g"]]
        codes, scales, wire = s["grad"], s["scales"], case["wire"]
        if wire == "fp16":
            codes = codes.view(torch.float16)
        grad = codes.double()
        if wire == "i8":
            # a decoded element is one rounded 32-bit product
            grad = (codes.float() * scales.repeat_interleave(BLOCK)[:codes.numel()]).double()
        x, m, mu = s["x"].double(), s["m"].double(), MUON["momentum"]
        for at, r, c in s["layout"]:
            g = grad[at:at + r * c]
            m[at:at + r * c] = mu * m[at:at + r * c] + g
            u = mu * m[at:at + r * c] + g if case["nesterov"] else m[at:at + r * c]
            step = MUON["rms"] * max(r, c) ** 0.5 * polar(u.reshape(r, c)).reshape(-1)
            x[at:at + r * c] -= MUON["lr"] * (MUON["weight_decay"] * x[at:at + r * c] + step)
        return dict(x=x, m=m)
    if case["tokens"] * case["width"] > 1 << 27:
        return None
    ids = s["ids"].cpu().numpy()
    if kind == "embed":
        named = torch.from_numpy(ids[ids >= 0]).cuda().long()
        out = torch.zeros(len(ids), case["width"], dtype=torch.float64, device="cuda")
        out[torch.from_numpy(np.flatnonzero(ids >= 0)).cuda()] = s["scale"] * s["table"].double()[named]
        return out
    dy = s["dy"].double()
    acc = s["acc"].double()
    order = np.argsort(ids, kind="stable")
    order = torch.from_numpy(order[ids[order] >= 0]).cuda()
    if order.numel():
        tok = torch.from_numpy(ids).cuda().long()[order]
        sums = torch.cumsum(dy[order], 0)  # sums of runs of equal tokens, as differences of running sums
        last = torch.nonzero(torch.cat([tok[1:] != tok[:-1], tok.new_ones(1, dtype=torch.bool)])).view(-1)
        run_sum = sums[last]
        run_sum[1:] -= sums[last[:-1]]
        acc[tok[last]] += s["scale"] * s["samples"] * run_sum
    return acc
