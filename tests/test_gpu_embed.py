"""dedloc_embed and dedloc_embed_grad against their definitions in 64 bits.

The lookup is one fp32 product rounded once more to a 16-bit output: it is
compared bit for bit with the same two roundings.  The gradient's tolerance: a
token's sum of k values in fp32 in any order is off by at most (k - 1) 2^-24
sum |dy|, the factor's product, the fma and the factor's own rounding add
3 * 2^-24 of the magnitudes."""

import numpy as np
import pytest

from paper_2106_10207_amd import dedloc as D

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def rows(n, width, dtype, seed, pad=0, offset=0, fill=float("nan")):
    """n rows of width, `pad` apart, `offset` elements into a buffer whose gaps hold `fill`."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.full((n * (width + pad) + offset + 1,), fill, dtype=dtype, device=DEV)
    v = buf[offset:offset + n * (width + pad)].view(n, width + pad)[:, :width]
    v.copy_(torch.randn(n, width, generator=g, device=DEV))
    return v, buf


def tokens(n, vocab, seed, kind="zipf", wide=True):
    rng = np.random.default_rng(seed)
    if kind == "zipf":
        ids = (np.exp(rng.random(n) * np.log(vocab + 1)) - 1).astype(np.int64).clip(0, vocab - 1)
    elif kind == "one":
        ids = np.full(n, vocab // 2)
    elif kind == "two":  # runs that cut every chunk, and one token between them
        ids = np.where(np.arange(n) % 3 == 0, 0, vocab - 1)
    else:  # "masked": nothing names a row
        ids = np.where(np.arange(n) % 2 == 0, -1, vocab)
    if kind == "zipf":
        out = rng.random(n) < 0.2
        ids[out] = rng.choice([-1, -7, vocab, vocab + 5, 2 ** 31 - 1, -2 ** 31], int(out.sum()))
        if wide and n:
            ids[rng.integers(0, n)] = 2 ** 32 + 1  # low half names a row
    return torch.from_numpy(ids.astype(np.int64 if wide else np.int32)).to(DEV)


def embed_ref(table, ids, scale, dtype):
    t, i = table.float().cpu(), ids.cpu().long()
    ok = (i >= 0) & (i < t.shape[0])
    r = t[torch.where(ok, i, 0)] * np.float32(scale)
    return torch.where(ok[:, None], r, 0.0).to(dtype)


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("table", TYPES)
@pytest.mark.parametrize("n,vocab,width,pad,offset", [(1, 1, 1, 0, 0), (1, 50, 128, 0, 0), (70, 33, 7, 0, 1),
                                                      (257, 100, 333, 5, 3), (64, 9, 2050, 1, 0), (5, 40, 4096, 0, 0)])
def test_embed(table, out, n, vocab, width, pad, offset):
    t, _ = rows(vocab, width, table, seed=n + width, pad=pad, offset=offset)
    ids = tokens(n, vocab, seed=n, wide=n % 2 == 1)
    o, buf = rows(n, width, out, seed=1, pad=pad + 1, offset=offset, fill=7.0)
    scale = float(np.sqrt(width))
    D.dedloc_embed(t, ids, scale, out=o)
    want = embed_ref(t, ids, scale, out)
    assert torch.equal(o.cpu(), want)
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[offset:offset + n * (width + pad + 1)].view(n, -1)[:, :width] = False
    assert bool((buf[rest] == 7.0).all())


def test_embed_infinities_stay_in_their_rows():
    t, _ = rows(4, 70, torch.float32, seed=1)
    t[2] = float("nan")
    t[3, 5] = float("inf")
    ids = torch.tensor([0, 2, -1, 3, 9, 1], device=DEV)
    o = D.dedloc_embed(t, ids, 2.0)
    assert bool(torch.isnan(o[1]).all()) and float(o[3, 5]) == float("inf")
    assert torch.equal(o[[0, 5]], 2 * t[[0, 1]]) and bool((o[[2, 4]] == 0).all())


def test_embed_empty():
    t, _ = rows(4, 8, torch.float32, seed=1)
    assert D.dedloc_embed(t, torch.zeros(0, dtype=torch.int64, device=DEV)).shape == (0, 8)
    none = torch.empty(0, 8, device=DEV)
    assert bool((D.dedloc_embed(none, torch.zeros(3, dtype=torch.int32, device=DEV)) == 0).all())
    acc = t.clone()
    D.dedloc_embed_grad(acc, torch.zeros(0, dtype=torch.int64, device=DEV), torch.empty(0, 8, device=DEV))
    assert torch.equal(acc, t)


def grad_case(dy_dtype, n, vocab, width, pad, offset, kind, wide, seed):
    dy, _ = rows(n, width, dy_dtype, seed=seed, pad=pad, offset=offset)
    acc, buf = rows(vocab, width, torch.float32, seed=seed + 1, pad=pad, offset=offset, fill=7.0)
    ids = tokens(n, vocab, seed, kind, wide)
    before = acc.double().cpu().numpy()
    ws = D.make_embed_workspace(n, vocab, width)
    ws.fill_(255)
    scale, samples = float(np.float32(np.sqrt(width))), 12.0
    D.dedloc_embed_grad(acc, ids, dy, scale, samples, ws)
    i, d = ids.cpu().numpy(), dy.double().cpu().numpy()
    ok = (i >= 0) & (i < vocab)
    total, size, count = (np.zeros_like(before) for _ in range(3))
    np.add.at(total, i[ok], d[ok])
    np.add.at(size, i[ok], np.abs(d[ok]))
    np.add.at(count, i[ok], 1.0)
    f = scale * samples
    got = acc.double().cpu().numpy()
    bound = 2.0 ** -24 * (f * size * (count + 2) + np.abs(before) + np.abs(before + f * total))
    assert (np.abs(got - (before + f * total)) <= bound).all()
    assert np.array_equal(got[count == 0], before[count == 0])
    rest = torch.ones_like(buf, dtype=torch.bool)
    rest[offset:offset + vocab * (width + pad)].view(vocab, -1)[:, :width] = False
    assert bool((buf[rest] == 7.0).all())


@pytest.mark.parametrize("dy", TYPES)
@pytest.mark.parametrize("n,vocab,width,pad,offset", [(1, 1, 1, 0, 0), (3, 2, 5, 0, 1), (31, 300, 64, 0, 0), (32, 7, 130, 3, 1),
                                                      (33, 255, 128, 0, 0), (64, 256, 33, 0, 0), (2047, 257, 9, 1, 0),
                                                      (2049, 65535, 40, 0, 0), (4500, 65536, 24, 0, 2),
                                                      (9000, 70000, 16, 0, 0), (700, 1 << 20, 4, 0, 0),
                                                      (100, 40, 1100, 0, 0), (16384, 40000, 2, 0, 0), (16385, 1000, 8, 0, 0), (70001, 3000, 3, 0, 0),
                                                      (16500, 100000, 3, 0, 0), (17000, 1000000, 2, 0, 0),
                                                      (17000, (1 << 21) + 5, 1, 0, 0)])
def test_embed_grad(dy, n, vocab, width, pad, offset):
    grad_case(dy, n, vocab, width, pad, offset, "zipf", n % 2 == 0, n)


@pytest.mark.parametrize("kind", ["one", "two", "masked"])
@pytest.mark.parametrize("n", [1, 32, 64, 65, 3000, 20000])
def test_embed_grad_runs(kind, n):
    """Every position of one token, long runs side by side, nothing but masked positions."""
    grad_case(torch.bfloat16, n, 500, 20, 0, 0, kind, True, n)


def test_embed_grad_same_bits():
    """Twice, on a workspace of other contents, through 32-bit ids: the same bits; NaN stays in its token's row."""
    ids = tokens(5000, 300, 3)
    dy, _ = rows(5000, 70, torch.bfloat16, seed=4)
    ids[17] = 299
    dy[17, 3] = float("nan")
    ws = D.make_embed_workspace(5000, 300, 70)
    out = []
    for fill in (0, 171):
        ws.fill_(fill)
        for i in (ids, ids.clamp(-1, 300).int()):
            out.append(D.dedloc_embed_grad(torch.zeros(300, 70, device=DEV), i, dy, 2.0, 3.0, ws))
    for o in out[1:]:
        assert torch.equal(o.view(torch.int32), out[0].view(torch.int32))
    bad = torch.isnan(out[0])
    assert bool(bad[299, 3]) and int(bad.sum()) == 1


def test_embed_grad_is_the_lookups_gradient():
    """Against differences of the lookup: L = sum(w * embed(table)) is linear in the table, so a difference of any
    width is its gradient but for roundings (fp32: 2^-20 of the sums' magnitudes)."""
    ids = tokens(60, 6, 9)
    table, _ = rows(6, 10, torch.float32, seed=2)
    w, _ = rows(60, 10, torch.float32, seed=3)
    scale = 1.75
    grad = D.dedloc_embed_grad(torch.zeros(6, 10, device=DEV), ids, w, scale, 1.0).cpu().double()

    def loss(t):
        return float((D.dedloc_embed(t, ids, scale).double() * w.double()).sum())

    size = float((D.dedloc_embed(table, ids, scale).double() * w.double()).abs().sum())
    for v in range(6):
        for c in range(10):
            up, down = table.clone(), table.clone()
            up[v, c] += 4.0
            down[v, c] -= 4.0
            step = float(up[v, c]) - float(down[v, c])
            assert abs((loss(up) - loss(down)) / step - float(grad[v, c])) <= 2.0 ** -20 * (size + 16 * 60)


def test_embed_graph_and_stream():
    """Lookup and gradient on another stream, and replayed in a graph with new ids between the replays."""
    vocab, width, n = 200, 48, 3000
    table, _ = rows(vocab, width, torch.float32, seed=5)
    dy, _ = rows(n, width, torch.float32, seed=6)
    sets = [tokens(n, vocab, k) for k in range(3)]
    want = []
    acc = torch.zeros(vocab, width, device=DEV)
    for ids in sets:
        out = D.dedloc_embed(table, ids, 3.0)
        D.dedloc_embed_grad(acc, ids, dy, 3.0, 2.0)
        want.append((out, acc.clone()))
    ids, out, acc, ws = sets[0].clone(), torch.empty(n, width, device=DEV), torch.zeros(vocab, width, device=DEV), \
        D.make_embed_workspace(n, vocab, width)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        D.dedloc_embed(table, ids, 3.0, out=out)
        D.dedloc_embed_grad(acc, ids, dy, 3.0, 2.0, ws)
    for new, (o, g) in zip(sets, want):
        ids.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(acc, g)
        (acc * 2).sum().item()
    s = torch.cuda.Stream()
    acc = torch.zeros(vocab, width, device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    for new, (o, g) in zip(sets, want):
        D.dedloc_embed(table, new, 3.0, out=out, stream=s)
        D.dedloc_embed_grad(acc, new, dy, 3.0, 2.0, ws, stream=s)
        s.synchronize()
        assert torch.equal(out, o) and torch.equal(acc, g)
        torch.cuda.synchronize()


def test_lookup_of_more_rows_than_a_grid_takes():
    """2^23 rows of 256 threads make 2^31 threads; the rows after them, and 16 GiB of output."""
    n, vocab, width = (1 << 23) + 5, 300, 1021
    gen = torch.Generator(device=DEV).manual_seed(3)
    table = torch.randn(vocab, width, generator=gen, device=DEV)
    ids = torch.randint(-1, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    out = D.dedloc_embed(table, ids, 0.5, out_dtype=torch.bfloat16)
    rows = torch.cat([0.5 * table, torch.zeros(1, width, device=DEV)]).to(torch.bfloat16)  # row -1: zeros
    for i in range(0, n, 1 << 20):
        assert torch.equal(out[i:i + (1 << 20)], rows[ids[i:i + (1 << 20)].long()])


def test_gradient_of_more_chunks_than_a_grid_takes():
    """2^24 + 31 chunks of 32 positions.  Sums of ones below 2^24 are exact in fp32, whatever their order."""
    n, vocab = (1 << 29) + 1000, 1 << 20
    gen = torch.Generator(device=DEV).manual_seed(4)
    ids = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    ids[:1 << 22] = 5
    acc = torch.zeros(vocab, 1, device=DEV)
    D.dedloc_embed_grad(acc, ids, torch.ones(n, 1, dtype=torch.float16, device=DEV), 2.0, 3.0)
    want = torch.zeros(vocab, dtype=torch.int64, device=DEV)
    for i in range(0, n, 1 << 26):
        want += torch.bincount(ids[i:i + (1 << 26)], minlength=vocab)
    assert int(want.max()) < 1 << 24 and torch.equal(acc[:, 0].double(), 6.0 * want.double())


@pytest.mark.parametrize("vocab", [(1 << 24) - 1, 1 << 24, (1 << 24) + 5, 1 << 30])
@pytest.mark.parametrize("n", [1, 100, 3000, 16384, 17000])
def test_embed_grad_of_tokens_past_24_bits(n, vocab):
    """Three or four digits of 8 bits in the short sorts, of 8 or 9 in the long one.  Sums of small integers are exact in
    fp32, whatever their order."""
    rng = np.random.default_rng(n)
    ends = np.concatenate([np.arange(5), vocab - 1 - np.arange(5), [vocab // 2, (1 << 24) - 1, (1 << 16), 255, 256]])
    ids = np.where(rng.random(n) < 0.5, rng.choice(ends, n), rng.integers(0, vocab, n))
    ids = np.where(rng.random(n) < 0.1, rng.choice([-1, vocab, vocab + 3, -vocab], n), ids)
    if n == 1:
        ids[:] = vocab - 1
    dy = rng.integers(-3, 4, (n, 1))
    acc = torch.zeros(vocab, 1, device=DEV)
    D.dedloc_embed_grad(acc, torch.from_numpy(ids).to(DEV), torch.from_numpy(dy).half().to(DEV), 2.0, 3.0)
    ok = (ids >= 0) & (ids < vocab)
    named, place = np.unique(ids[ok], return_inverse=True)
    want = 6.0 * np.bincount(place, dy[ok, 0], len(named))
    assert np.array_equal(acc[torch.from_numpy(named).to(DEV), 0].double().cpu().numpy(), want)
    assert int(torch.count_nonzero(acc)) == np.count_nonzero(want)


@pytest.mark.parametrize("n,width", [(8192, 128), (32768, 256), (32768, 1024)])
def test_one_workspace_for_fewer_positions_and_narrower_rows(n, width):
    """A last micro-batch that is shorter, on the workspace of the others, whose end nothing passes.  A token's values
    are small integers, so that its sum is exact."""
    vocab = 700
    gen = torch.Generator(device=DEV).manual_seed(n)
    size = D.make_embed_workspace(n, vocab, width).numel()
    buf = torch.full((size + 4096,), 171, dtype=torch.uint8, device=DEV)
    ws = buf[:size]
    for k, w in ((n, width), (n - 1, width), (n // 2, width), (4353, width), (n - 1, width - 1), (n // 2 + 1, width // 2), (3, 5)):
        ids = torch.randint(-1, vocab, (k,), generator=gen, device=DEV)
        ids[k // 3: k // 2] = 5  # runs over many chunks
        dy = torch.randint(-8, 9, (k, w), generator=gen, device=DEV).to(torch.bfloat16)
        acc = D.dedloc_embed_grad(torch.zeros(vocab, w, device=DEV), ids, dy, 2.0, 3.0, ws)
        want = torch.zeros(vocab + 1, w, dtype=torch.float64, device=DEV)
        want.index_add_(0, torch.where(ids < 0, vocab, ids), dy.double())
        assert torch.equal(acc.double(), 6.0 * want[:vocab])
        assert bool((buf[size:] == 171).all())
