"""Calls on a stream of the caller's that make their own workspace and results:
tensors that the current stream allocates while such a call still waits must
not share its memory."""

import pytest

from paper_2106_10207_amd import dedloc as D

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DEV = "cuda"


def orthogonalize(stream):
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = torch.randn(200, 300, generator=gen, device=DEV)
    return g, lambda: D.dedloc_orthogonalize([g], stream=stream)[0]


def muon(stream):
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, m, g = torch.randn(3, 256 * 512, generator=gen, device=DEV)
    return (x, m, g), lambda: (D.dedloc_muon_step(x, m, g, [0, 256 * 512], [(256, 512)], [3], D.muon_cfg(), stream=stream), x)[1]


def embed(stream):
    gen = torch.Generator(device=DEV).manual_seed(3)
    table, ids = torch.randn(500, 128, generator=gen, device=DEV), torch.randint(0, 500, (3000,), generator=gen, device=DEV)
    return (table, ids), lambda: D.dedloc_embed(table, ids, 2.0, stream=stream)


def embed_grad(stream):
    gen = torch.Generator(device=DEV).manual_seed(4)
    ids = torch.randint(0, 500, (30000,), generator=gen, device=DEV)
    dy, acc = torch.randn(30000, 64, generator=gen, device=DEV), torch.zeros(500, 64, device=DEV)
    return (ids, dy), lambda: D.dedloc_embed_grad(acc, ids, dy, stream=stream)


@pytest.mark.parametrize("make", [orthogonalize, muon, embed, embed_grad])
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
