"""A small language model trained by a collaboration, with every step of the
training around the model in the library.

Each peer looks its tokens up (dedloc_embed), runs the model's own layers
(plain torch here), and adds its gradients into its accumulator: the table's
by the lookup's gradient (dedloc_embed_grad), the matrices' by
dedloc_accumulate.  When the global batch is full the peers' messages
(dedloc_finalize) are averaged (dedloc_reduce_shard), and the averaged
message updates the one set of parameters all peers share: the matrices by
Muon (dedloc_muon_step), the table and the gains by LAMB (dedloc_lamb_step).

The flat vector holds the matrices first, then the rest, so that each
optimizer takes its part of the vector and of the message.

    python examples/train_lm.py [--rounds 60] [--peers 4]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2106_10207_amd import dedloc as D  # noqa: E402

VOCAB, WIDTH, HIDDEN = 500, 64, 128
MATRICES = [(HIDDEN, 2 * WIDTH), (VOCAB, HIDDEN)]  # two tokens in, one out
REST = [VOCAB * WIDTH, HIDDEN]                     # the embedding table, the hidden layer's gain
SCALE = WIDTH ** 0.5
MASK = -1                                          # a position before the text: no row, no gradient


class Model:
    """The parameters, shared by the peers, in one flat vector, and the optimizers' state."""

    def __init__(self, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.split = sum(r * c for r, c in MATRICES)
        self.x = torch.randn(self.split + sum(REST), generator=g, device=device) * 0.05
        self.x[-HIDDEN:] = 1.0
        self.momentum = torch.zeros(self.split, device=device)
        self.m, self.v = (torch.zeros(sum(REST), device=device) for _ in range(2))
        self.matrix_offsets, self.rest_offsets = [0], [0]
        for r, c in MATRICES:
            self.matrix_offsets.append(self.matrix_offsets[-1] + r * c)
        for n in REST:
            self.rest_offsets.append(self.rest_offsets[-1] + n)
        self.ws_muon = D.make_muon_workspace(MATRICES, device)
        self.ws_lamb = D.make_workspace(sum(REST), self.rest_offsets, device)

    def views(self, flat):
        """(first matrix, second matrix, table, gain) of a flat vector."""
        o = self.matrix_offsets
        return (flat[:o[1]].view(MATRICES[0]), flat[o[1]:o[2]].view(MATRICES[1]),
                flat[self.split:self.split + REST[0]].view(VOCAB, WIDTH), flat[-HIDDEN:])

    def gradients(self, ids, target, acc):
        """The mean loss of a micro-batch (ids: [samples, 2], MASK where there is
        no token); its gradients, times the samples, are added into acc."""
        w1, w2, table, gain = (p.detach() for p in self.views(self.x))
        rows = D.dedloc_embed(table, ids, SCALE).requires_grad_()
        params = [p.clone().requires_grad_() for p in (w1, w2, gain)]
        hidden = torch.tanh(rows.view(len(ids), 2 * WIDTH) @ params[0].t()) * params[2]
        loss = torch.nn.functional.cross_entropy(hidden @ params[1].t(), target)
        loss.backward()
        a1, a2, a_table, a_gain = self.views(acc)
        for a, p in zip((a1, a2, a_gain), params):
            D.dedloc_accumulate(a.reshape(-1), p.grad.reshape(-1), len(ids))
        D.dedloc_embed_grad(a_table, ids, rows.grad, SCALE, len(ids))
        return float(loss.detach())

    def update(self, message, step, lr=0.02):
        """One step from the averaged fp16 message."""
        D.dedloc_muon_step(self.x[:self.split], self.momentum, message[:self.split], self.matrix_offsets, MATRICES,
                           [3] * len(MATRICES), D.muon_cfg(lr=lr, weight_decay=0.01), D.DEDLOC_CODEC_FP16, ws=self.ws_muon)
        D.dedloc_lamb_step(self.x[self.split:], self.m, self.v, message[self.split:], self.rest_offsets, [3, 2],
                           D.lamb_cfg(lr=lr, weight_decay=0.01, step=step), D.DEDLOC_CODEC_FP16, ws=self.ws_lamb)


def text(samples, generator):
    """Two tokens of a text and the one that follows: a fixed rule of the two."""
    ids = torch.randint(0, VOCAB, (samples, 2), generator=generator, device=generator.device)
    ids[:, 0][torch.rand(samples, generator=generator, device=generator.device) < 0.1] = MASK
    return ids, (3 * ids[:, 1] + 7) % VOCAB


def train(rounds=60, peers=4, micro_batches=2, samples=256, device="cuda", seed=1):
    """The mean loss of every round."""
    model, losses = Model(device), []
    accs = [torch.zeros_like(model.x) for _ in range(peers)]
    gens = [torch.Generator(device=device).manual_seed(seed + p) for p in range(peers)]
    for step in range(1, rounds + 1):
        total = 0.0
        for acc, gen in zip(accs, gens):
            for _ in range(micro_batches):
                total += model.gradients(*text(samples, gen), acc)
        counts = [micro_batches * samples] * peers
        messages = [D.dedloc_finalize(acc, n, D.DEDLOC_CODEC_FP16)[0] for acc, n in zip(accs, counts)]
        mean, _ = D.dedloc_reduce_shard(messages, counts, model.x.numel(), D.DEDLOC_CODEC_FP16)
        model.update(mean, step)
        losses.append(total / (peers * micro_batches))
    return losses


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--rounds", type=int, default=60)
    p.add_argument("--peers", type=int, default=4)
    a = p.parse_args()
    for i, loss in enumerate(train(a.rounds, a.peers)):
        if i % 5 == 0 or i + 1 == a.rounds:
            print(f"round {i + 1:3d}  loss {loss:.4f}", flush=True)
