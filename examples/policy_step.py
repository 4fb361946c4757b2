"""A trainer's step from tokens to receivers, on the framework's operators.

A minimal policy (embedding, one hidden matrix, output layer) is kept as the
framework keeps any trainer state: one flat binary32 shard of weights and its
moments.  Each step

  embedding -> hidden matrix -> linear cross entropy     (train.embedding, linear_ce)
  their gradients, one weight per token's loss           (train.linear_ce_grad, embedding_grad)
  AdamW on the two vocabulary tables                     (dte_adamw_forward)
  Muon on the hidden matrix                              (train.muon_forward)
  the BF16-visible change, without a snapshot, into the  (DeltaPipeline: extract, remap, apply)
  shards of two tensor-parallel receivers

The hidden layer's own products are torch's.  The Muon range is inverted like
the AdamW ranges, with the update in place of the first moment and ones in
place of the second (train.MuonStep.inverse).

    python examples/policy_step.py [--steps 20] [--vocab 6002] [--hidden 256] [--tokens 1024]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_00455_amd import binding as B  # noqa: E402
from paper_2608_00455_amd import train  # noqa: E402
from paper_2608_00455_amd.layouts import Piece, PlanSpec, SenderSeg, SPiece, View  # noqa: E402
from paper_2608_00455_amd.pipeline import DeltaPipeline  # noqa: E402
from synth.workloads import StepHP  # noqa: E402


def receiver_plan(vocab, hidden, ranks=2):
    """Vocabulary rows of both tables and input columns of the matrix split
    over the receivers."""
    shapes = [("embed", (vocab, hidden)), ("matrix", (hidden, hidden)), ("head", (vocab, hidden))]
    begins, pos = [], 0
    for _, s in shapes:
        begins.append(pos)
        pos += math.prod(s)
    senders = [SenderSeg(n, s, [SPiece((0, 0), s, k, (0, 0))]) for k, (n, s) in enumerate(shapes)]
    views, numel = [], []
    for r in range(ranks):
        at, mine = 0, []
        for k, (n, (rows, cols)) in enumerate(shapes):
            split = (rows, cols // ranks) if n == "matrix" else (rows // ranks, cols)
            lo = (0, r * split[1]) if n == "matrix" else (r * split[0], 0)
            mine.append((at, View(n, split, [Piece(k, lo, split, (0, 0))])))
            at += math.prod(split)
        views.append(mine)
        numel.append(at)
    return PlanSpec([(b, s) for b, (_, s) in zip(begins, shapes)], views, numel, senders)


class Policy:
    def __init__(self, vocab, hidden, lr=1e-3, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.hidden = vocab, hidden
        self.scale = math.sqrt(hidden)          # of the embedding's rows
        n = vocab * hidden
        self.ranges = {"embed": (0, n), "matrix": (n, n + hidden ** 2),
                       "head": (n + hidden ** 2, 2 * n + hidden ** 2)}
        total = 2 * n + hidden ** 2
        self.p = 0.02 * torch.randn(total, generator=gen, device=device)
        self.p[slice(*self.ranges["matrix"])] *= 1.0 / (0.02 * math.sqrt(hidden))
        self.m, self.v, self.g = (torch.zeros_like(self.p) for _ in range(3))
        self.ones = torch.ones(hidden ** 2, device=device)
        self.step_no = 0
        self.adamw = StepHP(lr=lr, weight_decay=0.01, step=1)
        self.muon = train.MuonStep(lr=lr, update_scale=0.2 * math.sqrt(hidden))
        self.pipe = DeltaPipeline(receiver_plan(vocab, hidden), capacity=total)
        self.publish_dense()

    def part(self, t, name):
        b, e = self.ranges[name]
        return t[b:e].view(-1, self.hidden)

    def publish_dense(self):
        """The receivers' first weights."""
        rows = self.vocab // 2
        cols = self.hidden // 2
        for r, shard in enumerate(self.pipe.shards):
            w = {n: self.part(self.p, n).bfloat16() for n in self.ranges}
            shard.copy_(torch.cat([w["embed"][r * rows:(r + 1) * rows].reshape(-1),
                                   w["matrix"][:, r * cols:(r + 1) * cols].reshape(-1),
                                   w["head"][r * rows:(r + 1) * rows].reshape(-1)]).view(
                                       torch.int16))

    def step(self, tokens, targets, weights, temperature=1.0):
        """One step on tokens and targets (int64 [T]; -1 is padding) with one
        weight per token's loss; returns the losses and the number of BF16
        weights that changed."""
        w = self.p.bfloat16()
        E, M, H = (self.part(w, n) for n in ("embed", "matrix", "head"))
        x = train.embedding(E, tokens, scale=self.scale)
        h = x @ M.t()
        loss, lse = train.linear_ce(h, H, targets, scale=1.0 / temperature)
        gh, _ = train.linear_ce_grad(h, H, targets, lse, weights, self.part(self.g, "head"),
                                     scale=1.0 / temperature)
        self.part(self.g, "matrix").copy_(gh.t() @ x)
        train.embedding_grad(gh @ M, tokens, self.part(self.g, "embed"), scale=self.scale)

        self.step_no += 1
        hp = StepHP(lr=self.adamw.lr, weight_decay=self.adamw.weight_decay, step=self.step_no)
        s = torch.cuda.current_stream().cuda_stream
        for name in ("embed", "head"):
            b, e = self.ranges[name]
            B.dte_adamw_forward(*(t[b:].data_ptr() for t in (self.p, self.m, self.v, self.g)),
                                e - b, hp, s)
        update = train.muon_forward(*(self.part(t, "matrix") for t in (self.p, self.m, self.g)),
                                    self.muon)

        self.pipe.reset()
        for name in ("embed", "matrix", "head"):
            b, e = self.ranges[name]
            if name == "matrix":
                self.pipe.extract(self.p[b:e], update.float().view(-1), self.ones,
                                  self.muon.inverse(), index_base=b)
            else:
                self.pipe.extract(self.p[b:e], self.m[b:e], self.v[b:e], hp, index_base=b)
        self.pipe.remap()
        self.pipe.apply()
        return loss, int(self.pipe.cursor.item())

    def stale(self):
        """Receiver weights that differ from the trainer's in BF16."""
        old = [s.clone() for s in self.pipe.shards]
        self.publish_dense()
        return sum(int((a != b).sum()) for a, b in zip(old, self.pipe.shards))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--vocab", type=int, default=6002)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=1024)
    a = ap.parse_args()
    policy = Policy(a.vocab, a.hidden)
    gen = torch.Generator(device="cuda").manual_seed(1)
    weights = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")
    for k in range(a.steps):
        tokens = torch.randint(0, 64, (a.tokens,), generator=gen, device="cuda")
        loss, changed = policy.step(tokens, (tokens * 31 + 7) % a.vocab, weights)
        print("step %2d  loss %.4f  changed %d of %d (%.2f %%)" % (
            k, float(loss.mean()), changed, policy.p.numel(), 100.0 * changed / policy.p.numel()),
            flush=True)
    print("receiver weights that differ from the trainer's: %d" % policy.stale())


if __name__ == "__main__":
    main()
