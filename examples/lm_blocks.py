"""A data-parallel training step of a next-token model with residual blocks on one
GPU, with K workers as K gradient replicas:

  h = E[token], y = N(h) * v0
  block i: b = y W_i^T, h += s * sigmoid(g_i) * v_i * N(b), y = N(h) * u_i
  loss = cross entropy of y U^T with the next token

The residual h is fp32, the blocks' side fp16.  The blocks' products, forward and
for their inputs' gradient, are of 4-bit numbers (Mxfp4); each block's input is kept
in 8 bits (Checkpoint), from which its weight's gradient is taken; norms, gates and
residuals and their gradients are Norm's.  As in lm_step.py, every gradient goes
straight into the worker's replica, Plan sums the replicas in reduction-tree order
and steps tables and vectors, Muon steps the matrices.

  python examples/lm_blocks.py [--steps 30] [--blocks 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1511_00175_amd as fc  # noqa: E402

SCALE = 0.5  # of a block's residual


class Model:
    """Weights, velocity and replicas as flat vectors in the framework's layout."""

    def __init__(self, vocab=512, dim=128, blocks=2, workers=4, tokens=1024, device="cuda:0", seed=0):
        self.vocab, self.dim, self.blocks, self.workers, self.tokens = vocab, dim, blocks, workers, tokens
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        shapes = {"E": (vocab, dim), "U": (vocab, dim), "v": (dim,)}  # v: the first norm's weight
        for i in range(blocks):
            shapes.update({f"v{i}": (dim,), f"g{i}": (dim,), f"u{i}": (dim,)})
        shapes.update({f"W{i}": (dim, dim) for i in range(blocks)})
        self.places, at = {}, 0
        for name, shape in shapes.items():
            self.places[name] = at, shape
            at += -(-torch.Size(shape).numel() // 4) * 4
        self.total = at
        self.w = torch.zeros(at, device=device)
        for name in shapes:
            p = self.part(self.w, name)
            p.copy_(torch.randn(p.shape, generator=g, device=device) * dim ** -0.5 if p.dim() > 1 else
                    torch.zeros_like(p) if name[0] == "g" else torch.ones_like(p))
        self.v, self.sum = torch.zeros_like(self.w), torch.zeros_like(self.w)
        self.replicas = torch.zeros((workers, at), device=device)
        # every worker's gradients are summed by one plan; tables and vectors, and the matrices, are stepped by two
        self.reduce = fc.Plan([(0, at)], workers)
        self.rest = fc.Plan([(p, torch.Size(s).numel()) for n, (p, s) in self.places.items() if n[0] != "W"], workers)
        self.matrices = fc.Muon([(p, *s) for n, (p, s) in self.places.items() if n[0] == "W"])
        self.embed = fc.Embedding(vocab, dim, tokens)
        self.xent = fc.CrossEntropy(vocab, dim, tokens, "f16")
        self.norm = fc.Norm(dim, tokens, "f16", "f32", gate="sigmoid")
        self.keep = fc.Checkpoint(dim, tokens, dim, "f16")
        self.four = fc.Mxfp4(dim, dim, tokens)

    def part(self, flat, name):
        at, shape = self.places[name]
        return flat[at:at + torch.Size(shape).numel()].view(shape)

    def gradients(self, worker, tokens, targets):
        """One worker's losses; its gradients' sums go into its replica."""
        n, dim, dev = len(tokens), self.dim, self.w.device
        w = {name: self.part(self.w, name) for name in self.places}
        grad = {name: self.part(self.replicas[worker], name) for name in self.places}
        half, full = (lambda: torch.empty((n, dim), dtype=torch.float16, device=dev)), (lambda: torch.empty((n, dim), device=dev))

        h, y, loss = full(), half(), torch.empty(n, device=dev)
        self.embed.lookup(w["E"], tokens, h)
        self.norm.before(h, y, weight=w["v"])
        kept, first = [], h
        weight = self.four.empty(dim)
        for i in range(self.blocks):
            b, out, codes, then = half(), full(), self.keep.empty(n), half()
            self.keep.pack(y, *codes)
            self.four.pack(w[f"W{i}"], *weight)
            self.four.linear(y, *weight, b)
            self.norm.between(h, b, out, then, weight=w[f"v{i}"], gate=w[f"g{i}"], next_weight=w[f"u{i}"], scale=SCALE)
            kept.append((codes, b, out))
            h, y = out, then

        dy, dh, U = half(), None, w["U"].half()
        self.xent.loss_grad(y, U, targets, loss, dy, grad["U"])
        for i in reversed(range(self.blocks)):
            codes, b, out = kept.pop()
            db, dx, before = half(), full(), half()
            self.norm.between_grad(out, b, dy, dx, db, dout=dh, weight=w[f"v{i}"], dweight=grad[f"v{i}"], gate=w[f"g{i}"],
                                   dgate=grad[f"g{i}"], next_weight=w[f"u{i}"], dnext=grad[f"u{i}"], scale=SCALE)
            self.keep.grad(db, *codes, grad[f"W{i}"])
            self.four.pack(w[f"W{i}"], *weight, transpose=True)
            self.four.linear(db, *weight, before)
            dh, dy = dx, before
        dx = full()
        self.norm.before_grad(first, dy, dx, dout=dh, weight=w["v"], dweight=grad["v"])
        self.embed.grad(dx, tokens, grad["E"])
        return loss

    def step(self, batches, lr=1.0, matrix_lr=0.02, mu=0.9, wd=1e-4):
        """One step on every worker's (tokens, targets); the mean loss."""
        losses = [self.gradients(k, *batch) for k, batch in enumerate(batches)]
        count = self.workers * self.tokens
        self.reduce.tree_reduce(self.replicas, self.sum)
        self.rest.sgd_step(self.w, self.v, self.sum, lr, mu, wd, count)
        self.matrices.step(self.w, self.v, self.sum, matrix_lr, mu, wd, count)
        return torch.cat(losses).mean()


def batches(model, seed):
    """Text in which a token mostly says what comes next; a few positions are
    padding."""
    g = torch.Generator(device=model.w.device)
    g.manual_seed(seed)

    def uniform(high):
        return torch.randint(0, high, (model.tokens,), generator=g, device=model.w.device)

    got = []
    for _ in range(model.workers):
        tokens = uniform(model.vocab)
        targets = torch.where(uniform(10) == 0, uniform(model.vocab), (7 * tokens + 3) % model.vocab)
        got.append((tokens, torch.where(uniform(50) == 0, -1, targets)))
    return got


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--blocks", type=int, default=2)
    a = ap.parse_args()
    model = Model(blocks=a.blocks)
    for k in range(a.steps):
        print(f"step {k:3d}  loss {float(model.step(batches(model, k))):.4f}", flush=True)


if __name__ == "__main__":
    main()
