"""A data-parallel training step of a small next-token model on one GPU, with
K workers as K gradient replicas:

  h = E[token], z = h M, logits = z U^T, loss = cross entropy with the next token

Each worker's gradients go straight into its replica: the table E's from
Embedding.grad, the vocabulary rows U's from CrossEntropy.loss_grad, the matrix
M's from a plain product.  Plan sums the replicas in reduction-tree order and
steps the two tables by momentum SGD; Muon steps the matrix from the same sum.

  python examples/lm_step.py [--steps 30]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1511_00175_amd as fc  # noqa: E402


class Model:
    """Weights, velocity and replicas as flat vectors in the framework's layout."""

    def __init__(self, vocab=512, dim=128, workers=4, tokens=1024, device="cuda:0", seed=0):
        self.vocab, self.dim, self.workers, self.tokens = vocab, dim, workers, tokens
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        table, square = vocab * dim, dim * dim
        self.places = {"E": (0, (vocab, dim)), "U": (table, (vocab, dim)), "M": (2 * table, (dim, dim))}
        self.total = 2 * table + square
        self.w = torch.randn(self.total, generator=g, device=device) * dim ** -0.5
        self.v = torch.zeros_like(self.w)
        self.replicas = torch.zeros((workers, self.total), device=device)
        self.sum = torch.zeros_like(self.w)
        # every worker's gradients are summed by one plan; the tables and the matrix are stepped by two
        self.reduce = fc.Plan([(0, self.total)], workers)
        self.tables = fc.Plan([(0, table), (table, table)], workers)
        self.matrix = fc.Muon([(2 * table, dim, dim)])
        self.embed = fc.Embedding(vocab, dim, tokens)
        self.xent = fc.CrossEntropy(vocab, dim, tokens, "f16")

    def part(self, flat, name):
        at, (rows, cols) = self.places[name]
        return flat[at:at + rows * cols].view(rows, cols)

    def gradients(self, worker, tokens, targets):
        """One worker's losses; its gradients' sums go into its replica."""
        E, U, M = (self.part(self.w, n).half() for n in ("E", "U", "M"))  # the 16-bit copies that the products read
        grad = self.replicas[worker]
        h, dz = (torch.empty((len(tokens), self.dim), dtype=torch.float16, device=self.w.device) for _ in range(2))
        loss = torch.empty(len(tokens), device=self.w.device)
        self.embed.lookup(E, tokens, h)
        z = h @ M
        self.xent.loss_grad(z, U, targets, loss, dz, self.part(grad, "U"))
        self.part(grad, "M").copy_(h.t() @ dz)
        self.embed.grad(dz @ M.t().contiguous(), tokens, self.part(grad, "E"))
        return loss

    def step(self, batches, lr=2.0, matrix_lr=0.02, mu=0.9, wd=1e-4):
        """One step on every worker's (tokens, targets); the mean loss."""
        losses = [self.gradients(k, *batch) for k, batch in enumerate(batches)]
        count = self.workers * self.tokens
        self.reduce.tree_reduce(self.replicas, self.sum)
        self.tables.sgd_step(self.w, self.v, self.sum, lr, mu, wd, count)
        self.matrix.step(self.w, self.v, self.sum, matrix_lr, mu, wd, count)
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
    a = ap.parse_args()
    model = Model()
    for k in range(a.steps):
        print(f"step {k:3d}  loss {float(model.step(batches(model, k))):.4f}", flush=True)


if __name__ == "__main__":
    main()
