"""A small token model trained with the natural gradient: embedding, dropout, experts with a residual, a read-out layer.

    python examples/token_experts.py [--steps 30] [--dtype bf16]

The model learns a fixed map from tokens to tokens.  Every row h of the dropped-out embedding goes to two of the experts, chosen by
a fixed random projection, z = h + sum_j gate_j W_{e_j} h, and the read-out layer scores the classes.  Each layer has Kronecker
factors of its inputs and of the gradients at its outputs: the embedding a diagonal A (token frequencies) and a dense G, an expert
those of the rows that it received, the read-out those of a fully-connected layer.  The library does everything that touches the
embedding, the experts and the factors; the read-out's products, the softmax and the routing scores are torch's.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_06015_amd import kfac, workloads as wl  # noqa: E402

FAN = 2


class Model:
    def __init__(self, vocab=512, dim=64, experts=8, classes=512, tokens=4096, dtype=torch.float32, p=0.1, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.gen, self.vocab, self.dim, self.experts, self.classes, self.tokens = g, vocab, dim, experts, classes, tokens
        self.dtype, self.p, self.seed, self.step_no, self.scale = dtype, p, seed, 0, dim ** 0.5
        new = dict(device="cuda")
        n = tokens * FAN
        self.expert_layer, self.out_layer = wl.fc_layer(1, dim, dim, 0), wl.fc_layer(tokens, dim, classes, 0)
        # the inverse of the embedding's G, and its weights as a layer of the update
        self.table_g, self.table_layer = wl.fc_layer(tokens, 1, dim, 0), wl.fc_layer(1, dim, vocab, 0)
        rand = lambda *s: torch.randn(*s, generator=g, **new)  # noqa: E731
        self.table, self.W, self.Wout = rand(vocab, dim) / self.scale, rand(experts, dim, dim) * 0.5 / self.scale, rand(classes, dim) / self.scale
        self.router = rand(dim, experts)
        self.target_of = torch.randperm(max(vocab, classes), generator=g, **new)[:vocab] % classes
        self.previous = [w.clone() for w in (self.table, self.W, self.Wout)]
        # running averages and inverses
        self.A_table = torch.zeros(vocab, **new)
        self.A = [torch.zeros(experts, dim, dim, **new), torch.zeros(dim, dim, **new), torch.zeros(1, 1, **new)]
        self.G = [torch.zeros(experts, dim, dim, **new), torch.zeros(classes, classes, **new), torch.zeros(dim, dim, **new)]
        self.Ai, self.Gi = [torch.zeros_like(a) for a in self.A], [torch.zeros_like(b) for b in self.G]
        self.info = torch.zeros(2 * (experts + 2), dtype=torch.int32, **new)
        self.pi = torch.zeros(experts + 2, **new)
        # activations and gradients
        self.h, self.x0 = torch.empty(tokens, dim, dtype=dtype, **new), torch.empty(tokens, dim, dtype=dtype, **new)
        self.y, self.dy = torch.empty(n, dim, dtype=dtype, **new), torch.empty(n, dim, dtype=dtype, **new)
        self.dx, self.dx0 = torch.empty(n, dim, dtype=dtype, **new), torch.empty(tokens, dim, dtype=dtype, **new)
        self.dtable, self.dW = torch.empty(vocab, dim, **new), torch.empty(experts, dim, dim, **new)
        self.order, self.offsets = torch.empty(n, dtype=torch.int32, **new), torch.empty(experts + 1, dtype=torch.int32, **new)
        self.all_rows = torch.tensor([0, vocab], dtype=torch.int32, **new)
        self.layers = [self.expert_layer] * experts + [self.out_layer, self.table_g]
        need = max(kfac.kfac_workspace_bytes(self.layers), kfac.kfac_workspace_bytes([self.out_layer, self.table_layer]),
                   kfac.kfac_embedding_workspace_bytes(tokens, vocab, dim), kfac.kfac_segments_workspace_bytes(n, experts),
                   kfac.kfac_expert_workspace_bytes(self.expert_layer, experts, n))
        self.ctx = kfac.Context([self.expert_layer], workspace_bytes=need)

    def forward(self, ids):
        """The classes' scores [tokens, classes]."""
        kfac.kfac_embedding(self.ctx, ids, self.table, self.scale, self.x0)
        kfac.kfac_dropout(self.ctx, self.x0, self.p, self.seed, self.step_no, self.h)
        score = self.h.float() @ self.router
        best = score.topk(FAN, dim=1)
        self.gate, self.choice = best.values.softmax(1), best.indices.to(torch.int32).reshape(-1)
        kfac.kfac_segments(self.ctx, self.choice, self.experts, self.order, self.offsets)
        self.Wd = self.W.to(self.dtype)
        kfac.kfac_expert_forward(self.ctx, self.expert_layer, self.order, self.offsets, self.h, self.Wd, self.y, fan=FAN)
        self.z = self.h.float() + (self.gate[:, :, None] * self.y.float().view(self.tokens, FAN, self.dim)).sum(1)
        return self.z @ self.Wout.T

    def backward(self, ids, dlogits):
        """Gradients of the table, the experts and the read-out from those of every token's loss at its scores, summed over tokens."""
        dz = dlogits @ self.Wout
        self.dWout = dlogits.T @ self.z
        self.dy.copy_((self.gate[:, :, None] * dz[:, None, :]).view(-1, self.dim))
        kfac.kfac_expert_grad_input(self.ctx, self.expert_layer, self.order, self.offsets, self.dy, self.Wd, self.dx)
        kfac.kfac_expert_grad_weight(self.ctx, self.expert_layer, self.order, self.offsets, self.h, self.dy, self.dW, fan=FAN)
        dh = (dz + self.dx.float().view(self.tokens, FAN, self.dim).sum(1)).to(self.dtype)
        kfac.kfac_dropout(self.ctx, dh, self.p, self.seed, self.step_no, self.dx0)
        decay = 0.0 if self.step_no == 0 else 0.95
        kfac.kfac_embedding_grad(self.ctx, ids, self.dx0, self.scale, self.dtable, A_diag=self.A_table, decay=decay)
        return decay

    def statistics(self, dlogits, decay):
        kfac.kfac_stats_expert(self.ctx, self.expert_layer, self.order, self.offsets, self.h, self.dy, decay, self.A[0], self.G[0], fan=FAN)
        kfac.kfac_stats(self.ctx, [self.out_layer, self.table_g], kfac.KFAC_F32, [self.z, None], [dlogits, self.dx0.float() * self.scale], decay, False,
                        [self.A[1], None], [self.G[1], self.G[2]])
        self.A[2].copy_(self.A_table.mean().view(1, 1))      # the mean of the diagonal: what the split of the damping asks of A

    def step(self, ids, eta=0.3, momentum=0.5, gamma=0.03):
        """One iteration; returns the mean loss."""
        target = self.target_of[ids]
        logits = self.forward(ids)
        logp = logits.log_softmax(1)
        loss = -logp.gather(1, target[:, None]).mean()
        dlogits = logp.exp()
        dlogits.scatter_add_(1, target[:, None], torch.full((self.tokens, 1), -1.0, device="cuda"))
        decay = self.backward(ids, dlogits)
        self.statistics(dlogits, decay)
        E, c = self.experts, self.ctx
        A, G = list(self.A[0]) + self.A[1:], list(self.G[0]) + self.G[1:]
        Ai, Gi = list(self.Ai[0]) + self.Ai[1:], list(self.Gi[0]) + self.Gi[1:]
        kfac.kfac_invert(c, self.layers, A, G, gamma, Ai, Gi, self.pi, self.info)
        grads = list(self.dW / self.tokens) + [self.dWout / self.tokens]
        U = [torch.empty_like(w) for w in grads]
        kfac.kfac_precondition(c, self.layers[:E + 1], Gi[:E + 1], Ai[:E + 1], grads, U)
        # the table: rows over the diagonal of A, then the symmetric inverse of G as the weights of one expert that has all rows
        rows = self.dtable / self.tokens / (self.A_table + self.pi[E + 1] * gamma)[:, None]
        U_table = torch.empty_like(rows)
        kfac.kfac_expert_forward(c, self.expert_layer, None, self.all_rows, rows, self.Gi[2][None], U_table)
        kfac.kfac_update_weights(c, self.layers[:E] + [self.out_layer, self.table_layer], U + [U_table], eta, momentum, False, 0.0,
                                 list(self.W) + [self.Wout, self.table], list(self.previous[1]) + [self.previous[2], self.previous[0]])
        self.step_no += 1
        return loss

    def batch(self):
        return torch.randint(0, self.vocab, (self.tokens,), generator=self.gen, device="cuda")


def train(steps=30, **options):
    """The losses of `steps` iterations."""
    m = Model(**options)
    losses = [m.step(m.batch()) for _ in range(steps)]
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    a = ap.parse_args()
    for i, v in enumerate(train(a.steps, dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16)):
        print("step %3d  loss %.4f" % (i, v))
