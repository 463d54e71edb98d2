"""Trains the token tables of a toy language model, answers from them in 8 bits and
generates from them in 4.

The model is its token interface alone: the embedding of a token is the hidden
state, a part of that of the one before it the residual stream, and they go
through the final norm into the LM head.  A training step makes every call a real model's
would:

  final norm            HeadNorm: s = x + r, h = norm(s)
  logits, their loss    a library product, a softmax
  back through the norm HeadNorm.grad
  gradients             dY^T h for the head, coalesced rows for the embedding
  clipping              GradClipper over both tables and the norm's gains
  steps                 EmberTable, the embedding's with its row count on the device

with no value read back to the host.  Answering takes the norm's 8-bit output and
the head in 8 bits (HeadQ8), which takes the table's present rows once after the steps
on it.  Generating holds both tables in 4 bits (HeadQ4): a step reads the last tokens' rows,
goes through the norm and the head and draws the next tokens (Sampler), all of it in one
HIP graph that is replayed for every token.

    python examples/token_interface.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_01455_amd import ember  # noqa: E402


class TokenInterface:
    BEFORE = 0.25    # of the embedding of the token before

    def __init__(self, V=2048, D=256, tokens=512, lr=0.02, max_norm=1.0, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.V, self.D, self.T, self.max_norm, self.lr = V, D, tokens, max_norm, lr
        bf = dict(dtype=torch.bfloat16, device=device)
        self.E = (torch.randn(V, D, generator=g, device=device) * 0.02).to(torch.bfloat16)
        self.W = (torch.randn(V, D, generator=g, device=device) * 0.02).to(torch.bfloat16)
        self.gain = torch.ones(D, device=device)
        self.follows = torch.randperm(V, generator=g, device=device)   # the language: what comes after a token
        self.norm = ember.HeadNorm(self.gain, max_tokens=tokens)
        self.head = ember.EmberTable(V, D, device=device, lr=lr)
        self.embedding = ember.EmberTable(V, D, device=device, lr=lr)
        self.head8 = ember.HeadQ8.from_table(self.W)
        self.head8_step = 0      # of the head's steps, that it was rounded after
        self.coalescer = ember.Coalescer(2 * tokens, V, D, device=device)
        self.G = torch.empty(V, D, **bf)
        self.S, self.H, self.dX = (torch.empty(tokens, D, **bf) for _ in range(3))
        self.rstd = torch.empty(tokens, device=device)
        self.dgain = torch.empty(D, device=device)
        self.clip = ember.GradClipper([self.G, self.coalescer.G_rows, self.dgain],
                                      counts=[None, self.coalescer.n_out, None])
        self.g = g

    def batch(self):
        """Token pairs and what follows them: a fixed successor of the later one, now and then anything."""
        before, token = (torch.randint(0, self.V, (self.T,), generator=self.g, device=self.E.device) for _ in range(2))
        target = self.follows[token]
        noise = torch.rand(self.T, generator=self.g, device=self.E.device) < 0.05
        target = torch.where(noise, torch.randint(0, self.V, (self.T,), generator=self.g, device=self.E.device), target)
        return before, token, target

    def step(self, before, token, target, lr=None):
        """One training step; returns the loss, a scalar on the device."""
        lr = self.lr if lr is None else lr
        self.head.lr = self.embedding.lr = lr
        X, R = self.E[token], self.E[before] * self.BEFORE
        self.norm(X, R, S=self.S, Y=self.H, rstd=self.rstd)
        logits = (self.H @ self.W.t()).float()
        logp = torch.log_softmax(logits, dim=1)
        at = torch.arange(self.T, device=X.device)
        dY = logp.exp()
        dY[at, target] -= 1.0
        dY = (dY / self.T).to(torch.bfloat16)

        self.norm.grad(dY @ self.W, self.S, self.rstd, self.dX, self.dgain)
        torch.mm(dY.t().contiguous(), self.H, out=self.G)
        # the sum's gradient is that of both embeddings it was made of
        co = self.coalescer
        co.enqueue(torch.cat([token, before]), torch.cat([self.dX, self.dX * self.BEFORE]))
        self.clip(self.max_norm)

        self.head.step(self.W, self.G)
        t = self.embedding
        ember.ember_step_sparse_rows_devn(self.E, co.G_rows, co.idx, co.n_out, t.r, t.c, t.t + 1, t.lr, t.beta2,
                                          t.eps, t.maximize, t.ws)
        t.t += 1
        self.gain.sub_(self.dgain, alpha=lr)
        return -logp[at, target].mean()

    def answer(self, before, token):
        """Logits of the next token for any number of pairs, from 8-bit states and an 8-bit head."""
        X, R = self.E[token], self.E[before] * self.BEFORE
        n = token.numel()
        S = torch.empty_like(X)
        Q = torch.empty(n, (self.D + 15) // 16 * 16, dtype=torch.int8, device=X.device)[:, :self.D]   # 16-byte rows
        scale = torch.empty(n, device=X.device)
        logits = torch.empty(n, self.V, dtype=torch.bfloat16, device=X.device)
        if self.head8_step != self.head.t:
            self.head8.load(self.W)
            self.head8_step = self.head.t
        self.norm(X, R, S=S, Q=Q, qscale=scale)
        self.head8.logits(Q, scale, logits)
        return logits

    def generate(self, before, token, u, temperature=None, top_k=None, top_p=None, min_p=None):
        """Tokens that follow n pairs, one after the other, from both tables in 4 bits: u (steps x n)
        holds the random numbers, the others are the sampler's, a value a sequence.  Returns the tokens and
        their log-probabilities, steps x n each."""
        steps, n = u.shape
        dev = self.E.device
        tables = [ember.HeadQ4.from_table(t, group=64) for t in (self.E, self.W)]
        sampler = ember.Sampler(n, self.V, device=dev)
        D8 = (self.D + 15) // 16 * 16
        X, R, S = (torch.empty(n, D8, dtype=torch.bfloat16, device=dev)[:, :self.D] for _ in range(3))     # 16-byte rows
        Q = torch.empty(n, D8, dtype=torch.int8, device=dev)[:, :self.D]
        L = torch.empty(n, (self.V + 7) // 8 * 8, dtype=torch.bfloat16, device=dev)[:, :self.V]
        scale, logp, u_now = (torch.empty(n, device=dev) for _ in range(3))
        last, ids = before.clone(), token.clone()
        norm = ember.HeadNorm(self.gain, eps=self.norm.eps)

        def step():
            tables[0].rows(ids, X)
            tables[0].rows(last, R)
            R.mul_(self.BEFORE)
            norm(X, R, S=S, Q=Q, qscale=scale)
            tables[1].logits(Q, scale, L)
            last.copy_(ids)
            sampler(L, u_now, ids, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, logp=logp)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        out, out_logp = torch.empty(steps, n, dtype=torch.int64, device=dev), torch.empty(steps, n, device=dev)
        for i in range(steps):
            u_now.copy_(u[i])
            graph.replay()
            out[i], out_logp[i] = ids, logp
        return out, out_logp


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    a = ap.parse_args()
    m = TokenInterface()
    for i in range(a.steps):
        loss = m.step(*m.batch(), lr=m.lr * (1 - i / a.steps))
        if i % 50 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {loss.item():.3f}, gradient norm {m.clip.norm.item():.3f}, "
                  f"factor {m.clip.factor.item():.3f}", flush=True)
    before, token, _ = m.batch()
    right = (m.answer(before, token).argmax(dim=1) == m.follows[token]).float().mean().item()
    one = m.answer(before[:1], token[:1]).argmax(dim=1).item()
    print(f"answers in 8 bits: {right:.3f} right; after token {token[0].item()} comes {one} "
          f"(the language's: {m.follows[token[0]].item()})")
    n, steps = 4, 8
    u = torch.rand(steps, n, generator=m.g, device=m.E.device)
    ids, logp = m.generate(before[:n], token[:n], u, top_p=torch.full((n,), 0.9, device=m.E.device))
    chain = torch.cat([token[None, :n], ids])
    right = (m.follows[chain[:-1]] == ids).float().mean().item()
    print(f"generated from tables in 4 bits: {ids[:, 0].tolist()}, {right:.3f} of {n} x {steps} as the language has them, "
          f"log-probability {logp.mean().item():.2f} a token")


if __name__ == "__main__":
    main()
