"""Answering token by token from tables in 4 bits: rows, the final norm in 8 bits, logits and
sampling one after the other, as a program calls them, and the example that does so."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F = torch.bfloat16, torch.float32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def em():
    from paper_2607_01455_amd import ember
    return ember


class Chain:
    def __init__(self, em, V, D, group, T, seed, dtype=BF):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.V, self.D, self.T = V, D, T
        W, E = (self.mat(V, D, BF).copy_(torch.randn(V, D, generator=g, device=DEV) * s) for s in (0.3, 0.02))
        bias = torch.randn(V, generator=g, device=DEV)
        self.head, self.embed = em.HeadQ4.from_table(W, group, bias), em.HeadQ4.from_table(E, group)
        self.norm = em.HeadNorm(0.5 + torch.rand(D, generator=g, device=DEV))
        self.sampler = em.Sampler(T, V)
        self.X, self.R, self.S = (self.mat(T, D, BF) for _ in range(3))
        self.R.copy_(torch.randn(T, D, generator=g, device=DEV) * 0.02)
        self.Q, self.L = self.mat(T, D, torch.int8), self.mat(T, V, dtype)
        self.scale, self.logp = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        self.ids = torch.randint(0, V, (T,), generator=g, device=DEV)
        self.kept = torch.empty(T, dtype=torch.int32, device=DEV)
        self.u = torch.rand(T, generator=g, device=DEV)
        self.ask = dict(temperature=torch.full((T,), 0.7, device=DEV), top_p=torch.full((T,), 0.9, device=DEV),
                        top_k=torch.full((T,), 100, dtype=torch.int32, device=DEV))

    @staticmethod
    def mat(rows, cols, dtype):
        q = 16 // torch.empty(0, dtype=dtype).element_size()
        return torch.zeros(rows, (cols + q - 1) // q * q, dtype=dtype, device=DEV)[:, :cols]

    def step(self):
        self.embed.rows(self.ids, self.X)
        self.norm(self.X, self.R, S=self.S, Q=self.Q, qscale=self.scale)
        self.head.logits(self.Q, self.scale, self.L)
        self.sampler(self.L, self.u, self.ids, logp=self.logp, kept=self.kept, **self.ask)


@pytest.mark.parametrize("V,D,group,T,dtype", [(3000, 200, 64, 1, BF), (20000, 1000, 128, 3, F), (9000, 513, 32, 20, BF),
                                               (33000, 256, 64, 70, F)])
def test_every_link_reads_what_the_one_before_wrote(em, V, D, group, T, dtype):
    """Each output against float64 from the step's own inputs: none is read before it is written,
    on one stream with no wait in between."""
    print(f"answer V={V} D={D} group={group} T={T} {dtype}", flush=True)
    c = Chain(em, V, D, group, T, V, dtype)
    E, W = c.mat(V, D, F), c.mat(V, D, F)
    c.embed.rows(None, E)
    c.head.rows(None, W)
    for i in range(3):
        before = c.ids.clone()
        c.step()
        torch.cuda.synchronize()
        assert torch.equal(c.X, E[before].to(BF))
        s = c.X.double() + c.R.double()
        y = s * (s.square().mean(dim=1, keepdim=True) + c.norm.eps).rsqrt() * c.norm.gain.double()
        top = y.abs().amax(dim=1, keepdim=True)
        # codes to the nearest of 127 steps; fp32 may tip one over
        assert ((c.Q.double() * c.scale.double()[:, None] - y).abs() <= top / 127 * 0.5001).all()
        want = c.Q.double() * c.scale.double()[:, None] @ W.double().t().contiguous() + c.head.bias.double()
        size = (c.Q.double().abs() * c.scale.double()[:, None]) @ W.double().abs().t().contiguous() + c.head.bias.double().abs()
        n = (D + group - 1) // group
        bar = 2.0 ** -24 * (2 * n + 5) * size + (2.0 ** -8 * want.abs() if dtype == BF else 0)
        assert ((c.L.double() - want).abs() <= bar).all()
        for t in range(T):
            l = c.L[t].double().cpu()
            e = torch.exp((l - l.max()) / c.ask["temperature"][t].item())
            order = torch.argsort(l, descending=True, stable=True)[:100]
            w = e[order]
            order = order[torch.cumsum(w, 0) - w < c.ask["top_p"][t].item() * w.sum()]
            left = torch.sort(order).values
            run = torch.cumsum(e[left], 0)
            at = left[int((run <= c.u[t].item() * run[-1]).sum())]
            assert c.ids[t].item() == at.item() and c.kept[t].item() == len(left)
        c.u.copy_(torch.rand(T, device=DEV))


def test_a_captured_step_is_the_eager_one(em):
    """A graph of the whole step, replayed with eager steps of another chain on the same tables between."""
    a, b = (Chain(em, 20000, 384, 128, 5, 7) for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i in range(6):
        u = torch.rand(5, device=DEV)
        a.u.copy_(u)
        b.u.copy_(u)
        graph.replay()
        b.step()
        if i % 2:
            torch.cuda.synchronize()
        for x in ("X", "S", "Q", "scale", "L", "ids", "logp", "kept"):
            assert torch.equal(getattr(a, x), getattr(b, x)), (i, x)


def test_a_row_without_a_token_stays_without(em):
    """A sequence whose state is not finite has NaN logits, so no token (-1), and -1 gives a row of NaN
    again; its neighbours go on."""
    c, d = (Chain(em, 5000, 200, 64, 4, 9) for _ in range(2))
    c.R[2, 7] = float("inf")
    for i in range(3):
        c.step()
        d.step()
        torch.cuda.synchronize()
        assert c.ids[2] == -1 and torch.isnan(c.L[2].float()).all() and torch.isnan(c.logp[2])
        rest = [0, 1, 3]
        assert torch.equal(c.ids[rest], d.ids[rest]) and torch.equal(c.L[rest], d.L[rest])
        if i == 0:
            c.R[2] = d.R[2]
    assert torch.isnan(c.X[2].float()).all()


def test_one_table_for_both_ends(em):
    """A head and an embedding that are one table: the largest logit of a token's own row is its own."""
    c = Chain(em, 2000, 256, 128, 8, 3, F)
    c.embed, c.norm = c.head, em.HeadNorm(torch.ones(256, device=DEV))
    c.head.bias = None
    c.R.zero_()
    start = c.ids.clone()
    c.ask = dict(temperature=torch.zeros(8, device=DEV))
    c.step()
    assert torch.equal(c.ids, start) and (c.kept == 1).all()


def test_generating_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import token_interface
    finally:
        sys.path.pop(0)
    m = token_interface.TokenInterface(V=1024, D=104, tokens=256, max_norm=0.3)
    before, token, _ = m.batch()
    n, steps = 5, 6
    u = torch.rand(steps, n, device=DEV)
    ids, logp = m.generate(before[:n], token[:n], u, top_k=torch.full((n,), 50, dtype=torch.int32, device=DEV))
    assert ids.shape == (steps, n) and ((ids >= 0) & (ids < 1024)).all()
    assert torch.isfinite(logp).all() and (logp <= 0).all()
    again, _ = m.generate(before[:n], token[:n], u, top_k=torch.full((n,), 50, dtype=torch.int32, device=DEV))
    assert torch.equal(ids, again)
    greedy, _ = m.generate(before[:n], token[:n], u, temperature=torch.zeros(n, device=DEV))
    other, _ = m.generate(before[:n], token[:n], 1 - u.clamp(min=0.01), temperature=torch.zeros(n, device=DEV))
    assert torch.equal(greedy, other)          # without temperature the random numbers do not matter
