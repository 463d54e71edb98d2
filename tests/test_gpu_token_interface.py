"""The example that trains a toy model's token tables and answers in 8 bits: its
loss falls, its gradients are clipped to the limit, and the 8-bit answers are
those of the unrounded ones."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_token_interface_learns_and_answers():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import token_interface
    finally:
        sys.path.pop(0)
    m = token_interface.TokenInterface(V=1024, D=104, tokens=256, max_norm=0.3)
    losses, clipped = [], 0
    for i in range(150):
        before = [t.clone() for t in (m.E, m.W)] if i == 0 else None
        losses.append(m.step(*m.batch(), lr=0.02 * (1 - i / 150)).item())
        n = torch.linalg.vector_norm(torch.cat([m.G.double().reshape(-1), m.dgain.double(),
                                                m.coalescer.G_rows[:int(m.coalescer.n_out)].double().reshape(-1)]))
        assert n.item() <= 0.3 * (1 + 2.0 ** -7)     # rounded to bf16 once clipped
        clipped += m.clip.factor.item() < 1.0
        if before is not None:
            assert not torch.equal(before[0], m.E) and not torch.equal(before[1], m.W)
    print("losses", losses[0], losses[-1], "steps clipped", clipped, flush=True)
    assert clipped > 0
    assert sum(losses[-10:]) / 10 < 0.25 * losses[0]
    before, token, _ = m.batch()
    logits = m.answer(before, token).float()
    X, R = m.E[token].float(), (m.E[before] * m.BEFORE).float()
    s = X + R
    y = s * torch.rsqrt(s.square().mean(dim=1, keepdim=True) + m.norm.eps) * m.gain
    plain = y @ m.W.float().t()
    # rounding y and W to 8 bits moves a logit by about sqrt(D) rounding errors of each: a few percent of its scale
    assert (logits - plain).square().mean().sqrt() <= 0.03 * plain.square().mean().sqrt()
    assert (logits.argmax(dim=1) == plain.argmax(dim=1)).float().mean() >= 0.95
    assert (logits.argmax(dim=1) == m.follows[token]).float().mean() >= 0.9
    # one token at a time gives what the batch gives
    for i in (0, 100, 255):
        assert torch.equal(m.answer(before[i:i + 1], token[i:i + 1]), m.answer(before, token)[i:i + 1])


def test_answers_round_the_head_once_after_its_steps(monkeypatch):
    """The 8-bit head is made of the table once for any number of answers, and anew after a step."""
    from paper_2607_01455_amd import ember
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import token_interface
    finally:
        sys.path.pop(0)
    m = token_interface.TokenInterface(V=512, D=64, tokens=128)
    before, token, target = m.batch()
    rounded = []
    quantize = ember.ember_quantize_rows
    monkeypatch.setattr(ember, "ember_quantize_rows", lambda *a: (rounded.append(1), quantize(*a)))
    first = m.answer(before, token)
    assert torch.equal(m.answer(before, token), first) and len(rounded) <= 1
    m.step(before, token, target)
    rounded.clear()
    after = m.answer(before, token)
    assert torch.equal(m.answer(before, token), after) and len(rounded) == 1
    fresh = ember.HeadQ8.from_table(m.W)
    assert torch.equal(m.head8.Wq, fresh.Wq) and torch.equal(m.head8.wscale, fresh.wscale)
    assert not torch.equal(after, first)
