"""examples/rollout.py: what its steps write one by one is what a model gives on the whole sequences at once."""
from __future__ import annotations

import importlib.util
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "rollout.py"
    spec = importlib.util.spec_from_file_location("rollout_example", path)
    m = importlib.util.module_from_spec(spec)
    import sys

    sys.modules[spec.name] = m  # (its dataclasses look themselves up)
    spec.loader.exec_module(m)
    return m


def test_rollouts(example, capsys):
    """The sampler's log-probs of the steps, against those of the whole sequence as one chain through a fresh cache, under the
    same cuts.  Both run the bf16 model: their logits differ by some bf16 steps of 2^-8 of their size (up to about 12)."""
    import torch

    B, turn_len, prompt = 6, 4, 21
    student, teacher, prompts, first, second = example.main(B=B, turn_len=turn_len, turns=3, prompt=prompt)
    assert "rollouts" in capsys.readouterr().out
    fresh = example.Model(student.s, B, 1)
    for b in range(B):
        tokens = torch.tensor(prompts[b].tolist() + first.tokens[b], dtype=torch.int32, device="cuda")
        n = len(tokens) - 1
        counts = torch.zeros(B, dtype=torch.int64, device="cuda")
        counts[b] = n
        ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
        logits = fresh(tokens[:-1].contiguous(), example.chain(ctx, counts), ctx, example.offsets(counts))
        x = logits[prompt - 1:].double() / 0.9
        x = x.masked_fill(x < x.topk(50, dim=1).values[:, -1:], float("-inf"))
        p, order = x.softmax(1).sort(dim=1, descending=True)
        p = torch.where(p.cumsum(1) - p < 0.95, p, 0.0)
        p = torch.zeros_like(p).scatter_(1, order, p / p.sum(1, keepdim=True))
        got = p.gather(1, tokens[prompt:].long()[:, None])[:, 0].log()
        want = torch.tensor(first.logp[b], dtype=torch.float64, device="cuda")
        finite = torch.isfinite(got)  # (a token at the cuts' edge may fall on either side)
        assert finite.double().mean() > 0.9
        assert (got - want)[finite].abs().max() < 0.25


def test_drafted_tree(example):
    """Logits of a tree's tokens equal those of each path taken as a chain, and the accepted path continues as if it had been."""
    import torch

    B = 5
    model, other = example.Model(example.Shape(), B, 1), example.Model(example.Shape(), B, 1)
    g = torch.Generator(device="cuda").manual_seed(4)
    prompts = torch.randint(0, 4096, (B, 30), generator=g, device="cuda").int()
    ctx, counts = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), 30, device="cuda")
    for m in (model, other):
        m(prompts.reshape(-1), example.chain(ctx, counts), ctx, example.offsets(counts))
    ctx += 30
    start = ctx.clone()
    last = torch.randint(0, 4096, (B,), generator=g, device="cuda").int()
    token, accepted, logits = example.draft_step(model, ctx, last, seed=1)
    guess = (model.embed[last.long()] @ model.head.T).topk(2, dim=1).indices.int()
    for j in range(2):  # last, guess j as a chain of two
        pair = torch.stack([last, guess[:, j]], 1).view(-1)
        two = torch.full((B,), 2, device="cuda")
        want = other(pair, example.chain(start, two), start, example.offsets(two))
        assert (want[::2].float() - logits[::3].float()).abs().max() < 0.2
        assert (want[1::2].float() - logits[1 + j::3].float()).abs().max() < 0.2
    assert torch.equal(ctx, start + 1 + (accepted > 0).int())
    # the next token over what was kept, against the kept tokens as a chain from the start
    nxt, one = token, torch.ones(B, dtype=torch.int64, device="cuda")
    got = model(nxt, example.chain(ctx, one), ctx, example.offsets(one))
    kept = [[int(last[b])] + ([int(guess[b, int(accepted[b]) - 1])] if accepted[b] else []) + [int(nxt[b])] for b in range(B)]
    n = torch.tensor([len(k) for k in kept], device="cuda")
    flat = torch.tensor([t for k in kept for t in k], dtype=torch.int32, device="cuda")
    want = other(flat, example.chain(start, n), start, example.offsets(n))[n.cumsum(0) - 1]
    assert (got.float() - want.float()).abs().max() < 0.2


def test_gradients(example):
    """The student's gradients with the kernels in its layers, against those with the plain norm and rotation in bf16 steps: a
    gradient that went through some tens of bf16 roundings (2^-8 each, of random sign) on either side is off by less than 0.05
    of its norm."""
    import torch

    def plain(q, k, qn, kn, pos, cos, sin):
        def one(x, w):
            y = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6) * w.float()
            a, b = y.chunk(2, dim=-1)
            c, s = cos[pos.long()][:, None], sin[pos.long()][:, None]
            return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)

        return one(q, qn), one(k, kn)

    model = example.Model(example.Shape(), 1, 1)
    tokens = torch.randint(0, 4096, (77,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").int()
    weights = [w.requires_grad_(True) for layer in model.layers for w in layer.values()]
    grads = []
    for qk in (example.QkNormRope.apply, plain):
        logp = example.sequence_logits(model, tokens, qk)[:-1].float().log_softmax(-1)
        grads.append(torch.autograd.grad(-logp.gather(1, tokens[1:].long()[:, None]).mean(), weights))
    for a, b in zip(*grads):
        assert (a.float() - b.float()).norm() <= 0.05 * b.float().norm()
