"""A rollout engine in small: a student writes, a teacher scores every token as it
comes, rollouts whose running score falls below lambda stop, and restarts resume
from the cached prefix.  Random weights; every step of attention, cache, sampling
and scoring is the library's:

    projections -> stride_kv_append (norm, rotation, paged cache) -> stride_tree_attention
    -> logits -> stride_sample -> stride_score_step_compact -> (stop, restart)

The student then learns from what it wrote (the OPD loss over the kept tokens), with
stride_qk_norm_rope and its backward pass in its layers.

    python examples/rollout.py
"""
from __future__ import annotations

import sys
from dataclasses import dataclass, field
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2609_14636_gb300 as stride  # noqa: E402


@dataclass
class Shape:
    vocab: int = 4096
    width: int = 512
    layers: int = 2
    heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    page: int = 16
    longest: int = 512  # tokens of a sequence


class Model:
    """A decoder with normed, rotated queries and keys.  Sequences live in a paged cache of `slots` sequences; a call
    takes the new tokens of any of them."""

    def __init__(self, shape: Shape, slots: int, seed: int, device="cuda"):
        self.s, self.slots, self.device = shape, slots, device
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *n: (torch.randn(n, generator=g, device=device) * n[-1] ** -0.5).bfloat16()  # noqa: E731
        qkv = (shape.heads + 2 * shape.kv_heads) * shape.head_dim
        self.embed = torch.randn(shape.vocab, shape.width, generator=g, device=device).bfloat16()
        self.head = w(shape.vocab, shape.width) * 3
        self.layers = [dict(qkv=w(qkv, shape.width), out=w(shape.width, shape.heads * shape.head_dim), up=w(2 * shape.width, shape.width),
                            down=w(shape.width, 2 * shape.width), qn=1 + 0.1 * w(shape.head_dim), kn=1 + 0.1 * w(shape.head_dim))
                       for _ in range(shape.layers)]
        angle = torch.arange(shape.longest, device=device)[:, None] * 1e4 ** (-torch.arange(0, shape.head_dim, 2, device=device) / shape.head_dim)
        self.cos, self.sin = angle.cos(), angle.sin()
        pages = -(-shape.longest // shape.page)
        pool = (slots * pages, shape.page, shape.kv_heads, shape.head_dim)
        self.cache = [(torch.empty(pool, dtype=torch.bfloat16, device=device), torch.empty(pool, dtype=torch.bfloat16, device=device))
                      for _ in range(shape.layers)]
        self.table = torch.randperm(slots * pages, generator=g, device=device).int().view(slots, pages)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def __call__(self, tokens, position, ctx_len, tok_off, tree_mask=None):
        """Logits [N, vocab] of the new tokens; their keys and values are in the slots from each ctx_len on."""
        s, N = self.s, len(tokens)
        x, self.kv = self.embed[tokens.long()], []
        q_out = torch.empty(N, s.heads, s.head_dim, dtype=torch.bfloat16, device=self.device)
        out = torch.empty_like(q_out)
        work = torch.empty(stride.stride_tree_attention_workspace_size(N, s.heads, s.kv_heads, s.head_dim), dtype=torch.uint8, device=self.device)
        norm = lambda x: x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).bfloat16()  # noqa: E731
        for layer, (k_cache, v_cache) in zip(self.layers, self.cache):
            q, k, v = (norm(x) @ layer["qkv"].T).view(N, -1, s.head_dim).split([s.heads, s.kv_heads, s.kv_heads], dim=1)
            self.kv.append((k, v))
            stride.stride_kv_append(k, v, k_cache, v_cache, self.table, ctx_len, tok_off, pos=position, cos=self.cos, sin=self.sin,
                                    k_weight=layer["kn"], q=q, q_out=q_out, q_weight=layer["qn"], dev_status=self.status)
            stride.stride_tree_attention(q_out, k_cache, v_cache, self.table, ctx_len, tok_off, tree_mask, s.head_dim ** -0.5, out,
                                         workspace=work, dev_status=self.status)
            x = x + out.view(N, -1) @ layer["out"].T
            x = x + torch.nn.functional.silu(norm(x) @ layer["up"].T) @ layer["down"].T
        return norm(x) @ self.head.T

    def keep(self, rows, position, ctx_len, tok_off):
        """Writes the last call's tokens `rows` (an accepted path through a tree) from each ctx_len on."""
        for layer, (k, v), (k_cache, v_cache) in zip(self.layers, self.kv, self.cache):
            stride.stride_kv_append(k[rows], v[rows], k_cache, v_cache, self.table, ctx_len, tok_off, pos=position, cos=self.cos,
                                    sin=self.sin, k_weight=layer["kn"], dev_status=self.status)


def offsets(counts):
    return torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()


def chain(ctx_len, counts):
    """Positions of each sequence's next tokens."""
    rows = torch.repeat_interleave(torch.arange(len(counts), device=counts.device), counts)
    return (ctx_len.long()[rows] + torch.arange(len(rows), device=counts.device) - offsets(counts).long()[rows]).int()


@dataclass
class Rollouts:
    """What a call of roll() leaves of its B rollouts."""
    state: object
    tokens: list = field(default_factory=list)     # per rollout
    logp: list = field(default_factory=list)       # of the sampler, per rollout
    turn_mean: torch.Tensor = None                 # [B, turns], the turns that were closed
    turns: torch.Tensor = None


def roll(student, teacher, ctx_len, last, turn_len, turns, lam, seed, temperature=0.9, top_k=50, top_p=0.95):
    """Writes up to turns * turn_len tokens per rollout, one a step, from the cached prefixes; `last`: each one's last
    token, not in the cache yet.  ctx_len is moved on in place."""
    dev, B, V = ctx_len.device, len(ctx_len), student.s.vocab
    g = torch.Generator(device=dev).manual_seed(seed)
    r = Rollouts(stride.new_state(B), [[] for _ in range(B)], [[] for _ in range(B)], torch.zeros(B, turns, device=dev),
                 torch.zeros(B, dtype=torch.int32, device=dev))
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    live, last = torch.arange(B, device=dev), last.clone()
    for step in range(turns * turn_len):
        counts = torch.zeros(B, dtype=torch.int64, device=dev)
        counts[live] = 1
        tok_off, pos = offsets(counts), ctx_len[live].contiguous()
        s_logits, t_logits = (m(last[live], pos, ctx_len, tok_off) for m in (student, teacher))
        ctx_len += counts.int()
        n = len(live)
        token, logp = torch.empty(n, dtype=torch.int32, device=dev), torch.empty(n, device=dev)
        stride.stride_sample(s_logits, torch.empty(n, V, device=dev).exponential_(generator=g), token, temperature=temperature,
                             top_k=top_k, top_p=top_p, logp=logp, dev_status=status)
        closes = (step + 1) % turn_len == 0
        turn_end = torch.full((n,), int(closes), dtype=torch.uint8, device=dev)
        stopped, turn_out = torch.empty(n, dtype=torch.uint8, device=dev), stride.new_turn_stats(n)
        stride.stride_score_step_compact(s_logits, t_logits, token, turn_end, live.int(), stride.TURN_MEAN, lam, r.state,
                                         stopped_now=stopped, turn_out=turn_out, dev_status=status)
        last[live] = token
        for b, t, lp in zip(live.tolist(), token.tolist(), logp.tolist()):
            r.tokens[b].append(t)
            r.logp[b].append(lp)
        if closes:
            r.turn_mean[live, step // turn_len] = turn_out.view(torch.float32)[:n, 8]  # stride_turn_stats.mean_t
            r.turns[live] += 1
            live = live[stopped == 0]
            if not len(live):
                break
    assert int(status) == 0 and int(student.status) == 0 and int(teacher.status) == 0
    return r


def draft_step(model, ctx_len, last, seed):
    """One step with drafted continuations: after each rollout's last token two guesses at the next one (the likeliest by the
    embeddings alone) go through the model as a tree with it; where the sampled token is one of them, its own logits are
    there already.  Returns the sampled tokens and which of them were guessed; the accepted tokens are in the cache."""
    dev, B = ctx_len.device, len(ctx_len)
    guess = (model.embed[last.long()] @ model.head.T).topk(2, dim=1).indices.int()
    tree = torch.cat([last[:, None], guess], dim=1).view(-1)          # per rollout: last, guess, guess
    mask = torch.tensor([0b001, 0b011, 0b101], device=dev).repeat(B)
    counts = torch.full((B,), 3, dtype=torch.int64, device=dev)
    depth = torch.tensor([0, 1, 1], dtype=torch.int32, device=dev).repeat(B)
    pos = ctx_len.repeat_interleave(3) + depth
    logits = model(tree, pos, ctx_len, offsets(counts), mask)
    g = torch.Generator(device=dev).manual_seed(seed)
    token = torch.empty(B, dtype=torch.int32, device=dev)
    stride.stride_sample(logits[::3].contiguous(), torch.empty(B, model.s.vocab, device=dev).exponential_(generator=g), token, top_k=4)
    hit = guess == token[:, None]
    accepted = torch.where(hit[:, 0], 1, torch.where(hit[:, 1], 2, 0))  # the tree's row that is kept after the first
    rows = torch.stack([torch.arange(B, device=dev) * 3, torch.arange(B, device=dev) * 3 + accepted], 1)
    counts = torch.where(accepted > 0, 2, 1)
    keep = rows.view(-1)[(torch.arange(2, device=dev)[None] < counts[:, None]).view(-1)]
    model.keep(keep, pos[keep].contiguous(), ctx_len, offsets(counts))
    ctx_len += counts.int()
    return token, accepted, logits


class QkNormRope(torch.autograd.Function):
    """stride_qk_norm_rope where gradients flow; q, k [N, heads, D] of a layer, norm weights [D]."""

    @staticmethod
    def forward(ctx, q, k, qn, kn, pos, cos, sin):
        ctx.save_for_backward(q, k, qn, kn, pos, cos, sin)
        q_out, k_out = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        stride.stride_qk_norm_rope(q, k, q_out, k_out, pos, cos, sin, qn, kn)
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, qn, kn, pos, cos, sin = ctx.saved_tensors
        dq, dk = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
        dqn, dkn = (torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in (qn, kn))
        work = torch.empty(stride.stride_qk_norm_rope_backward_workspace_size(len(q), q.shape[1], k.shape[1], q.shape[2]), dtype=torch.uint8, device=q.device)
        stride.stride_qk_norm_rope_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, dq, dk, pos, cos, sin, qn, kn,
                                            dq_weight=dqn, dk_weight=dkn, workspace=work)
        return dq, dk, dqn.to(qn.dtype), dkn.to(kn.dtype), None, None, None


def sequence_logits(model, tokens, qk=QkNormRope.apply):
    """Logits [n, vocab] of one whole sequence, with gradients."""
    s, n = model.s, len(tokens)
    pos = torch.arange(n, dtype=torch.int32, device=tokens.device)
    x, rows = model.embed[tokens.long()], lambda t: t.transpose(0, 1)[None]
    norm = lambda x: x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).bfloat16()  # noqa: E731
    for layer in model.layers:
        q, k, v = (norm(x) @ layer["qkv"].T).view(n, -1, s.head_dim).split([s.heads, s.kv_heads, s.kv_heads], dim=1)
        q, k = qk(q, k, layer["qn"], layer["kn"], pos, model.cos, model.sin)
        y = torch.nn.functional.scaled_dot_product_attention(rows(q), rows(k), rows(v), is_causal=True, enable_gqa=True)
        x = x + y[0].transpose(0, 1).reshape(n, -1) @ layer["out"].T
        x = x + torch.nn.functional.silu(norm(x) @ layer["up"].T) @ layer["down"].T
    return norm(x) @ model.head.T


def learn(student, teacher, prompts, written, rate):
    """One step of gradient descent on the OPD loss, -logp_S (logp_T - logp_S) over the written tokens; returns the mean
    of logp_S - logp_T."""
    weights = [w for layer in student.layers for w in layer.values()]
    for w in weights:
        w.requires_grad_(True)
        w.grad = None
    total, n = 0.0, sum(map(len, written))
    for prompt, new in zip(prompts, written):
        tokens = torch.cat([prompt, torch.tensor(new, dtype=torch.int32, device=prompt.device)])
        at = slice(len(prompt) - 1, len(tokens) - 1)
        logp = lambda x: x[at].float().log_softmax(-1).gather(1, tokens[len(prompt):].long()[:, None])[:, 0]  # noqa: E731
        own = logp(sequence_logits(student, tokens))
        with torch.no_grad():
            d = own - logp(sequence_logits(teacher, tokens))
        (own * d).sum().div(n).backward()
        total += float(d.sum())
    with torch.no_grad():
        for w in weights:
            w -= rate * w.grad
            w.requires_grad_(False)
    return total / n


def main(B=16, turn_len=8, turns=6, prompt=40):
    shape = Shape()
    student, teacher = Model(shape, B, 1), Model(shape, B, 1)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(3)
    for a, b in zip(student.layers, teacher.layers):  # the teacher: a student that has moved a little
        for name in ("qkv", "down"):
            b[name] += 0.3 * torch.randn(b[name].shape, generator=g, device=dev).bfloat16() * a[name].std()
    prompts = torch.randint(0, shape.vocab, (B, prompt), generator=g, device=dev).int()
    ctx_len, counts = torch.zeros(B, dtype=torch.int32, device=dev), torch.full((B,), prompt - 1, device=dev)
    for m in (student, teacher):  # the prompts' first tokens, as chains
        m(prompts[:, :-1].reshape(-1), chain(ctx_len, counts), ctx_len, offsets(counts))
    ctx_len += counts.int()
    first = roll(student, teacher, ctx_len, prompts[:, -1].contiguous(), turn_len, turns, lam=-17.0, seed=5)
    stops = stride.state_to_numpy(first.state)["stop_turn"]
    print(f"{B} rollouts, {sum(map(len, first.tokens))} tokens, {int((stops >= 0).sum())} stopped early")

    # restart from the weakest turn: the tokens before it are in the cache already
    k_star, k_max = torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev)
    stride.stride_select_restart(first.turn_mean, first.turns, None, -17.0, k_star, k_max)
    reused = k_star * turn_len
    ctx_len.copy_(prompt - 1 + reused)
    last = torch.tensor([(prompts[b].tolist() + t)[prompt - 1 + int(n)] for b, (t, n) in enumerate(zip(first.tokens, reused.tolist()))],
                        dtype=torch.int32, device=dev)
    second = roll(student, teacher, ctx_len, last, turn_len, 2, lam=-17.0, seed=6)
    print(f"restarted after {reused.tolist()} reused tokens, {sum(map(len, second.tokens))} new ones")
    token, accepted, _ = draft_step(student, ctx_len, torch.tensor([t[-1] for t in second.tokens], dtype=torch.int32, device=dev), seed=7)
    print(f"drafted step: {int((accepted > 0).sum())} of {B} guesses accepted")
    gap = [learn(student, teacher, prompts, first.tokens, rate=0.02) for _ in range(2)]
    print(f"mean of log p_S - log p_T over the rollouts: {gap[0]:.4f}, after a step {gap[1]:.4f}")
    return student, teacher, prompts, first, second


if __name__ == "__main__":
    main()
