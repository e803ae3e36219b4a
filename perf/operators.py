"""The measured cases of the decode-step operators: what a rollout engine and a trainer ask of them.

Four kinds of pass:

* ``qk``      norms of queries and keys per head with the position rotation, forward and backward: a training step's
              (stride_qk_norm_rope, stride_qk_norm_rope_backward);
* ``append``  keys and values into a paged cache, norm and rotation on the way, the queries with them
              (stride_kv_append);
* ``attn``    attention of drafted tokens, a chain or a tree, over the paged cache (stride_tree_attention);
* ``sample``  tokens from logits with temperature, top-k, top-p and min-p (stride_sample).

The plain forms are elementary torch operations in 32 bits, rounded once at the end.  ``exact`` states the same
definitions in 64 bits, per sequence or row, apart from them.
"""
import math

import numpy as np
import torch

own = False

V0 = 151_936  # the vocabulary of the repository's bf16 workloads
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
MAX_KV = 256 * 2100 * 8 * 128  # cached elements of K that a drawn case reads at most
MAX_PAIRS = 4 * 511 * 32 * 6700 * 128  # multiply-adds of a drawn case's scores


def listed():
    return [
        # A training step's queries and keys: views of the fused projection, rotary halves, bf16.
        dict(name="qk_train_16384", kind="qk", tokens=16_384, Hq=32, Hk=8, D=128, R=128, norm=True, inter=False, dtype="bf16"),
        # An odd number of tokens and heads, 96 components of which 64 rotate in interleaved pairs, fp32.
        dict(name="qk_odd_1021_f32", kind="qk", tokens=1021, Hq=9, Hk=3, D=96, R=64, norm=True, inter=True, dtype="f32"),
        # One decode step of 256 rollouts: a token each.  Latency counts.
        dict(name="append_256_steps", kind="append", seqs=256, new=1, Hq=32, Hk=8, D=128, R=128, page=16, ctx=512,
             norm=True, inter=False, heads_first=False, dtype="bf16"),
        # Restarted rollouts: their prefixes' tokens go into the cache, pages ordered heads first.
        dict(name="append_13_restarts", kind="append", seqs=13, new=640, Hq=28, Hk=4, D=128, R=128, page=64, ctx=700,
             norm=False, inter=False, heads_first=True, dtype="bf16"),
        # The smallest call: one rollout's one token over a few cached ones.
        dict(name="attn_1x1_short", kind="attn", seqs=1, new=1, tree=False, Hq=16, Hk=2, D=128, page=16, ctx=37,
             ragged=False, heads_first=False, dtype="bf16"),
        # A decode step of 256 rollouts of unequal lengths.
        dict(name="attn_256_steps", kind="attn", seqs=256, new=1, tree=False, Hq=32, Hk=8, D=128, page=16, ctx=4096,
             ragged=True, heads_first=False, dtype="bf16"),
        # One long agentic trajectory: few rows, a long axis.
        dict(name="attn_1_long", kind="attn", seqs=1, new=1, tree=False, Hq=32, Hk=8, D=128, page=64, ctx=131_072,
             ragged=False, heads_first=True, dtype="bf16"),
        # Drafted trees of up to 13 tokens over unequal prefixes.
        dict(name="attn_32_trees_13", kind="attn", seqs=32, new=13, tree=True, Hq=32, Hk=8, D=128, page=16, ctx=8000,
             ragged=True, heads_first=False, dtype="bf16"),
        # A restart's new observation tokens, a chain, over the reused prefix: arithmetic counts.
        dict(name="attn_4_chains_511", kind="attn", seqs=4, new=511, tree=False, Hq=32, Hk=8, D=128, page=32, ctx=6000,
             ragged=True, heads_first=False, dtype="bf16"),
        # The last live rollout's token.
        dict(name="sample_1", kind="sample", rows=1, V=V0, ld=V0, dtype="bf16", sharp=True, cut="mixed"),
        # A step's tokens of 256 rollouts, each row with parameters of its own.
        dict(name="sample_256_mixed", kind="sample", rows=256, V=V0, ld=V0, dtype="bf16", sharp=True, cut="mixed"),
        # The tiny reference's logits, nothing cut off.
        dict(name="sample_512_f32_all", kind="sample", rows=512, V=32_000, ld=32_000, dtype="f32", sharp=False, cut="none"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["qk", "append", "attn", "attn", "attn", "sample", "sample"])
    if kind == "sample":
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        V = rng.choice([V0, V0, 32_000, _log_int(rng, 1000, 152_064)])
        if rng.random() < 0.3:
            V -= rng.randint(1, 7)  # rows that no vector divides ...
        ld = V if rng.random() < 0.6 else (V + 63) // 64 * 64  # ... packed, or padded to aligned rows
        return dict(kind=kind, rows=_log_int(rng, 1, 300), V=V, ld=ld, dtype=dtype, sharp=rng.random() < 0.7,
                    cut=rng.choice(["mixed", "mixed", "top_k", "top_p", "min_p", "none"]))
    Hk = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 3, 4, 4, 7, 8])
    if kind == "qk":
        D = rng.choice([64, 128, 128, 96, 80, 256])
        return dict(kind=kind, tokens=max(1, _log_int(rng, 1, 16_384) * 128 // (D * max(1, Hk * (G + 1) // 40))), Hq=Hk * G, Hk=Hk,
                    D=D, R=D if rng.random() < 0.7 else D // 4 * 2, norm=rng.random() < 0.8, inter=rng.random() < 0.3,
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    D = rng.choice([128, 128, 64])
    page = rng.choice([16, 32, 64, 24])
    first = rng.random() < 0.5
    dtype = rng.choice(["bf16", "bf16", "f16"])
    seqs = _log_int(rng, 1, 256)
    if kind == "append":
        return dict(kind=kind, seqs=seqs, new=_log_int(rng, 1, max(1, 8320 // seqs)), Hq=Hk * G, Hk=Hk, D=D,
                    R=D if rng.random() < 0.7 else D // 2, page=page, ctx=rng.randint(1, 700), norm=rng.random() < 0.6,
                    inter=rng.random() < 0.3, heads_first=first, dtype=dtype)
    ctx = _log_int(rng, 16, 131_072)
    what = rng.choice(["one", "one", "tree", "chain"])
    new = 1 if what == "one" else rng.randint(2, 64) if what == "tree" else _log_int(rng, 2, 511)
    while seqs > 1 and (seqs * ctx * Hk * D > MAX_KV or seqs * new * Hk * G * (ctx + new) * D > MAX_PAIRS):
        seqs = (seqs + 1) // 2 if seqs > 2 else 1
    while ctx * Hk * D > MAX_KV or new * Hk * G * (ctx + new) * D > MAX_PAIRS:
        ctx = ctx // 2
    return dict(kind=kind, seqs=seqs, new=new, tree=what == "tree", Hq=Hk * G, Hk=Hk, D=D, page=page, ctx=ctx,
                ragged=rng.random() < 0.7, heads_first=first, dtype=dtype)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _lengths(case, seed):
    """Cached and new tokens per sequence.  Unequal ones reach from nothing cached to the case's longest; the case sets
    the lengths (outputs of all seeds have one shape), the seed which sequence has which."""
    B, ctx, new = case["seqs"], case["ctx"], case["new"]
    rng = np.random.default_rng([B, ctx, new])
    n_ctx = np.full(B, ctx, np.int64)
    n_new = np.full(B, new, np.int64)
    if case.get("ragged", True):
        n_ctx = (ctx * np.sqrt(rng.random(B))).astype(np.int64) * (rng.random(B) > 0.02)
        n_ctx[0] = ctx
        if new > 1:
            n_new = np.maximum(1, new - rng.integers(0, max(1, new // 3) + 1, B))
    at = np.random.default_rng([seed, 3]).permutation(B)
    return n_ctx[at], n_new[at]


def _cache(case, seed, n_ctx, n_new, g, dev):
    """A page pool in random order, its block table, and the two caches of it, [pages, page, heads, D] as views."""
    page, Hk, D, dt = case["page"], case["Hk"], case["D"], DT[case["dtype"]]
    need = -(-(n_ctx + n_new) // page)
    pool = int(need.sum()) + 3
    rng = np.random.default_rng([seed, 5])
    perm, table, at = rng.permutation(pool).astype(np.int32), np.full((len(need), int(need.max())), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    shape = (pool, Hk, page, D) if case["heads_first"] else (pool, page, Hk, D)
    kv = []
    for _ in range(2):
        c = torch.empty(shape, dtype=dt, device=dev)
        for a in range(0, pool, 4096):  # (generated in pieces: the fp32 draws take twice the room)
            c[a:a + 4096] = torch.randn((min(4096, pool - a),) + shape[1:], generator=g, device=dev)
        kv.append(c.transpose(1, 2) if case["heads_first"] else c)
    to = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, t)).to(dev)  # noqa: E731
    return dict(k_cache=kv[0], v_cache=kv[1], block_table=to(table, np.int32), ctx_len=to(n_ctx, np.int32),
                tok_off=to(np.concatenate([[0], np.cumsum(n_new)]), np.int32))


def _tables(rows, R, dev):
    inv = 1.0 / (1e6 ** (torch.arange(0, R, 2, dtype=torch.float64, device=dev) / R))
    a = torch.arange(rows, dtype=torch.float64, device=dev)[:, None] * inv
    return a.cos().float(), a.sin().float()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    kind, dt = case["kind"], DT[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    s = dict(case=case)
    if kind == "sample":
        rows, V, ld = case["rows"], case["V"], case["ld"]
        rng = np.random.default_rng([seed, 7])
        x = torch.empty((rows, ld), dtype=dt, device=dev)
        noise = torch.empty((rows, V), device=dev)
        for a in range(0, rows, 128):
            n = min(128, rows - a)
            z = randn(n, ld) * 3.0
            if case["sharp"]:  # the few dozen tokens that a model's context calls for
                z *= 0.8
                at = torch.randint(0, V, (n, 48), generator=g, device=dev)
                z.scatter_add_(1, at, 6.0 + 4.0 * torch.rand((n, 48), generator=g, device=dev) + 4.0 * torch.rand((n, 1), generator=g, device=dev))
            x[a:a + n] = z
            noise[a:a + n].exponential_(generator=g)
        noise.clamp_(min=1e-30)
        x[:, ::97] = float("-inf") if seed % 2 else torch.finfo(dt).min  # tokens that a grammar rules out
        cut = case["cut"]
        pick = lambda v, t: torch.from_numpy(rng.choice(np.array(v, t), rows)).to(dev)  # noqa: E731
        mixed = cut == "mixed"
        s.update(x=x, V=V, noise=noise, temperature=pick([0.0, 0.6, 0.8, 1.0, 1.0], np.float32) if mixed else 1.0,
                 top_k=pick([0, 20, 50, 1], np.int32) if mixed else 50 if cut == "top_k" else 0,
                 top_p=pick([0.8, 0.95, 1.0], np.float32) if mixed else 0.9 if cut == "top_p" else 1.0,
                 min_p=pick([0.0, 0.0, 0.05], np.float32) if mixed else 0.05 if cut == "min_p" else 0.0)
        if mixed and rows == 1:  # the lone row is an ordinary one, neither greedy nor uncut
            s.update(temperature=torch.full_like(s["temperature"], 0.8), top_k=torch.full_like(s["top_k"], 20), top_p=torch.full_like(s["top_p"], 0.95))
        s.update(tokens=torch.empty(rows, dtype=torch.int32, device=dev), logp=torch.empty(rows, device=dev))
        return s
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if kind == "attn":
        n_ctx, n_new = _lengths(case, seed)
        s.update(_cache(case, seed, n_ctx, n_new, g, dev), max_ctx=int((n_ctx + n_new).max()), max_new=int(n_new.max()))
        N = int(n_new.sum())
        s["q"] = (randn(N, Hq, D) * 2.0).to(dt)
        s["tree_mask"] = None
        if case["tree"]:
            rng = np.random.default_rng([seed, 11])
            bits = np.zeros((case["seqs"], int(n_new.max())), np.uint64)
            for j in range(bits.shape[1]):  # the parent is one of the four drafted before, or the last cached token
                parent = j - 1 - rng.integers(0, 4, case["seqs"])
                up = np.where(parent >= 0, bits[np.arange(case["seqs"]), np.maximum(parent, 0)], np.uint64(0))
                bits[:, j] = up | np.uint64(1 << j)
            s["tree_mask"] = torch.from_numpy(np.concatenate([bits[b, :n] for b, n in enumerate(n_new)]).view(np.int64)).to(dev)
        s.update(scale=D ** -0.5, out=torch.empty((N, Hq, D), dtype=dt, device=dev), lse=torch.empty((N, Hq), device=dev))
        return s
    if kind == "append":
        n_ctx, n_new = _lengths(case, seed)
        s.update(_cache(case, seed, n_ctx, n_new, g, dev))
        N = int(n_new.sum())
        pos = np.concatenate([c + np.arange(n) for c, n in zip(n_ctx, n_new)])
    else:
        N = case["tokens"]
        pos = np.concatenate([np.arange(N // 2), np.arange(N - N // 2)])  # two packed sequences
    qkv = randn(N, (Hq + 2 * Hk) * D).to(dt)  # the fused projection, of which q, k and v are views
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], dim=1))
    cos, sin = _tables(int(pos.max()) + 1, case["R"], dev)
    s.update(q=q, k=k, v=v, pos=torch.from_numpy(pos.astype(np.int32)).to(dev), cos=cos, sin=sin, q_weight=None, k_weight=None,
             eps=1e-6, q_out=torch.empty((N, Hq, D), dtype=dt, device=dev))
    if case["norm"]:
        s.update(q_weight=(1 + 0.2 * randn(D)).to(dt), k_weight=(1 + 0.2 * randn(D)).to(dt))
    if kind == "qk":
        s.update(k_out=torch.empty((N, Hk, D), dtype=dt, device=dev), dq_out=randn(N, Hq, D).to(dt), dk_out=randn(N, Hk, D).to(dt))
        d = torch.empty_like(qkv)
        s["dq"], s["dk"], _ = (t.unflatten(1, (-1, D)) for t in d.split([Hq * D, Hk * D, Hk * D], dim=1))
        if case["norm"]:
            s.update(dq_weight=torch.empty(D, device=dev), dk_weight=torch.empty(D, device=dev))
        else:
            s.update(dq_weight=None, dk_weight=None)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["kind"]](s)


def _workspace(s, size, *sizes):
    """The scratch that such a program allocates once."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(size(*sizes), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_qk(s):
    import paper_2609_14636_gb300 as stride

    ws = _workspace(s, stride.stride_qk_norm_rope_backward_workspace_size, *s["q"].shape[:2], s["k"].shape[1], s["q"].shape[2])
    rope = dict(pos=s["pos"], cos=s["cos"], sin=s["sin"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                interleaved=s["case"]["inter"])
    stride.stride_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], **rope)
    stride.stride_qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["dq"], s["dk"], **rope,
                                        dq_weight=s["dq_weight"], dk_weight=s["dk_weight"], workspace=ws)
    return [s["q_out"], s["k_out"], s["dq"], s["dk"]] + ([s["dq_weight"], s["dk_weight"]] if s["case"]["norm"] else [])


def _own_append(s):
    import paper_2609_14636_gb300 as stride

    stride.stride_kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"], s["tok_off"],
                            pos=s["pos"], cos=s["cos"], sin=s["sin"], k_weight=s["k_weight"], q=s["q"], q_out=s["q_out"],
                            q_weight=s["q_weight"], eps=s["eps"], interleaved=s["case"]["inter"])
    return [s["q_out"], s["k_cache"], s["v_cache"]]


def _own_attn(s):
    import paper_2609_14636_gb300 as stride

    ws = _workspace(s, stride.stride_tree_attention_workspace_size, *s["q"].shape[:2], s["k_cache"].shape[2], s["q"].shape[2])
    stride.stride_tree_attention(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"], s["tok_off"],
                                 s["tree_mask"], s["scale"], s["out"], lse=s["lse"], workspace=ws)
    return [s["out"], s["lse"]]


def _own_sample(s):
    import paper_2609_14636_gb300 as stride

    stride.stride_sample(s["x"], s["noise"], s["tokens"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                         min_p=s["min_p"], logp=s["logp"], V=s["V"])
    return [s["tokens"], s["logp"]]


def _rotate(x, cos, sin, inter):
    R = 2 * cos.shape[-1]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if inter else (x[..., :R // 2], x[..., R // 2:R])
    a, b = a * cos - b * sin, a * sin + b * cos
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1), x[..., R:]], -1)


def _norm_rope(x, w, cos, sin, s):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * w.float()
    return _rotate(x, cos, sin, s["case"]["inter"])


def _norm_rope_backward(dy, x, w, cos, sin, s):
    du = _rotate(dy.float(), cos, -sin, s["case"]["inter"])
    if w is None:
        return du, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"])
    n, g = x * r, du * w.float()
    return r * (g - n * (g * n).mean(-1, keepdim=True)), (du * n).sum((0, 1))


def _plain_qk(s):
    at = s["pos"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    s["q_out"].copy_(_norm_rope(s["q"], s["q_weight"], cos, sin, s))
    s["k_out"].copy_(_norm_rope(s["k"], s["k_weight"], cos, sin, s))
    dq, dqw = _norm_rope_backward(s["dq_out"], s["q"], s["q_weight"], cos, sin, s)
    dk, dkw = _norm_rope_backward(s["dk_out"], s["k"], s["k_weight"], cos, sin, s)
    s["dq"].copy_(dq)
    s["dk"].copy_(dk)
    return [s["q_out"], s["k_out"], s["dq"], s["dk"]] + ([dqw, dkw] if s["case"]["norm"] else [])


def _token_places(s, N):
    """Sequence, place among its new tokens and cache slot (page, row) of each new token."""
    off, i = s["tok_off"].long(), torch.arange(N, device=s["tok_off"].device)
    b = torch.searchsorted(off, i, right=True) - 1
    j = i - off[b]
    slot = s["ctx_len"].long()[b] + j
    page = s["k_cache"].shape[1]
    return b, j, s["block_table"][b, slot // page].long(), slot % page


def _plain_append(s):
    at = s["pos"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    _, _, page, row = _token_places(s, len(at))
    s["k_cache"][page, row] = _norm_rope(s["k"], s["k_weight"], cos, sin, s).to(s["k_cache"].dtype)
    s["v_cache"][page, row] = s["v"]
    s["q_out"].copy_(_norm_rope(s["q"], s["q_weight"], cos, sin, s))
    return [s["q_out"], s["k_cache"], s["v_cache"]]


def _plain_attn(s):
    q, page = s["q"], s["k_cache"].shape[1]
    N, Hq, D = q.shape
    Hk = s["k_cache"].shape[2]
    B, G, L, n = len(s["ctx_len"]), Hq // Hk, s["max_ctx"], s["max_new"]
    b, j, _, _ = _token_places(s, N)
    ctx, off = s["ctx_len"].long(), s["tok_off"].long()
    slot = torch.arange(L, device=q.device)
    have = slot < (ctx + off[1:] - off[:-1])[:, None]  # [B, L]
    pages = s["block_table"][:, slot // page].long().clamp(min=0)
    K = torch.where(have[:, :, None, None], s["k_cache"][pages, slot % page].float(), 0.0)  # [B, L, Hk, D]
    V = torch.where(have[:, :, None, None], s["v_cache"][pages, slot % page].float(), 0.0)
    Q = torch.zeros((B, n, Hk, G, D), device=q.device)
    Q[b, j] = q.float().unflatten(1, (Hk, G)) * s["scale"]
    S = torch.matmul(Q.permute(0, 2, 1, 3, 4).reshape(B, Hk, n * G, D), K.permute(0, 2, 3, 1)).unflatten(2, (n, G))
    back = slot - ctx[:, None]  # the slot's place among the new tokens
    if s["tree_mask"] is None:
        new_ok = back[:, None] <= torch.arange(n, device=q.device)[:, None]  # [B, n, L]
    else:
        bits = torch.zeros((B, n), dtype=torch.int64, device=q.device)
        bits[b, j] = s["tree_mask"]
        new_ok = (bits[:, :, None] >> back[:, None].clamp(0, 63)) & 1 != 0
    ok = have[:, None] & ((back < 0)[:, None] | new_ok)
    S = S.masked_fill(~ok[:, None, :, None], float("-inf"))
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    S = torch.exp(S - m)
    l = S.sum(-1, keepdim=True)  # noqa: E741
    O = torch.matmul(S.flatten(2, 3), V.transpose(1, 2)).unflatten(2, (n, G)) / torch.where(l == 0, 1.0, l)  # noqa: E741
    s["out"].copy_(O.permute(0, 2, 1, 3, 4)[b, j].flatten(1, 2))
    s["lse"].copy_((m + l.log())[..., 0].permute(0, 2, 1, 3)[b, j].flatten(1, 2))
    return [s["out"], s["lse"]]


def _plain_sample(s):
    x = s["x"][:, :s["V"]].float()
    col = lambda v: v[:, None] if isinstance(v, torch.Tensor) else v  # noqa: E731
    V, T = x.shape[1], torch.as_tensor(col(s["temperature"]), device=x.device)
    top_k, top_p, min_p = col(s["top_k"]), col(s["top_p"]), col(s["min_p"])
    d = (x - x.amax(1, keepdim=True)) / torch.where(T == 0, 1.0, T)
    w = d.exp()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices  # ties: lowest index first
    ws = w.gather(1, order)
    rank = torch.arange(V, device=x.device)
    most = torch.as_tensor(top_k, device=x.device)
    most = torch.where(most <= 0, V, most)
    most = torch.where(T == 0, 1, most)
    ws = torch.where(rank < most, ws, 0.0)
    mass = ws.cumsum(1)
    limit = torch.as_tensor(top_p, device=x.device)
    keep = (rank < most) & (ws >= min_p) & ((mass - ws < limit * mass[:, -1:]) | (limit >= 1))
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0.0))
    race = torch.zeros_like(w).scatter_(1, order, torch.where(keep, 1.0, -1.0))
    race = torch.where(race > 0, w / s["noise"], -1.0)
    best = race.amax(1, keepdim=True)
    token = torch.where(race == best, rank, V).amin(1)
    s["tokens"].copy_(token)
    s["logp"].copy_(d.gather(1, token[:, None])[:, 0] - w.sum(1).log())
    return [s["tokens"], s["logp"]]


_run_own = dict(qk=_own_qk, append=_own_append, attn=_own_attn, sample=_own_sample)
_run_plain = dict(qk=_plain_qk, append=_plain_append, attn=_plain_attn, sample=_plain_sample)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind == "sample":
        n = case["rows"] * case["V"]
        return {"bytes": n * (e + (4 if case["cut"] == "none" else 0)) + 24 * case["rows"], "flops": 4 * n}
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if kind == "qk":  # forward: rows in and out; backward: rows and gradients in, gradients out; the tables twice
        n = case["tokens"] * (Hq + Hk) * D
        return {"bytes": 5 * n * e + case["tokens"] * (8 * case["R"] + 8), "flops": 30 * n}
    n_ctx, n_new = _lengths(case, 0)
    N = int(n_new.sum())
    if kind == "append":
        return {"bytes": 2 * N * (Hq + 2 * Hk) * D * e + N * (4 * case["R"] + 4), "flops": 10 * N * (Hq + Hk) * D}
    pairs = n_new * n_ctx + (0 if case["tree"] else n_new * (n_new + 1) // 2)  # a tree's own pairs are few
    return {"bytes": int((n_ctx + n_new).sum()) * Hk * D * 2 * e + N * Hq * (2 * D * e + 4), "flops": 4 * D * Hq * int(pairs.sum())}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(qk=_exact_qk, append=_exact_append, attn=_exact_attn, sample=_exact_sample)[case["kind"]](case, s)


def _pairs(case, s):
    """Index of each rotated component's partner, its sign in the rotation, and cos, sin per token and component."""
    D, R = case["D"], case["R"]
    i = torch.arange(D, device="cuda")
    if case["inter"]:
        partner, sign, angle = i ^ 1, torch.where(i % 2 == 0, -1.0, 1.0), i // 2
    else:
        partner, sign, angle = torch.where(i < R // 2, i + R // 2, i - R // 2), torch.where(i < R // 2, -1.0, 1.0), i % (R // 2)
    turned = i < R
    angle = torch.where(turned, angle, 0)
    rows = s["pos"].long()
    c = torch.where(turned, s["cos"].double()[rows][:, angle], 1.0)[:, None]
    n = torch.where(turned, s["sin"].double()[rows][:, angle] * sign, 0.0)[:, None]
    return torch.where(turned, partner, i), c, n


def _exact_forward(case, s, x, w):
    x = x.double()
    if w is not None:
        x = w.double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["D"] + s["eps"])
    partner, c, n = _pairs(case, s)
    return c * x + n * x[..., partner]


def _exact_qk(case, s):
    out, grads, weights = [], [], []
    partner, c, n = _pairs(case, s)
    for x, w, dy in ((s["q"], s["q_weight"], s["dq_out"]), (s["k"], s["k_weight"], s["dk_out"])):
        out.append(_exact_forward(case, s, x, w))
        dy = dy.double()
        du = c * dy - n * dy[..., partner]  # the inverse rotation
        if w is None:
            grads.append(du)
            continue
        x = x.double()
        ms = (x * x).sum(-1, keepdim=True) / case["D"] + s["eps"]
        weights.append((du * x / ms.sqrt()).sum((0, 1)))
        g = du * w.double()
        grads.append(g / ms.sqrt() - x * (g * x).sum(-1, keepdim=True) / (case["D"] * ms ** 1.5))
    return out + grads + weights


def _exact_append(case, s):
    k, v = s["k_cache"].double(), s["v_cache"].double()
    rows = _exact_forward(case, s, s["k"], s["k_weight"])
    off, ctx, table = s["tok_off"].tolist(), s["ctx_len"].tolist(), s["block_table"].long()
    for b in range(case["seqs"]):
        slot = ctx[b] + torch.arange(off[b + 1] - off[b], device="cuda")
        at = table[b][slot // case["page"]], slot % case["page"]
        k[at] = rows[off[b]:off[b + 1]]
        v[at] = s["v"][off[b]:off[b + 1]].double()
    return [_exact_forward(case, s, s["q"], s["q_weight"]), k, v]


def _exact_attn(case, s):
    off, ctx, table = s["tok_off"].tolist(), s["ctx_len"].tolist(), s["block_table"].long()
    N, Hq, D = s["q"].shape
    Hk, page = case["Hk"], case["page"]
    out = torch.zeros((N, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((N, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        n = off[b + 1] - off[b]
        slot = torch.arange(ctx[b] + n, device="cuda")
        at = table[b][slot // page], slot % page
        i, back = torch.arange(n, device="cuda"), slot - ctx[b]
        if s["tree_mask"] is None:
            ok = back[None] <= i[:, None]
        else:
            mask = s["tree_mask"][off[b]:off[b + 1]]
            ok = (back < 0)[None] | ((mask[:, None] >> back.clamp(0, 63)[None]) & 1).bool()
        K, V = s["k_cache"][at].double(), s["v_cache"][at].double()
        for h in range(Hq):
            z = s["q"][off[b]:off[b + 1], h].double() @ K[:, h // (Hq // Hk)].T * s["scale"]
            z = z.masked_fill(~ok, -math.inf)
            lse[off[b]:off[b + 1], h] = torch.logsumexp(z, 1)
            out[off[b]:off[b + 1], h] = torch.softmax(z, 1).nan_to_num(0.0) @ V[:, h // (Hq // Hk)]
    return [out, lse]


def _exact_sample(case, s):
    rows = case["rows"]
    each = lambda v: v.tolist() if isinstance(v, torch.Tensor) else [v] * rows  # noqa: E731
    T, k, p, mp = (each(s[n]) for n in ("temperature", "top_k", "top_p", "min_p"))
    tokens, logp = [], []
    for r in range(rows):
        x = s["x"][r, :s["V"]].double()
        if T[r] == 0:
            tokens.append(torch.nonzero(x == x.max())[0, 0])
            logp.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        x, at = torch.sort(x, descending=True, stable=True)
        n = k[r] if 0 < k[r] < len(x) else len(x)
        prob = torch.softmax(x[:n] / T[r], 0)
        if p[r] < 1:
            n = max(1, int((prob.cumsum(0) - prob < p[r]).sum()))
        n = min(n, max(1, int((prob >= mp[r] * prob[0]).sum())))
        prob = prob[:n] / prob[:n].sum()
        race = prob / s["noise"][r].double()[at[:n]]
        win = at[:n][race == race.max()].min()
        tokens.append(win)
        logp.append(prob[torch.nonzero(at[:n] == win)[0, 0]].log())
    return [torch.stack(tokens).int(), torch.stack(logp)]
