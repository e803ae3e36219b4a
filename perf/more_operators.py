"""The measured cases of the operators around a rollout's cache and its logits: what is kept and what may be sampled.

Three kinds of pass:

* ``mass``      attention weight that each cached slot got, added up over steps (stride_attention_mass);
* ``evict``     the slots of most weight, the first and the last ones, copied in order into other pages
                (stride_kv_evict);
* ``controls``  penalties for repeated tokens, biases and grammar masks on logits (stride_logit_controls).

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
        # The smallest call: one rollout's one token over a few cached ones.  Latency counts.
        dict(name="mass_1x1_short", kind="mass", seqs=1, new=1, tree=False, Hq=16, Hk=2, D=128, page=16, ctx=37,
             ragged=False, heads_first=False, decay=1.0, dtype="bf16"),
        # A decode step of 256 rollouts of unequal lengths.
        dict(name="mass_256_steps", kind="mass", seqs=256, new=1, tree=False, Hq=32, Hk=8, D=128, page=16, ctx=4096,
             ragged=True, heads_first=False, decay=1.0, dtype="bf16"),
        # One long agentic trajectory: few rows, a long axis; older weight fades.
        dict(name="mass_1_long", kind="mass", seqs=1, new=1, tree=False, Hq=32, Hk=8, D=128, page=64, ctx=131_072,
             ragged=False, heads_first=True, decay=0.99, dtype="bf16"),
        # Drafted trees of up to 13 tokens over unequal prefixes, half precision.
        dict(name="mass_32_trees_13", kind="mass", seqs=32, new=13, tree=True, Hq=32, Hk=8, D=128, page=16, ctx=8000,
             ragged=True, heads_first=False, decay=1.0, dtype="f16"),
        # Observations' new tokens, chains over the reused prefixes, whose weights start anew: arithmetic counts.
        dict(name="mass_4_chains_511", kind="mass", seqs=4, new=511, tree=False, Hq=32, Hk=8, D=128, page=32, ctx=6000,
             ragged=True, heads_first=False, decay=0.0, dtype="bf16"),
        # A few short rollouts make room: odd sizes, pages that end inside a vector of slots, fp32 caches.
        dict(name="evict_3_odd_f32", kind="evict", seqs=3, Hk=3, D=80, page=24, ctx=323, budget=101, sink=3, recent=17,
             ragged=True, heads_first=True, dtype="f32"),
        # 256 rollouts of unequal lengths, those over 1,024 tokens cut to that.
        dict(name="evict_256", kind="evict", seqs=256, Hk=8, D=128, page=16, ctx=4096, budget=1024, sink=4, recent=256,
             ragged=True, heads_first=False, dtype="bf16"),
        # One long agentic trajectory, an eighth of it kept.
        dict(name="evict_1_long", kind="evict", seqs=1, Hk=8, D=128, page=64, ctx=131_072, budget=16_384, sink=64, recent=4096,
             ragged=False, heads_first=True, dtype="bf16"),
        # The last live rollout's logits: everything at once.
        dict(name="controls_1", kind="controls", rows=1, V=V0, ld=V0, hist=2000, bias=40, mask=True, dtype="bf16"),
        # A step of 256 rollouts inside tool calls' grammars, with penalties over up to 4,096 tokens and biases.
        dict(name="controls_256_all", kind="controls", rows=256, V=V0, ld=V0, hist=4096, bias=100, mask=True, dtype="bf16"),
        # The tiny reference's logits, penalties alone.
        dict(name="controls_512_f32", kind="controls", rows=512, V=32_000, ld=32_000, hist=1500, bias=0, mask=False, dtype="f32"),
        # A vocabulary that no vector divides, packed rows, half precision.
        dict(name="controls_33_odd_f16", kind="controls", rows=33, V=50_257, ld=50_257, hist=700, bias=7, mask=True, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["mass", "mass", "evict", "controls", "controls"])
    if kind == "controls":
        V = rng.choice([V0, V0, 32_000, _log_int(rng, 1000, 152_064)])
        if rng.random() < 0.3:
            V -= rng.randint(1, 7)  # rows that no vector divides ...
        ld = V if rng.random() < 0.6 else (V + 63) // 64 * 64  # ... packed, or padded to aligned rows
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        return dict(kind=kind, rows=_log_int(rng, 1, 300 if SIZE[dtype] == 2 else 128), V=V, ld=ld, hist=rng.choice([0, _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)]),
                    bias=rng.choice([0, _log_int(rng, 1, 300)]), mask=rng.random() < 0.6, dtype=dtype)
    Hk = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 24])
    first = rng.random() < 0.5
    ctx = _log_int(rng, 16, 131_072)
    seqs = _log_int(rng, 1, 256)
    if kind == "evict":
        D = rng.choice([128, 128, 64, 80, 256])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        while seqs > 1 and seqs * ctx * Hk * D * SIZE[dtype] > MAX_KV * 2:
            seqs = seqs // 2
        budget = max(1, int(ctx * rng.choice([0.1, 0.25, 0.25, 0.5])) - rng.randint(0, 3))
        return dict(kind=kind, seqs=seqs, Hk=Hk, D=D, page=page, ctx=ctx, budget=budget, sink=rng.randint(0, min(64, budget)),
                    recent=rng.randint(0, budget // 2), ragged=rng.random() < 0.7, heads_first=first, dtype=dtype)
    G = rng.choice([1, 3, 4, 4, 7, 8])
    D = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    what = rng.choice(["one", "one", "tree", "chain"])
    new = 1 if what == "one" else rng.randint(2, 64) if what == "tree" else _log_int(rng, 2, 511)
    while seqs > 1 and (seqs * ctx * Hk * D > MAX_KV or seqs * new * Hk * G * (ctx + new) * D > MAX_PAIRS):
        seqs = (seqs + 1) // 2 if seqs > 2 else 1
    while ctx * Hk * D > MAX_KV or new * Hk * G * (ctx + new) * D > MAX_PAIRS:
        ctx = ctx // 2
    return dict(kind=kind, seqs=seqs, new=new, tree=what == "tree", Hq=Hk * G, Hk=Hk, D=D, page=page, ctx=ctx,
                ragged=rng.random() < 0.7, heads_first=first, decay=rng.choice([1.0, 1.0, 0.99, 0.0]), dtype=dtype)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _lengths(case, seed):
    """Cached and new tokens per sequence.  Unequal ones reach from nothing cached to the case's longest; the case sets
    the lengths (outputs of all seeds have one shape), the seed which sequence has which."""
    B, ctx, new = case["seqs"], case["ctx"], case.get("new", 0)
    rng = np.random.default_rng([B, ctx, new])
    n_ctx = np.full(B, ctx, np.int64)
    n_new = np.full(B, new, np.int64)
    if case["ragged"]:
        n_ctx = (ctx * np.sqrt(rng.random(B))).astype(np.int64) * (rng.random(B) > 0.02)
        n_ctx[0] = ctx
        if new > 1:
            n_new = np.maximum(1, new - rng.integers(0, max(1, new // 3) + 1, B))
    at = np.random.default_rng([seed, 3]).permutation(B)
    return n_ctx[at], n_new[at]


def _pool(case, lengths, order, g, dev, fill=True):
    """A page pool in random order as [pages, page, heads, D] and the block table of sequences of these lengths."""
    page, Hk, D = case["page"], case["Hk"], case["D"]
    need = -(-lengths // page)
    pool = int(need.sum()) + 3
    perm, table, at = order.permutation(pool).astype(np.int32), np.full((len(need), max(1, int(need.max()))), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    shape = (pool, Hk, page, D) if case["heads_first"] else (pool, page, Hk, D)
    kv = []
    for _ in range(2):
        c = torch.zeros(shape, dtype=DT[case["dtype"]], device=dev)
        for a in range(0, pool if fill else 0, 4096):  # (generated in pieces: the fp32 draws take twice the room)
            c[a:a + 4096] = torch.randn((min(4096, pool - a),) + shape[1:], generator=g, device=dev)
        kv.append(c.transpose(1, 2) if case["heads_first"] else c)
    return kv[0], kv[1], torch.from_numpy(table).to(dev)


def _int32(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(dev)


def _fresh_mass(randn, shape):
    """Weights that slots have got so far: most little, a few nearly all of it, many none that 32 bits hold."""
    m = torch.exp(2.5 * randn(*shape) - 4.0)
    return torch.where(m < 1e-3, 0.0, m)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng([seed, 5])
    kind, dt = case["kind"], DT[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    s = dict(case=case)
    if kind == "controls":
        rows, V, ld, hist, n_bias = case["rows"], case["V"], case["ld"], case["hist"], case["bias"]
        x = torch.empty((rows, ld), dtype=dt, device=dev)
        for a in range(0, rows, 128):
            x[a:a + 128] = randn(min(128, rows - a), ld) * 3.0
        s.update(x=x, V=V, out=torch.empty_like(x), history=None, history_len=None, prompt_len=None, repetition=1.0, frequency=0.0,
                 presence=0.0, bias_off=None, bias_token=None, bias=None, allowed=None)
        pick = lambda v: torch.from_numpy(rng.choice(np.array(v, np.float32), rows)).to(dev)  # noqa: E731
        if hist:  # words repeat: some tokens often, most once; what lies past a row's length is padding
            n = np.random.default_rng([rows, hist]).integers((hist + 1) // 2, hist + 1, rows)
            t = (V * torch.rand((rows, hist), generator=g, device=dev) ** 4).int().clamp(max=V - 1)
            far = torch.randint(0, V, (rows, hist), generator=g, device=dev, dtype=torch.int32)
            t = torch.where(torch.rand((rows, hist), generator=g, device=dev) < 0.5, t, far)
            t = torch.where(torch.arange(hist, device=dev) < _int32(n, dev)[:, None], t, -1)
            s.update(history=t, history_len=_int32(n, dev), prompt_len=_int32(n * rng.random(rows), dev),
                     repetition=pick([1.0, 1.05, 1.2]), frequency=pick([0.0, 0.1, 0.5]), presence=pick([0.0, 0.0, 0.7]))
        if n_bias:  # tokens nudged, a few banned
            n = np.random.default_rng([rows, n_bias, 1]).integers(0, n_bias + 1, rows)
            n[0] = n_bias
            total = int(n.sum())
            b = 4.0 * randn(total)
            b[::11] = float("-inf")
            s.update(bias_off=_int32(np.concatenate([[0], np.cumsum(n)]), dev), bias=b,
                     bias_token=torch.randint(0, V, (total,), generator=g, device=dev, dtype=torch.int32))
        if case["mask"]:  # a free state of the grammar rules out little, a strict one all but a few
            words = (V + 31) // 32
            bits = lambda: torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=g, device=dev, dtype=torch.int64)  # noqa: E731
            few, many = bits() & bits() & bits() & bits() & bits(), bits() | bits() | bits() | bits() | bits()
            allow = torch.where(torch.from_numpy(rng.random(rows) < 0.5).to(dev)[:, None], few, many)
            allow[torch.from_numpy(rng.random(rows) < 0.2).to(dev)] = -1  # outside a tool call: everything
            s["allowed"] = allow.int()
        return s
    n_ctx, n_new = _lengths(case, seed)
    Hk, D = case["Hk"], case["D"]
    s["k_cache"], s["v_cache"], s["block_table"] = _pool(case, n_ctx + n_new, rng, g, dev)
    s["ctx_len"], s["max_len"] = _int32(n_ctx, dev), int((n_ctx + n_new).max())
    s["mass"] = _fresh_mass(randn, (case["seqs"], Hk, (s["max_len"] + 31) // 32 * 32))
    if kind == "evict":
        m = np.minimum(n_ctx, case["budget"])
        s["k_to"], s["v_to"], s["to_table"] = _pool(case, m, rng, g, dev, fill=False)
        s.update(new_len=torch.empty(case["seqs"], dtype=torch.int32, device=dev),
                 kept=torch.full((case["seqs"], Hk, case["budget"]), -1, dtype=torch.int32, device=dev),
                 mass_to=torch.zeros((case["seqs"], Hk, case["budget"]), device=dev))
        return s
    N, Hq = int(n_new.sum()), case["Hq"]
    s["tok_off"], s["max_new"] = _int32(np.concatenate([[0], np.cumsum(n_new)]), dev), int(n_new.max())
    s["q"] = (randn(N, Hq, D) * 2.0).to(dt)
    s["tree_mask"] = None
    if case["tree"]:
        bits = np.zeros((case["seqs"], int(n_new.max())), np.uint64)
        for j in range(bits.shape[1]):  # the parent is one of the four drafted before, or the last cached token
            parent = j - 1 - rng.integers(0, 4, case["seqs"])
            up = np.where(parent >= 0, bits[np.arange(case["seqs"]), np.maximum(parent, 0)], np.uint64(0))
            bits[:, j] = up | np.uint64(1 << j)
        s["tree_mask"] = torch.from_numpy(np.concatenate([bits[b, :n] for b, n in enumerate(n_new)]).view(np.int64)).to(dev)
    # what attention leaves: ln sum exp of scores of variance 4 over the slots that a token sees
    seen = np.concatenate([c + 1 + np.arange(n) for c, n in zip(n_ctx, n_new)])
    s["lse"] = torch.from_numpy(np.log(seen).astype(np.float32)).to(dev)[:, None] + 2.0 + 0.2 * randn(N, Hq)
    s["scale"] = D ** -0.5
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["case"]["kind"]](s)


def _own_mass(s):
    import paper_2609_14636_gb300 as stride

    stride.stride_attention_mass(s["q"], s["lse"], s["k_cache"], s["block_table"], s["ctx_len"], s["tok_off"], s["tree_mask"],
                                 s["scale"], s["mass"], decay=s["case"]["decay"])
    return [s["mass"]]


def _own_evict(s):
    import paper_2609_14636_gb300 as stride

    c = s["case"]
    stride.stride_kv_evict(s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"], s["mass"], c["budget"], s["k_to"], s["v_to"],
                           s["to_table"], s["new_len"], s["kept"], mass_to=s["mass_to"], sink=c["sink"], recent=c["recent"])
    return [s["k_to"], s["v_to"], s["new_len"], s["kept"], s["mass_to"]]


def _own_controls(s):
    import paper_2609_14636_gb300 as stride

    stride.stride_logit_controls(s["x"], s["out"], history=s["history"], history_len=s["history_len"], prompt_len=s["prompt_len"],
                                 repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias_off=s["bias_off"],
                                 bias_token=s["bias_token"], bias=s["bias"], allowed=s["allowed"], V=s["V"])
    return [s["out"][:, :s["V"]]]


def _cached(s, cache, slot, have):
    """The cache's rows of these slots of every sequence in 32 bits, [B, L, heads, D]; zeros where there are none."""
    page = cache.shape[1]
    pages = s["block_table"][:, slot // page].long().clamp(min=0)
    return torch.where(have[:, :, None, None], cache[pages, slot % page].float(), 0.0)


def _plain_mass(s):
    q, Hk = s["q"], s["case"]["Hk"]
    N, Hq, D = q.shape
    B, G, L, n, dev = len(s["ctx_len"]), Hq // Hk, s["max_len"], s["max_new"], q.device
    ctx, off = s["ctx_len"].long(), s["tok_off"].long()
    i = torch.arange(N, device=dev)
    b = torch.searchsorted(off, i, right=True) - 1
    j = i - off[b]
    slot = torch.arange(L, device=dev)
    have = slot < (ctx + off[1:] - off[:-1])[:, None]
    K = _cached(s, s["k_cache"], slot, have)
    Q = torch.zeros((B, n, Hk, G, D), device=dev)
    Q[b, j] = q.float().unflatten(1, (Hk, G)) * s["scale"]
    S = torch.matmul(Q.permute(0, 2, 1, 3, 4).reshape(B, Hk, n * G, D), K.permute(0, 2, 3, 1)).unflatten(2, (n, G))
    lse = torch.full((B, n, Hk, G), float("inf"), device=dev)  # (tokens that a sequence does not have add nothing)
    lse[b, j] = s["lse"].unflatten(1, (Hk, G))
    S = S.sub_(lse.permute(0, 2, 1, 3)[..., None]).exp_()
    back = slot - ctx[:, None]  # the slot's place among the new tokens
    if s["tree_mask"] is None:
        new_ok = back[:, None] <= torch.arange(n, device=dev)[:, None]
    else:
        bits = torch.zeros((B, n), dtype=torch.int64, device=dev)
        bits[b, j] = s["tree_mask"]
        new_ok = (bits[:, :, None] >> back[:, None].clamp(0, 63)) & 1 != 0
    ok = have[:, None] & ((back < 0)[:, None] | new_ok)  # [B, n, L]
    S = S.sum(3)  # over the heads of a group
    got = torch.where(ok[:, None], S, 0.0).sum(2)  # [B, Hk, L]
    old = s["mass"][..., :L]
    before = torch.where((back < 0)[:, None], old * s["case"]["decay"], 0.0)
    s["mass"][..., :L] = torch.where(have[:, None], before + got, old)
    return [s["mass"]]


def _plain_evict(s):
    c, dev, L = s["case"], s["mass"].device, s["max_len"]
    most, n = c["budget"], s["ctx_len"].long()[:, None, None]
    slot = torch.arange(L, device=dev)
    m = n.clamp(max=most)
    first = m.clamp(max=c["sink"])
    last = (m - first).clamp(max=c["recent"])
    mass = s["mass"][..., :L]
    rank = torch.where((slot < first) | ((slot >= n - last) & (slot < n)), float("inf"), mass)
    rank = torch.where(slot < n, rank, float("-inf"))
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices  # ties: lowest slot first
    keep = torch.zeros(mass.shape, dtype=torch.bool, device=dev).scatter_(2, order, (slot < m).expand_as(order))
    b, h, at = torch.nonzero(keep, as_tuple=True)  # in the slots' order
    to = (keep.cumsum(2) - 1)[b, h, at]
    s["kept"][b, h, to] = at.int()
    s["mass_to"][b, h, to] = mass[b, h, at]
    page, page_to = s["k_cache"].shape[1], s["k_to"].shape[1]
    where = s["block_table"][b, at // page].long(), at % page, h
    there = s["to_table"][b, to // page_to].long(), to % page_to, h
    s["k_to"][there] = s["k_cache"][where]
    s["v_to"][there] = s["v_cache"][where]
    s["new_len"].copy_(m.view(-1))
    return [s["k_to"], s["v_to"], s["new_len"], s["kept"], s["mass_to"]]


def _plain_controls(s):
    V, dev = s["V"], s["x"].device
    y = s["x"][:, :V].float()
    rows = len(y)
    col = lambda v: v[:, None] if isinstance(v, torch.Tensor) else v  # noqa: E731
    if s["history"] is not None:
        t, place = s["history"].long(), torch.arange(s["history"].shape[1], device=dev)
        have = place < s["history_len"][:, None]
        t = torch.where(have, t, V)  # (one more column takes the padding)
        seen = torch.zeros((rows, V + 1), device=dev).scatter_(1, t, 1.0)[:, :V] > 0
        made = have & (place >= s["prompt_len"][:, None])
        count = torch.zeros((rows, V + 1), device=dev).scatter_add_(1, t, made.float())[:, :V]
        r = col(s["repetition"])
        y = torch.where(seen, torch.where(y > 0, y / r, y * r), y)
        y = y - col(s["frequency"]) * count - torch.where(count > 0, col(s["presence"]), 0.0)
    if s["bias"] is not None:
        i = torch.arange(len(s["bias"]), device=dev)
        row = torch.searchsorted(s["bias_off"].long(), i, right=True) - 1
        entry = torch.full((rows * V,), -1, dtype=torch.int64, device=dev)
        entry = entry.scatter_reduce_(0, row * V + s["bias_token"], i, "amax").view(rows, V)  # the last of a token counts
        y = torch.where(entry >= 0, y + s["bias"][entry.clamp(min=0)], y)
    if s["allowed"] is not None:
        j = torch.arange(V, device=dev)
        y = torch.where((s["allowed"][:, j // 32] >> (j % 32)) & 1 != 0, y, float("-inf"))
    s["out"][:, :V] = y
    return [s["out"][:, :V]]


_run_own = dict(mass=_own_mass, evict=_own_evict, controls=_own_controls)
_run_plain = dict(mass=_plain_mass, evict=_plain_evict, controls=_plain_controls)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind == "controls":
        n = case["rows"] * case["V"]
        lists = 4 * case["rows"] * case["hist"] * 3 // 4 + 8 * case["rows"] * case["bias"] // 2
        return {"bytes": 2 * n * e + (n // 8 if case["mask"] else 0) + lists, "flops": 2 * n}
    Hk, D = case["Hk"], case["D"]
    n_ctx, n_new = _lengths(case, 0)
    if kind == "evict":  # masses in; kept rows of keys and values in and out, their slots and masses out
        kept = int(np.minimum(n_ctx, case["budget"]).sum()) * Hk
        return {"bytes": 4 * int(n_ctx.sum()) * Hk + kept * (4 * D * e + 8), "flops": 4 * int(n_ctx.sum()) * Hk}
    N, Hq, slots = int(n_new.sum()), case["Hq"], int((n_ctx + n_new).sum())
    pairs = n_new * n_ctx + (0 if case["tree"] else n_new * (n_new + 1) // 2)  # a tree's own pairs are few
    return {"bytes": slots * Hk * (D * e + (8 if case["decay"] else 4)) + N * Hq * (D * e + 4), "flops": 2 * D * Hq * int(pairs.sum())}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return dict(mass=_exact_mass, evict=_exact_evict, controls=_exact_controls)[case["kind"]](case, s)


def _exact_mass(case, s):
    mass = s["mass"].double()
    off, ctx, table = s["tok_off"].tolist(), s["ctx_len"].tolist(), s["block_table"].long()
    G = case["Hq"] // case["Hk"]
    for b in range(case["seqs"]):
        n = off[b + 1] - off[b]
        slot = torch.arange(ctx[b] + n, device="cuda")
        K = s["k_cache"][table[b][slot // case["page"]], slot % case["page"]].double()
        i, back = torch.arange(n, device="cuda"), slot - ctx[b]
        if s["tree_mask"] is None:
            sees = i[:, None] >= back
        else:
            sees = (back < 0) | ((s["tree_mask"][off[b]:off[b + 1], None] >> back.clamp(0, 63)) & 1).bool()
        mass[b, :, :ctx[b]] *= case["decay"]
        mass[b, :, ctx[b]:ctx[b] + n] = 0
        for h in range(case["Hq"]):
            z = s["q"][off[b]:off[b + 1], h].double() @ K[:, h // G].T * s["scale"] - s["lse"][off[b]:off[b + 1], h, None].double()
            mass[b, h // G, :len(slot)] += z.masked_fill(~sees, -math.inf).exp().sum(0)
    return [mass]


def _exact_evict(case, s):
    k, v, kept, mass = s["k_to"].double(), s["v_to"].double(), s["kept"].clone(), s["mass_to"].double()
    lengths, table, to_table = s["ctx_len"].tolist(), s["block_table"].long(), s["to_table"].long()
    got = []
    for b, n in enumerate(lengths):
        m = min(n, case["budget"])
        got.append(m)
        a = min(m, case["sink"])
        z = min(m - a, case["recent"])
        page, i = case["page"], torch.arange(m, device="cuda")
        for h in range(case["Hk"]):
            w = s["mass"][b, h, a:n - z].double()
            by = torch.argsort(-w, stable=True)[:m - a - z] + a
            all_kept = torch.cat([torch.arange(a, device="cuda"), by, torch.arange(n - z, n, device="cuda")]).sort().values
            kept[b, h, :m] = all_kept.int()
            mass[b, h, :m] = s["mass"][b, h, all_kept].double()
            at, to = (table[b][all_kept // page], all_kept % page, h), (to_table[b][i // page], i % page, h)
            k[to], v[to] = s["k_cache"][at].double(), s["v_cache"][at].double()
    return [k, v, torch.tensor(got, dtype=torch.int32), kept, mass]


def _exact_controls(case, s):
    rows, V = case["rows"], s["V"]
    each = lambda v: v.tolist() if isinstance(v, torch.Tensor) else [v] * rows  # noqa: E731
    rep, freq, pres = (each(s[n]) for n in ("repetition", "frequency", "presence"))
    out = torch.empty((rows, V), dtype=torch.float64, device="cuda")
    for r in range(rows):
        y = s["x"][r, :V].double()
        if s["history"] is not None:
            n, p = int(s["history_len"][r]), int(s["prompt_len"][r])
            everything, made = s["history"][r, :n].long(), s["history"][r, p:n].long()
            seen = everything.unique()
            y[seen] = torch.where(y[seen] > 0, y[seen] / rep[r], y[seen] * rep[r])
            token, times = made.unique(return_counts=True)
            y[token] -= freq[r] * times.double() + pres[r]
        if s["bias"] is not None:
            a, z = int(s["bias_off"][r]), int(s["bias_off"][r + 1])
            last = dict(zip(s["bias_token"][a:z].tolist(), s["bias"][a:z].tolist()))
            if last:
                at = torch.tensor(list(last), device="cuda")
                y[at] += torch.tensor(list(last.values()), dtype=torch.float64, device="cuda")
        if s["allowed"] is not None:
            words = s["allowed"][r].long() & 0xFFFFFFFF
            ok = ((words[:, None] >> torch.arange(32, device="cuda")) & 1).bool().view(-1)[:V]
            y[~ok] = -math.inf
        out[r] = y
    return [out]
