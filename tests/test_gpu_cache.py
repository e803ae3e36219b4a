"""Attention weight per slot and eviction by it against their plain forms in 64
bits (tests/cache_reference.py, which states the tolerances)."""
from __future__ import annotations

import numpy as np
import pytest

import cache_reference as ref
import decode_reference as dec

pytestmark = pytest.mark.gpu

BAD_LAYOUT = 0x2


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


def gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(torch, a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def pool(torch, pages, page, Hk, D, dtype, order, g):
    """[pages, page, heads, D]: rows first, heads first, or rows of more components than a head has."""
    shape = {"rows": (pages, page, Hk, D), "heads": (pages, Hk, page, D), "wide": (pages, page, Hk, D + 8)}[order]
    x = torch.randn(shape, generator=g, device="cuda").to(dec.torch_dtype(dtype))
    return x.transpose(1, 2) if order == "heads" else x[..., :D]


def block_table(need, rng):
    """Pages of sequences of so many pages, in random order among a few others."""
    perm, at = rng.permutation(int(sum(need)) + 3), 0
    table = np.full((len(need), max(1, max(need))), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, len(perm)


def slots(cache, table, b, n):
    """Rows [n, heads, D] of a sequence's first n slots in 64 bits."""
    page = cache.shape[1]
    i = np.arange(n)
    return dec.f64(cache[list(table[b, i // page]), list(i % page)]) if n else np.zeros((0,) + tuple(cache.shape[2:]))


# ---------------------------------------------------------------------------------------------------------------------
# attention weights
# ---------------------------------------------------------------------------------------------------------------------
MASS = [
    # sequences (committed, new), Hq, Hk, D, page, order, tree, decay, dtype
    ([(0, 1)], 1, 1, 64, 16, "rows", False, 1.0, "bf16"),
    ([(37, 1)], 16, 2, 128, 16, "rows", False, 1.0, "bf16"),
    ([(15, 1), (16, 1), (17, 1), (0, 0), (31, 1), (1, 1)], 8, 2, 128, 16, "heads", False, 0.9, "f16"),
    ([(100, 1), (3, 0), (64, 1)], 7, 1, 64, 24, "rows", False, 0.0, "bf16"),
    ([(200, 1), (129, 1)], 24, 8, 80, 7, "wide", False, 1.0, "bf16"),
    ([(50, 1)], 16, 1, 40, 1, "rows", False, 1.0, "f16"),
    ([(50, 1)], 32, 1, 8, 64, "rows", False, 0.5, "bf16"),
    ([(20, 3), (0, 5), (77, 1), (40, 0)], 4, 4, 128, 32, "rows", False, 1.0, "bf16"),
    ([(20, 13), (130, 6), (5, 1)], 8, 2, 128, 16, "heads", True, 1.0, "bf16"),
    ([(0, 64), (10, 33)], 4, 1, 64, 48, "rows", True, 0.0, "f16"),
    ([(60, 64)], 3, 3, 24, 5, "rows", True, 1.0, "bf16"),
    ([(300, 130)], 8, 2, 128, 32, "rows", False, 1.0, "bf16"),
    ([(0, 257), (33, 40), (500, 1)], 4, 1, 64, 16, "heads", False, 0.0, "f16"),
    ([(129, 100), (0, 0), (7, 300)], 6, 2, 120, 8, "wide", False, 0.99, "bf16"),
    ([(70, 90)], 2, 1, 128, 20, "rows", False, 1.0, "f16"),
    ([(1000, 1)] * 40 + [(20, 90)], 4, 2, 64, 16, "rows", False, 1.0, "bf16"),
    # a chain of many blocks among units of one; pages of a tile and more, of which a warp looks up many at once
    ([(700, 3)] * 12 + [(300, 200)], 16, 2, 128, 16, "rows", False, 1.0, "bf16"),
    ([(5000, 9), (0, 0), (64, 64), (9000, 30)], 8, 2, 64, 128, "heads", False, 0.9, "f16"),
    ([(5000, 90), (1, 1), (9000, 120)], 8, 2, 128, 256, "rows", False, 1.0, "bf16"),
    # several tiles for each CTA, odd numbers of them among them, of one block of rows or more
    ([(3900, 40), (1200, 33), (5000, 45), (130, 60)], 32, 8, 128, 32, "rows", False, 0.9, "bf16"),
    ([(3900, 140), (1200, 33), (5000, 145), (130, 60)], 32, 8, 128, 32, "rows", False, 0.9, "f16"),
    ([(3900, 13), (1200, 9), (5000, 11), (130, 2)], 16, 8, 120, 24, "heads", True, 1.0, "f16"),
]


def mass_inputs(torch, case, seed=1, spare=9):
    lengths, Hq, Hk, D, page, order, tree, decay, dtype = case
    g, rng = gen(torch, seed), np.random.default_rng(seed)
    total = [c + n for c, n in lengths]
    table, pages = block_table([-(-t // page) for t in total], rng)
    k = pool(torch, pages, page, Hk, D, dtype, order, g)
    N = sum(n for _, n in lengths)
    q = (torch.randn(N, Hq, D + 8, generator=g, device="cuda") * 2).to(dec.torch_dtype(dtype))[..., :D]
    off = np.concatenate([[0], np.cumsum([n for _, n in lengths])])
    mask = None
    if tree:  # some tokens see nothing of the new ones, themselves among them
        bits = [0] * N
        for b, (_, n) in enumerate(lengths):
            for j in range(n):
                bits[off[b] + j] = int(rng.integers(0, 2 ** 63)) & ((1 << n) - 1) if rng.random() < 0.8 else 0
        mask = torch.tensor(np.array(bits, np.uint64).view(np.int64), device="cuda")
    m = torch.rand(len(lengths), Hk, max(total) + spare, generator=g, device="cuda") * 3
    lse = torch.randn(N, Hq, generator=g, device="cuda") * 0.5 + 3
    return dict(k=k, q=q, table=table, off=off, mask=mask, mass=m, lse=lse, scale=D ** -0.5)


def call_mass(stride, torch, x, case, status=None, mass=None, **kw):
    stride.stride_attention_mass(x["q"], x["lse"], x["k"], i32(torch, x["table"]), i32(torch, [c for c, _ in case[0]]), i32(torch, x["off"]),
                                 x["mask"], x["scale"], x["mass"] if mass is None else mass, decay=case[7], dev_status=status, **kw)


def sees_of(x, case, b):
    c, n = case[0][b]
    back = np.arange(c + n) - c
    if x["mask"] is None:
        return back[None] <= np.arange(n)[:, None]
    bits = x["mask"].cpu().numpy().view(np.uint64)[x["off"][b]:x["off"][b] + n]
    return (back < 0)[None] | ((bits[:, None] >> np.clip(back, 0, 63).astype(np.uint64)[None]) & np.uint64(1)).astype(bool)


def check_mass(x, case, before, after, skip=()):
    lengths, Hq, Hk, D, *_, decay, _ = case
    G = Hq // Hk
    q, lse = dec.f64(x["q"]), dec.f64(x["lse"])
    for b, (c, n) in enumerate(lengths):
        L = c + n if n else 0
        assert np.array_equal(after[b, :, L:], before[b, :, L:], equal_nan=True), b
        if not n or b in skip:
            continue
        K = np.nan_to_num(slots(x["k"], x["table"], b, L), posinf=0, neginf=0)
        sees, rows = sees_of(x, case, b), slice(x["off"][b], x["off"][b] + n)
        for h in range(Hk):
            heads = slice(h * G, (h + 1) * G)
            want, tol = ref.mass(before[b, h], q[rows, heads], lse[rows, heads], K[:, h], c, sees, x["scale"], decay)
            bad = ~(np.abs(after[b, h, :L] - want) <= tol)
            assert not bad.any(), (b, h, np.flatnonzero(bad)[:5], after[b, h, :L][bad][:3], want[bad][:3], tol[bad][:3])


@pytest.mark.parametrize("case", MASS, ids=str)
def test_attention_mass(env, case):
    torch, stride, dev = env
    x = mass_inputs(torch, case)
    before = x["mass"].double().cpu().numpy()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    first = x["mass"].clone()
    call_mass(stride, torch, x, case, status)
    call_mass(stride, torch, x, case, mass=first)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.equal(first, x["mass"])  # the same call, the same bits
    check_mass(x, case, before, x["mass"].double().cpu().numpy())


@pytest.mark.parametrize("case", [MASS[3], MASS[8], MASS[9], MASS[12], MASS[13]], ids=str)
def test_what_no_row_sees(env, case):
    """NaN and infinities past a sequence's end, in new tokens' keys that no row sees, and, without a decay, in the masses."""
    torch, stride, dev = env
    x = mass_inputs(torch, case)
    page = x["k"].shape[1]
    for b, (c, n) in enumerate(case[0]):
        unseen = [j for j in range(c + n) if n and not sees_of(x, case, b)[:, j].any()]
        past = range(c + n, -(-(c + n) // page) * page)
        for i, j in enumerate([*unseen, *past]):
            x["k"][int(x["table"][b, j // page]), j % page] = (float("nan"), float("inf"))[i % 2]
    used = set(x["table"][x["table"] >= 0].tolist())
    for p in range(len(x["k"])):
        if p not in used:
            x["k"][p] = float("nan")
    if case[7] == 0:
        x["mass"].fill_(float("nan"))
    before = x["mass"].double().cpu().numpy()
    call_mass(stride, torch, x, case)
    check_mass(x, case, before, x["mass"].double().cpu().numpy())


def test_rows_that_see_nothing(env):
    """An lse of -inf adds nothing; keys with infinities, whose scores are infinite, are the formula's."""
    torch, stride, dev = env
    for case in (([(37, 1)], 4, 2, 64, 16, "rows", False, 1.0, "bf16"), ([(140, 70)], 4, 2, 64, 16, "rows", False, 1.0, "bf16")):
        x = mass_inputs(torch, case)
        x["lse"][::2, 1] = float("-inf")
        x["lse"][-1, 2:] = float("-inf")
        before = x["mass"].double().cpu().numpy()
        call_mass(stride, torch, x, case)
        check_mass(x, case, before, x["mass"].double().cpu().numpy())
        x["q"].copy_(x["q"].abs() + 0.1)
        x["k"][int(x["table"][0, 1]), 3] = float("-inf")  # (weight 0)
        x["mass"].zero_()
        call_mass(stride, torch, x, case)
        assert (x["mass"][0, :, 19] == 0).all() and torch.isfinite(x["mass"]).all()


def test_infinite_keys_that_rows_see(env):
    """Weights of 0 and nothing else, where a block's rows do not fill the products' columns."""
    torch, stride, dev = env
    for case in (([(37, 1)], 3, 1, 64, 16, "rows", False, 1.0, "bf16"), ([(140, 9), (300, 11)], 5, 1, 128, 16, "rows", False, 1.0, "bf16"),
                 ([(300, 37)], 6, 2, 64, 16, "rows", False, 1.0, "f16"), ([(130, 13), (20, 7)], 4, 2, 128, 16, "rows", True, 1.0, "bf16")):
        x = mass_inputs(torch, case)
        x["q"].copy_(x["q"].abs() + 0.1)
        lost = (3, 19, case[0][0][0] - 1)
        for j in lost:
            x["k"][int(x["table"][0, j // 16]), j % 16, :, 5] = float("-inf")
        before = x["mass"].double().cpu().numpy()
        call_mass(stride, torch, x, case)
        after = x["mass"].double().cpu().numpy()
        for j in lost:
            assert np.array_equal(after[0, :, j], before[0, :, j]), (case, j)
        x["k"].nan_to_num_(neginf=0.0)
        got = after.copy()
        got[0][:, list(lost)] = 0
        again = x["mass"]
        again.copy_(torch.from_numpy(before))
        call_mass(stride, torch, x, case)
        rest = again.double().cpu().numpy()
        rest[0][:, list(lost)] = 0
        assert np.array_equal(rest, got), case  # (other slots: the same bits)


def test_mass_layouts(env):
    """Masses of other strides; a slot without a page, lengths that do not fit, trees of too many tokens."""
    torch, stride, dev = env
    for case in (([(40, 1), (90, 1), (33, 1)], 8, 2, 64, 16, "rows", False, 1.0, "bf16"),
                 ([(40, 20), (90, 31), (33, 70)], 8, 2, 64, 16, "rows", False, 1.0, "bf16")):
        x = mass_inputs(torch, case)
        wide = torch.full((2, 4, x["mass"].shape[2] + 13), -1.0, device=dev)  # heads first, unaligned rows
        view = wide[:, 1:, 5:5 + x["mass"].shape[2]].transpose(0, 1)
        view.copy_(x["mass"])
        before = x["mass"].double().cpu().numpy()
        call_mass(stride, torch, x, case, mass=view)
        check_mass(x, case, before, view.double().cpu().numpy())
        rest = wide.clone()
        rest[:, 1:, 5:5 + x["mass"].shape[2]] = -1
        assert (rest == -1).all()
        # a slot without a page
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        kept = x["table"].copy()
        x["table"][1, 2] = len(x["k"])
        m = x["mass"].clone()
        call_mass(stride, torch, x, case, status, m)
        assert int(status) == BAD_LAYOUT
        got = m.double().cpu().numpy()
        assert np.isnan(got[1, :, 32:48]).all() and np.isfinite(got[1, :, :32]).all() and np.isfinite(got[1, :, 48:]).all()
        x["table"] = kept
        # masses that a sequence does not fit in
        status.zero_()
        longest = max(c + n for c, n in case[0])
        m = x["mass"][..., :longest - 1].clone()
        call_mass(stride, torch, x, case, status, m)
        assert int(status) == BAD_LAYOUT
        b = [c + n for c, n in case[0]].index(longest)
        assert torch.equal(m[b], x["mass"][b, :, :longest - 1])
        check_mass(x, case, before[..., :longest - 1], m.double().cpu().numpy(), skip=(b,))
        # a negative length, one that the table does not hold
        for wrong in (-3, x["table"].shape[1] * 16):
            status.zero_()
            m = x["mass"].clone()
            bad = (([(wrong, case[0][0][1])] + case[0][1:]),) + case[1:]
            call_mass(stride, torch, x, bad, status, m)
            assert int(status) == BAD_LAYOUT and torch.equal(m[0], x["mass"][0])
            assert not torch.equal(m[1], x["mass"][1])
    # more drafted tokens than a tree's mask holds
    case = ([(5, 65), (9, 3)], 2, 1, 64, 16, "rows", False, 1.0, "bf16")
    x = mass_inputs(torch, case)
    x["mask"] = torch.full((68,), 7, dtype=torch.int64, device=dev)
    status, m = torch.zeros(1, dtype=torch.int32, device=dev), x["mass"].clone()
    call_mass(stride, torch, x, case, status, m)
    assert int(status) == BAD_LAYOUT and torch.equal(m[0], x["mass"][0]) and not torch.equal(m[1], x["mass"][1])


def test_attention_weights_add_up(env):
    """With attention's own lse, a row's weights over its slots sum to 1."""
    torch, stride, dev = env
    for case in (MASS[2], MASS[8], MASS[11], MASS[12]):
        x = mass_inputs(torch, case)
        N, Hq, D = x["q"].shape
        Hk = case[2]
        args = i32(torch, x["table"]), i32(torch, [c for c, _ in case[0]]), i32(torch, x["off"])
        q = x["q"].contiguous()
        out = torch.empty_like(q)
        ws = torch.empty(stride.stride_tree_attention_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
        stride.stride_tree_attention(q, x["k"], x["k"], *args, x["mask"], x["scale"], out, lse=x["lse"], workspace=ws)
        x["mass"].zero_()
        call_mass(stride, torch, x, case)
        for b, (c, n) in enumerate(case[0]):
            rows = torch.isfinite(x["lse"][x["off"][b]:x["off"][b] + n]).unflatten(1, (Hk, -1)).sum((0, 2)).double()
            # lse is D 2^-24 scale sum |q k| and 4e-6 off, a weight twice that and 2^-22 and its sums' roundings; sum |q k| <= |q| |k|
            size = D * 2.0 ** -24 * x["scale"] * float(x["q"].double().norm(dim=-1).max()) * float(x["k"].double().norm(dim=-1).max())
            off = 3 * size + 4e-6 + 2.0 ** -22 + (c + n + n * Hq) * 2.0 ** -24
            assert ((x["mass"][b].double().sum(-1) - rows).abs() <= off * rows).all()


# ---------------------------------------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------------------------------------
EVICT = [
    # lengths, budgets (a number: all), Hk, D, page, page of the new pages, order, sink, recent, dtype
    ([1], 1, 1, 64, 16, 16, "rows", 0, 0, "bf16"),
    ([5, 0, 1], 0, 2, 64, 16, 16, "rows", 1, 1, "bf16"),
    ([37, 16, 17, 0, 90], 16, 2, 128, 16, 16, "rows", 0, 0, "bf16"),
    ([37, 16, 17, 0, 90], [20, 3, -1, 5, 89], 3, 80, 24, 16, "heads", 2, 3, "f16"),
    ([100, 33], 31, 1, 51, 7, 5, "rows", 31, 9, "f32"),
    ([100, 33], 31, 1, 6, 7, 5, "wide", 4, 31, "bf16"),
    ([640, 513, 512], 200, 2, 64, 64, 32, "heads", 4, 64, "bf16"),
    ([5000], 1234, 2, 64, 16, 16, "rows", 3, 77, "bf16"),
    ([20000, 3], 7777, 1, 32, 64, 64, "rows", 0, 0, "f16"),
    ([300000], 100, 1, 8, 64, 16, "rows", 10, 10, "bf16"),
    ([50] * 200, 13, 3, 16, 8, 8, "rows", 1, 2, "bf16"),
    ([9, 9], 9, 2, 1024, 4, 4, "rows", 0, 0, "f32"),
]
VALUES = ("spread", "ties", "equal", "wild")


def evict_inputs(torch, case, values, seed=2):
    lengths, budget, Hk, D, page, page_to, order, sink, recent, dtype = case
    g, rng = gen(torch, seed), np.random.default_rng(seed)
    B = len(lengths)
    budgets = [budget] * B if isinstance(budget, int) else budget
    m = [min(n, max(0, k)) for n, k in zip(lengths, budgets)]
    table, pages = block_table([-(-n // page) for n in lengths], rng)
    to_table, to_pages = block_table([-(-n // page_to) for n in m], rng)
    wide = max(max(lengths), 1) + 3
    mass = torch.exp(2 * torch.randn(B, Hk, wide, generator=g, device="cuda"))
    if values == "ties":
        mass = (4 * torch.rand(B, Hk, wide, generator=g, device="cuda")).floor()
    elif values == "equal":
        mass = torch.full_like(mass, 0.25)
    elif values == "wild":
        pick = torch.tensor([0.0, -0.0, float("inf"), float("-inf"), float("nan"), -1.5, 1e-42, 3e38], device="cuda")
        mass = torch.where(torch.rand(mass.shape, generator=g, device="cuda") < 0.4,
                           pick[torch.randint(0, 8, mass.shape, generator=g, device="cuda")], mass - 1)
    x = dict(mass=mass, table=table, to_table=to_table, m=m, budgets=budgets, most=max(max(m), 1) + 2)
    for name in ("k", "v"):
        x[name] = pool(torch, pages, page, Hk, D, dtype, order, g)
    for name in ("k_to", "v_to"):
        x[name] = pool(torch, to_pages, page_to, Hk, D, dtype, "rows" if order == "heads" else "heads", g)
    x["new_len"] = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    x["kept"] = torch.full((B, Hk, x["most"]), -7, dtype=torch.int32, device="cuda")
    x["mass_to"] = torch.full((Hk, B, x["most"] + 1), -7.0, device="cuda").transpose(0, 1)
    return x


def call_evict(stride, torch, x, case, status=None, mass_to=True, **kw):
    lengths, budget = case[:2]
    stride.stride_kv_evict(x["k"], x["v"], i32(torch, x["table"]), i32(torch, lengths), x["mass"],
                           budget if isinstance(budget, int) else i32(torch, budget), x["k_to"], x["v_to"], i32(torch, x["to_table"]),
                           x["new_len"], x["kept"], mass_to=x["mass_to"] if mass_to else None, sink=case[7], recent=case[8],
                           dev_status=status, **kw)


def check_evict(torch, x, case, before, skip=()):
    lengths, _, Hk, D, page, page_to, order, sink, recent, dtype = case
    want = {k: v.clone() for k, v in before.items()}
    mass = x["mass"].cpu().numpy()
    for b, n in enumerate(lengths):
        if b in skip:
            continue
        want["new_len"][b] = n if x["budgets"][b] < 0 else x["m"][b]
        if x["budgets"][b] < 0 or not x["m"][b]:
            continue
        i = np.arange(x["m"][b])
        there = x["to_table"][b, i // page_to], i % page_to
        for h in range(Hk):
            at = ref.remaining(mass[b, h], n, x["budgets"][b], sink, recent)
            want["kept"][b, h, :len(at)] = i32(torch, at)
            want["mass_to"][b, h, :len(at)] = x["mass"][b, h, list(at)]
            for name in ("k", "v"):
                want[name + "_to"][list(there[0]), list(there[1]), h] = x[name][list(x["table"][b, at // page]), list(at % page), h]
    for name, w in want.items():
        assert torch.equal(x[name].nan_to_num(nan=-99.0) if w.is_floating_point() else x[name],
                           w.nan_to_num(nan=-99.0) if w.is_floating_point() else w), name


def outputs(x):
    return {k: x[k].clone() for k in ("k_to", "v_to", "new_len", "kept", "mass_to")}


@pytest.mark.parametrize("case", EVICT, ids=lambda c: str(c) if len(c[0]) < 9 else f"{len(c[0])} x {c[0][0]}")
@pytest.mark.parametrize("values", VALUES)
def test_evict(env, case, values):
    torch, stride, dev = env
    x = evict_inputs(torch, case, values)
    before, source = outputs(x), (x["k"].clone(), x["v"].clone(), x["mass"].clone())
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    call_evict(stride, torch, x, case, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check_evict(torch, x, case, before)
    assert torch.equal(x["k"], source[0]) and torch.equal(x["v"], source[1])
    assert torch.equal(x["mass"].nan_to_num(nan=-99.0), source[2].nan_to_num(nan=-99.0))


def test_evict_within_a_pool(env):
    """The new pages are others of the same pools; no masses are asked for; the pages that two sequences share stay."""
    torch, stride, dev = env
    case = ([70, 64], 20, 2, 64, 16, 16, "rows", 2, 5, "bf16")
    x = evict_inputs(torch, case, "ties")
    x["table"][1, :3] = x["table"][0, :3]
    both = {}
    for name in ("k", "v"):
        both[name] = torch.cat([x[name], x[name + "_to"].contiguous()])
    first = len(x["k"])
    x["to_table"] = np.where(x["to_table"] >= 0, x["to_table"] + first, -1)
    x["k"] = x["k_to"] = both["k"]
    x["v"] = x["v_to"] = both["v"]
    before = outputs(x)
    source = x["k"].clone(), x["v"].clone()
    call_evict(stride, torch, x, case, mass_to=False)

    mass = x["mass"].cpu().numpy()
    for b in range(2):
        for h in range(2):
            at = ref.remaining(mass[b, h], case[0][b], 20, 2, 5)
            assert x["kept"][b, h, :20].tolist() == at.tolist()
            i = np.arange(20)
            got = x["k"][list(x["to_table"][b, i // 16]), list(i % 16), h]
            assert torch.equal(got, source[0][list(x["table"][b, at // 16]), list(at % 16), h])
    assert torch.equal(x["k"][:first], source[0][:first]) and torch.equal(x["v"][:first], source[1][:first])
    assert (x["mass_to"] == -7).all()


def test_evict_layouts(env):
    """Lengths and budgets that do not fit, slots without a page."""
    torch, stride, dev = env
    case = ([70, 64, 40], 20, 2, 64, 16, 16, "rows", 2, 5, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device=dev)

    def refused(change, b=1, status_of=BAD_LAYOUT):
        x = evict_inputs(torch, case, "ties")
        lengths = list(case[0])
        change(x, lengths)
        before = outputs(x)
        status.zero_()
        call_evict(stride, torch, x, (lengths,) + case[1:], status)
        assert int(status) == status_of
        before["new_len"][b] = -1
        check_evict(torch, x, (lengths,) + case[1:], before, skip=(b,))

    refused(lambda x, n: n.__setitem__(1, -1))
    refused(lambda x, n: n.__setitem__(1, 5 * 16 + 1))  # more than the table holds
    refused(lambda x, n: x.__setitem__("mass", x["mass"][..., :69].contiguous()), b=0)
    x = evict_inputs(torch, case, "ties")  # more remain than a row of kept holds
    x["kept"] = torch.full((3, 2, 19), -7, dtype=torch.int32, device=dev)
    status.zero_()
    call_evict(stride, torch, x, case, status)
    assert int(status) == BAD_LAYOUT and x["new_len"].tolist() == [-1, -1, -1] and (x["kept"] == -7).all()
    x = evict_inputs(torch, case, "ties")  # ... or than the new pages
    x["to_table"] = x["to_table"][:, :1]
    status.zero_()
    call_evict(stride, torch, x, case, status)
    assert int(status) == BAD_LAYOUT and x["new_len"].tolist() == [-1, -1, -1] and (x["kept"] == -7).all()
    for where in ("table", "to_table"):  # a slot without a page: all other rows are copied
        x = evict_inputs(torch, case, "ties")
        good, before = x[where].copy(), outputs(x)
        for wrong in (-1, 10 ** 6):
            x[where] = good.copy()
            x[where][2, 0] = wrong
            status.zero_()
            for name, t in before.items():
                x[name].copy_(t)
            call_evict(stride, torch, x, case, status)
            assert int(status) == BAD_LAYOUT
            lost = {k: v.clone() for k, v in before.items()}
            got = {k: x[k].clone() for k in before}
            x[where] = good
            if where == "table":
                at = [ref.remaining(x["mass"].cpu().numpy()[2, h], 40, 20, 2, 5) for h in range(2)]
                rows = [np.flatnonzero(a < 16) for a in at]
            else:
                rows = [np.arange(16)] * 2
            for name in ("k_to", "v_to"):  # (put right what was left out, after a look that it was)
                for h in range(2):
                    p, r = x["to_table"][2, rows[h] // 16], rows[h] % 16
                    assert torch.equal(got[name][list(p), list(r), h], lost[name][list(p), list(r), h])
                    a = ref.remaining(x["mass"].cpu().numpy()[2, h], 40, 20, 2, 5)[rows[h]]
                    x[name][list(p), list(r), h] = x[name[0]][list(x["table"][2, a // 16]), list(a % 16), h]
            check_evict(torch, x, case, before)
