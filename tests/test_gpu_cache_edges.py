"""Attention weight per slot and eviction where a call's parts are missing, infinite or laid out backwards, against
the same call on whole inputs or their plain forms in 64 bits (tests/cache_reference.py, which states the
tolerances)."""
from __future__ import annotations

import ctypes
import importlib.util
import sys
from pathlib import Path

import numpy as np
import pytest

import decode_reference as dec
from test_gpu_cache import BAD_LAYOUT, call_evict, call_mass, check_mass, evict_inputs, i32, mass_inputs, outputs, sees_of, slots

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


# ---------------------------------------------------------------------------------------------------------------------
# attention weights
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page", [128, 256, 16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [13, 90], ids=["52 rows", "360 rows"])
@pytest.mark.parametrize("lost", ["first", "last", "all of one", "all", "many"])
def test_tiles_without_pages(env, page, D, new, lost):
    """Whole tiles of 128 slots have no page, in a call of several tiles for each CTA: NaN there, all other slots as if the
    pages were there (a slot's sum is its own: the same bits)."""
    torch, stride, dev = env
    case = ([(20000, new), (700, new), (0, new), (130, new)], 32, 8, D, page, "rows", False, 0.9, "bf16")
    x = mass_inputs(torch, case)
    before = x["mass"].clone()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    call_mass(stride, torch, x, case, status)
    assert int(status) == 0
    whole = x["mass"].double().cpu().numpy()
    check_mass(x, case, before.double().cpu().numpy(), whole, skip=(0,))
    # the pages of those runs of 128 slots (or of a page, where it is longer)
    run, rng = max(128, page), np.random.default_rng(page)
    total = [c + n for c, n in case[0]]
    runs = [(b, r) for b, t in enumerate(total) for r in range(-(-t // run))]
    gone = {"first": [(0, 0)], "last": [(3, -(-total[3] // run) - 1), (0, -(-total[0] // run) - 1)],
            "all of one": [r for r in runs if r[0] == 1], "all": runs,
            "many": [r for r in runs if rng.random() < 0.5]}[lost]
    nan = np.zeros(whole.shape, bool)
    for b, r in gone:
        x["table"][b, r * run // page:(r + 1) * run // page] = (-1, len(x["k"]), 2 ** 31 - 1)[r % 3]
        nan[b, :, r * run:min((r + 1) * run, total[b])] = True
    for _ in range(3):
        m = before.clone()
        status.zero_()
        call_mass(stride, torch, x, case, status, m)
        assert int(status) == BAD_LAYOUT
        got = m.double().cpu().numpy()
        assert np.isnan(got[nan]).all() and np.array_equal(got[~nan], whole[~nan])


# sequences whose last block of rows (128 / group tokens) has a ragged run of 32 columns after a whole one: new tokens, Hq, Hk, D, tree
RAGGED = [
    # up to 256 rows a sequence: 40, 34, 63, 126 = 96 + 30 columns, 40 and 100 under trees
    (20, 4, 2, 64, False), (17, 2, 1, 128, False), (21, 3, 1, 64, False), (42, 3, 1, 128, False), (20, 4, 2, 128, True), (25, 4, 1, 64, True),
    # more: a last block of 40, 68, 116 columns; of 36 and 112 under trees (groups of 8, 9, 14)
    (74, 8, 2, 64, False), (81, 4, 1, 128, False), (93, 4, 1, 64, False), (53, 8, 1, 128, True), (46, 9, 1, 64, True), (35, 14, 1, 128, True),
]


def ragged(torch, shape, decay=1.0, dtype="bf16"):
    """Two sequences, of whose slots a warp's 32 have committed and new ones, all seen by a block's later rows; q of either sign."""
    new, Hq, Hk, D, tree = shape
    case = ([(120, new), (1000, new)], Hq, Hk, D, 16, "rows", tree, decay, dtype)
    x = mass_inputs(torch, case)
    if tree:  # a block's first token sees itself alone, the others all
        tokens, bits = 128 // (Hq // Hk), np.full(2 * new, (1 << new) - 1, np.uint64)
        for i in range(2 * new):
            if i % new % tokens == 0:
                bits[i] = 1 << (i % new)
        x["mask"] = torch.tensor(bits.view(np.int64), device="cuda")
    return case, x


@pytest.mark.parametrize("shape", RAGGED, ids=str)
def test_rows_of_any_values_that_do_not_vote(env, shape):
    """An lse of -inf: the row may hold NaN and infinities, wherever in a block it is."""
    torch, stride, dev = env
    new, Hq, Hk, D, _ = shape
    tokens = 128 // (Hq // Hk)
    for some in ([0], list(range(0, new, tokens)), [new - 1], [min(new // tokens * tokens, new - 1)], list(range(0, new, 3))):
        case, x = ragged(torch, shape)
        for i, t in enumerate(some):
            for b in range(2):
                x["lse"][b * new + t] = float("-inf")
                x["q"][b * new + t] = (float("nan"), float("inf"), float("-inf"))[i % 3]
        before = x["mass"].double().cpu().numpy()
        call_mass(stride, torch, x, case)
        check_mass(x, case, before, x["mass"].double().cpu().numpy())


@pytest.mark.parametrize("shape", RAGGED, ids=str)
def test_infinite_new_keys(env, shape):
    """A new key whose scores are -inf for the rows that see it and +inf or NaN for those that do not: weights of 0, and all other
    slots as if it were finite, with the same bits.  And one whose scores are +inf for the rows that see it: that slot is infinite."""
    torch, stride, dev = env
    new, Hq, Hk, D, tree = shape
    tokens = 128 // (Hq // Hk)
    at = [3] if tree else [t for t in (*range(1, 8), tokens + 1, 2 * tokens + 2) if t < new]
    for value, j in [(v, j) for v in ("-inf", "+inf") for j in at]:
        case, x = ragged(torch, shape)
        x["q"][..., 5] = x["q"][..., 5].abs() + 0.1
        sees = (np.arange(new) >= j) if not tree else np.arange(new) % tokens != 0
        for b in range(2):
            for i in np.flatnonzero(~sees):
                x["q"][b * new + int(i), :, 5] *= (-1, 0)[int(i) % 2]  # (+inf, NaN)
        finite = x["mass"].clone()
        call_mass(stride, torch, x, case, mass=finite)
        for b, (c, _) in enumerate(case[0]):
            x["k"][int(x["table"][b, (c + j) // 16]), (c + j) % 16, :, 5] = float(value)
        call_mass(stride, torch, x, case)
        for b, (c, _) in enumerate(case[0]):
            assert (x["mass"][b, :, c + j] == (0.0 if value == "-inf" else float("inf"))).all(), (value, j, x["mass"][b, :, c + j])
            x["mass"][b, :, c + j] = finite[b, :, c + j]
        assert torch.equal(x["mass"], finite), (value, j)
        assert finite.isfinite().all()


@pytest.mark.parametrize("case", [
    # trees (and a chain) of more than 256 rows a sequence: several blocks, whose columns' halves are of two warps; last blocks of few
    # columns; groups that do not divide 128, and one of a token a block
    ([(700, 64), (130, 60), (0, 50)], 32, 4, 128, 16, "rows", True, 0.9, "bf16"),
    ([(700, 64), (0, 0), (130, 33), (5, 64)], 32, 4, 64, 8, "heads", True, 1.0, "f16"),
    ([(300, 64), (40, 61), (0, 11)], 24, 1, 64, 16, "rows", True, 1.0, "bf16"),
    ([(1000, 64), (90, 55), (127, 37)], 14, 2, 128, 24, "wide", True, 0.5, "f16"),
    ([(90, 64), (64, 63), (3, 1)], 40, 4, 24, 32, "rows", True, 0.0, "bf16"),
    ([(200, 13), (129, 3)], 128, 1, 64, 16, "rows", True, 1.0, "bf16"),
    ([(200, 13), (129, 3), (0, 2)], 200, 2, 128, 16, "rows", False, 1.0, "f16"),
    ([(2000, 64)] * 24, 16, 2, 128, 64, "rows", True, 0.9, "bf16"),
], ids=str)
def test_trees_of_many_rows(env, case):
    torch, stride, dev = env
    x = mass_inputs(torch, case)
    before = x["mass"].double().cpu().numpy()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    again = x["mass"].clone()
    call_mass(stride, torch, x, case, status)
    call_mass(stride, torch, x, case, mass=again)
    assert int(status) == 0 and torch.equal(again, x["mass"])
    check_mass(x, case, before, x["mass"].double().cpu().numpy(), skip=() if len(case[0]) < 9 else range(3, 23))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,Hq,Hk,D", [(1, 8, 2, 64), (13, 8, 2, 128), (20, 6, 1, 64), (90, 8, 2, 64), (81, 4, 1, 128)], ids=str)
def test_large_scores(env, new, Hq, Hk, D, dtype):
    """Scores of about 2,048 that are whole eighths, lse that are whole sixteenths, both exact in 32 bits: what is left of a weight's
    error is what the header states.  Its factors scale log2 e and lse log2 e are rounded once each, 2^-24 (|s| + |lse|); the constant's
    rounding is common to both, 2^-24 |s - lse|, and so is that of their difference; the exponential's is 2^-22.  A sum of R weights
    and the masses' last one: (R + 2) 2^-24."""
    torch, stride, dev = env
    case = ([(300, new), (37, new)], Hq, Hk, D, 16, "rows", False, 1.0, dtype)
    x = mass_inputs(torch, case)
    for name in ("q", "k"):
        x[name].copy_(torch.where(x[name] > 0.5, 1.0, torch.where(x[name] < -0.5, -1.0, 0.0)))
        x[name][..., 0] = 128
    x["scale"] = 0.125
    x["lse"].copy_(2048 + 3 + torch.arange(Hq, device=dev) * 0.4375)  # (alike for all of a head's rows: roundings do not cancel)
    x["mass"].zero_()
    call_mass(stride, torch, x, case)
    got, G = x["mass"].double().cpu().numpy(), Hq // Hk
    q, lse = dec.f64(x["q"]), dec.f64(x["lse"])
    for b, (c, n) in enumerate(case[0]):
        K, sees = slots(x["k"], x["table"], b, c + n), sees_of(x, case, b)
        for h in range(Hk):
            rows, heads = slice(x["off"][b], x["off"][b] + n), slice(h * G, (h + 1) * G)
            d = q[rows, heads] @ K[:, h].T * 0.125 - lse[rows, heads, None]  # [n, G, slots]
            assert np.array_equal(d * 16, np.round(d * 16)) and np.abs(d).max() < 2.0 ** 8
            e = np.exp(d) * sees[:, None]
            want, R = e.sum((0, 1)), n * G
            off = 2.0 ** -24 * (np.abs(d + lse[rows, heads, None]) + np.abs(lse[rows, heads, None])) + 2.0 ** -23 * np.abs(d) + 2.0 ** -22
            tol = (e * np.expm1(off)).sum((0, 1)) + (R + 2) * 2.0 ** -24 * want
            error = np.abs(got[b, h, :c + n] - want)
            assert (error <= tol).all(), (b, h, (error / want).max(), (tol / want).min())


# ---------------------------------------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("budget", [-1, [-1, 8, -7]], ids=str)
def test_the_example_keeps_all_slots_of_a_negative_budget(env, budget):
    """Such a sequence's slots and their masses go along to the new pages: with all kept, the next logits are the same bits."""
    torch, stride, dev = env
    path = Path(__file__).resolve().parents[1] / "examples" / "rollout.py"
    spec = importlib.util.spec_from_file_location("rollout_example_edges", path)
    example = importlib.util.module_from_spec(spec)
    sys.modules[spec.name] = example
    spec.loader.exec_module(example)
    counts = torch.tensor([37, 20, 5], device=dev)
    tokens = torch.randint(0, 4096, (int(counts.sum()),), generator=torch.Generator(device="cuda").manual_seed(6), device=dev).int()
    zero, more = torch.zeros(3, dtype=torch.int32, device=dev), torch.tensor([7, 8, 9], dtype=torch.int32, device=dev)
    models = [example.Model(example.Shape(), 3, 1) for _ in range(2)]
    for m in models:
        m.watch()
        m(tokens, example.chain(zero, counts), zero, example.offsets(counts))
    ctx = counts.int()
    m, other = models
    new_len = m.evict(ctx, budget if isinstance(budget, int) else i32(torch, budget))
    left = torch.where(torch.tensor(budget, device=dev) < 0, ctx, torch.tensor(budget, device=dev))
    assert torch.equal(new_len, left.int()) and int(m.status) == 0
    page = m.s.page
    for layer in range(m.s.layers):
        for b in range(3):
            if int(left[b]) < int(ctx[b]):
                continue
            i = torch.arange(int(ctx[b]), device=dev)
            at = m.table[b].long()[i // page], i % page
            for a, c in zip(m.cache[layer], other.cache[layer]):
                assert torch.equal(a[at], c[at])
            assert torch.equal(m.mass[layer][b, :, :len(i)], other.mass[layer][b, :, :len(i)])
    step = example.offsets(torch.ones_like(counts))
    a, c = m(more, ctx, new_len, step), other(more, ctx, ctx, step)
    assert a.isfinite().all()
    if isinstance(budget, int):
        assert torch.equal(a, c)


@pytest.mark.parametrize("backwards", ["heads", "rows", "pages", "all"])
@pytest.mark.parametrize("side", ["from", "to", "both"])
@pytest.mark.parametrize("D", [64, 51], ids=["vectors", "elements"])
def test_evict_pools_of_negative_strides(env, backwards, side, D):
    """A pool whose base is its last head, row or page, through the C entry: the same rows as in a pool that is flipped in memory."""
    torch, stride, dev = env
    from paper_2609_14636_gb300 import decode

    case = ([70, 64, 90], 20, 3, D, 16, 8, "rows", 2, 5, "bf16")
    dims = {"pages": [0], "rows": [1], "heads": [2], "all": [0, 1, 2]}[backwards]

    def call(flip):
        """Outputs, in the order of the pools that are not flipped."""
        x = evict_inputs(torch, case, "spread")
        i = dict(table=i32(torch, x["table"]), to=i32(torch, x["to_table"]), n=i32(torch, case[0]))
        held = []

        def cache(names, table, turned):
            pools = [x[n].contiguous() for n in names]
            strides, base = list(pools[0].stride()[:3]), 0
            if turned:
                pools = [p.flip(dims) for p in pools]
                for d in dims:
                    base += (pools[0].shape[d] - 1) * strides[d] * pools[0].element_size()
                    strides[d] = -strides[d]
            held.append((pools, turned))
            return decode._PagedCache(pools[0].data_ptr() + base, pools[1].data_ptr() + base, *strides, *pools[0].shape[:3], 3, table.data_ptr(),
                                      table.shape[1], i["n"].data_ptr(), None)

        source, to = cache("kv", i["table"], flip and side != "to"), cache(["k_to", "v_to"], i["to"], flip and side != "from")
        m, m2 = decode._slot_mass(x["mass"], "mass", 3, 3), decode._slot_mass(x["mass_to"], "mass_to", 3, 3)
        how = decode._EvictParams(None, case[1], case[7], case[8], x["most"])
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()
        assert stride.lib().stride_kv_evict(ctypes.byref(source), ctypes.byref(m), ctypes.byref(to), 0, D, ctypes.byref(how),
                                            x["new_len"].data_ptr(), x["kept"].data_ptr(), ctypes.byref(m2), status.data_ptr(), None) == 0
        torch.cuda.synchronize()
        assert int(status) == 0
        pools, turned = held[1]
        return [p.flip(dims) if turned else p for p in pools] + [x["new_len"], x["kept"], x["mass_to"]]

    for got, want in zip(call(True), call(False)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 40, -2 ** 31 - 1, 10 ** 30], ids=str)
@pytest.mark.parametrize("name", ["budget", "sink", "recent"])
def test_evict_numbers_past_32_bits(env, name, big):
    """Refused, not cut: 2^40 slots would be none, 2^31 a sequence that is left out."""
    torch, stride, dev = env
    case = ([70, 64], 20, 2, 64, 16, 16, "rows", 2, 5, "bf16")
    x = evict_inputs(torch, case, "spread")
    before = outputs(x)
    case = case[:1] + (big if name == "budget" else 20,) + case[2:7] + (big if name == "sink" else 2, big if name == "recent" else 5) + case[9:]
    with pytest.raises(ValueError, match=f"{name} is {big}, beyond 32 bits"):
        call_evict(stride, torch, x, case)
    torch.cuda.synchronize()
    for k, t in before.items():
        assert torch.equal(x[k], t)
