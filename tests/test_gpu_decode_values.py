"""The decode step's operators on values, masks and sizes at the ends of what they
accept (tolerances: tests/decode_reference.py)."""
from __future__ import annotations

import numpy as np
import pytest

import decode_reference as ref
from test_gpu_decode_step import Paged, check_attention, check_sample, env, gen, logits, qk_inputs, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(torch, stride, c, q, scale, mask=None):
    """out, lse, status of a call."""
    N, Hq, D = q.shape
    out, lse = torch.full_like(q, 7.0), torch.full((N, Hq), 7.0, device=q.device)
    ws = torch.empty(stride.stride_tree_attention_workspace_size(N, Hq, c.k.shape[2], D), dtype=torch.uint8, device=q.device)
    status = torch.zeros(1, dtype=torch.int32, device=q.device)
    stride.stride_tree_attention(q, *c.args, mask, scale, out, lse=lse, workspace=ws, dev_status=status)
    torch.cuda.synchronize()
    return out, lse, int(status)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
def test_every_new_value_has_a_component_that_is_not_finite(env, dtype, D):  # noqa: F811
    """Rows of 16 and fewer: each new token's value is infinite in a component of its own, which the rows before it keep finite."""
    torch, stride, dev = env
    n_ctx, n_new, Hq = [5 * b % 41 for b in range(70)], [1 + b % 4 for b in range(70)], 4
    c = Paged(torch, n_ctx, n_new, 1, D, 16, dtype, False, 1)
    c.put(torch, gen(torch, 2))
    for b, (have, n) in enumerate(zip(n_ctx, n_new)):
        pg, row = c.slots(b, have + n)
        for j in range(n):
            c.v[int(pg[have + j]), int(row[have + j]), 0, (17 * b + 9 * j) % D] = float("inf")
    q = torch.randn((sum(n_new), Hq, D), generator=gen(torch, 3), device=dev).to(ref.torch_dtype(dtype))
    first, _, status = attend(torch, stride, c, q, D ** -0.5)
    assert status == 0
    for _ in range(20):
        assert torch.equal(attend(torch, stride, c, q, D ** -0.5)[0], first)
    Q, K, V, got, u, at = ref.f64(q), ref.f64(c.k), ref.f64(c.v), ref.f64(first), ref.UNIT[dtype], 0
    for b, (have, n) in enumerate(zip(n_ctx, n_new)):
        pg, row = c.slots(b, have + n)
        for i in range(n):
            for h in range(Hq):
                o, _, size = ref.attention(Q[at + i, h], K[pg, row, 0], V[pg, row, 0], np.arange(have + n) <= have + i, D ** -0.5)
                y, good = got[at + i, h], np.isfinite(o)
                assert good.sum() == D - i - 1 and (y[~good] == np.inf).all()
                assert (np.abs(y[good] - o[good]) <= u * size[good] + u * np.abs(o[good]) + 8 * 2e-6 * size[good] + 1e-30).all()
        at += n


@pytest.mark.parametrize("page", [8, 16, 64])
def test_missing_page_among_many_rows(env, page):  # noqa: F811
    """Wherever in a tile the page is missing, its sequence's rows are NaN and the other sequences' keep their bits."""
    torch, stride, dev = env
    c = Paged(torch, [300, 700, 200], [40, 40, 40], 2, 128, page, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = torch.randn((120, 8, 128), generator=gen(torch, 3), device=dev).bfloat16()
    good, good_lse, status = attend(torch, stride, c, q, 0.1)
    assert status == 0 and torch.isfinite(good).all()
    table = c.args[2].clone()
    for entry in {0, 1, 7, 650 // page, 699 // page}:
        for spoil in (-1, c.k.shape[0]):
            c.args[2].copy_(table)
            c.args[2][1, entry] = spoil
            out, lse, status = attend(torch, stride, c, q, 0.1)
            assert status == stride.DEV_BAD_LAYOUT
            assert torch.isnan(out[40:80]).all() and torch.isnan(lse[40:80]).all()
            for at in (slice(0, 40), slice(80, 120)):
                assert torch.equal(out[at], good[at]) and torch.equal(lse[at], good_lse[at])


def test_sample_of_more_columns_than_there_are(env):  # noqa: F811
    torch, stride, dev = env
    x = torch.zeros((4, 128), device=dev)[:, 28:]
    tokens = torch.full((4,), 7, dtype=torch.int32, device=dev)
    for V in (101, 128):
        with pytest.raises(ValueError, match="V"):
            stride.stride_sample(x, None, tokens, temperature=0, V=V)
    assert (tokens == 7).all()
    stride.stride_sample(x, None, tokens, temperature=0, V=100)
    assert not tokens.any()


# N, Hq, Hk, D, R, interleaved, norm, dtype, layout
PASS_THROUGH = [
    (5, 3, 1, 128, 64, False, False, "bf16", "plain"),
    (5, 3, 1, 128, 64, True, False, "bf16", "fused"),
    (7, 2, 2, 96, 36, True, False, "f16", "plain"),
    (7, 2, 2, 80, 16, False, False, "f32", "fused"),
    (6, 2, 1, 64, 0, False, False, "bf16", "plain"),
    (6, 5, 1, 64, 10, True, False, "f32", "plain"),
    (5, 3, 1, 128, 64, False, True, "bf16", "plain"),
    (5, 3, 1, 128, 64, True, True, "f16", "fused"),
    (9, 2, 1, 80, 40, True, True, "f32", "plain"),
    (4, 2, 1, 51, 22, False, False, "bf16", "odd"),
    (4, 2, 1, 51, 22, True, True, "f32", "odd"),
]


def the_same(got, want, tol):
    got, good = ref.f64(got), np.isfinite(want)
    assert np.array_equal(got[~good], want[~good], equal_nan=True), (got[~good], want[~good])
    bad = ~(np.abs(got[good] - want[good]) <= np.broadcast_to(tol, want.shape)[good])
    assert not bad.any(), (int(bad.sum()), got[good][bad][:4], want[good][bad][:4])


@pytest.mark.parametrize("case", PASS_THROUGH, ids=str)
def test_components_that_are_not_rotated_and_not_finite(env, case):  # noqa: F811
    """An infinity or NaN past rot_dim changes nothing else, but through the norm; forward, backward and append."""
    torch, stride, dev = env
    N, Hq, Hk, D, R, inter, norm, dtype, layout = case
    rows = [qk_inputs(torch, N, Hq, Hk, D, dtype, layout, s) for s in (1, 2)]
    for t in (t for x in rows for t in x):
        for token, comp, value in ((0, D - 1, np.inf), (1, R, -np.inf), (2, D - 3, np.nan), (2, D - 2, np.inf)):
            t[token, -1, comp] = value
    (q, k, v), (dyq, dyk, _) = rows
    dt, u, g = ref.torch_dtype(dtype), ref.UNIT[dtype], gen(torch, 3)
    cos, sin = tables(torch, N + 5, R)
    pos = torch.randint(1, N + 5, (N,), generator=g, device=dev).int() if R else None
    w = [(1 + 0.3 * torch.randn(D, generator=g, device=dev)).to(dt) if norm else None for _ in range(2)]
    how = dict(pos=pos, cos=cos, sin=sin, q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=inter)
    out, grads = ([torch.zeros_like(t, memory_format=torch.contiguous_format) for t in (q, k)] for _ in range(2))
    dw = [torch.zeros(D, device=dev) if norm else None for _ in range(2)]
    ws = torch.empty(stride.stride_qk_norm_rope_backward_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
    stride.stride_qk_norm_rope(q, k, *out, **how)
    clean = [qk_inputs(torch, N, Hq, Hk, D, dtype, layout, s)[:2] for s in (1, 2)]  # (rows without them)
    # (x finite, dy not: a gradient of an infinite x is NaN throughout)
    stride.stride_qk_norm_rope_backward(dyq, dyk, *clean[0], *grads, **how, dq_weight=dw[0], dk_weight=dw[1], workspace=ws)
    c = Paged(torch, [3], [N], Hk, D, 4, dtype, False, 1, fill=0.0)
    q_out = torch.zeros_like(out[0])
    stride.stride_kv_append(k, v, *c.args, q=q, q_out=q_out, **how)
    torch.cuda.synchronize()
    pg, row = (torch.from_numpy(a[3:]).to(dev).long() for a in c.slots(0, 3 + N))
    assert torch.equal(torch.nan_to_num(c.k[pg, row], 9.0), torch.nan_to_num(out[1], 9.0))
    assert torch.equal(torch.nan_to_num(c.v[pg, row], 9.0), torch.nan_to_num(v, 9.0))
    assert torch.equal(torch.nan_to_num(q_out, 9.0), torch.nan_to_num(out[0], 9.0))
    cs, sn = (ref.f64(t[pos.long()]) for t in (cos, sin)) if R else (None, None)
    with np.errstate(invalid="ignore"):
        for x, dy, x0, wt, y, dx, dwt, H in ((q, dyq, clean[0][0], w[0], out[0], grads[0], dw[0], Hq),
                                             (k, dyk, clean[0][1], w[1], out[1], grads[1], dw[1], Hk)):
            wt = None if wt is None else ref.f64(wt)
            want, size = ref.norm_rope(ref.f64(x), wt, 1e-5, cs, sn, inter)
            the_same(y, want, u * np.abs(want) + (D + 20) * 2.0 ** -24 * size)
            want, wantw, size, sizew = ref.norm_rope_backward(ref.f64(dy), ref.f64(x0), wt, 1e-5, cs, sn, inter)
            the_same(dx, want, u * np.abs(want) + (D + 20) * 2.0 ** -24 * size)
            if norm:
                the_same(dwt, wantw, 2.0 ** -24 * (D + 40 + np.sqrt(N * H)) * sizew)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n_new", [1, 40], ids=["few", "many"])
@pytest.mark.parametrize("nats", [0, 10, 18])
@pytest.mark.parametrize("sink", ["first", "last"])
def test_attention_of_a_long_tail_under_one_large_score(env, dtype, n_new, nats, sink):  # noqa: F811
    """One committed slot scores far above the others and has no value: the output is the tail's."""
    torch, stride, dev = env
    have, D = 20_000, 64
    c = Paged(torch, [have], [n_new], 1, D, 16, dtype, False, 1)
    pg, row = (torch.from_numpy(a).to(dev).long() for a in c.slots(0, have + n_new))
    c.k[pg, row], c.v[pg, row] = 0.0, (1 + 0.2 * torch.rand((have + n_new, 1, D), generator=gen(torch, 2), device=dev)).to(c.v.dtype)
    at = 0 if sink == "first" else have - 1
    c.k[pg[at], row[at], 0, 0], c.v[pg[at], row[at]] = float(nats), 0.0
    q = torch.zeros((n_new, 2, D), device=dev).to(c.k.dtype)
    q[..., 0] = 1.0
    check_attention(torch, stride, c, q, None, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_of_scores_as_large_as_their_steps(env, dtype):  # noqa: F811
    """Scores of 2^27 in units of ln 2, where 32 bits step by 16: a row's reference follows each step."""
    torch, stride, dev = env
    have, n_new, D, page = 40_000, 40, 64, 16
    scale = np.float32(16 * np.log(2))
    scale2 = np.float32(scale * np.float32(1.4426950408889634))
    m = [float(np.float32(np.float32(2 ** 23 + b) * scale2)) for b in range(8)]
    low = next(b for b in range(7) if (m[b] / 16) % 2 == 1 and m[b + 1] - m[b] == 16)
    c = Paged(torch, [have], [n_new], 1, D, page, dtype, False, 1)
    c.put(torch, gen(torch, 2))
    pg, row = (torch.from_numpy(a).to(dev).long() for a in c.slots(0, have + n_new))
    c.k[pg, row] = 0.0
    c.k[pg, row, 0, 0], c.k[pg, row, 0, 1] = 4096.0, float(low)
    tiles = np.random.default_rng(5).permutation(have // 64)[:have // 64 // 3]
    at = torch.from_numpy(tiles * 64 + 17).to(dev)
    c.k[pg[at], row[at], 0, 1] = float(low + 1)
    q = torch.zeros((n_new, 2, D), device=dev).to(c.k.dtype)
    q[..., 0], q[..., 1] = 2048.0, 1.0
    check_attention(torch, stride, c, q, None, float(scale), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_top_p_of_the_largest_flat_row(env, dtype):  # noqa: F811
    """Equal logits: top_p keeps the first of them, whose masses add up to nearly 2^63 units."""
    torch, stride, dev = env
    V, top_p = stride.MAX_TOP_P_VOCAB, [0.8, 0.9, 0.95]
    x = torch.full((3, V), 1.5, device=dev).to(ref.torch_dtype(dtype))
    noise = 1 + torch.rand((3, V), generator=gen(torch, 2), device=dev)
    kept = [int(np.ceil(p * V)) for p in top_p]
    for r, n in enumerate(kept):  # (a hundred-thousandth to either side of the last one)
        noise[r, n - 90], noise[r, n + 90] = 0.5, 0.1
    tokens, logp = torch.zeros(3, dtype=torch.int32, device=dev), torch.zeros(3, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    stride.stride_sample(x, noise, tokens, top_p=torch.tensor(top_p, device=dev), logp=logp, dev_status=status)
    assert int(status) == 0
    assert tokens.tolist() == [n - 90 for n in kept]
    assert (np.abs(ref.f64(logp) + np.log(kept)) <= 3e-5).all()  # (ln's own error, and the hundred-thousandth)


def test_sample_top_p_of_what_a_top_k_leaves_of_ties(env):  # noqa: F811
    """The last of top_k tokens is the second of four equal ones, which lie far apart, and many that are hardly smaller follow; a
    top_p of nearly 1 keeps all that top_k leaves.  The tokens that come next would win if they were kept."""
    torch, stride, dev = env
    rows, V, top_k, below = 32, 40_000, 2001, 1500
    rng = np.random.default_rng(6)
    x, noise = torch.full((rows, V), -30.0), torch.empty((rows, V)).exponential_(generator=torch.Generator().manual_seed(7)) + 0.1
    for r in range(rows):
        value = np.concatenate([0.001 + rng.random(top_k - 2), np.zeros(4), -0.001 - 0.02 * rng.random(below)])
        ties = 10 + r, 50 + r, V - 5000 - r, V - 10 - r
        at = np.concatenate([rng.choice(np.arange(5100, V - 10_000), top_k - 2, replace=False), ties, rng.choice(np.arange(100, 4900), below, replace=False)])
        x[r, at] = torch.from_numpy(value.astype(np.float32))
        noise[r, at[top_k:]] = 1e-4  # (not kept)
    check_sample(torch, stride, x.to(dev), noise.to(dev), 1.0, [top_k] * rows, [float(np.float32(1 - 2.0 ** -24))] * rows, 0.0)


@pytest.mark.parametrize("rows,min_p,top_p", [(1, 0.5, 1.0), (305, 0.5, 1.0), (305, 0.5, 0.999)])
def test_sample_equal_ratios(env, rows, min_p, top_p):  # noqa: F811
    """Equal logits and equal noise, wherever they lie in a row: the lowest index is drawn."""
    torch, stride, dev = env
    V, rng = 151_936, np.random.default_rng(rows)
    x = torch.randn((rows, V), generator=gen(torch, 4), device=dev).clamp_(max=4).bfloat16()
    at = rng.integers(0, V, (rows, 3))
    for r in range(rows):  # (in half of the rows in places that one thread comes to out of order)
        if r % 2 == 0:
            lane = r // 2 % 6
            at[r] = 8 * (16_384 + 512 * lane), 8 * (512 * lane + 1) + 3, 8 * (512 * lane + 2) + 1
    x[torch.arange(rows, device=dev)[:, None], torch.from_numpy(at).to(dev)] = 8.0
    tokens = torch.zeros(rows, dtype=torch.int32, device=dev)
    stride.stride_sample(x, torch.ones((rows, V), device=dev), tokens, min_p=min_p, top_p=top_p)
    assert tokens.tolist() == at.min(1).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [1e-45, 1e-40, 4e-39, 2e-38])
def test_sample_at_the_smallest_temperatures(env, dtype, T):  # noqa: F811
    """The largest logits alone, by their noise."""
    torch, stride, dev = env
    x, noise = logits(torch, 8, 5003, dtype, 5)
    x = x.round()
    x[::2] -= x[::2].amax(1, keepdim=True)  # (rows whose largest is 0, and others)
    for k, p, m in ((0, 1.0, 0.0), (3, 1.0, 0.0), (2000, 0.5, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.3)):
        check_sample(torch, stride, x, noise, [T] * 8, [k] * 8, [p] * 8, [m] * 8)


@pytest.mark.parametrize("T", [1.0, 600.0, 1000.0, 60_000.0])
def test_sample_lowest_value_of_half(env, T):  # noqa: F811
    """A mask of -65504 is a logit: its weight is 0 up to a temperature of 600, and counts from some 630 on."""
    torch, stride, dev = env
    x, noise = logits(torch, 12, 3001, "f16", 8)
    x[:, ::3] = torch.finfo(x.dtype).min
    noise[:, ::3] = 1e-30
    for k, p, m in ((0, 1.0, 0.0), (2500, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 1e-4)):
        tokens, _ = check_sample(torch, stride, x, noise, [T] * 12, [k] * 12, [p] * 12, [m] * 12)
        if T <= 600:
            assert (tokens % 3 != 0).all()
