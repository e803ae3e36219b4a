"""The decode step's operators against their plain forms in 64 bits
(tests/decode_reference.py, which states the tolerances)."""
from __future__ import annotations

import numpy as np
import pytest

import decode_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


def gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def tables(torch, rows, R):
    if R == 0:
        return None, None
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    return a.cos().float().contiguous(), a.sin().float().contiguous()


def close(got, want, tol):
    got = ref.f64(got)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], np.broadcast_to(tol, want.shape)[bad][:4])


# ---------------------------------------------------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------------------------------------------------
QK = [
    # N, Hq, Hk, D, R, interleaved, norm, dtype, layout
    (1, 1, 1, 128, 128, False, True, "bf16", "plain"),
    (3, 8, 2, 128, 128, True, True, "bf16", "fused"),
    (37, 5, 1, 64, 32, False, True, "f16", "fused"),
    (33, 4, 4, 96, 96, False, True, "bf16", "fused"),
    (9, 7, 1, 80, 40, False, True, "bf16", "fused"),
    (9, 7, 1, 80, 40, True, True, "f16", "plain"),
    (5, 3, 2, 256, 128, False, True, "bf16", "fused"),
    (5, 3, 2, 512, 256, False, True, "bf16", "plain"),
    (5, 3, 2, 512, 512, True, True, "f32", "plain"),
    (2, 2, 1, 1024, 1024, False, True, "f32", "fused"),
    (2, 2, 1, 1024, 64, True, True, "bf16", "plain"),
    (21, 3, 1, 50, 22, False, True, "f32", "plain"),
    (21, 3, 1, 51, 22, True, True, "bf16", "odd"),
    (300, 9, 3, 128, 64, True, True, "f32", "odd"),
    (11, 2, 2, 128, 0, False, True, "bf16", "plain"),
    (11, 2, 2, 128, 128, False, False, "bf16", "fused"),
    (2000, 4, 1, 64, 64, False, True, "bf16", "fused"),
    (1, 1, 1, 1, 0, False, True, "f32", "plain"),
    (4, 1, 1, 2, 2, False, True, "f32", "plain"),
]


def qk_inputs(torch, N, Hq, Hk, D, dtype, layout, seed):
    g, dt = gen(torch, seed), ref.torch_dtype(dtype)
    if layout == "plain":
        return [torch.randn((N, h, D), generator=g, device="cuda").to(dt) for h in (Hq, Hk, Hk)]
    pad = 3 if layout == "odd" else 8  # "odd": rows that start at no vector's boundary
    x = torch.randn((N, (Hq + 2 * Hk) * D + pad), generator=g, device="cuda").to(dt)
    x = x[:, pad:] if layout == "odd" else x[:, :-pad]
    return [t.unflatten(1, (-1, D)) for t in x.split([Hq * D, Hk * D, Hk * D], dim=1)]


@pytest.mark.parametrize("case", QK, ids=str)
def test_norm_rope_and_backward(env, case):
    torch, stride, dev = env
    N, Hq, Hk, D, R, inter, norm, dtype, layout = case
    q, k, _ = qk_inputs(torch, N, Hq, Hk, D, dtype, layout, 1)
    dyq, dyk, _ = qk_inputs(torch, N, Hq, Hk, D, dtype, layout, 2)
    g, dt, u = gen(torch, 3), ref.torch_dtype(dtype), ref.UNIT[dtype]
    cos, sin = tables(torch, N + 5, R)
    pos = torch.randint(0, N + 5, (N,), generator=g, device=dev).int() if R else None
    w = [(1 + 0.3 * torch.randn(D, generator=g, device=dev)).to(dt) if norm else None for _ in range(2)]
    out = [torch.full_like(t, float("nan"), memory_format=torch.contiguous_format) for t in (q, k)]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    how = dict(pos=pos, cos=cos, sin=sin, q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=inter)
    stride.stride_qk_norm_rope(q, k, *out, **how, dev_status=status)
    grads = [torch.full_like(t, float("nan"), memory_format=torch.contiguous_format) for t in (q, k)]
    dw = [torch.full((D,), float("nan"), device=dev) if norm else None for _ in range(2)]
    ws = torch.empty(stride.stride_qk_norm_rope_backward_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
    stride.stride_qk_norm_rope_backward(dyq, dyk, q, k, *grads, **how, dq_weight=dw[0], dk_weight=dw[1], workspace=ws, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    c = s = None
    if R:
        at = pos.long()
        c, s = ref.f64(cos[at]), ref.f64(sin[at])
    for x, dy, wt, y, dx, dwt, H in ((q, dyq, w[0], out[0], grads[0], dw[0], Hq), (k, dyk, w[1], out[1], grads[1], dw[1], Hk)):
        wt = None if wt is None else ref.f64(wt)
        want, size = ref.norm_rope(ref.f64(x), wt, 1e-5, c, s, inter)
        close(y, want, u * np.abs(want) + (D + 20) * 2.0 ** -24 * size)
        want, wantw, size, sizew = ref.norm_rope_backward(ref.f64(dy), ref.f64(x), wt, 1e-5, c, s, inter)
        close(dx, want, u * np.abs(want) + (D + 20) * 2.0 ** -24 * size)
        if norm:
            close(dwt, wantw, 2.0 ** -24 * (D + 40 + np.sqrt(N * H)) * sizew)


def test_gradient_against_differences():
    """The reference's gradient (which the kernel is held to above) against central differences of its forward form."""
    rng = np.random.default_rng(5)
    x, dy, w = rng.standard_normal((3, 2, 12)), rng.standard_normal((3, 2, 12)), 1 + rng.standard_normal(12)
    a = rng.standard_normal((3, 4))
    for inter in (False, True):
        f = lambda x, w: float((ref.norm_rope(x, w, 1e-3, np.cos(a), np.sin(a), inter)[0] * dy).sum())  # noqa: B023, E731
        dx, dw, _, _ = ref.norm_rope_backward(dy, x, w, 1e-3, np.cos(a), np.sin(a), inter)
        h = 1e-5
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = h
            assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[i]) < 1e-7
        for i in range(12):
            e = np.zeros(12)
            e[i] = h
            assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[i]) < 1e-7


def test_gradient_kernel_against_differences(env):
    """dq of the fp32 kernel against differences of the forward kernel's sums (64-bit sums of 32-bit results)."""
    torch, stride, dev = env
    N, H, D = 2, 3, 64
    q, k, _ = qk_inputs(torch, N, H, 1, D, "f32", "plain", 7)
    dyq, dyk, _ = qk_inputs(torch, N, H, 1, D, "f32", "plain", 8)
    cos, sin = tables(torch, 9, 32)
    how = dict(pos=torch.tensor([3, 8], dtype=torch.int32, device=dev), cos=cos, sin=sin,
               q_weight=torch.linspace(0.5, 1.5, D, device=dev), k_weight=torch.linspace(1.5, 0.5, D, device=dev))
    dq, dk, dwq = torch.empty_like(q), torch.empty_like(k), torch.empty(D, device=dev)
    ws = torch.empty(stride.stride_qk_norm_rope_backward_workspace_size(N, H, 1, D), dtype=torch.uint8, device=dev)
    stride.stride_qk_norm_rope_backward(dyq, dyk, q, k, dq, dk, **how, dq_weight=dwq, workspace=ws)

    def value(q, k):
        a, b = torch.empty_like(q), torch.empty_like(k)
        stride.stride_qk_norm_rope(q, k, a, b, **how)
        return float((a.double() * dyq).sum() + (b.double() * dyk).sum())

    g, h = gen(torch, 9), 2.0 ** -7
    for _ in range(6):
        eq, ek = torch.randn(q.shape, generator=g, device=dev), torch.randn(k.shape, generator=g, device=dev)
        diff = (value(q + h * eq, k + h * ek) - value(q - h * eq, k - h * ek)) / (2 * h)
        want = float((dq.double() * eq).sum() + (dk.double() * ek).sum())
        # second-order truncation h^2 and 32-bit results (2^-24 of sums of about 25) over h
        assert abs(diff - want) < 0.02 * (1 + abs(want)), (diff, want)


def test_norm_rope_in_place_position_and_stream(env):
    """Outputs may be the inputs; a position outside the tables makes that token's rows NaN; any stream."""
    torch, stride, dev = env
    q, k, _ = qk_inputs(torch, 4, 2, 1, 128, "bf16", "plain", 4)
    cos, sin = tables(torch, 8, 128)
    pos = torch.tensor([0, 8, -1, 7], dtype=torch.int32, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    want = [torch.empty_like(q), torch.empty_like(k)]
    stride.stride_qk_norm_rope(q, k, *want, pos=pos, cos=cos, sin=sin, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == stride.DEV_POSITION
    for t in want:
        assert torch.isnan(t[1:3]).all() and not torch.isnan(t[0]).any() and not torch.isnan(t[3]).any()
    side = torch.cuda.Stream()
    stride.stride_qk_norm_rope(q, k, q, k, pos=pos, cos=cos, sin=sin, stream=side)
    side.synchronize()
    assert torch.equal(torch.nan_to_num(q), torch.nan_to_num(want[0])) and torch.equal(torch.nan_to_num(k), torch.nan_to_num(want[1]))


def test_norm_rope_without_tokens(env):
    torch, stride, dev = env
    q, k = torch.empty((0, 2, 64), device=dev), torch.empty((0, 1, 64), device=dev)
    w = torch.ones(64, device=dev)
    dw = torch.full((64,), 5.0, device=dev)
    stride.stride_qk_norm_rope(q, k, q, k)
    stride.stride_qk_norm_rope_backward(q, k, q, k, q, k, q_weight=w, dq_weight=dw)
    assert not dw.any()  # no rows: the sum is zero


# ---------------------------------------------------------------------------------------------------------------------
# a paged cache
# ---------------------------------------------------------------------------------------------------------------------
class Paged:
    """Sequences of the given lengths in a pool of pages in random order, with pages to spare."""

    def __init__(self, torch, n_ctx, n_new, Hk, D, page, dtype, heads_first, seed, fill=float("nan")):
        self.n_ctx, self.n_new, self.page = n_ctx, n_new, page
        dt, rng = ref.torch_dtype(dtype), np.random.default_rng(seed)
        need = [max(1, -(-(c + n) // page)) for c, n in zip(n_ctx, n_new)]
        pool = sum(need) + 2
        perm, self.table = rng.permutation(pool), np.full((len(need), max(need) + 1), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        shape = (pool, Hk, page, D) if heads_first else (pool, page, Hk, D)
        self.k, self.v = (torch.full(shape, fill, dtype=dt, device="cuda") for _ in range(2))
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.args = (self.k, self.v, torch.from_numpy(self.table).cuda(), torch.tensor(n_ctx, dtype=torch.int32, device="cuda"),
                     torch.tensor(np.concatenate([[0], np.cumsum(n_new)]), dtype=torch.int32, device="cuda"))

    def slots(self, b, n):
        s = np.arange(n)
        return self.table[b, s // self.page], s % self.page

    def put(self, torch, g):
        """Committed and new tokens' keys and values, N(0, 1); all other slots stay as they are."""
        for b, (c, n) in enumerate(zip(self.n_ctx, self.n_new)):
            pg, row = (torch.from_numpy(a).cuda().long() for a in self.slots(b, c + n))
            for t in (self.k, self.v):
                t[pg, row] = torch.randn((c + n,) + tuple(t.shape[2:]), generator=g, device="cuda").to(t.dtype)


APPEND = [
    # n_ctx, n_new, Hq, Hk, D, R, page, heads_first, dtype, norm, inter
    ([5], [1], 4, 1, 128, 128, 16, False, "bf16", True, False),
    ([0, 15, 16, 31, 3], [1, 1, 1, 1, 1], 8, 2, 64, 64, 16, True, "f16", True, False),
    ([0, 7, 100], [40, 0, 3], 6, 3, 96, 48, 24, False, "bf16", True, True),
    ([9] * 70, [2, 0] * 35, 2, 2, 64, 32, 1, True, "f32", False, False),
    ([2, 3], [5, 6], 0, 5, 50, 20, 7, False, "f32", True, False),
    ([1000, 1], [3, 300], 7, 1, 128, 0, 64, False, "bf16", False, False),
]


@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(env, case):
    torch, stride, dev = env
    n_ctx, n_new, Hq, Hk, D, R, page, first, dtype, norm, inter = case
    c = Paged(torch, n_ctx, n_new, Hk, D, page, dtype, first, 1, fill=7.0)
    N, g, dt, u = sum(n_new), gen(torch, 2), ref.torch_dtype(dtype), ref.UNIT[dtype]
    q, k, v = qk_inputs(torch, N, max(Hq, 1), Hk, D, dtype, "fused", 3)
    cos, sin = tables(torch, 2000, R)
    pos = torch.randint(0, 2000, (N,), generator=g, device=dev).int()
    w = [(1 + 0.3 * torch.randn(D, generator=g, device=dev)).to(dt) if norm else None for _ in range(2)]
    q_out = torch.full((N, Hq, D), float("nan"), dtype=dt, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    with_q = dict(q=q, q_out=q_out, q_weight=w[0]) if Hq else {}
    stride.stride_kv_append(k, v, *c.args, pos=pos if R else None, cos=cos, sin=sin, k_weight=w[1], eps=1e-5,
                            interleaved=inter, dev_status=status, **with_q)
    torch.cuda.synchronize()
    assert int(status) == 0
    cs, sn = (ref.f64(cos[pos.long()]), ref.f64(sin[pos.long()])) if R else (None, None)
    want_k, size = ref.norm_rope(ref.f64(k), None if w[1] is None else ref.f64(w[1]), 1e-5, cs, sn, inter)
    K, V = np.full(c.k.shape, 7.0), np.full(c.v.shape, 7.0)
    tol = np.zeros(c.k.shape)
    at = 0
    for b, (have, n) in enumerate(zip(n_ctx, n_new)):
        pg, row = (a[have:] for a in c.slots(b, have + n))
        K[pg, row], V[pg, row] = want_k[at:at + n], ref.f64(v)[at:at + n]
        tol[pg, row] = u * np.abs(want_k[at:at + n]) + (D + 20) * 2.0 ** -24 * size[at:at + n]
        at += n
    close(c.k, K, tol)  # (all other slots are as they were)
    close(c.v, V, 0.0)
    if Hq:
        want, size = ref.norm_rope(ref.f64(q), None if w[0] is None else ref.f64(w[0]), 1e-5, cs, sn, inter)
        close(q_out, want, u * np.abs(want) + (D + 20) * 2.0 ** -24 * size)


def test_append_without_a_page(env):
    """Slots that the block table does not hold are not written; the other tokens are."""
    torch, stride, dev = env
    for spoil in (-1, 10 ** 6, None):
        c = Paged(torch, [3, 3], [2, 1], 1, 64, 4, "bf16", False, 1, fill=0.0)
        k, v = torch.ones((3, 1, 64), dtype=torch.bfloat16, device=dev), torch.ones((3, 1, 64), dtype=torch.bfloat16, device=dev)
        table = c.args[2].clone()
        if spoil is None:
            table = table[:, :1].contiguous()  # slot 4 of sequence 0 lies past the table
        else:
            table[0, 1] = spoil
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        stride.stride_kv_append(k, v, c.k, c.v, table, *c.args[3:], dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == stride.DEV_BAD_LAYOUT
        assert float(c.k.sum()) == 2 * 64  # token 0 (slot 3) of the first, token 0 of the second


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
def random_tree(rng, n):
    bits = []
    for j in range(n):
        parent = j - 1 - int(rng.integers(0, 3))
        bits.append((bits[parent] if parent >= 0 else 0) | (1 << j))
    return bits


def check_attention(torch, stride, c, q, mask, scale, dtype, out_like=None, workspace=None):
    N, Hq, D = q.shape
    Hk = c.k.shape[2]
    dev = q.device
    out = torch.full_like(q, float("nan"), memory_format=torch.contiguous_format) if out_like is None else out_like
    lse = torch.full((N, Hq), float("nan"), device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = workspace if workspace is not None else torch.empty(stride.stride_tree_attention_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
    tm = None if mask is None else torch.from_numpy(np.array(mask, np.uint64).view(np.int64)).to(dev)
    stride.stride_tree_attention(q, *c.args, tm, scale, out, lse=lse, workspace=ws, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    Q, K, V, u = ref.f64(q), ref.f64(c.k), ref.f64(c.v), ref.UNIT[dtype]
    got, got_lse = ref.f64(out), ref.f64(lse)
    at = 0
    for b, (have, n) in enumerate(zip(c.n_ctx, c.n_new)):
        pg, row = c.slots(b, have + n)
        for i in range(n):
            seen = np.zeros(have + n, bool)
            seen[:have] = True
            for j in range(n):
                seen[have + j] = j <= i if mask is None else bool((int(mask[at + i]) >> j) & 1)
            for h in range(Hq):
                kk, vv = K[pg, row, h // (Hq // Hk)], V[pg, row, h // (Hq // Hk)]
                o, e, size = ref.attention(Q[at + i, h], kk, vv, seen, scale)
                tol = u * size + u * np.abs(o) + 8 * 2e-6 * size + 1e-30
                assert (np.abs(got[at + i, h] - o) <= tol).all(), (b, i, h, np.abs(got[at + i, h] - o).max(), tol.max())
                if e == -np.inf:
                    assert got_lse[at + i, h] == -np.inf
                else:
                    reach = (np.abs(kk[seen]) @ np.abs(Q[at + i, h])).max() * abs(scale)
                    assert abs(got_lse[at + i, h] - e) <= D * 2.0 ** -24 * reach + 4e-6, (b, i, h, got_lse[at + i, h], e)
        at += n
    return out, lse


ATTN = [
    # n_ctx, n_new, Hq, Hk, D, page, heads_first, dtype, tree
    ([0], [1], 1, 1, 64, 16, False, "bf16", False),
    ([37], [1], 16, 2, 128, 16, False, "bf16", False),
    ([63, 64, 65, 0, 1, 127], [1] * 6, 8, 2, 128, 16, True, "f16", False),
    ([1000, 3, 500], [1, 0, 1], 7, 1, 128, 24, False, "bf16", False),
    ([5000], [1], 4, 4, 64, 64, True, "bf16", False),
    ([200, 10, 0, 64], [13, 1, 5, 64], 8, 2, 128, 16, False, "bf16", True),
    ([130, 0], [64, 64], 3, 3, 64, 1, True, "f16", True),
    ([100], [7], 16, 1, 128, 32, False, "bf16", True),
    ([100, 0, 40], [100, 70, 1], 4, 1, 128, 16, False, "bf16", False),
    ([0], [200], 2, 1, 64, 128, True, "bf16", False),
    ([61, 200], [3, 2], 4, 2, 96, 20, False, "bf16", True),
    ([61, 200], [1, 1], 4, 2, 8, 16, False, "f16", False),
    ([10] * 400, [1] * 400, 4, 2, 64, 16, False, "bf16", False),
    ([3000, 0, 0, 0, 2], [2, 1, 1, 1, 1], 24, 3, 80, 16, True, "bf16", True),
]


@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"{len(c[0])}x{max(c[1])}-{c[2]}x{c[3]}x{c[4]}-{c[5]}-{c[7]}-{'tree' if c[8] else 'chain'}")
def test_attention(env, case):
    """Slots past each sequence's end hold NaN."""
    torch, stride, dev = env
    n_ctx, n_new, Hq, Hk, D, page, first, dtype, tree = case
    c = Paged(torch, n_ctx, n_new, Hk, D, page, dtype, first, 1)
    g, rng, N = gen(torch, 2), np.random.default_rng(3), sum(n_new)
    c.put(torch, g)
    q = (1.5 * torch.randn((N, Hq, D), generator=g, device=dev)).to(ref.torch_dtype(dtype))
    mask = [m for n in n_new for m in random_tree(rng, n)] if tree else None
    check_attention(torch, stride, c, q, mask, D ** -0.5, dtype)


def test_attention_rows_that_see_nothing(env):
    """Masks without a bit: nothing cached, out 0 and lse -inf; else the cached tokens alone."""
    torch, stride, dev = env
    c = Paged(torch, [0, 70, 0], [3, 2, 1], 2, 64, 16, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = torch.randn((6, 4, 64), generator=gen(torch, 3), device=dev).bfloat16()
    out, lse = check_attention(torch, stride, c, q, [0, 2, 0, 0, 0, 0], 0.125, "bf16")
    assert not out[0].any() and (lse[0] == float("-inf")).all()


def test_attention_unseen_tokens_may_hold_anything(env):
    """A drafted token that no row sees (padding of the tree) holds NaN and infinities."""
    torch, stride, dev = env
    c = Paged(torch, [20], [4], 1, 128, 16, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = torch.randn((4, 8, 128), generator=gen(torch, 3), device=dev).bfloat16()
    pg, row = c.slots(0, 24)
    for j, x in ((2, float("nan")), (3, float("inf"))):
        c.k[int(pg[20 + j]), int(row[20 + j])] = x
        c.v[int(pg[20 + j]), int(row[20 + j])] = x
    with np.errstate(invalid="ignore"):
        check_attention(torch, stride, c, q, [1, 3, 1, 3], 0.1, "bf16")


def test_attention_strides(env):
    """q and out as views of wider buffers, k and v as the halves of one pool."""
    torch, stride, dev = env
    g = gen(torch, 4)
    c = Paged(torch, [90, 33], [2, 3], 2, 64, 16, "bf16", False, 1)
    pool = torch.full((c.k.shape[0], 16, 2, 2 * 64), float("nan"), dtype=torch.bfloat16, device=dev)
    c.k, c.v = pool[..., :64], pool[..., 64:]
    c.args = (c.k, c.v) + c.args[2:]
    c.put(torch, g)
    q = torch.randn((5, 3, 4, 64), generator=g, device=dev).bfloat16()[:, 1]
    out = torch.zeros((4, 5, 72), dtype=torch.bfloat16, device=dev).transpose(0, 1)[..., :64]
    check_attention(torch, stride, c, q, None, 0.125, "bf16", out_like=out)


def test_attention_large_offsets(env):
    """Pages more than 2^31 elements into a pool."""
    torch, stride, dev = env
    Hk, D, page = 8, 128, 64
    pool = torch.empty((2 ** 31 // (Hk * D * page) + 40, page, Hk, D), dtype=torch.bfloat16, device=dev)
    c = Paged(torch, [150], [2], Hk, D, page, "bf16", False, 1)
    c.table[0, :3] = pool.shape[0] - np.array([1, 5, 17])
    c.k = c.v = pool
    c.args = (c.k, c.v, torch.from_numpy(c.table).to(dev)) + c.args[3:]
    c.put(torch, gen(torch, 2))
    q = torch.randn((2, 8, D), generator=gen(torch, 3), device=dev).bfloat16()

    class Few:  # the reference reads the few pages alone
        pass

    few = Few()
    few.n_ctx, few.n_new, few.page = c.n_ctx, c.n_new, page
    few.slots = lambda b, n: (np.arange(n) // page, np.arange(n) % page)
    few.k = few.v = pool[torch.from_numpy(c.table[0, :3]).to(dev).long()]
    few.args = c.args
    check_attention(torch, stride, few, q, None, 0.1, "bf16")
    k1 = torch.randn((2, Hk, D), generator=gen(torch, 5), device=dev).bfloat16()
    stride.stride_kv_append(k1, k1, *c.args)
    pg, row = c.slots(0, 152)
    assert torch.equal(pool[int(pg[151]), int(row[151])], k1[1])


def test_attention_is_repeatable_and_leaves_nothing_between_calls(env):
    """The same bits from a workspace of any contents, on another stream, and in a graph."""
    torch, stride, dev = env
    c = Paged(torch, [3000, 100], [5, 2], 2, 128, 16, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = torch.randn((7, 8, 128), generator=gen(torch, 3), device=dev).bfloat16()
    ws = torch.full((stride.stride_tree_attention_workspace_size(7, 8, 2, 128),), 255, dtype=torch.uint8, device=dev)
    a = torch.empty_like(q)
    stride.stride_tree_attention(q, *c.args, None, 0.1, a, workspace=ws)
    other = Paged(torch, [17], [7], 2, 128, 16, "bf16", False, 2)
    other.put(torch, gen(torch, 5))
    stride.stride_tree_attention(q, *other.args, None, 0.1, torch.empty_like(q), workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = torch.empty_like(q)
    with torch.cuda.stream(side):
        stride.stride_tree_attention(q, *c.args, None, 0.1, b, workspace=ws)
    side.synchronize()
    assert torch.equal(a, b)
    graph, d = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        stride.stride_tree_attention(q, *c.args, None, 0.1, d, workspace=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, d)


def test_attention_bad_layouts(env):
    """A missing page, a tree of more than 64 tokens, a slot past the table: that sequence's rows are NaN, the others right."""
    torch, stride, dev = env
    for what in ("page", "big page", "tree", "table"):
        n_new = [1, 65 if what == "tree" else 2, 1]
        c = Paged(torch, [40, 100, 30], n_new, 1, 64, 16, "bf16", False, 1)
        c.put(torch, gen(torch, 2))
        N = sum(n_new)
        q = torch.randn((N, 2, 64), generator=gen(torch, 3), device=dev).bfloat16()
        mask = torch.ones(N, dtype=torch.int64, device=dev) if what == "tree" else None
        good, bad = torch.empty_like(q), torch.empty_like(q)
        lse = torch.empty((N, 2), device=dev)
        ws = torch.empty(stride.stride_tree_attention_workspace_size(N, 2, 1, 64), dtype=torch.uint8, device=dev)
        args = list(c.args)
        stride.stride_tree_attention(q, *args, None, 0.125, good, workspace=ws)
        if what == "page":
            args[2][1, 3] = -1
        elif what == "big page":
            args[2][1, 3] = args[0].shape[0]
        elif what == "table":
            args[3][1] = args[2].shape[1] * 16
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        stride.stride_tree_attention(q, *args, mask, 0.125, bad, lse=lse, workspace=ws, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == stride.DEV_BAD_LAYOUT
        assert torch.isnan(bad[1:-1]).all() and torch.isnan(lse[1:-1]).all()
        assert torch.equal(bad[0], good[0]) and torch.equal(bad[-1], good[-1])


# ---------------------------------------------------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------------------------------------------------
def check_sample(torch, stride, x, noise, T, top_k, top_p, min_p, V=None):
    rows, dev = x.shape[0], x.device
    V = x.shape[1] if V is None else V
    tokens = torch.full((rows,), -7, dtype=torch.int32, device=dev)
    logp = torch.full((rows,), 7.0, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    each = lambda v, t: torch.tensor(v, dtype=t, device=dev) if isinstance(v, (list, np.ndarray)) else v  # noqa: E731
    stride.stride_sample(x, noise, tokens, temperature=each(T, torch.float32), top_k=each(top_k, torch.int32),
                         top_p=each(top_p, torch.float32), min_p=each(min_p, torch.float32), logp=logp, dev_status=status, V=V)
    torch.cuda.synchronize()
    X, E = ref.f64(x)[:, :V], np.ones((rows, V)) if noise is None else ref.f64(noise)
    row = lambda v, r: float(np.float32(v[r])) if isinstance(v, (list, np.ndarray)) else float(np.float32(v))  # noqa: E731
    none = 0
    for r in range(rows):
        a = X[r], E[r], row(T, r), int(row(top_k, r)), row(top_p, r), row(min_p, r)
        ok, got = ref.acceptable(*a), int(tokens[r])
        assert got in ok, (r, got, ok)
        near, token, lp = ref.sample(*a)
        if token < 0:
            none += 1
            assert torch.isnan(logp[r])
        elif got == token and ok == {token}:
            assert abs(float(logp[r]) - lp) <= 2e-5, (r, float(logp[r]), lp)
    assert int(status) == (stride.DEV_NO_TOKEN if none else 0)
    return tokens, logp


def logits(torch, rows, V, dtype, seed, sigma=3.0, ld=None):
    g = gen(torch, seed)
    x = (sigma * torch.randn((rows, ld or V), generator=g, device="cuda")).to(ref.torch_dtype(dtype))
    noise = torch.empty((rows, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    return x, noise


CUTS = [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.3, 0, 1.0, 0.1), (0.8, 50, 0.95, 0.02), (2.0, 1, 0.5, 0.0),
        (0.0, 3, 0.5, 0.5), (1.0, 0, 0.0, 0.0), (1.0, 10 ** 9, 0.999999, 2.0), (0.01, 0, 0.99, 0.0), (50.0, 700, 0.3, 0.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 4099, 32_000, 151_936])
def test_sample(env, V, dtype):
    """Each row with parameters of its own; rows that start at odd places."""
    torch, stride, dev = env
    x, noise = logits(torch, len(CUTS), V, dtype, V, ld=V + (V % 3))
    T, k, p, m = (list(v) for v in zip(*CUTS))
    check_sample(torch, stride, x, noise, T, k, p, m, V=V)


@pytest.mark.parametrize("cut", CUTS, ids=str)
def test_sample_one_parameter_for_all(env, cut):
    torch, stride, dev = env
    x, noise = logits(torch, 33, 5003, "bf16", 5)
    check_sample(torch, stride, x, None if cut[0] == 0 else noise, *cut)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_ties(env, dtype):
    """Rows of few distinct values, of one value, of both zeros: the first by index are kept."""
    torch, stride, dev = env
    x, noise = logits(torch, 24, 30_011, dtype, 9)
    x[:8] = (x[:8] / 4).round() * 4
    x[8:16] = 1.5
    x[16:] = torch.where(x[16:] > 0, 0.0, -0.0).to(x.dtype)
    k = [0, 1, 2, 50, 3000, 20_000, 30_010, 30_012] * 3
    check_sample(torch, stride, x, noise, 1.0, k, 1.0, 0.0)
    check_sample(torch, stride, x, noise, 1.0, k, 0.4, 0.0)
    check_sample(torch, stride, x, noise, 0.5, 0, [0.01, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.999] * 3, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_sample_ruled_out_tokens(env, dtype):
    """-inf and the type's lowest value are never drawn, whatever is asked for; rows without a token."""
    torch, stride, dev = env
    x, noise = logits(torch, 20, 2000, dtype, 11)
    low = torch.finfo(x.dtype).min
    x[:, ::2] = float("-inf")
    x[5:, 1::4] = low
    x[10] = float("-inf")
    x[11, 7] = float("nan")
    x[12, 7] = float("inf")
    x[13] = low
    x[14] = float("-inf")
    x[14, 1234] = -3.0
    x[15] = float("-inf")
    x[15, 3] = low
    noise[16] = float("nan")
    noise[17] = float("inf")
    noise[18, :1000] = 0.0
    T = [1.0] * 20
    T[2], T[3], T[4] = float("nan"), -1.0, float("inf")
    p = [1.0, 0.9] * 10
    p[1] = float("nan")
    for k in (0, 3, 1500):
        tokens, _ = check_sample(torch, stride, x, noise, T, k, p, 0.0)
        assert int(tokens[14]) == 1234 and int(tokens[15]) == 3
        assert all(int(tokens[r]) == -1 for r in (1, 2, 3, 4, 10, 11, 12, 16, 17))
        assert all(float(x[r, int(tokens[r])]) > low for r in (0, 5, 6, 7, 8, 9, 14, 19))


def test_sample_extreme_spread(env):
    """Logits of all sizes: a range of bit patterns that takes every level of the search."""
    torch, stride, dev = env
    g = gen(torch, 3)
    x = torch.randn((12, 9001), generator=g, device=dev) * 10.0 ** torch.randint(-30, 3, (12, 9001), generator=g, device=dev).float()
    noise = torch.empty_like(x).exponential_(generator=g)
    for k, p in ((0, 0.9), (100, 1.0), (4000, 0.7), (0, 0.2)):
        check_sample(torch, stride, x, noise, 1.0, k, p, 0.0)


def test_sample_frequencies(env):
    """Tokens come with their probabilities: 200,000 rows of one distribution, each count within 5 standard deviations."""
    torch, stride, dev = env
    V, rows = 40, 200_000
    g = gen(torch, 17)
    one = torch.randn(V, generator=g, device=dev) * 1.5
    x = one.expand(rows, V).contiguous()
    noise = torch.empty((rows, V), device=dev).exponential_(generator=g)
    tokens = torch.empty(rows, dtype=torch.int32, device=dev)
    stride.stride_sample(x, noise, tokens, temperature=0.9, top_k=20, top_p=0.9)
    p = torch.softmax(one.double() / 0.9, 0)
    p, at = p.sort(descending=True)
    p[20:] = 0
    p /= p.sum()
    p[p.cumsum(0) - p >= 0.9] = 0
    p /= p.sum()
    n = torch.bincount(tokens.long(), minlength=V)[at].double()
    assert ((n - rows * p).abs() <= 5 * (rows * p * (1 - p)).sqrt() + 1e-9).all()


def test_sample_feeds_the_step(env):
    """The sampled tokens are what stride_score_step takes: its student log-prob is the untruncated one of the token."""
    torch, stride, dev = env
    x, noise = logits(torch, 8, 4000, "bf16", 21)
    tokens, logp = torch.empty(8, dtype=torch.int32, device=dev), torch.empty(8, device=dev)
    stride.stride_sample(x, noise, tokens, logp=logp)
    state, out = stride.new_state(8), {"logp_s": torch.empty(8, device=dev)}
    stride.stride_score_step(x, x, tokens, torch.zeros(8, dtype=torch.uint8, device=dev), stride.TURN_MEAN, -1e9, state, out=out)
    torch.cuda.synchronize()
    assert (out["logp_s"] - logp).abs().max() < 1e-4
