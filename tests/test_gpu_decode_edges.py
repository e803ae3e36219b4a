"""The decode step's operators at the places where a mask, a scale, a number of
sequences or of rows changes how they work (tolerances: tests/decode_reference.py)."""
from __future__ import annotations

import numpy as np
import pytest

import decode_reference as ref
from test_gpu_decode_step import Paged, check_attention, check_sample, env, gen, logits, random_tree  # noqa: F401

pytestmark = pytest.mark.gpu

WILD = [
    # n_ctx, n_new, Hq, Hk, D, page, heads_first, dtype, tree
    ([40, 0], [5, 3], 4, 2, 128, 16, False, "bf16", False),
    ([40, 30], [4, 4], 4, 1, 64, 16, False, "f16", True),
    ([500], [6], 2, 1, 96, 24, True, "bf16", True),
    ([70, 5], [150, 60], 4, 1, 128, 16, False, "bf16", False),
    ([130], [64], 6, 2, 64, 16, False, "f16", True),
    ([3000, 60], [50, 40], 4, 2, 96, 64, True, "bf16", True),
    ([0], [300], 1, 1, 64, 8, False, "bf16", False),
]


@pytest.mark.parametrize("case", WILD, ids=str)
def test_values_that_are_not_finite_reach_the_rows_that_see_them_alone(env, case):  # noqa: F811
    """Single components of new tokens' values are NaN or infinite, and one new token's key is NaN."""
    torch, stride, dev = env
    n_ctx, n_new, Hq, Hk, D, page, first, dtype, tree = case
    c = Paged(torch, n_ctx, n_new, Hk, D, page, dtype, first, 1)
    g, rng, N = gen(torch, 2), np.random.default_rng(3), sum(n_new)
    c.put(torch, g)
    for b, (have, n) in enumerate(zip(n_ctx, n_new)):
        pg, row = c.slots(b, have + n)
        for j, comp, x in ((n // 3, 1, np.nan), (n // 2, 7, np.inf), (n // 2, 6, -np.inf), (2 * n // 3, 7, -np.inf), (n - 1, D - 1, np.nan)):
            c.v[int(pg[have + j]), int(row[have + j]), :, comp] = x
        c.k[int(pg[have + n - 2]), int(row[have + n - 2]), Hk - 1] = np.nan
    q = torch.randn((N, Hq, D), generator=g, device=dev).to(ref.torch_dtype(dtype))
    mask = [m for n in n_new for m in random_tree(rng, n)] if tree else None
    out, lse = torch.zeros_like(q), torch.zeros((N, Hq), device=dev)
    tm = None if mask is None else torch.from_numpy(np.array(mask, np.uint64).view(np.int64)).to(dev)
    ws = torch.empty(stride.stride_tree_attention_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    stride.stride_tree_attention(q, *c.args, tm, D ** -0.5, out, lse=lse, workspace=ws, dev_status=status)
    assert int(status) == 0
    Q, K, V, u, got, got_lse = ref.f64(q), ref.f64(c.k), ref.f64(c.v), ref.UNIT[dtype], ref.f64(out), ref.f64(lse)
    at, kinds = 0, set()
    for b, (have, n) in enumerate(zip(n_ctx, n_new)):
        pg, row = c.slots(b, have + n)
        for i in range(n):
            seen = np.arange(have + n) < have
            for j in range(n):
                seen[have + j] = j <= i if mask is None else bool((mask[at + i] >> j) & 1)
            for h in range(Hq):
                kk, vv = K[pg, row, h // (Hq // Hk)], V[pg, row, h // (Hq // Hk)]
                with np.errstate(invalid="ignore"):
                    o, e, size = ref.attention(Q[at + i, h], kk, vv, seen, D ** -0.5)
                y, good = got[at + i, h], np.isfinite(o)
                assert np.array_equal(y[~good], o[~good], equal_nan=True), (b, i, h, y[~good], o[~good])
                tol = u * size[good] + u * np.abs(o[good]) + 8 * 2e-6 * size[good] + 1e-30
                assert (np.abs(y[good] - o[good]) <= tol).all(), (b, i, h)
                assert np.isnan(got_lse[at + i, h]) == np.isnan(e)
                kinds.add((bool(good.all()), bool(np.isnan(e))))
        at += n
    assert {(True, False), (False, False), (False, True)} <= kinds  # rows of every kind were there


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("n_new", [[1, 2], [70, 30]], ids=str)
def test_attention_scales(env, scale, n_new):  # noqa: F811
    torch, stride, dev = env
    c = Paged(torch, [90, 200], n_new, 2, 64, 16, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = (0.3 * torch.randn((sum(n_new), 4, 64), generator=gen(torch, 3), device=dev)).bfloat16()
    check_attention(torch, stride, c, q, None, scale, "bf16")


@pytest.mark.parametrize("n_new", [1, 9], ids=["few", "many"])
def test_attention_of_more_sequences_than_fit_in_shared_memory(env, n_new):  # noqa: F811
    torch, stride, dev = env
    rng, B = np.random.default_rng(4), 1500
    n_ctx = rng.integers(0, 20, B).tolist()
    new = [int(n_new * (b % 3 > 0)) for b in range(B)]
    c = Paged(torch, n_ctx, new, 1, 64, 8, "bf16", False, 1)
    c.put(torch, gen(torch, 2))
    q = torch.randn((sum(new), 2 if n_new == 1 else 4, 64), generator=gen(torch, 3), device=dev).bfloat16()
    check_attention(torch, stride, c, q, None, 0.125, "bf16")


@pytest.mark.parametrize("D,dtype,page", [(64, "f16", 64), (96, "bf16", 16), (128, "f16", 8), (32, "bf16", 128)])
def test_attention_of_many_rows_over_long_prefixes(env, D, dtype, page):  # noqa: F811
    """Units cut between many workers, and joined."""
    torch, stride, dev = env
    n_new = [33, 2, 64]
    c = Paged(torch, [9000, 40, 2000], n_new, 2, D, page, dtype, page == 64, 1)
    c.put(torch, gen(torch, 2))
    q = (1.5 * torch.randn((sum(n_new), 4, D), generator=gen(torch, 3), device=dev)).to(ref.torch_dtype(dtype))
    rng = np.random.default_rng(3)
    check_attention(torch, stride, c, q, [m for n in n_new for m in random_tree(rng, n)], D ** -0.5, dtype)


def test_rotation_tables_anywhere(env):  # noqa: F811
    """Tables that start between 16-byte vectors give the same bits, forward and backward."""
    torch, stride, dev = env
    N, D, g = 37, 128, gen(torch, 4)
    q, k, dq_out, dk_out = ((torch.randn((N, h, D), generator=g, device=dev)).bfloat16() for h in (3, 1, 3, 1))
    w, pos = torch.randn(D, generator=g, device=dev).bfloat16(), torch.randint(0, 50, (N,), generator=g, device=dev).int()
    angle = torch.arange(50, device=dev)[:, None] * torch.linspace(1, 0.01, D // 2, device=dev)
    cos, sin = angle.cos(), angle.sin()
    got = []
    for shift in (0, 1):
        c, s = (torch.cat([t.new_zeros(shift), t.flatten()])[shift:].view(t.shape) for t in (cos, sin))
        assert c.data_ptr() % 16 == 4 * shift
        out = [torch.empty_like(t) for t in (q, k, q, k)]
        ws = torch.empty(stride.stride_qk_norm_rope_backward_workspace_size(N, 3, 1, D), dtype=torch.uint8, device=dev)
        stride.stride_qk_norm_rope(q, k, *out[:2], pos, c, s, w, w)
        stride.stride_qk_norm_rope_backward(dq_out, dk_out, q, k, *out[2:], pos, c, s, w, w, workspace=ws)
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_append_of_a_negative_length(env):  # noqa: F811
    """Its tokens are not written, not those either that a sum would put into a slot; the other sequences' are."""
    torch, stride, dev = env
    c = Paged(torch, [2, 3, 4], [3, 4, 1], 1, 64, 4, "bf16", False, 1, fill=0.0)
    k = torch.ones((8, 1, 64), dtype=torch.bfloat16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    ctx = torch.tensor([2, -2, 4], dtype=torch.int32, device=dev)
    stride.stride_kv_append(k, k, *c.args[:3], ctx, c.args[4], dev_status=status)
    assert int(status) == stride.DEV_BAD_LAYOUT
    assert float(c.k.sum()) == float(c.v.sum()) == 4 * 64


@pytest.mark.parametrize("rows", [39, 304, 305, 700])
def test_sample_numbers_of_rows(env, rows):  # noqa: F811
    """A row's share of the GPU changes with their number: the tokens do not."""
    torch, stride, dev = env
    V = 4001
    rng = np.random.default_rng(rows)
    x, noise = logits(torch, rows, V, "bf16", rows)
    T = rng.choice([0.0, 0.5, 1.0, 2.0], rows).astype(np.float32)
    top_k = rng.choice([0, 1, 40, 900, V], rows)
    top_p = rng.choice([0.2, 0.9, 0.999, 1.0], rows)
    min_p = rng.choice([0.0, 0.01], rows)
    check_sample(torch, stride, x, noise, T, top_k, top_p, min_p)


@pytest.mark.parametrize("rows", [130, 512])
def test_sample_rows_without_top_k_among_others(env, rows):  # noqa: F811
    """More rows than the GPU takes at once, in any order of kinds."""
    torch, stride, dev = env
    V = 20_001
    rng = np.random.default_rng(rows)
    x, noise = logits(torch, rows, V, "bf16", rows)
    top_k = rng.choice([0, 1, 40, V, V - 1, -3], rows, p=[0.3, 0.2, 0.3, 0.1, 0.05, 0.05])
    top_k[0] = top_k[-1] = 0
    T, top_p = np.full(rows, 0.9, np.float32), rng.choice([0.5, 0.95, 1.0], rows)
    check_sample(torch, stride, x, noise, T, top_k, top_p, 0.0)
