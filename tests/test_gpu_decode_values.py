"""The decode step's operators on values, masks and sizes at the ends of what they
accept (tolerances: tests/decode_reference.py)."""
from __future__ import annotations

import numpy as np
import pytest

import decode_reference as ref
from test_gpu_decode_step import Paged, env, gen  # noqa: F401

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
