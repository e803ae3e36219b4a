"""Controls on logits against their plain form in 64 bits
(tests/cache_reference.py, which states the tolerances)."""
from __future__ import annotations

import numpy as np
import pytest

import cache_reference as ref
import decode_reference as dec

pytestmark = pytest.mark.gpu

TOKEN_RANGE, BAD_LAYOUT, BAD_CONTROL = 0x1, 0x2, 0x20


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


def i32(torch, a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def bits_of(allowed):
    """[rows, V] bool as int32 words, the bits past V set."""
    rows, V = allowed.shape
    b = np.ones((rows, -(-V // 32) * 32), bool)
    b[:, :V] = allowed
    return np.packbits(b, axis=1, bitorder="little").view(np.int32)


CASES = [
    # rows, V, ld (0: V), history, biases, mask, dtype
    (1, 1, 0, 3, 2, False, "f32"),
    (1, 7, 0, 0, 0, True, "bf16"),
    (2, 33, 40, 5, 0, True, "bf16"),
    (3, 1000, 0, 200, 20, True, "bf16"),
    (3, 1001, 0, 200, 20, True, "f16"),
    (2, 4099, 4104, 60, 0, False, "f32"),
    (4, 4099, 0, 0, 9, True, "f32"),
    (2, 32_000, 0, 5000, 0, True, "f32"),
    (2, 50_257, 0, 9000, 300, True, "bf16"),
    (2, 151_936, 0, 3000, 100, True, "f16"),
    (1, 151_936, 151_940, 4097, 0, False, "bf16"),
    (5, 24_577, 0, 100, 0, True, "bf16"),
    (2, 12_289, 0, 100, 5, True, "f32"),
    (1, 300_001, 0, 700, 3, True, "bf16"),
    (2, 257, 260, 20_000, 5000, True, "bf16"),
]


def inputs(torch, case, seed=1):
    rows, V, ld, hist, n_bias, mask, dtype = case
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, ld or V, generator=g, device="cuda") * 4).to(dec.torch_dtype(dtype))
    x[:, ::13] = float("-inf")
    x[:, 1::29] = 0.0
    d = dict(x=x, V=V, kw={}, history=[np.zeros(0, int)] * rows, prompt=[0] * rows, rep=[1.0] * rows, freq=[0.0] * rows, pres=[0.0] * rows,
             biases=[[]] * rows, allowed=None)
    if hist:
        h = (V * rng.random((rows, hist)) ** 3).astype(np.int64).clip(0, V - 1)
        h[rng.random(h.shape) < 0.05] = -1
        n = rng.integers(0, hist + 1, rows)
        n[0] = hist
        p = (n * rng.random(rows)).astype(int)
        each = lambda v: torch.tensor(rng.choice(np.array(v, np.float32), rows), device="cuda")  # noqa: E731
        d["kw"] = dict(history=i32(torch, h), history_len=i32(torch, n), prompt_len=i32(torch, p), repetition=each([1.0, 1.3, 0.7]),
                       frequency=each([0.0, 0.3, -0.2]), presence=each([0.0, 0.6]))
        for r, (name, got) in enumerate(zip(("rep", "freq", "pres"), ("repetition", "frequency", "presence"))):
            d[name] = d["kw"][got].double().tolist()
        d["history"], d["prompt"] = [h[r, :n[r]] for r in range(rows)], p.tolist()
    if n_bias:
        n = rng.integers(0, n_bias + 1, rows)
        n[-1] = n_bias
        off, t = np.concatenate([[0], np.cumsum(n)]), rng.integers(-1, V, int(n.sum()))
        t[::3] = np.minimum(t[::3], 3)  # several entries for a token
        b = (rng.standard_normal(len(t)) * 3).astype(np.float32)
        b[::7] = -np.inf
        d["kw"] |= dict(bias_off=i32(torch, off), bias_token=i32(torch, t), bias=torch.tensor(b, device="cuda"))
        d["biases"] = [list(zip(t[off[r]:off[r + 1]].tolist(), b[off[r]:off[r + 1]].astype(float).tolist())) for r in range(rows)]
    if mask:
        a = rng.random((rows, V)) < np.array([0.02, 0.98, 1.1])[rng.integers(0, 3, rows)][:, None]
        if rows > 1:
            a[1] = False  # nothing is allowed
        d["allowed"] = a
        d["kw"]["allowed"] = torch.tensor(bits_of(a), device="cuda")
    return d


def check(d, x, out, dtype, rows=None):
    got, x = dec.f64(out), dec.f64(x)
    for r in range(len(x)) if rows is None else rows:
        with np.errstate(invalid="ignore"):
            want, size = ref.controls(x[r, :d["V"]], d["history"][r], d["prompt"][r], d["rep"][r], d["freq"][r], d["pres"][r], d["biases"][r],
                                      None if d["allowed"] is None else d["allowed"][r % len(d["allowed"])])
        fin = np.isfinite(want)
        y = got[r, :d["V"]]
        assert np.array_equal(y[~fin], want[~fin], equal_nan=True), r
        tol = dec.UNIT[dtype] * np.abs(want[fin]) + 5 * 2.0 ** -24 * size[fin]
        bad = ~(np.abs(y[fin] - want[fin]) <= tol)
        assert not bad.any(), (r, np.flatnonzero(fin)[bad][:5], y[fin][bad][:3], want[fin][bad][:3])


@pytest.mark.parametrize("case", CASES, ids=str)
def test_controls(env, case):
    torch, stride, dev = env
    d = inputs(torch, case)
    rows, V, dtype = case[0], case[1], case[-1]
    out = torch.full_like(d["x"], 77.0)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    stride.stride_logit_controls(d["x"], out, **d["kw"], V=V, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(d, d["x"], out, dtype)
    assert (out[:, V:] == 77).all()
    # in place
    again = d["x"].clone()
    stride.stride_logit_controls(again, again, **d["kw"], V=V)
    assert torch.equal(again[:, :V], out[:, :V]) and torch.equal(again[:, V:], d["x"][:, V:])
    # rows of another alignment
    wide = torch.full((rows, V + 11), 77.0, dtype=out.dtype, device=dev)
    stride.stride_logit_controls(d["x"], wide[:, 3:], **d["kw"], V=V)
    assert torch.equal(wide[:, 3:3 + V], out[:, :V]) and (wide[:, :3] == 77).all() and (wide[:, 3 + V:] == 77).all()


def test_one_value_for_all_and_one_mask(env):
    torch, stride, dev = env
    case = (3, 1000, 0, 100, 0, True, "bf16")
    d = inputs(torch, case)
    d["allowed"] = d["allowed"][:1]
    d["rep"], d["freq"], d["pres"], d["prompt"] = [1.25] * 3, [0.5] * 3, [0.25] * 3, [0] * 3
    out = torch.empty_like(d["x"])
    kw = dict(history=d["kw"]["history"], history_len=d["kw"]["history_len"], allowed=d["kw"]["allowed"][:1])
    stride.stride_logit_controls(d["x"], out, **kw, repetition=1.25, frequency=0.5, presence=0.25)
    check(d, d["x"], out, "bf16")
    # nothing to do: a copy
    stride.stride_logit_controls(d["x"], out)
    assert torch.equal(out, d["x"])
    # no rows; a history without columns
    stride.stride_logit_controls(d["x"][:0], out[:0], **{k: v[:0] if k != "allowed" else v for k, v in kw.items()})
    out.zero_()
    stride.stride_logit_controls(d["x"], out, history=kw["history"][:, :0], history_len=torch.zeros(3, dtype=torch.int32, device=dev))
    assert torch.equal(out, d["x"])


def test_wild_logits(env):
    """Infinities and NaN go through the formula; a mask hides them."""
    torch, stride, dev = env
    x = torch.tensor([[float("inf"), float("-inf"), float("nan"), 0.0, -0.0, 1e30, 3.0, float("nan")]], device=dev)
    d = dict(V=8, history=[[0, 1, 2, 3, 4, 5]], prompt=[6], rep=[2.0], freq=[0.0], pres=[0.0], biases=[[(0, -np.inf), (6, np.inf)]],
             allowed=np.array([[True] * 7 + [False]]))
    out = torch.empty_like(x)
    stride.stride_logit_controls(x, out, history=i32(torch, d["history"]), history_len=i32(torch, [6]), prompt_len=i32(torch, [6]), repetition=2.0,
                                 bias_off=i32(torch, [0, 2]), bias_token=i32(torch, [0, 6]), bias=torch.tensor([-np.inf, np.inf], device=dev),
                                 allowed=torch.tensor(bits_of(d["allowed"]), device=dev))
    check(d, x, out, "f32")


def test_what_is_refused_on_the_device(env):
    torch, stride, dev = env
    case = (5, 1000, 0, 60, 10, True, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device=dev)

    def run(bit, row, **change):
        d = inputs(torch, case)
        d["kw"] |= {k: d["kw"][k].clone() for k in change}
        for k, v in change.items():
            d["kw"][k][row] = v
        for place in (False, True):
            out = d["x"].clone() if place else torch.empty_like(d["x"])
            status.zero_()
            stride.stride_logit_controls(out if place else d["x"], out, **d["kw"], dev_status=status)
            assert int(status) == bit, change
            assert torch.isnan(out[row]).all()
            check(d, d["x"], out, "bf16", [r for r in range(5) if r != row])

    for v in (0.0, -1.0, float("nan"), float("inf")):
        run(BAD_CONTROL, 2, repetition=v)
    for v in (float("nan"), float("-inf")):
        run(BAD_CONTROL, 1, frequency=v)
        run(BAD_CONTROL, 4, presence=v)
    for v in (-1, 61, 2 ** 31 - 1):
        run(BAD_LAYOUT, 3, history_len=v)
    d = inputs(torch, case)  # lists that end before they begin, or past all entries
    off = d["kw"]["bias_off"].clone()
    for r, v in ((5, 10 ** 6), (0, -1)):
        d["kw"]["bias_off"] = off.clone()
        d["kw"]["bias_off"][r] = v
        out = torch.empty_like(d["x"])
        status.zero_()
        stride.stride_logit_controls(d["x"], out, **d["kw"], dev_status=status)
        bad = min(r, 4)
        assert int(status) == BAD_LAYOUT and torch.isnan(out[bad]).all()
        check(d, d["x"], out, "bf16", [i for i in range(5) if i != bad])
    # tokens past the vocabulary are told of and left out
    for name in ("history", "bias_token"):
        d = inputs(torch, case)
        t = d["kw"][name].clone()
        if name == "history":
            t[0, 7] = 1000
            d["history"][0][7] = 10 ** 9
        else:
            t[0], d["biases"][0] = 2 ** 31 - 1, d["biases"][0][1:]
            assert int(d["kw"]["bias_off"][1]) > 0
        d["kw"][name] = t
        out = torch.empty_like(d["x"])
        status.zero_()
        stride.stride_logit_controls(d["x"], out, **d["kw"], dev_status=status)
        assert int(status) == TOKEN_RANGE
        check(d, d["x"], out, "bf16")
    d = inputs(torch, case)
    with pytest.raises(ValueError):
        stride.stride_logit_controls(d["x"], torch.empty_like(d["x"]), bias=d["kw"]["bias"])
    with pytest.raises(ValueError):
        stride.stride_logit_controls(d["x"], torch.empty_like(d["x"]), allowed=d["kw"]["allowed"][:, :31])
    with pytest.raises(ValueError):
        stride.stride_logit_controls(d["x"], torch.empty_like(d["x"])[:4])
    with pytest.raises(stride.StrideError):
        stride.stride_logit_controls(d["x"], torch.empty_like(d["x"]), history=d["kw"]["history"][:1].expand(5, -1),
                                     history_len=d["kw"]["history_len"])
