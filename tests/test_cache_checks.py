"""What the calls around a rollout's cache and its logits refuse, before any CUDA
call (CPU only; the pointers are never dereferenced on these paths), and their plain
forms by hand."""
import ctypes
import math

import numpy as np
import pytest

import cache_reference as ref
from test_decode_checks import DUMMY, cache, env, rows  # noqa: F401


def mass(decode, **kw):
    d = dict(data=DUMMY, seq_stride=128, head_stride=64, slots=64)
    d.update(kw)
    return decode._SlotMass(*[d[n] for n, _ in decode._SlotMass._fields_])


def of(fields, bad):
    return {k: v for k, v in bad.items() if k in dict(fields)}


def test_names_match_the_header(env):  # noqa: F811
    stride, decode, L = env
    src = (stride._build.INCLUDE / "stride_decode.h").read_text()
    assert f"#define STRIDE_DEV_BAD_CONTROL {hex(decode.DEV_BAD_CONTROL)} " in src
    for name in ("stride_attention_mass", "stride_kv_evict", "stride_logit_controls"):
        assert callable(getattr(stride, name)) and name in decode.__all__


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=1), 2), (dict(dtype=3), 2), (dict(D=60), 1), (dict(D=136), 1), (dict(D=0), 1), (dict(scale=math.nan), 1),
    (dict(scale=math.inf), 1), (dict(decay=-0.5), 1), (dict(decay=math.nan), 1), (dict(decay=math.inf), 1), (dict(heads=3), 1),
    (dict(rows=DUMMY + 2), 1), (dict(token=4 * 64 + 4), 1), (dict(head=68), 1), (dict(k=None), 1), (dict(k=DUMMY + 8), 1),
    (dict(row_stride=129), 1), (dict(page_stride=4), 1), (dict(head_stride=4), 1), (dict(tok_off=None), 1), (dict(ctx_len=None), 1),
    (dict(lse=None), 1), (dict(lse=DUMMY + 2), 1), (dict(mass=None), 1), (dict(mass_data=None), 1), (dict(mass_data=DUMMY + 2), 1),
    (dict(slots=0), 1), (dict(seq=127, n_seqs=2), 1), (dict(mass_head=63), 1), (dict(mass_head=0), 1), (dict(mass_head=-64, n_seqs=2, N=0), 0),
    (dict(seq=64, mass_head=128, n_seqs=2, N=0), 0), (dict(seq=64, mass_head=127, n_seqs=2), 1), (dict(N=-1), 1), (dict(N=2 ** 29 + 1), 1), (dict(N=0), 0), (dict(N=0, lse=None), 0), (dict(N=0, v=None), 0)])
def test_attention_mass(env, bad, code):  # noqa: F811
    stride, decode, L = env
    q = rows(decode, heads=bad.get("heads", 4), data=bad.get("rows", DUMMY), token=bad.get("token"), head=bad.get("head"))
    c = cache(decode, **of(decode._PagedCache._fields_, bad))
    m = mass(decode, data=bad.get("mass_data", DUMMY), slots=bad.get("slots", 64), seq_stride=bad.get("seq", 128),
             head_stride=bad.get("mass_head", 64))
    assert L.stride_attention_mass(ctypes.byref(q), bad.get("lse", DUMMY), bad.get("dtype", 0), bad.get("N", 5), bad.get("D", 64),
                                   bad.get("scale", 0.1), None, ctypes.byref(c), bad.get("decay", 1.0),
                                   ctypes.byref(m) if "mass" not in bad else None, None, None) == code


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(D=0), dict(D=1025), dict(sink=-1), dict(recent=-1), dict(most=0), dict(new_len=None), dict(new_len=DUMMY), dict(budget=3 * DUMMY), dict(to_slots=65), dict(kept=None),
    dict(k=None), dict(v=None), dict(n_pages=0), dict(block_table=None), dict(ctx_len=None), dict(n_seqs=0), dict(to_heads=3),
    dict(to_seqs=2), dict(to_k=DUMMY + 1), dict(mass_data=None), dict(to_slots=15), dict(to_mass=DUMMY)], ids=str)
def test_evict(env, bad):  # noqa: F811
    stride, decode, L = env
    f = cache(decode, **of(decode._PagedCache._fields_, bad))
    t = cache(decode, ctx_len=None, tok_off=None, n_heads=bad.get("to_heads", 2), n_seqs=bad.get("to_seqs", f.n_seqs or 1),
              k=bad.get("to_k", DUMMY))
    d = dict(budget=None, budget_all=8, sink=1, recent=2, most=16)
    d.update(of(decode._EvictParams._fields_, bad))
    how = decode._EvictParams(*[d[n] for n, _ in decode._EvictParams._fields_])
    m, m2 = mass(decode, data=bad.get("mass_data", DUMMY)), mass(decode, data=bad.get("to_mass", DUMMY * 2), slots=bad.get("to_slots", 16))
    assert L.stride_kv_evict(ctypes.byref(f), ctypes.byref(m), ctypes.byref(t), bad.get("dtype", 0), bad.get("D", 64),
                             ctypes.byref(how), bad.get("new_len", 3 * DUMMY), bad.get("kept", DUMMY), ctypes.byref(m2), None,
                             None) == (2 if "dtype" in bad else 1)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), 2), (dict(V=0), 1), (dict(V=2 ** 30 + 1, ld=2 ** 31, ld_out=2 ** 31), 1), (dict(ld=99), 1), (dict(ld_out=99), 1),
    (dict(rows=-1), 1), (dict(logits=None), 1), (dict(out=None), 1), (dict(logits=DUMMY + 1), 1), (dict(out=DUMMY + 1), 1),
    (dict(out=DUMMY, ld_out=104), 1), (dict(history_len=None), 1), (dict(history_most=-1), 1), (dict(history_most=2 ** 30, history_stride=2 ** 30), 1), (dict(history_stride=9), 1),
    (dict(repetition_all=0.0), 1), (dict(repetition_all=-1.0), 1), (dict(repetition_all=math.nan), 1), (dict(repetition_all=math.inf), 1),
    (dict(frequency_all=math.nan), 1), (dict(presence_all=math.inf), 1), (dict(n_bias=-1), 1), (dict(bias=None), 1),
    (dict(bias_token=None), 1), (dict(allowed_stride=3), 1), (dict(rows=0), 0), (dict(rows=0, logits=None, out=None), 0)])
def test_logit_controls(env, bad, code):  # noqa: F811
    stride, decode, L = env
    d = dict(history=DUMMY, history_stride=10, history_most=10, history_len=DUMMY, prompt_len=None, repetition=None, repetition_all=1.1,
             frequency=None, frequency_all=0.1, presence=None, presence_all=0.1, bias_off=DUMMY, bias_token=DUMMY, bias=DUMMY, n_bias=3,
             allowed=DUMMY, allowed_stride=4)
    d.update(of(decode._LogitRules._fields_, bad))
    r = decode._LogitRules(*[d[n] for n, _ in decode._LogitRules._fields_])
    assert L.stride_logit_controls(bad.get("logits", DUMMY), bad.get("ld", 100), bad.get("out", 2 * DUMMY), bad.get("ld_out", 100),
                                   bad.get("dtype", 0), bad.get("V", 100), bad.get("rows", 2), ctypes.byref(r), None, None) == code


def test_python_refuses_host_tensors(env):  # noqa: F811
    import torch

    stride, decode, L = env
    x = torch.zeros(2, 2, 64)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_attention_mass(x, x, x, x, x, x, None, 1.0, x)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_kv_evict(x[None], x[None], x, x, x, 4, x[None], x[None], x, x, x)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_logit_controls(x[0], x[0])
    with pytest.raises(TypeError):
        stride.stride_attention_mass(x)


def test_plain_forms():
    """The plain forms against cases worked by hand."""
    q, K = np.array([[[1.0, 0.0], [0.0, 2.0]], [[1.0, 1.0], [0.0, 0.0]]]), np.array([[0.0, 1.0], [2.0, 0.0], [1.0, 1.0]])
    lse = np.array([[0.0, 1.0], [0.5, -np.inf]])
    sees = np.array([[True, True, False], [True, True, True]])
    got, tol = ref.mass(np.array([10.0, 20.0, 30.0]), q, lse, K, 2, sees, 0.5, 0.5)
    want = [5 + math.exp(0) + math.exp(1 - 1) + math.exp(0.5 - 0.5), 10 + math.exp(1) + math.exp(0 - 1) + math.exp(1 - 0.5), math.exp(1 - 0.5)]
    assert np.allclose(got, want, rtol=1e-12) and (tol > 0).all() and (tol < 1e-4).all()
    m = np.array([1.0, 5.0, 5.0, np.nan, 0.0, 7.0, -np.inf, 5.0, 2.0], np.float32)
    assert ref.remaining(m, 9, 9, 0, 0).tolist() == list(range(9))
    assert ref.remaining(m, 9, 3, 0, 0).tolist() == [1, 2, 5]
    assert ref.remaining(m, 9, 4, 1, 1).tolist() == [0, 1, 5, 8]
    assert ref.remaining(m, 9, 8, 0, 0).tolist() == [0, 1, 2, 4, 5, 6, 7, 8]  # the NaN goes first
    assert ref.remaining(m, 9, 2, 3, 3).tolist() == [0, 1] and ref.remaining(m, 9, 3, 2, 5).tolist() == [0, 1, 8]
    assert ref.remaining(m, 4, 9, 1, 1).tolist() == [0, 1, 2, 3] and ref.remaining(m, 0, 9, 1, 1).tolist() == []
    y, _ = ref.controls(np.array([2.0, -2.0, 4.0, 1.0, -np.inf]), [0, 1, 2, 2, 0, -1, 9], 2, 2.0, 0.5, 0.25, [(3, 5.0), (2, 1.0), (3, -1.0)],
                        np.array([True, True, True, True, False]))
    assert y.tolist() == [1 - 0.5 - 0.25, -4.0, 2 - 1.0 - 0.25 + 1.0, 0.0, -np.inf]
