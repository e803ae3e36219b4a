"""What the decode step's calls refuse, before any CUDA call (CPU only; the
pointers are never dereferenced on these paths)."""
import ctypes
import math

import pytest

DUMMY = 4096  # non-null, aligned


@pytest.fixture(scope="module")
def env():
    import paper_2609_14636_gb300 as stride
    from paper_2609_14636_gb300 import decode

    return stride, decode, stride.lib()


def rows(decode, heads=4, D=64, data=DUMMY, token=None, head=None):
    return decode._HeadRows(data, heads * D if token is None else token, D if head is None else head, heads)


def how(decode, **kw):
    d = dict(q_weight=DUMMY, k_weight=DUMMY, eps=1e-6, interleaved=0, rot_dim=64, pos=DUMMY, cos_table=DUMMY, sin_table=DUMMY,
             table_rows=10)
    d.update(kw)
    return decode._NormRope(*[d[n] for n, _ in decode._NormRope._fields_])


def cache(decode, **kw):
    d = dict(k=DUMMY, v=DUMMY, page_stride=16 * 2 * 64, row_stride=2 * 64, head_stride=64, n_pages=4, page_size=16, n_heads=2,
             n_seqs=1, block_table=DUMMY, table_stride=4, ctx_len=DUMMY, tok_off=DUMMY)
    d.update(kw)
    return decode._PagedCache(*[d[n] for n, _ in decode._PagedCache._fields_])


def params(decode, **kw):
    d = dict(temperature=None, temperature_all=1.0, top_k=None, top_k_all=0, top_p=None, top_p_all=1.0, min_p=None, min_p_all=0.0)
    d.update(kw)
    return decode._SampleParams(*[d[n] for n, _ in decode._SampleParams._fields_])


def test_sizes_match_the_header(env):
    stride, decode, L = env
    src = (stride._build.INCLUDE / "stride_decode.h").read_text()
    for name, value in (("STRIDE_DTYPE_F16 ", decode.DTYPE_F16), ("STRIDE_MAX_HEAD_DIM ", decode.MAX_HEAD_DIM),
                        ("STRIDE_MAX_ATTENTION_DIM ", decode.MAX_ATTENTION_DIM), ("STRIDE_MAX_TREE ", decode.MAX_TREE),
                        ("STRIDE_DEV_POSITION ", hex(decode.DEV_POSITION)), ("STRIDE_DEV_NO_TOKEN ", hex(decode.DEV_NO_TOKEN))):
        assert f"#define {name}{value} " in src, name
    assert stride.stride_qk_norm_rope_backward_workspace_size(0, 4, 2, 64) == 0
    assert stride.stride_qk_norm_rope_backward_workspace_size(5, 4, 2, 64) % 256 == 0
    assert stride.stride_tree_attention_workspace_size(5, 4, 3, 64) == 0
    assert stride.stride_tree_attention_workspace_size(5, 4, 2, 64) > 0


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), 2), (dict(N=-1), 1), (dict(N=2 ** 31), 1), (dict(D=0), 1), (dict(D=1025), 1), (dict(data=None), 1),
    (dict(out_heads=3), 1), (dict(rot_dim=63), 1), (dict(rot_dim=66), 1), (dict(rot_dim=-2), 1), (dict(pos=None), 1),
    (dict(cos_table=None), 1), (dict(table_rows=0), 1), (dict(eps=math.nan), 1), (dict(eps=-1.0), 1), (dict(N=0), 0)])
def test_norm_rope(env, bad, code):
    stride, decode, L = env
    dtype, N, D = bad.get("dtype", 0), bad.get("N", 0 if code == 0 else 5), bad.get("D", 64)
    r, o = rows(decode, data=bad.get("data", DUMMY)), rows(decode, heads=bad.get("out_heads", 4))
    h = how(decode, **{k: v for k, v in bad.items() if k in ("rot_dim", "pos", "cos_table", "table_rows", "eps")})
    p = [ctypes.byref(x) for x in (r, r, o, o)]
    assert L.stride_qk_norm_rope(*p, dtype, N, D, ctypes.byref(h), None, None) == code
    assert L.stride_qk_norm_rope_backward(p[0], p[1], p[0], p[1], p[2], p[3], dtype, N, D, ctypes.byref(h), None, None, None, DUMMY,
                                          1 << 30, None) == code


def test_norm_rope_backward_workspace(env):
    stride, decode, L = env
    r, h = ctypes.byref(rows(decode)), how(decode)
    need = stride.stride_qk_norm_rope_backward_workspace_size(5, 4, 4, 64)
    call = lambda ws, n, h=h, dw=None: L.stride_qk_norm_rope_backward(r, r, r, r, r, r, 0, 5, 64, ctypes.byref(h), dw, None, None, ws, n, None)  # noqa: E731
    for ws, n in ((None, need), (DUMMY, need - 1), (DUMMY + 128, need)):
        assert call(ws, n) == stride.ERR_WORKSPACE
    assert call(DUMMY, need, how(decode, q_weight=None), DUMMY) == stride.ERR_INVALID_ARG  # a gradient of no weight


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=7), 2), (dict(k=None), 1), (dict(v=None), 1), (dict(n_pages=0), 1), (dict(page_size=0), 1), (dict(n_heads=3), 1),
    (dict(n_seqs=0), 1), (dict(table_stride=0), 1), (dict(block_table=None), 1), (dict(ctx_len=None), 1), (dict(tok_off=None), 1),
    (dict(rot_dim=1), 1), (dict(N=0), 0)])
def test_append(env, bad, code):
    stride, decode, L = env
    r = rows(decode, heads=2)
    c = cache(decode, **{k: v for k, v in bad.items() if k in dict(decode._PagedCache._fields_)})
    h = how(decode, rot_dim=bad.get("rot_dim", 64))
    assert L.stride_kv_append(ctypes.byref(r), ctypes.byref(r), None, None, bad.get("dtype", 0), bad.get("N", 3), 64, ctypes.byref(h),
                              ctypes.byref(c), None, None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=1), 2), (dict(D=60), 1), (dict(D=136), 1), (dict(D=0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
    (dict(heads=3), 1), (dict(data=DUMMY + 2), 1), (dict(token=4 * 64 + 4), 1), (dict(head=68), 1), (dict(k=DUMMY + 8), 1),
    (dict(row_stride=129), 1), (dict(page_stride=4), 1), (dict(head_stride=4), 1), (dict(workspace=None), 3), (dict(bytes=-1), 3),
    (dict(workspace=DUMMY + 16), 3), (dict(N=-1), 1), (dict(N=0), 0)])
def test_attention(env, bad, code):
    stride, decode, L = env
    q = rows(decode, heads=bad.get("heads", 4), data=bad.get("data", DUMMY), token=bad.get("token"), head=bad.get("head"))
    c = cache(decode, **{k: v for k, v in bad.items() if k in dict(decode._PagedCache._fields_)})
    D, N = bad.get("D", 64), bad.get("N", 5)
    need = stride.stride_tree_attention_workspace_size(5, 4, 2, 64)
    assert L.stride_tree_attention(ctypes.byref(q), ctypes.byref(q), None, bad.get("dtype", 0), N, D, bad.get("scale", 0.1), None,
                                   ctypes.byref(c), None, bad.get("workspace", DUMMY), need + bad.get("bytes", 0), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), 2), (dict(V=0), 1), (dict(V=2 ** 30 + 1, ld=2 ** 31), 1), (dict(ld=99), 1), (dict(rows=-1), 1),
    (dict(logits=None), 1), (dict(tokens=None), 1), (dict(noise=None), 1), (dict(ld_noise=99), 1), (dict(temperature_all=-1.0), 1),
    (dict(temperature_all=math.nan), 1), (dict(temperature_all=math.inf), 1), (dict(top_p_all=math.nan), 1),
    (dict(min_p_all=math.nan), 1), (dict(rows=0), 0), (dict(rows=0, temperature_all=0.0, noise=None, ld_noise=0), 0)])
def test_sample(env, bad, code):
    stride, decode, L = env
    p = params(decode, **{k: v for k, v in bad.items() if k in dict(decode._SampleParams._fields_)})
    assert L.stride_sample(bad.get("logits", DUMMY), bad.get("dtype", 0), bad.get("ld", 100), bad.get("V", 100), bad.get("rows", 2),
                           bad.get("noise", DUMMY), bad.get("ld_noise", 100), ctypes.byref(p), bad.get("tokens", DUMMY), None, None,
                           None) == code


def test_python_refuses_host_tensors(env):
    import torch

    stride, decode, L = env
    x = torch.zeros(2, 2, 64)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_qk_norm_rope(x, x, x, x)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_kv_append(x, x, x, x, x, x, x)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_tree_attention(x, x, x, x, x, x, None, 1.0, x)
    with pytest.raises(TypeError, match="CUDA"):
        stride.stride_sample(x[0], None, x, temperature=0)
    for fn in (stride.stride_qk_norm_rope_backward, stride.stride_qk_norm_rope):
        with pytest.raises(TypeError):
            fn(x)


def test_data_between_elements(env):
    """Rows, caches, logits and noise that no element of their type can start at."""
    stride, decode, L = env
    odd, r, h, c, s = ctypes.byref(rows(decode, data=DUMMY + 1)), ctypes.byref(rows(decode, heads=2)), how(decode), cache(decode), params(decode)
    h, c, s = ctypes.byref(h), ctypes.byref(c), ctypes.byref(s)
    assert L.stride_qk_norm_rope(odd, r, odd, r, 0, 5, 64, h, None, None) == 1
    assert L.stride_qk_norm_rope_backward(odd, r, odd, r, odd, r, 0, 5, 64, h, None, None, None, DUMMY, 1 << 30, None) == 1
    assert L.stride_kv_append(r, r, odd, odd, 0, 5, 64, h, c, None, None) == 1
    assert L.stride_kv_append(r, r, None, None, 0, 5, 64, h, ctypes.byref(cache(decode, k=DUMMY + 1)), None, None) == 1
    assert L.stride_tree_attention(r, odd, None, 0, 5, 64, 1.0, None, c, None, DUMMY, 1 << 30, None) == 1
    for x, noise, dtype in ((DUMMY + 1, DUMMY, 0), (DUMMY + 2, DUMMY, 1), (DUMMY, DUMMY + 2, 0)):
        assert L.stride_sample(x, dtype, 100, 100, 2, noise, 100, s, DUMMY, None, None, None) == 1
