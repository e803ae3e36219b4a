"""The rollout's decode step around the scoring path (include/stride_decode.h):
norms of queries and keys with the position rotation, the append to a paged
cache, attention of drafted tokens over it, and sampling.

The functions keep the C names; they take torch CUDA tensors as those of the
package do and are part of it (``stride.stride_sample`` and so on).  Head rows
are ``[tokens, heads, D]`` tensors with unit stride along D and any other
strides, so q, k and v may be views of one fused projection; caches are
``[pages, page_size, heads, D]`` with any strides of the first three (a pool
stored heads first is passed as its transposed view).
"""
from __future__ import annotations

import ctypes

import paper_2609_14636_gb300 as _s

__all__ = [
    "DTYPE_F16", "DEV_POSITION", "DEV_NO_TOKEN", "MAX_HEAD_DIM", "MAX_ATTENTION_DIM", "MAX_TREE", "MAX_TOP_P_VOCAB",
    "stride_qk_norm_rope", "stride_qk_norm_rope_backward", "stride_qk_norm_rope_backward_workspace_size", "stride_kv_append",
    "stride_tree_attention", "stride_tree_attention_workspace_size", "stride_sample",
]

DTYPE_F16 = 2
DEV_POSITION, DEV_NO_TOKEN = 0x8, 0x10
MAX_HEAD_DIM = 1024  # STRIDE_MAX_HEAD_DIM
MAX_ATTENTION_DIM = 128  # STRIDE_MAX_ATTENTION_DIM
MAX_TREE = 64  # STRIDE_MAX_TREE
MAX_TOP_P_VOCAB = 1 << 23  # STRIDE_MAX_TOP_P_VOCAB

_P, _i32, _i64, _f32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class _HeadRows(ctypes.Structure):
    _fields_ = [("data", _P), ("token_stride", _i64), ("head_stride", _i64), ("n_heads", _i32)]


class _NormRope(ctypes.Structure):
    _fields_ = [("q_weight", _P), ("k_weight", _P), ("eps", _f32), ("interleaved", _i32), ("rot_dim", _i32), ("pos", _P),
                ("cos_table", _P), ("sin_table", _P), ("table_rows", _i64)]


class _PagedCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("page_stride", _i64), ("row_stride", _i64), ("head_stride", _i64), ("n_pages", _i32),
                ("page_size", _i32), ("n_heads", _i32), ("n_seqs", _i32), ("block_table", _P), ("table_stride", _i64),
                ("ctx_len", _P), ("tok_off", _P)]


class _SampleParams(ctypes.Structure):
    _fields_ = [("temperature", _P), ("temperature_all", _f32), ("top_k", _P), ("top_k_all", _i32), ("top_p", _P),
                ("top_p_all", _f32), ("min_p", _P), ("min_p_all", _f32)]


def declare(L) -> None:
    """The argument types of the library's functions."""
    rows, how, cache = ctypes.POINTER(_HeadRows), ctypes.POINTER(_NormRope), ctypes.POINTER(_PagedCache)
    for fn, args, res in (
            ("stride_qk_norm_rope", [rows] * 4 + [_i32, _i64, _i32, how, _P, _P], ctypes.c_int),
            ("stride_qk_norm_rope_backward", [rows] * 6 + [_i32, _i64, _i32, how, _P, _P, _P, _P, _sz, _P], ctypes.c_int),
            ("stride_qk_norm_rope_backward_workspace_size", [_i64, _i32, _i32, _i32], _sz),
            ("stride_kv_append", [rows] * 4 + [_i32, _i64, _i32, how, cache, _P, _P], ctypes.c_int),
            ("stride_tree_attention", [rows] * 2 + [_P, _i32, _i64, _i32, _f32, _P, cache, _P, _P, _sz, _P], ctypes.c_int),
            ("stride_tree_attention_workspace_size", [_i64, _i32, _i32, _i32], _sz),
            ("stride_sample", [_P, _i32, _i64, _i64, _i32, _P, _i64, ctypes.POINTER(_SampleParams), _P, _P, _P, _P], ctypes.c_int)):
        getattr(L, fn).argtypes = args
        getattr(L, fn).restype = res


# ---------------------------------------------------------------------------
# marshalling
# ---------------------------------------------------------------------------
def _dtype(t, name: str) -> int:
    torch = _s._torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    codes = {torch.bfloat16: _s.DTYPE_BF16, torch.float32: _s.DTYPE_F32, torch.float16: DTYPE_F16}
    if t.dtype not in codes:
        raise TypeError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
    return codes[t.dtype]


def _head_rows(t, name: str, like):
    """Checked head rows of the shape [like.shape[0], any, like.shape[2]] and like's type."""
    _dtype(t, name)
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be [tokens, heads, D] with unit stride along D")
    if t.dtype != like.dtype or t.shape[0] != like.shape[0] or t.shape[2] != like.shape[2]:
        raise ValueError(f"{name} must share dtype, tokens and D with the other rows")
    return _HeadRows(t.data_ptr(), t.stride(0), t.stride(1), t.shape[1])


def _norm_rope(like, N, pos, cos, sin, q_weight, k_weight, eps, interleaved):
    torch, D = _s._torch(), like.shape[2]
    h = _NormRope(_s._dev(q_weight, "q_weight", like.dtype, D, optional=True),
                  _s._dev(k_weight, "k_weight", like.dtype, D, optional=True), float(eps), int(bool(interleaved)), 0, None, None,
                  None, 0)
    if (cos is None) != (sin is None) or (cos is not None and pos is None):
        raise ValueError("a rotation takes pos, cos and sin together")
    if cos is not None:
        if cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must be [positions, rot_dim / 2]")
        h.rot_dim = 2 * cos.shape[1]
        h.pos = _s._dev(pos, "pos", torch.int32, N)
        h.cos_table, h.sin_table = _s._dev(cos, "cos", torch.float32), _s._dev(sin, "sin", torch.float32)
        h.table_rows = cos.shape[0]
    return h


def _paged_cache(k_cache, v_cache, block_table, ctx_len, tok_off, like):
    torch = _s._torch()
    for name, c in (("k_cache", k_cache), ("v_cache", v_cache)):
        if not isinstance(c, torch.Tensor) or not c.is_cuda or c.dim() != 4 or (c.shape[3] > 1 and c.stride(3) != 1):
            raise TypeError(f"{name} must be a CUDA tensor [pages, page_size, heads, D] with unit stride along D")
    if (k_cache.dtype != like.dtype or v_cache.dtype != like.dtype or k_cache.shape != v_cache.shape
            or k_cache.stride() != v_cache.stride() or k_cache.shape[3] != like.shape[2]):
        raise ValueError("the caches must share shape and strides with each other, dtype and D with the rows")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [sequences, pages]")
    n = block_table.shape[0]
    pages, page, heads, _ = k_cache.shape
    return _PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), *k_cache.stride()[:3], pages, page, heads, n,
                       _s._dev(block_table, "block_table", torch.int32), block_table.shape[1],
                       _s._dev(ctx_len, "ctx_len", torch.int32, n), _s._dev(tok_off, "tok_off", torch.int32, n + 1))


def _workspace(ws):
    return _s._dev(ws, "workspace", _s._torch().uint8, optional=True), 0 if ws is None else ws.numel()


def _each(value, name: str, dtype, rows: int, convert):
    """A parameter given per row (a tensor) or for all rows (a number): (pointer, number)."""
    if isinstance(value, _s._torch().Tensor):
        return _s._dev(value, name, dtype, rows), convert(0)
    return None, convert(value)


# ---------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------
def stride_qk_norm_rope(q, k, q_out, k_out, pos=None, cos=None, sin=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                        interleaved: bool = False, dev_status=None, stream=None) -> None:
    """Norms of queries and keys for each head, and their position rotation.

    q, k: [N, Hq, D], [N, Hk, D]; q_out, k_out likewise (may be q, k);
    q_weight, k_weight [D] of their type or None (not normalised); cos, sin
    float32 [positions, rot_dim / 2] with pos int32 [N], or None (not
    rotated).  interleaved: pairs (2i, 2i + 1) instead of halves."""
    rc = (_s._NATIVE or _s._native()).qk_norm_rope(q, k, q_out, k_out, pos, cos, sin, q_weight, k_weight, eps, interleaved,
                                                   dev_status, stream)
    if rc is not None:
        return _s._check("stride_qk_norm_rope", rc)
    dt, N, D = _dtype(q, "q"), q.shape[0], q.shape[-1]
    rc = _s.lib().stride_qk_norm_rope(
        *[ctypes.byref(_head_rows(t, n, q)) for n, t in (("q", q), ("k", k), ("q_out", q_out), ("k_out", k_out))], dt, N, D,
        ctypes.byref(_norm_rope(q, N, pos, cos, sin, q_weight, k_weight, eps, interleaved)),
        _s._dev(dev_status, "dev_status", _s._torch().int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_qk_norm_rope", rc)


def stride_qk_norm_rope_backward_workspace_size(n_tokens: int, Hq: int, Hk: int, D: int) -> int:
    return int(_s.lib().stride_qk_norm_rope_backward_workspace_size(int(n_tokens), int(Hq), int(Hk), int(D)))


def stride_qk_norm_rope_backward(dq_out, dk_out, q, k, dq, dk, pos=None, cos=None, sin=None, q_weight=None, k_weight=None,
                                 eps: float = 1e-6, interleaved: bool = False, dq_weight=None, dk_weight=None,
                                 workspace=None, dev_status=None, stream=None) -> None:
    """Gradients of :func:`stride_qk_norm_rope` at its inputs q, k: dq, dk, and
    float32 [D] dq_weight, dk_weight (None: not computed).  workspace: uint8
    of stride_qk_norm_rope_backward_workspace_size(N, Hq, Hk, D) bytes."""
    rc = (_s._NATIVE or _s._native()).qk_norm_rope_backward(dq_out, dk_out, q, k, dq, dk, pos, cos, sin, q_weight, k_weight,
                                                            eps, interleaved, dq_weight, dk_weight, workspace, dev_status,
                                                            stream)
    if rc is not None:
        return _s._check("stride_qk_norm_rope_backward", rc)
    torch, dt, N, D = _s._torch(), _dtype(q, "q"), q.shape[0], q.shape[-1]
    rows = (("dq_out", dq_out), ("dk_out", dk_out), ("q", q), ("k", k), ("dq", dq), ("dk", dk))
    rc = _s.lib().stride_qk_norm_rope_backward(
        *[ctypes.byref(_head_rows(t, n, q)) for n, t in rows], dt, N, D,
        ctypes.byref(_norm_rope(q, N, pos, cos, sin, q_weight, k_weight, eps, interleaved)),
        _s._dev(dq_weight, "dq_weight", torch.float32, D, optional=True),
        _s._dev(dk_weight, "dk_weight", torch.float32, D, optional=True),
        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), *_workspace(workspace), _s._stream(stream))
    _s._check("stride_qk_norm_rope_backward", rc)


def stride_kv_append(k, v, k_cache, v_cache, block_table, ctx_len, tok_off, pos=None, cos=None, sin=None, k_weight=None,
                     q=None, q_out=None, q_weight=None, eps: float = 1e-6, interleaved: bool = False, dev_status=None,
                     stream=None) -> None:
    """Writes the new tokens' keys (normed, rotated) and values into their
    sequences' slots; with q, q_out [N, Hq, D] also q_out = normed, rotated q.

    k, v: [N, Hk, D]; block_table int32 [sequences, pages]; ctx_len int32
    [sequences] tokens already cached; tok_off int32 [sequences + 1]: sequence
    b's new tokens are rows tok_off[b] .. tok_off[b + 1] - 1."""
    rc = (_s._NATIVE or _s._native()).kv_append(k, v, k_cache, v_cache, block_table, ctx_len, tok_off, pos, cos, sin, k_weight,
                                                q, q_out, q_weight, eps, interleaved, dev_status, stream)
    if rc is not None:
        return _s._check("stride_kv_append", rc)
    dt, N, D = _dtype(k, "k"), k.shape[0], k.shape[-1]
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    rows = [ctypes.byref(_head_rows(k, "k", k)), ctypes.byref(_head_rows(v, "v", k))]
    rows += [None, None] if q is None else [ctypes.byref(_head_rows(q, "q", k)), ctypes.byref(_head_rows(q_out, "q_out", k))]
    rc = _s.lib().stride_kv_append(
        *rows, dt, N, D, ctypes.byref(_norm_rope(k, N, pos, cos, sin, q_weight, k_weight, eps, interleaved)),
        ctypes.byref(_paged_cache(k_cache, v_cache, block_table, ctx_len, tok_off, k)),
        _s._dev(dev_status, "dev_status", _s._torch().int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_kv_append", rc)


def stride_tree_attention_workspace_size(n_tokens: int, Hq: int, Hk: int, D: int) -> int:
    return int(_s.lib().stride_tree_attention_workspace_size(int(n_tokens), int(Hq), int(Hk), int(D)))


def stride_tree_attention(q, k_cache, v_cache, block_table, ctx_len, tok_off, tree_mask, scale: float, out, lse=None,
                          workspace=None, dev_status=None, stream=None) -> None:
    """Attention of the new tokens' queries [N, Hq, D] over the paged cache
    (their own keys and values in it) into out [N, Hq, D], and float32 lse
    [N, Hq].  tree_mask int64 [N]: bit j of a token's word, it sees new token j
    of its sequence (at most MAX_TREE); None: each sees those up to itself.
    workspace: uint8 of stride_tree_attention_workspace_size(N, Hq, Hk, D)
    bytes."""
    rc = (_s._NATIVE or _s._native()).tree_attention(q, k_cache, v_cache, block_table, ctx_len, tok_off, tree_mask, scale, out,
                                                     lse, workspace, dev_status, stream)
    if rc is not None:
        return _s._check("stride_tree_attention", rc)
    torch, dt, N = _s._torch(), _dtype(q, "q"), q.shape[0]
    rc = _s.lib().stride_tree_attention(
        ctypes.byref(_head_rows(q, "q", q)), ctypes.byref(_head_rows(out, "out", q)),
        _s._dev(lse, "lse", torch.float32, N * q.shape[1], optional=True), dt, N, q.shape[2], float(scale),
        _s._dev(tree_mask, "tree_mask", torch.int64, N, optional=True),
        ctypes.byref(_paged_cache(k_cache, v_cache, block_table, ctx_len, tok_off, q)),
        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), *_workspace(workspace), _s._stream(stream))
    _s._check("stride_tree_attention", rc)


def stride_sample(logits, noise, tokens, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, logp=None, dev_status=None,
                  V: int | None = None, stream=None) -> None:
    """Samples a token of each row of logits [rows, ld] into int32 tokens, its
    log-probability under the distribution it was drawn from into float32 logp.

    noise: float32 [rows, >= V] of independent Exp(1) numbers
    (``torch.empty(rows, V).exponential_()``); None where temperature is the
    number 0.  temperature, top_p, min_p: numbers or float32 [rows]; top_k: a
    number or int32 [rows] (see include/stride_decode.h)."""
    rc = (_s._NATIVE or _s._native()).sample(logits, noise, tokens, temperature, top_k, top_p, min_p, logp, dev_status, V,
                                             stream)
    if rc is not None:
        return _s._check("stride_sample", rc)
    torch, dt = _s._torch(), _dtype(logits, "logits")
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, V] with unit column stride")
    rows, V = logits.shape[0], logits.shape[1] if V is None else int(V)
    if V > logits.shape[1]:
        raise ValueError(f"V is {V}, the logits have {logits.shape[1]} columns")
    if noise is not None:
        if not isinstance(noise, torch.Tensor) or not noise.is_cuda or noise.dtype != torch.float32:
            raise TypeError("noise must be a float32 CUDA tensor")
        if noise.dim() != 2 or noise.shape[0] < rows or noise.shape[1] < V or (noise.shape[1] > 1 and noise.stride(1) != 1):
            raise ValueError("noise must be [rows, V] with unit column stride")
    params = _SampleParams(*_each(temperature, "temperature", torch.float32, rows, float),
                           *_each(top_k, "top_k", torch.int32, rows, int), *_each(top_p, "top_p", torch.float32, rows, float),
                           *_each(min_p, "min_p", torch.float32, rows, float))
    rc = _s.lib().stride_sample(
        logits.data_ptr(), dt, max(logits.stride(0), logits.shape[1]) if rows <= 1 else logits.stride(0), V, rows,
        None if noise is None else noise.data_ptr(),
        0 if noise is None else max(noise.stride(0), noise.shape[1]) if rows <= 1 else noise.stride(0),
        ctypes.byref(params), _s._dev(tokens, "tokens", torch.int32, rows),
        _s._dev(logp, "logp", torch.float32, rows, optional=True),
        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_sample", rc)
