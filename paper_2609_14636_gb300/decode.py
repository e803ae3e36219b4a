"""The rollout's decode step around the scoring path (include/stride_decode.h):
norms of queries and keys with the position rotation, the append to a paged
cache, attention of drafted tokens over it, the weight that its slots got and
their eviction by it, controls on logits, and sampling.

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
    "DTYPE_F16", "DEV_POSITION", "DEV_NO_TOKEN", "DEV_BAD_CONTROL", "MAX_HEAD_DIM", "MAX_ATTENTION_DIM", "MAX_TREE", "MAX_TOP_P_VOCAB",
    "stride_qk_norm_rope", "stride_qk_norm_rope_backward", "stride_qk_norm_rope_backward_workspace_size", "stride_kv_append",
    "stride_tree_attention", "stride_tree_attention_workspace_size", "stride_attention_mass", "stride_kv_evict",
    "stride_logit_controls", "stride_sample",
]

DTYPE_F16 = 2
DEV_POSITION, DEV_NO_TOKEN, DEV_BAD_CONTROL = 0x8, 0x10, 0x20
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


class _SlotMass(ctypes.Structure):
    _fields_ = [("data", _P), ("seq_stride", _i64), ("head_stride", _i64), ("slots", _i64)]


class _EvictParams(ctypes.Structure):
    _fields_ = [("budget", _P), ("budget_all", _i32), ("sink", _i32), ("recent", _i32), ("most", _i32)]


class _LogitRules(ctypes.Structure):
    _fields_ = [("history", _P), ("history_stride", _i64), ("history_most", _i32), ("history_len", _P), ("prompt_len", _P), ("repetition", _P),
                ("repetition_all", _f32), ("frequency", _P), ("frequency_all", _f32), ("presence", _P), ("presence_all", _f32),
                ("bias_off", _P), ("bias_token", _P), ("bias", _P), ("n_bias", _i32), ("allowed", _P), ("allowed_stride", _i64)]


class _SampleParams(ctypes.Structure):
    _fields_ = [("temperature", _P), ("temperature_all", _f32), ("top_k", _P), ("top_k_all", _i32), ("top_p", _P),
                ("top_p_all", _f32), ("min_p", _P), ("min_p_all", _f32)]


def declare(L) -> None:
    """The argument types of the library's functions."""
    rows, how, cache = ctypes.POINTER(_HeadRows), ctypes.POINTER(_NormRope), ctypes.POINTER(_PagedCache)
    mass = ctypes.POINTER(_SlotMass)
    for fn, args, res in (
            ("stride_qk_norm_rope", [rows] * 4 + [_i32, _i64, _i32, how, _P, _P], ctypes.c_int),
            ("stride_qk_norm_rope_backward", [rows] * 6 + [_i32, _i64, _i32, how, _P, _P, _P, _P, _sz, _P], ctypes.c_int),
            ("stride_qk_norm_rope_backward_workspace_size", [_i64, _i32, _i32, _i32], _sz),
            ("stride_kv_append", [rows] * 4 + [_i32, _i64, _i32, how, cache, _P, _P], ctypes.c_int),
            ("stride_tree_attention", [rows] * 2 + [_P, _i32, _i64, _i32, _f32, _P, cache, _P, _P, _sz, _P], ctypes.c_int),
            ("stride_tree_attention_workspace_size", [_i64, _i32, _i32, _i32], _sz),
            ("stride_attention_mass", [rows, _P, _i32, _i64, _i32, _f32, _P, cache, _f32, mass, _P, _P], ctypes.c_int),
            ("stride_kv_evict", [cache, mass, cache, _i32, _i32, ctypes.POINTER(_EvictParams), _P, _P, mass, _P, _P], ctypes.c_int),
            ("stride_logit_controls", [_P, _i64, _P, _i64, _i32, _i64, _i32, ctypes.POINTER(_LogitRules), _P, _P], ctypes.c_int),
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
    c = _cache(k_cache, v_cache, block_table, like)
    c.ctx_len = _s._dev(ctx_len, "ctx_len", _s._torch().int32, c.n_seqs)
    c.tok_off = _s._dev(tok_off, "tok_off", _s._torch().int32, c.n_seqs + 1)
    return c


def _cache(k_cache, v_cache, block_table, like):
    """A checked pool and its block table, without lengths."""
    torch = _s._torch()
    for name, c in (("k_cache", k_cache), ("v_cache", v_cache)):
        if not isinstance(c, torch.Tensor) or not c.is_cuda or c.dim() != 4 or (c.shape[3] > 1 and c.stride(3) != 1):
            raise TypeError(f"{name} must be a CUDA tensor [pages, page_size, heads, D] with unit stride along D")
    if (k_cache.dtype != like.dtype or v_cache.dtype != like.dtype or k_cache.shape != v_cache.shape
            or k_cache.stride() != v_cache.stride() or k_cache.shape[3] != like.shape[-1]):
        raise ValueError("the caches must share shape and strides with each other, dtype and D with the rows")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [sequences, pages]")
    n = block_table.shape[0]
    pages, page, heads, _ = k_cache.shape
    return _PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), *k_cache.stride()[:3], pages, page, heads, n,
                       _s._dev(block_table, "block_table", torch.int32), block_table.shape[1], None, None)


def _slot_mass(t, name: str, seqs: int, heads: int):
    torch = _s._torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.float32:
        raise TypeError(f"{name} must be a float32 CUDA tensor")
    if t.dim() != 3 or t.shape[0] < seqs or t.shape[1] != heads or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name} must be [sequences, kv heads, slots] with unit stride along the slots")
    return _SlotMass(t.data_ptr(), t.stride(0), t.stride(1), t.shape[2])


def _logits_rows(t, name: str, V: int):
    """A row stride of logits [rows, >= V] (any, where there is one row)."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be [rows, V] with unit column stride")
    if V > t.shape[1]:
        raise ValueError(f"V is {V}, {name} has {t.shape[1]} columns")
    return max(t.stride(0), t.shape[1]) if t.shape[0] <= 1 else t.stride(0)


def _workspace(ws):
    return _s._dev(ws, "workspace", _s._torch().uint8, optional=True), 0 if ws is None else ws.numel()


def _each(value, name: str, dtype, rows: int, convert):
    """A parameter given per row (a tensor) or for all rows (a number): (pointer, number)."""
    if isinstance(value, _s._torch().Tensor):
        return _s._dev(value, name, dtype, rows), convert(0)
    return None, convert(value)


def _int32(value, name: str) -> int:
    """A number that the C structs hold in 32 bits (ctypes would cut it)."""
    v = int(value)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name} is {v}, beyond 32 bits")
    return v


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


def stride_attention_mass(q, lse, k_cache, block_table, ctx_len, tok_off, tree_mask, scale: float, mass, decay: float = 1.0,
                          dev_status=None, stream=None) -> None:
    """Adds the attention weights of the new tokens' queries [N, Hq, D] to their
    sequences' slots: q, the cache and lse [N, Hq] as of and after
    :func:`stride_tree_attention`.  mass float32 [sequences, kv heads, slots]
    with unit stride along the slots: mass = decay * mass + weights for the ctx_len
    committed slots (decay 0: whatever was there), the weights for the new
    tokens' own."""
    rc = (_s._NATIVE or _s._native()).attention_mass(q, lse, k_cache, block_table, ctx_len, tok_off, tree_mask, scale, mass, decay,
                                                     dev_status, stream)
    if rc is not None:
        return _s._check("stride_attention_mass", rc)
    torch, dt, N = _s._torch(), _dtype(q, "q"), q.shape[0]
    rows, cache = _head_rows(q, "q", q), _paged_cache(k_cache, k_cache, block_table, ctx_len, tok_off, q)
    rc = _s.lib().stride_attention_mass(
        ctypes.byref(rows), _s._dev(lse, "lse", torch.float32, N * q.shape[1]), dt, N, q.shape[2], float(scale),
        _s._dev(tree_mask, "tree_mask", torch.int64, N, optional=True), ctypes.byref(cache), float(decay),
        ctypes.byref(_slot_mass(mass, "mass", cache.n_seqs, cache.n_heads)),
        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_attention_mass", rc)


def stride_kv_evict(k_cache, v_cache, block_table, ctx_len, mass, budget, k_to, v_to, to_table, new_len, kept, mass_to=None,
                    sink: int = 0, recent: int = 0, dev_status=None, stream=None) -> None:
    """Copies of each sequence and kv head the slots that remain (up to `budget`:
    the first `sink`, the last `recent`, of the others those of the largest mass)
    in order into the pages of to_table in k_to, v_to (other pages of the same
    pools, or others).  budget: a number or int32 [sequences], negative: left
    out.  Written: int32 new_len [sequences], kept [sequences, kv heads, most]
    (the remaining slots), float32 mass_to [sequences, kv heads, >= most] or
    None (their masses)."""
    rc = (_s._NATIVE or _s._native()).kv_evict(k_cache, v_cache, block_table, ctx_len, mass, budget, k_to, v_to, to_table, new_len,
                                               kept, mass_to, sink, recent, dev_status, stream)
    if rc is not None:
        return _s._check("stride_kv_evict", rc)
    torch, dt = _s._torch(), _dtype(k_cache, "k_cache")
    if k_cache.dim() != 4 or k_to.dim() != 4:
        raise ValueError("caches must be [pages, page_size, heads, D]")
    like = k_cache[0]
    source = _cache(k_cache, v_cache, block_table, like)
    source.ctx_len = _s._dev(ctx_len, "ctx_len", torch.int32, source.n_seqs)
    to = _cache(k_to, v_to, to_table, like)
    if to.n_heads != source.n_heads or to.n_seqs != source.n_seqs:
        raise ValueError("both caches must have the same heads and sequences")
    if not isinstance(kept, torch.Tensor) or kept.dim() != 3 or kept.shape[1] != source.n_heads:
        raise ValueError("kept must be int32 [sequences, kv heads, most]")
    how = _EvictParams(*_each(budget, "budget", torch.int32, source.n_seqs, lambda v: _int32(v, "budget")), _int32(sink, "sink"),
                       _int32(recent, "recent"), _int32(kept.shape[2], "kept's row"))
    rc = _s.lib().stride_kv_evict(
        ctypes.byref(source), ctypes.byref(_slot_mass(mass, "mass", source.n_seqs, source.n_heads)), ctypes.byref(to), dt,
        k_cache.shape[3], ctypes.byref(how), _s._dev(new_len, "new_len", torch.int32, source.n_seqs),
        _s._dev(kept, "kept", torch.int32, source.n_seqs * source.n_heads * kept.shape[2]),
        None if mass_to is None else ctypes.byref(_slot_mass(mass_to, "mass_to", source.n_seqs, source.n_heads)),
        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_kv_evict", rc)


def stride_logit_controls(logits, out, history=None, history_len=None, prompt_len=None, repetition=1.0, frequency=0.0,
                          presence=0.0, bias_off=None, bias_token=None, bias=None, allowed=None, dev_status=None,
                          V: int | None = None, stream=None) -> None:
    """out = logits [rows, ld] with penalties for tokens that a row's sequence
    has, biases and a mask of allowed tokens (out may be logits).

    history int32 [rows, longest] with history_len int32 [rows], of which the
    first prompt_len (None: 0) are the prompt's: repetition divides (positive
    logits) or multiplies, frequency (times the count) and presence are taken
    off for the tokens past the prompt; numbers or float32 [rows].  bias_token
    int32, bias float32: row r's entries are bias_off[r] .. bias_off[r + 1] - 1
    (int32 [rows + 1]).  allowed int32 [rows or 1, words]: bit j % 32 of word
    j // 32 set, token j is allowed."""
    rc = (_s._NATIVE or _s._native()).logit_controls(logits, out, history, history_len, prompt_len, repetition, frequency, presence,
                                                     bias_off, bias_token, bias, allowed, dev_status, V, stream)
    if rc is not None:
        return _s._check("stride_logit_controls", rc)
    torch, dt = _s._torch(), _dtype(logits, "logits")
    V = logits.shape[-1] if V is None else int(V)
    if _dtype(out, "out") != dt or out.shape[0] != logits.shape[0]:
        raise ValueError("out must share dtype and rows with the logits")
    rows, ld, ld_out = logits.shape[0], _logits_rows(logits, "logits", V), _logits_rows(out, "out", V)
    r = _LogitRules()
    if history is not None:
        if not isinstance(history, torch.Tensor) or not history.is_cuda or history.dtype != torch.int32:
            raise TypeError("history must be an int32 CUDA tensor")
        if history.dim() != 2 or history.shape[0] < rows or (history.shape[1] > 1 and history.stride(1) != 1):
            raise ValueError("history must be [rows, longest] with unit column stride")
        r.history, r.history_stride = history.data_ptr(), history.stride(0)
        r.history_most = _int32(history.shape[1], "history's row")
        r.history_len = _s._dev(history_len, "history_len", torch.int32, rows)
        r.prompt_len = _s._dev(prompt_len, "prompt_len", torch.int32, rows, optional=True)
    elif history_len is not None or prompt_len is not None:
        raise ValueError("history_len and prompt_len go with a history")
    r.repetition, r.repetition_all = _each(repetition, "repetition", torch.float32, rows, float)
    r.frequency, r.frequency_all = _each(frequency, "frequency", torch.float32, rows, float)
    r.presence, r.presence_all = _each(presence, "presence", torch.float32, rows, float)
    if (bias_off is None) != (bias is None) or (bias_off is None) != (bias_token is None):
        raise ValueError("bias_off, bias_token and bias go together")
    if bias_off is not None:
        r.bias_off = _s._dev(bias_off, "bias_off", torch.int32, rows + 1)
        r.bias = _s._dev(bias, "bias", torch.float32)
        r.bias_token = _s._dev(bias_token, "bias_token", torch.int32, bias.numel())
        r.n_bias = _int32(bias.numel(), "biases")
    if allowed is not None:
        if not isinstance(allowed, torch.Tensor) or not allowed.is_cuda or allowed.dtype != torch.int32:
            raise TypeError("allowed must be an int32 CUDA tensor")
        if allowed.dim() != 2 or allowed.shape[0] not in (1, rows) or allowed.shape[1] < (V + 31) // 32 or (
                allowed.shape[1] > 1 and allowed.stride(1) != 1):
            raise ValueError("allowed must be [rows or 1, (V + 31) // 32] with unit column stride")
        r.allowed, r.allowed_stride = allowed.data_ptr(), 0 if allowed.shape[0] == 1 else allowed.stride(0)
    rc = _s.lib().stride_logit_controls(logits.data_ptr(), ld, out.data_ptr(), ld_out, dt, V, rows, ctypes.byref(r),
                                        _s._dev(dev_status, "dev_status", torch.int32, 1, optional=True), _s._stream(stream))
    _s._check("stride_logit_controls", rc)


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
