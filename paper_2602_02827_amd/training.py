"""ctypes binding of the training operators (include/colbandit_train.h), and their autograd forms.

The `colbandit_*` functions marshal arguments only, as those of `binding` do: torch supplies device
memory and the current stream, every step runs in the library's HIP kernels, and there is no
fallback.  Tensors must live on the current device.  `embedding`, `norm_rotate`, `attention`, `contrastive_maxsim`,
`clip_gradients_` and `orthogonal_step_` are the same operators as parts of a torch program.
"""
from __future__ import annotations

import ctypes
import math
from operator import index

import numpy as np
import torch

from . import binding
from .binding import BF16, F32, ColbanditError

EXPORTS = [
    "colbandit_sizeof_attn", "colbandit_bias_buckets", "colbandit_attention_workspace_bytes", "colbandit_attention",
    "colbandit_attention_backward", "colbandit_maxsim_scores", "colbandit_contrastive_loss", "colbandit_maxsim_backward",
    "colbandit_clip_workspace_bytes", "colbandit_clip_gradients",
    "colbandit_sizeof_window", "colbandit_attention_window_workspace_bytes", "colbandit_attention_window",
    "colbandit_attention_window_backward", "colbandit_embedding", "colbandit_embedding_workspace_bytes",
    "colbandit_embedding_backward", "colbandit_sizeof_rotation", "colbandit_rotary_table", "colbandit_norm_rotate",
    "colbandit_norm_rotate_workspace_bytes", "colbandit_norm_rotate_backward", "colbandit_orthogonalise_workspace_bytes",
    "colbandit_orthogonalise",
]

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}
_ERR_WORKSPACE = -5                                  # COLBANDIT_ERR_WORKSPACE


class ColbanditAttn(ctypes.Structure):
    _fields_ = [("dt", ctypes.c_int), ("n_seqs", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("d", ctypes.c_int), ("causal", ctypes.c_int), ("n_buckets", ctypes.c_int), ("max_distance", ctypes.c_int),
                ("scale", ctypes.c_float), ("total_q", ctypes.c_int64), ("total_k", ctypes.c_int64),
                ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_row", ctypes.c_int64), ("q_head", ctypes.c_int64), ("k_row", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("v_row", ctypes.c_int64), ("v_head", ctypes.c_int64),
                ("keep", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


class ColbanditWindow(ctypes.Structure):
    _fields_ = [("before", ctypes.c_int64), ("after", ctypes.c_int64), ("sinks", ctypes.c_int64)]


class ColbanditRotation(ctypes.Structure):
    _fields_ = [("dt", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int), ("d", ctypes.c_int),
                ("interleaved", ctypes.c_int), ("eps", ctypes.c_float), ("rows", ctypes.c_int64), ("n_positions", ctypes.c_int64),
                ("q", ctypes.c_void_p), ("k", ctypes.c_void_p),
                ("q_row", ctypes.c_int64), ("q_head", ctypes.c_int64), ("k_row", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("table", ctypes.c_void_p), ("positions", ctypes.c_void_p)]


_lib = None


def lib():
    """The library that `binding` loads, with the training calls' signatures."""
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, i, i64, sz, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        d = ctypes.c_double
        attn, window, rotation = (ctypes.POINTER(t) for t in (ColbanditAttn, ColbanditWindow, ColbanditRotation))
        for name, res, args in [
                ("colbandit_sizeof_attn", sz, []),
                ("colbandit_bias_buckets", i, [i, i, i, vp]),
                ("colbandit_attention_workspace_bytes", sz, [attn, i]),
                ("colbandit_attention", i, [attn, vp, vp, vp, sz, vp]),
                ("colbandit_attention_backward", i, [attn, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
                ("colbandit_maxsim_scores", i, [vp, i, i, i, i, vp, vp, i64, i64, vp, vp, vp]),
                ("colbandit_contrastive_loss", i, [vp, i, i64, vp, f, vp, vp, vp]),
                ("colbandit_maxsim_backward", i, [vp, vp, vp, i, i, i, i, vp, vp, i64, i64, vp, vp, vp]),
                ("colbandit_clip_workspace_bytes", sz, [i64, vp]),
                ("colbandit_clip_gradients", i, [i64, vp, vp, vp, vp, f, vp, vp, sz, vp]),
                ("colbandit_sizeof_window", sz, []),
                ("colbandit_attention_window_workspace_bytes", sz, [attn, window, i]),
                ("colbandit_attention_window", i, [attn, window, vp, vp, vp, sz, vp]),
                ("colbandit_attention_window_backward", i, [attn, window, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
                ("colbandit_embedding", i, [vp, i, i64, vp, i64, i64, i64, f, vp, i, vp]),
                ("colbandit_embedding_workspace_bytes", sz, [i64, i64, i64]),
                ("colbandit_embedding_backward", i, [vp, i, i64, vp, i64, i64, i64, f, vp, i, vp, sz, vp]),
                ("colbandit_sizeof_rotation", sz, []),
                ("colbandit_rotary_table", i, [i64, i, d, vp]),
                ("colbandit_norm_rotate", i, [rotation, vp, vp, vp]),
                ("colbandit_norm_rotate_workspace_bytes", sz, [rotation]),
                ("colbandit_norm_rotate_backward", i, [rotation, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
                ("colbandit_orthogonalise_workspace_bytes", sz, [i64, vp, vp]),
                ("colbandit_orthogonalise", i, [i64, vp, vp, vp, vp, vp, i, vp, vp, sz, vp])]:
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        if (L.colbandit_sizeof_attn(), L.colbandit_sizeof_window(), L.colbandit_sizeof_rotation()) != tuple(
                ctypes.sizeof(t) for t in (ColbanditAttn, ColbanditWindow, ColbanditRotation)):
            raise ImportError("libcolbandit.so was built from a different colbandit_train.h: rebuild it")
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(dev=None):
    # the handle alone: making a Stream object of it costs as much as a small call's kernels (2.8 us)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if dev is None else dev)


def _check(rc, what):
    if rc:
        raise ColbanditError(rc, what)


def _on_device(*tensors):
    """The current device, on which all of them must live."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors must live on the current device")
    return dev


def _offsets(off):
    if off.dtype != torch.int64 or off.dim() != 1 or not off.is_contiguous() or off.shape[0] < 2:
        raise ValueError("offsets must be a contiguous int64 vector of the sequences' number and one")
    return off


def _workspace(ws, need, device):
    if not need:
        return None, 0
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _on_device(ws)
        if not ws.is_contiguous():
            raise ValueError("the workspace must be contiguous")
    return ws, ws.numel() * ws.element_size()


def colbandit_bias_buckets(n_buckets, max_distance, causal=False) -> np.ndarray:
    """First distance of each bucket of one direction (computed by the library)."""
    starts = np.zeros(max(1, int(n_buckets)), dtype=np.int32)
    n = lib().colbandit_bias_buckets(int(n_buckets), int(max_distance), int(causal), starts.ctypes.data)
    if n < 0:
        raise ColbanditError(n, "colbandit_bias_buckets")
    return starts[:n]


def _attn(q, k, v, q_offsets, k_offsets, causal, scale, keep, bias, max_distance):
    if k_offsets is None:
        k_offsets = q_offsets
    dtype = q.dtype
    dt = _DTYPES.get(dtype)
    if dt is None or k.dtype != dtype or v.dtype != dtype:
        raise TypeError("q, k and v must be float32 or bfloat16, all of one type")
    k_shape = k.shape
    if q.dim() != 3 or len(k_shape) != 3 or v.shape != k_shape or q.shape[2] != k_shape[2]:
        raise ValueError("q is [total_q, heads, d], k and v are [total_k, kv_heads, d]")
    total_q, heads, d = q.shape
    total_k, kv_heads, _ = k_shape
    (q_row, q_head, q_last), (k_row, k_head, k_last), (v_row, v_head, v_last) = q.stride(), k.stride(), v.stride()
    if q_last != 1 or k_last != 1 or v_last != 1:
        raise ValueError("the values of a row and head must be consecutive")
    n = _offsets(q_offsets).shape[0]
    if k_offsets is not q_offsets and _offsets(k_offsets).shape[0] != n:
        raise ValueError("q_offsets and k_offsets must hold equally many sequences")
    if keep is not None:
        if keep.dtype not in (torch.bool, torch.uint8) or keep.shape != k_shape[:1] or not keep.is_contiguous():
            raise ValueError("keep is a contiguous bool or uint8 vector over the key rows")
    if bias is not None:
        if bias.dtype != dtype:
            raise TypeError("bias must have the type of q")
        if bias.dim() != 2 or bias.shape[1] != heads or not bias.is_contiguous():
            raise ValueError("bias is a contiguous [n_buckets, heads]")
    _on_device(q, k, v, q_offsets, k_offsets, keep, bias)
    return ColbanditAttn(
        dt, n - 1, heads, kv_heads, d, 1 if causal else 0, 0 if bias is None else bias.shape[0], _within(int(max_distance), 30),
        1.0 / math.sqrt(d) if scale is None else scale, total_q, total_k, q_offsets.data_ptr(), k_offsets.data_ptr(),
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_row, q_head, k_row, k_head, v_row, v_head, _ptr(keep), _ptr(bias))


def _within(x, bits):
    """A whole number, cut to what fits (ctypes would leave out its upper bits)."""
    return max(-1 << bits, min(index(x), 1 << bits))


def _window(window, sinks):
    """(before, after) and a number of first keys as the library takes them; None: all keys."""
    if window is None:
        if sinks:
            raise ValueError("sinks come with a window")
        return None
    before, after = window
    return ColbanditWindow(*(_within(x, 62) for x in (before, after, sinks)))


def _like(t):
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def _new(t, dtype, *shape):
    # without a type, and from numbers, it takes 1 us less, which small calls notice
    return t.new_empty(*shape) if dtype is t.dtype else t.new_empty(shape, dtype=dtype)


def _dense(t, shape, dtype, what):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


def colbandit_attention(q, k, v, q_offsets, k_offsets=None, *, causal=False, scale=None, keep=None, bias=None,
                        max_distance=128, window=None, sinks=0, workspace=None, out=None):
    """Attention over packed sequences, of all keys or, with window=(before, after), of those up to so far from a row's
    position and the first `sinks` of its sequence.  q [total_q, heads, d], k and v [total_k, kv_heads, d] (any
    row and head strides), offsets int64 [n+1]; `k_offsets` None: the queries' own; rows behind the last
    sequence get zeros.  `out`: tensors to write, as this returns them.  Returns dict(out [total_q, heads, d], lse float32
    [heads, total_q])."""
    w = _window(window, sinks)
    a = _attn(q, k, v, q_offsets, k_offsets, causal, scale, keep, bias, max_distance)
    L = lib()
    o, lse = (out["out"], out["lse"]) if out else (None, None)
    o = _like(q) if o is None else _dense(o, q.shape, q.dtype, "out")
    lse = _new(q, torch.float32, a.heads, a.total_q) if lse is None else _dense(lse, (a.heads, a.total_q), torch.float32, "lse")
    dev = _on_device(o, lse)
    if w is not None:
        ws, nb = _workspace(workspace, L.colbandit_attention_window_workspace_bytes(a, w, 0), q.device)
        _check(L.colbandit_attention_window(a, w, o.data_ptr(), lse.data_ptr(), _ptr(ws), nb, _stream(dev)), "colbandit_attention_window")
        return {"out": o, "lse": lse}
    ws, nb = _workspace(workspace, L.colbandit_attention_workspace_bytes(a, 0), q.device)
    _check(L.colbandit_attention(a, o.data_ptr(), lse.data_ptr(), _ptr(ws), nb, _stream(dev)), "colbandit_attention")
    return {"out": o, "lse": lse}


def colbandit_attention_backward(dout, q, k, v, out, lse, q_offsets, k_offsets=None, *, causal=False, scale=None,
                                 keep=None, bias=None, max_distance=128, window=None, sinks=0, workspace=None):
    """Gradients of colbandit_attention's inputs from that of its output.  Returns dict(dq, dk, dv,
    dbias), dense, `dbias` None without a bias."""
    w = _window(window, sinks)
    a = _attn(q, k, v, q_offsets, k_offsets, causal, scale, keep, bias, max_distance)
    L = lib()
    _dense(out, q.shape, q.dtype, "out")
    _dense(lse, (q.shape[1], q.shape[0]), torch.float32, "lse")
    _dense(dout, q.shape, q.dtype, "dout")
    _on_device(out, lse, dout)
    dq, dk, dv = _like(q), _like(k), _like(k)
    dbias = None if bias is None else torch.empty_like(bias)
    if w is not None:
        ws, nb = _workspace(workspace, L.colbandit_attention_window_workspace_bytes(a, w, 1), q.device)
        _check(L.colbandit_attention_window_backward(a, w, out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                                     dv.data_ptr(), _ptr(dbias), _ptr(ws), nb, _stream()),
               "colbandit_attention_window_backward")
        return {"dq": dq, "dk": dk, "dv": dv, "dbias": dbias}
    ws, nb = _workspace(workspace, L.colbandit_attention_workspace_bytes(a, 1), q.device)
    _check(L.colbandit_attention_backward(a, out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                          dv.data_ptr(), _ptr(dbias), _ptr(ws), nb, _stream()),
           "colbandit_attention_backward")
    return {"dq": dq, "dk": dk, "dv": dv, "dbias": dbias}


def _rows_of(t, what):
    """Type, shape and distance of the rows of a matrix whose rows may lie apart."""
    dt, shape = _DTYPES.get(t.dtype), t.shape
    if dt is None:
        raise TypeError(f"{what} must be float32 or bfloat16")
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{what} is [rows, width]")
    row, last = t.stride()
    if shape[0] <= 1:
        row = shape[1]
    if (last != 1 and shape[1] > 1) or row < shape[1]:
        raise ValueError(f"{what} has consecutive values, in rows that do not overlap")
    return dt, shape[0], shape[1], row


def _tokens(tokens):
    if tokens.dtype != torch.int64 or tokens.dim() != 1 or not tokens.is_contiguous():
        raise ValueError("tokens must be a contiguous int64 vector")
    return tokens.shape[0]


def _type_of_rows(dtype):
    dt = _DTYPES.get(dtype)
    if dt is None:
        raise TypeError("rows must be float32 or bfloat16")
    return dt


def colbandit_embedding(table, tokens, *, scale=1.0, dtype=None, out=None):
    """Rows of `table` [vocab, width] for `tokens` int64 [n], times scale; zeros for tokens outside of the table (padding).  `dtype`: of
    the rows, where it is not the table's; `out`: a tensor to write.  Returns dict(out [n, width])."""
    dt, vocab, width, row = _rows_of(table, "table")
    n = _tokens(tokens)
    if dtype is None:
        dtype = table.dtype
    to = _type_of_rows(dtype)
    out = _new(table, dtype, n, width) if out is None else _dense(out, (n, width), dtype, "out")
    dev = _on_device(table, tokens, out)
    _check(lib().colbandit_embedding(table.data_ptr(), dt, row, tokens.data_ptr(), n, vocab, width, scale, out.data_ptr(), to,
                                     _stream(dev)), "colbandit_embedding")
    return {"out": out}


def colbandit_embedding_backward(dout, tokens, vocab, *, scale=1.0, dtype=None, out=None, workspace=None):
    """Gradient of a table of `vocab` rows from that of the rows that were looked up, in the order of the tokens.  `dtype`: of the
    table; `out`: a tensor to write.  Returns dict(dtable [vocab, width])."""
    dt, n, width, row = _rows_of(dout, "dout")
    if _tokens(tokens) != n:
        raise ValueError("dout has a row for each token")
    if dtype is None:
        dtype = dout.dtype
    to = _type_of_rows(dtype)
    L = lib()
    out = _new(dout, dtype, vocab, width) if out is None else _dense(out, (vocab, width), dtype, "dtable")
    dev = _on_device(dout, tokens, out)
    ws, nb = _workspace(workspace, L.colbandit_embedding_workspace_bytes(n, vocab, width), dout.device)
    _check(L.colbandit_embedding_backward(dout.data_ptr(), dt, row, tokens.data_ptr(), n, vocab, width, scale, out.data_ptr(), to,
                                          _ptr(ws), nb, _stream(dev)), "colbandit_embedding_backward")
    return {"dtable": out}


def colbandit_rotary_table(n_positions, d, base=10000.0, device=None) -> torch.Tensor:
    """Cosine and sine of position * base^(-2i/d), float32 [n_positions, d/2, 2] (computed by the library on the host, in 64
    bits), on the current device or `device`."""
    table = torch.empty((n_positions, d // 2, 2), dtype=torch.float32)
    _check(lib().colbandit_rotary_table(n_positions, d, base, table.data_ptr()), "colbandit_rotary_table")
    return table.to(torch.device("cuda", torch.cuda.current_device()) if device is None else device)


def _rotation(q, k, positions, table, q_weight, k_weight, eps, interleaved, *more):
    """The library's arguments, and the current device (`more`: tensors that must live there too)."""
    dt, q_shape, k_shape = _DTYPES.get(q.dtype), q.shape, k.shape
    if dt is None or k.dtype != q.dtype:
        raise TypeError("q and k must be float32 or bfloat16, both of one type")
    if len(q_shape) != 3 or len(k_shape) != 3 or q_shape[0] != k_shape[0] or q_shape[2] != k_shape[2]:
        raise ValueError("q is [rows, heads, d], k [rows, kv_heads, d]")
    (q_row, q_head, q_last), (k_row, k_head, k_last) = q.stride(), k.stride()
    if q_last != 1 or k_last != 1:
        raise ValueError("the values of a row and head must be consecutive")
    rows, heads, d = q_shape
    n_positions = at = turns = wq = wk = None
    if q_weight is not None:
        wq = _dense(q_weight, (d,), torch.float32, "a weight").data_ptr()
    if k_weight is not None:
        wk = _dense(k_weight, (d,), torch.float32, "a weight").data_ptr()
    if table is not None:
        if positions is None:
            raise ValueError("a rotation needs positions")
        n_positions = table.shape[0]
        turns = _dense(table, (n_positions, d // 2, 2), torch.float32, "the table").data_ptr()
        at = _dense(positions, (rows,), torch.int64, "positions").data_ptr()
    dev = _on_device(q, k, None if table is None else positions, table, q_weight, k_weight, *more)
    return ColbanditRotation(dt, heads, k_shape[1], d, 1 if interleaved else 0, eps, rows, n_positions or 0, q.data_ptr(), k.data_ptr(),
                             q_row, q_head, k_row, k_head, wq, wk, turns, at), dev


def colbandit_norm_rotate(q, k, *, positions=None, table=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, out=None):
    """q [rows, heads, d] and k [rows, kv_heads, d] (any row and head strides), each head divided by its root mean square, times
    the weights float32 [d], and rotated by `table` (colbandit_rotary_table) at `positions` int64 [rows]; rows whose position is none
    of the table's get zeros.  `table` None: no rotation.  `out`: tensors to write, as this returns them (q and k themselves, where
    they are dense).  Returns dict(q, k), dense."""
    q_out, k_out = (_like(q), _like(k)) if out is None else (
        _dense(out["q"], q.shape, q.dtype, "q"), _dense(out["k"], k.shape, k.dtype, "k"))
    r, dev = _rotation(q, k, positions, table, q_weight, k_weight, eps, interleaved, q_out, k_out)
    _check(lib().colbandit_norm_rotate(r, q_out.data_ptr(), k_out.data_ptr(), _stream(dev)), "colbandit_norm_rotate")
    return {"q": q_out, "k": k_out}


def colbandit_norm_rotate_backward(dq_out, dk_out, q, k, *, positions=None, table=None, q_weight=None, k_weight=None, eps=1e-6,
                                   interleaved=False, workspace=None):
    """Gradients of colbandit_norm_rotate's inputs from those of its outputs.  Returns dict(dq, dk, dq_weight, dk_weight), the last two
    also where there are no weights."""
    _dense(dq_out, q.shape, q.dtype, "dq_out")
    _dense(dk_out, k.shape, k.dtype, "dk_out")
    r, dev = _rotation(q, k, positions, table, q_weight, k_weight, eps, interleaved, dq_out, dk_out)
    L = lib()
    dq, dk = _like(q), _like(k)
    dq_weight, dk_weight = _new(q, torch.float32, r.d), _new(q, torch.float32, r.d)
    ws, nb = _workspace(workspace, L.colbandit_norm_rotate_workspace_bytes(r), q.device)
    _check(L.colbandit_norm_rotate_backward(r, dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), dq_weight.data_ptr(),
                                            dk_weight.data_ptr(), _ptr(ws), nb, _stream(dev)), "colbandit_norm_rotate_backward")
    return {"dq": dq, "dk": dk, "dq_weight": dq_weight, "dk_weight": dk_weight}


def _maxsim(Q, docs, offsets):
    if Q.dtype not in _DTYPES or docs.dtype != Q.dtype:
        raise TypeError("Q and docs must be float32 or bfloat16, both of one type")
    if Q.dim() != 3 or docs.dim() != 2 or docs.shape[1] != Q.shape[2] or not Q.is_contiguous() or not docs.is_contiguous():
        raise ValueError("Q is a contiguous [n_queries, T, d], docs a contiguous [total_tokens, d]")
    _offsets(offsets)
    _on_device(Q, docs, offsets)
    return Q.shape[0], Q.shape[1], Q.shape[2], offsets.shape[0] - 1, docs.shape[0]


def colbandit_maxsim_scores(Q, docs, offsets):
    """MaxSim of all (query, document) pairs.  Returns dict(scores float32 [n_queries, N], argmax int32
    [n_queries, N, T])."""
    nq, T, d, N, total = _maxsim(Q, docs, offsets)
    scores = Q.new_empty((nq, N), dtype=torch.float32)
    argmax = Q.new_empty((nq, N, T), dtype=torch.int32)
    _check(lib().colbandit_maxsim_scores(Q.data_ptr(), nq, T, d, _DTYPES[Q.dtype], docs.data_ptr(), offsets.data_ptr(), N,
                                         total, scores.data_ptr(), argmax.data_ptr(), _stream()), "colbandit_maxsim_scores")
    return {"scores": scores, "argmax": argmax}


def colbandit_contrastive_loss(scores, targets, temperature=1.0):
    """Cross-entropy of each query's scores over all documents.  Returns dict(loss [n_queries], dscores
    [n_queries, N]: the gradient of the mean loss)."""
    nq, N = scores.shape
    _dense(scores, (nq, N), torch.float32, "scores")
    _dense(targets, (nq,), torch.int64, "targets")
    _on_device(scores, targets)
    loss = scores.new_empty(nq)
    dscores = torch.empty_like(scores)
    _check(lib().colbandit_contrastive_loss(scores.data_ptr(), nq, N, targets.data_ptr(), temperature, loss.data_ptr(),
                                            dscores.data_ptr(), _stream()), "colbandit_contrastive_loss")
    return {"loss": loss, "dscores": dscores}


def colbandit_maxsim_backward(dscores, argmax, Q, docs, offsets):
    """Gradients of the embeddings from those of the scores.  Returns dict(dQ, ddocs)."""
    nq, T, d, N, total = _maxsim(Q, docs, offsets)
    _dense(dscores, (nq, N), torch.float32, "dscores")
    _dense(argmax, (nq, N, T), torch.int32, "argmax")
    _on_device(dscores, argmax)
    dQ, ddocs = torch.empty_like(Q), torch.empty_like(docs)
    _check(lib().colbandit_maxsim_backward(dscores.data_ptr(), argmax.data_ptr(), Q.data_ptr(), nq, T, d, _DTYPES[Q.dtype],
                                           docs.data_ptr(), offsets.data_ptr(), N, total, dQ.data_ptr(), ddocs.data_ptr(),
                                           _stream()), "colbandit_maxsim_backward")
    return {"dQ": dQ, "ddocs": ddocs}


def colbandit_clip_gradients(grads, max_norm, out=None, workspace=None):
    """Global norm of `grads` (a list of contiguous float32 or bfloat16 tensors) and the tensors scaled by
    min(1, max_norm / (norm + 1e-6)): into `out` (a list alike), or in place.  Returns dict(norm float32
    scalar tensor, grads)."""
    grads = list(grads)
    to = grads if out is None else list(out)
    if not grads or len(to) != len(grads):
        raise ValueError("grads must be a list of tensors, and out one of as many")
    for g, o in zip(grads, to):
        if g.dtype not in _DTYPES or o.dtype != g.dtype:
            raise TypeError("gradients must be float32 or bfloat16, and outputs of their types")
        if not g.is_contiguous() or not o.is_contiguous() or o.shape != g.shape:
            raise ValueError("gradients and outputs must be contiguous, and outputs of their shapes")
    _on_device(*grads, *to)
    n = len(grads)
    pointers = ctypes.c_void_p * n
    sizes = (ctypes.c_int64 * n)(*[g.numel() for g in grads])
    L = lib()
    norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
    ws, nb = _workspace(workspace, L.colbandit_clip_workspace_bytes(n, sizes), norm.device)
    _check(L.colbandit_clip_gradients(n, pointers(*[g.data_ptr() for g in grads]), pointers(*[o.data_ptr() for o in to]),
                                      sizes, (ctypes.c_int32 * n)(*[_DTYPES[g.dtype] for g in grads]), max_norm,
                                      norm.data_ptr(), _ptr(ws), nb, _stream()), "colbandit_clip_gradients")
    return {"norm": norm, "grads": to}


POLYNOMIAL = (3.4445, -4.7750, 2.0315)               # takes singular values of any size to between 0.7 and 1.2 in five steps


def colbandit_orthogonalise(matrices, *, steps=5, coefficients=POLYNOMIAL, out=None, workspace=None):
    """Each of `matrices` (a list of contiguous 2-d float32 or bfloat16 tensors) with its singular values brought near to one by
    `steps` of s <- a s + b s^3 + c s^5, after a division by its Frobenius norm.  Into `out` (a list alike; it may be `matrices`), or
    new tensors.  Returns dict(out)."""
    to, call = _orthogonalise(matrices, steps, coefficients, out, workspace)
    _check(call(), "colbandit_orthogonalise")
    return {"out": to}


def _orthogonalise(matrices, steps, coefficients, out, workspace=None):
    """Outputs, and the library's call: without room for its work, which it asks for last, it checks all else and does nothing."""
    matrices = list(matrices)
    to = [torch.empty_like(m) for m in matrices] if out is None else list(out)
    if not matrices or len(to) != len(matrices):
        raise ValueError("matrices must be a list of tensors, and out one of as many")
    for m, o in zip(matrices, to):
        if m.dtype not in _DTYPES or o.dtype != m.dtype:
            raise TypeError("matrices must be float32 or bfloat16, and outputs of their types")
        if m.dim() != 2 or not m.is_contiguous() or not o.is_contiguous() or o.shape != m.shape:
            raise ValueError("matrices and outputs must be contiguous and two-dimensional, and outputs of their shapes")
    _on_device(*matrices, *to)
    n = len(matrices)
    pointers, sizes = ctypes.c_void_p * n, ctypes.c_int64 * n
    rows, cols = sizes(*[m.shape[0] for m in matrices]), sizes(*[m.shape[1] for m in matrices])
    L = lib()
    ws, nb = _workspace(workspace, L.colbandit_orthogonalise_workspace_bytes(n, rows, cols), matrices[0].device)
    args = (n, pointers(*[m.data_ptr() for m in matrices]), pointers(*[o.data_ptr() for o in to]), rows, cols,
            (ctypes.c_int32 * n)(*[_DTYPES[m.dtype] for m in matrices]), _within(steps, 30), (ctypes.c_float * 3)(*coefficients))
    return to, lambda room=True: L.colbandit_orthogonalise(*args, _ptr(ws), nb if room else 0, _stream())      # (and it holds ws)


# ---- as parts of a torch program ---------------------------------------------------------------------


class _FirstOrderOnly(torch.autograd.Function):
    """Gradients as they are; whatever is differentiated through them is an error and not left out."""
    @staticmethod
    def forward(ctx, n, *tensors):
        return tensors[:n]

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("second-order gradients of the training operators are not available")


def _first_order(grads, *inputs):
    """`grads` of a backward pass; where they are themselves to be differentiated (create_graph), tied to its inputs."""
    if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in inputs):
        return grads
    there = [g for g in grads if g is not None]
    tied = iter(_FirstOrderOnly.apply(len(there), *there, *(t for t in inputs if t is not None)))
    return tuple(None if g is None else next(tied) for g in grads)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, bias, q_offsets, k_offsets, keep, how):
        r = colbandit_attention(q, k, v, q_offsets, k_offsets, keep=keep, bias=bias, **how)
        ctx.save_for_backward(q, k, v, bias, q_offsets, k_offsets, keep, r["out"], r["lse"])
        ctx.how = how
        return r["out"]

    @staticmethod
    def backward(ctx, dout):
        q, k, v, bias, q_offsets, k_offsets, keep, out, lse = ctx.saved_tensors
        g = colbandit_attention_backward(dout.contiguous(), q, k, v, out, lse, q_offsets, k_offsets, keep=keep, bias=bias,
                                         **ctx.how)
        return *_first_order((g["dq"], g["dk"], g["dv"], g["dbias"]), q, k, v, bias, dout), None, None, None, None


def attention(q, k, v, q_offsets, k_offsets=None, *, causal=False, scale=None, keep=None, bias=None, max_distance=128, window=None,
              sinks=0):
    """colbandit_attention's output, differentiable in q, k, v and bias (once: second-order gradients are an error)."""
    how = dict(causal=causal, scale=scale, max_distance=max_distance)
    if window is not None or sinks:
        how.update(window=window, sinks=sinks)
    return _Attention.apply(q, k, v, bias, q_offsets, k_offsets, keep, how)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale, dtype):
        ctx.save_for_backward(tokens)
        ctx.how = (table.shape[0], scale, table.dtype)
        return colbandit_embedding(table, tokens, scale=scale, dtype=dtype)["out"]

    @staticmethod
    def backward(ctx, dout):
        tokens, = ctx.saved_tensors
        vocab, scale, dtype = ctx.how
        if dout.dim() != 2 or dout.stride(1) != 1 or dout.stride(0) < dout.shape[1]:
            dout = dout.contiguous()
        g = colbandit_embedding_backward(dout, tokens, vocab, scale=scale, dtype=dtype)["dtable"]
        return *_first_order((g,), dout), None, None, None


def embedding(table, tokens, *, scale=1.0, dtype=None):
    """colbandit_embedding's rows, differentiable in the table (once: second-order gradients are an error).  `tokens` of any shape:
    the rows have it, and the width as one more dimension."""
    out = _Embedding.apply(table, tokens.reshape(-1).contiguous(), float(scale), dtype)
    return out if tokens.dim() == 1 else out.view(*tokens.shape, table.shape[1])


class _NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, table, how):
        r = colbandit_norm_rotate(q, k, positions=positions, table=table, q_weight=q_weight, k_weight=k_weight, **how)
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, table)
        ctx.how = how
        return r["q"], r["k"]

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, q_weight, k_weight, positions, table = ctx.saved_tensors
        g = colbandit_norm_rotate_backward(dq.contiguous(), dk.contiguous(), q, k, positions=positions, table=table, q_weight=q_weight,
                                           k_weight=k_weight, **ctx.how)
        return *_first_order((g["dq"], g["dk"], None if q_weight is None else g["dq_weight"],
                              None if k_weight is None else g["dk_weight"]), q, k, q_weight, k_weight, dq, dk), None, None, None


def norm_rotate(q, k, *, positions=None, table=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """colbandit_norm_rotate's (q, k), differentiable in q, k and the weights (once: second-order gradients are an error)."""
    return _NormRotate.apply(q, k, q_weight, k_weight, positions, table, dict(eps=eps, interleaved=interleaved))


class _ContrastiveMaxSim(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, docs, offsets, targets, temperature):
        f = colbandit_maxsim_scores(Q, docs, offsets)
        l = colbandit_contrastive_loss(f["scores"], targets, temperature)
        ctx.save_for_backward(l["dscores"], f["argmax"], Q, docs, offsets)
        taking_part = ((targets >= 0) & (targets < f["scores"].shape[1])).sum().clamp(min=1)
        return l["loss"].sum() / taking_part

    @staticmethod
    def backward(ctx, dloss):
        dscores, argmax, Q, docs, offsets = ctx.saved_tensors
        g = colbandit_maxsim_backward(dscores * dloss, argmax, Q, docs, offsets)
        return *_first_order((g["dQ"], g["ddocs"]), Q, docs, dloss), None, None, None


def contrastive_maxsim(Q, docs, offsets, targets, temperature=1.0):
    """Mean contrastive loss of queries Q [n_queries, T, d] against packed documents, differentiable in
    Q and docs (once: second-order gradients are an error); targets int64 [n_queries], -1 leaves a query out."""
    return _ContrastiveMaxSim.apply(Q, docs, offsets, targets, float(temperature))


def clip_gradients_(parameters, max_norm):
    """Clips the parameters' gradients in place to a global norm of max_norm; returns the norm before (0 where no parameter
    has a gradient)."""
    parameters = list(dict.fromkeys(parameters))     # one that is listed twice has one gradient
    grads = [p.grad for p in parameters if p.grad is not None]
    if not grads:
        return torch.zeros((), device=parameters[0].device if parameters else None)
    return colbandit_clip_gradients(grads, float(max_norm))["norm"]


def orthogonal_step_(parameters, momenta, rate, momentum=0.95, steps=5, coefficients=POLYNOMIAL):
    """One step of descent along orthogonalised momenta, for 2-d parameters: of each that has a gradient the momentum becomes
    momentum * itself + gradient, and the parameter goes down `rate` times sqrt(max(1, rows / columns)) times
    colbandit_orthogonalise of gradient + momentum * itself.  `momenta`: a dict of the parameters' momenta, which this fills; they are
    float32 whatever the parameters' type.  A step that is refused changes nothing."""
    parameters = [p for p in dict.fromkeys(parameters) if p.grad is not None and p.numel()]
    if not parameters:
        return
    rate, momentum = float(rate), float(momentum)
    for p in parameters:
        if p.dim() != 2 or p.dtype not in _DTYPES:
            raise ValueError("parameters must be two-dimensional, and float32 or bfloat16")
        if p.grad.layout != torch.strided:
            raise ValueError("gradients must be dense")
        m = momenta.get(p)
        if m is not None and (m.shape != p.shape or m.layout != torch.strided or not m.is_floating_point()):
            raise ValueError("momenta must be dense, of floating point and their parameters' shapes")
    there = [m for m in map(momenta.get, parameters) if m is not None]
    _on_device(*parameters, *there)
    with torch.no_grad():
        # all memory is there, and the library has nothing against the call, before any momentum is changed
        updates = [torch.empty(p.shape, dtype=torch.float32, device=p.device) for p in parameters]
        new = {p: torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format) for p in parameters
               if momenta.get(p) is None}
        _, call = _orthogonalise(updates, steps, coefficients, updates)
        rc = call(room=False)
        if rc != _ERR_WORKSPACE:
            raise ColbanditError(rc, "colbandit_orthogonalise")
        momenta.update(new)
        for p, u in zip(parameters, updates):
            m = momenta[p]
            m.mul_(momentum).add_(p.grad)
            torch.add(p.grad, m, alpha=momentum, out=u)
        _check(call(), "colbandit_orthogonalise")
        for p, u in zip(parameters, updates):
            p.sub_(u, alpha=rate * math.sqrt(max(1.0, p.shape[0] / p.shape[1])))
