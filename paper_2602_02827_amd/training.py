"""ctypes binding of the training operators (include/colbandit_train.h), and their autograd forms.

The `colbandit_*` functions marshal arguments only, as those of `binding` do: torch supplies device
memory and the current stream, every step runs in the library's HIP kernels, and there is no
fallback.  Tensors must live on the current device.  `attention`, `contrastive_maxsim` and
`clip_gradients_` are the same operators as parts of a torch program.
"""
from __future__ import annotations

import ctypes
import math

import numpy as np
import torch

from . import binding
from .binding import BF16, F32, ColbanditError

EXPORTS = [
    "colbandit_sizeof_attn", "colbandit_bias_buckets", "colbandit_attention_workspace_bytes", "colbandit_attention",
    "colbandit_attention_backward", "colbandit_maxsim_scores", "colbandit_contrastive_loss", "colbandit_maxsim_backward",
    "colbandit_clip_workspace_bytes", "colbandit_clip_gradients",
]

_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}


class ColbanditAttn(ctypes.Structure):
    _fields_ = [("dt", ctypes.c_int), ("n_seqs", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("d", ctypes.c_int), ("causal", ctypes.c_int), ("n_buckets", ctypes.c_int), ("max_distance", ctypes.c_int),
                ("scale", ctypes.c_float), ("total_q", ctypes.c_int64), ("total_k", ctypes.c_int64),
                ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_row", ctypes.c_int64), ("q_head", ctypes.c_int64), ("k_row", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("v_row", ctypes.c_int64), ("v_head", ctypes.c_int64),
                ("keep", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


_lib = None


def lib():
    """The library that `binding` loads, with the training calls' signatures."""
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, i, i64, sz, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        attn = ctypes.POINTER(ColbanditAttn)
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
                ("colbandit_clip_gradients", i, [i64, vp, vp, vp, vp, f, vp, vp, sz, vp])]:
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        if L.colbandit_sizeof_attn() != ctypes.sizeof(ColbanditAttn):
            raise ImportError("libcolbandit.so was built from a different colbandit_train.h: rebuild it")
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    # the handle alone: making a Stream object of it costs as much as a small call's kernels (2.8 us)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(rc, what):
    if rc:
        raise ColbanditError(rc, what)


def _on_device(*tensors):
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors must live on the current device")


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
    if q.dtype not in _DTYPES or k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k and v must be float32 or bfloat16, all of one type")
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or q.shape[2] != k.shape[2]:
        raise ValueError("q is [total_q, heads, d], k and v are [total_k, kv_heads, d]")
    for t in (q, k, v):
        if t.stride(2) != 1:
            raise ValueError("the values of a row and head must be consecutive")
    if _offsets(q_offsets).shape != _offsets(k_offsets).shape:
        raise ValueError("q_offsets and k_offsets must hold equally many sequences")
    if keep is not None:
        if keep.dtype not in (torch.bool, torch.uint8) or keep.shape != k.shape[:1] or not keep.is_contiguous():
            raise ValueError("keep is a contiguous bool or uint8 vector over the key rows")
    if bias is not None:
        if bias.dtype != q.dtype:
            raise TypeError("bias must have the type of q")
        if bias.dim() != 2 or bias.shape[1] != q.shape[1] or not bias.is_contiguous():
            raise ValueError("bias is a contiguous [n_buckets, heads]")
    _on_device(q, k, v, q_offsets, k_offsets, keep, bias)
    return ColbanditAttn(
        _DTYPES[q.dtype], q_offsets.shape[0] - 1, q.shape[1], k.shape[1], q.shape[2], 1 if causal else 0,
        0 if bias is None else bias.shape[0], int(max_distance),
        1.0 / math.sqrt(q.shape[2]) if scale is None else scale, q.shape[0], k.shape[0],
        q_offsets.data_ptr(), k_offsets.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(),
        q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1), _ptr(keep), _ptr(bias))


def _dense(t, shape, dtype, what):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


def colbandit_attention(q, k, v, q_offsets, k_offsets=None, *, causal=False, scale=None, keep=None, bias=None,
                        max_distance=128, workspace=None, out=None):
    """Attention over packed sequences.  q [total_q, heads, d], k and v [total_k, kv_heads, d] (any
    row and head strides), offsets int64 [n+1]; `k_offsets` None: the queries' own; rows behind the last
    sequence get zeros.  `out`: tensors to write, as this returns them.  Returns dict(out [total_q, heads, d], lse float32
    [heads, total_q])."""
    a = _attn(q, k, v, q_offsets, k_offsets, causal, scale, keep, bias, max_distance)
    L = lib()
    o, lse = (out["out"], out["lse"]) if out else (None, None)
    o = q.new_empty(q.shape) if o is None else _dense(o, q.shape, q.dtype, "out")
    lse = q.new_empty((q.shape[1], q.shape[0]), dtype=torch.float32) if lse is None else \
        _dense(lse, (q.shape[1], q.shape[0]), torch.float32, "lse")
    _on_device(o, lse)
    ws, nb = _workspace(workspace, L.colbandit_attention_workspace_bytes(a, 0), q.device)
    _check(L.colbandit_attention(a, o.data_ptr(), lse.data_ptr(), _ptr(ws), nb, _stream()), "colbandit_attention")
    return {"out": o, "lse": lse}


def colbandit_attention_backward(dout, q, k, v, out, lse, q_offsets, k_offsets=None, *, causal=False, scale=None,
                                 keep=None, bias=None, max_distance=128, workspace=None):
    """Gradients of colbandit_attention's inputs from that of its output.  Returns dict(dq, dk, dv,
    dbias), dense, `dbias` None without a bias."""
    a = _attn(q, k, v, q_offsets, k_offsets, causal, scale, keep, bias, max_distance)
    L = lib()
    _dense(out, q.shape, q.dtype, "out")
    _dense(lse, (q.shape[1], q.shape[0]), torch.float32, "lse")
    _dense(dout, q.shape, q.dtype, "dout")
    _on_device(out, lse, dout)
    dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), k.new_empty(k.shape)
    dbias = None if bias is None else torch.empty_like(bias)
    ws, nb = _workspace(workspace, L.colbandit_attention_workspace_bytes(a, 1), q.device)
    _check(L.colbandit_attention_backward(a, out.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                          dv.data_ptr(), _ptr(dbias), _ptr(ws), nb, _stream()),
           "colbandit_attention_backward")
    return {"dq": dq, "dk": dk, "dv": dv, "dbias": dbias}


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


def attention(q, k, v, q_offsets, k_offsets=None, *, causal=False, scale=None, keep=None, bias=None, max_distance=128):
    """colbandit_attention's output, differentiable in q, k, v and bias (once: second-order gradients are an error)."""
    return _Attention.apply(q, k, v, bias, q_offsets, k_offsets, keep,
                            dict(causal=causal, scale=scale, max_distance=max_distance))


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
