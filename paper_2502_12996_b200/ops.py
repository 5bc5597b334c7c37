"""The decoder operators of the inner step on torch tensors: scaled embedding lookup, layer norm
(QKNorm included), causal attention over packed sequences and the distillation loss.

Functions named ``*_forward`` / ``*_backward`` are the library's calls: they check shapes, types and
strides (ValueError / TypeError), allocate outputs and workspaces from torch's allocator, and launch on
``stream`` (default: the current one).  Parameters are views into the replicas' flat vectors, [M, ...]
with any distance between replicas, and parameter gradients are written into views of the flat gradients
that ``State.inner_adamw`` takes, so nothing is copied between the two sides.  ``embedding``,
``layer_norm``, ``attention`` and ``distill`` are the same as torch.autograd functions, for programs that
leave the order of the backward pass to autograd.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
from contextlib import nullcontext
from typing import Optional, Tuple

import torch

from . import binding
from .binding import _check, _ptr

_DTYPES = {torch.float32: binding.DTYPE_F32, torch.bfloat16: binding.DTYPE_BF16}
_IDS = {torch.int32: 0, torch.int64: 1}


def _dtype(t: torch.Tensor, name: str) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"{name}: float32 or bfloat16 wanted, got {t.dtype}") from None


def _same_device(*named) -> None:
    dev = None
    for name, t in named:
        if t is None:
            continue
        if t.device.type != "cuda":
            raise ValueError(f"{name}: a CUDA tensor is wanted, got one on {t.device}")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"{name}: on {t.device}, the others on {dev}")


def _want(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


class _On:
    """The device and stream of one call: allocations inside belong to the stream that the kernels run on."""

    def __init__(self, t: torch.Tensor, stream):
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=t.device)
        index = t.device.index
        self.ctx = (torch.cuda.stream(stream) if stream is not None
                    else nullcontext() if index is None or index == torch.cuda.current_device() else torch.cuda.device(t.device))

    def __enter__(self) -> int:
        self.ctx.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        return self.ctx.__exit__(*exc)


def _workspace(nbytes: int, where: str, device) -> Tuple[torch.Tensor, int]:
    if nbytes < 0:
        raise binding.DilocoError(int(nbytes), where)
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device), int(nbytes)


def _replica_rows(t: torch.Tensor, name: str, shape) -> int:
    """A parameter or its gradient, [M, ...] with each replica's part contiguous: the distance between replicas."""
    _want(tuple(t.shape) == tuple(shape), f"{name}: shape {tuple(shape)} wanted, got {tuple(t.shape)}")
    _want(t.numel() == 0 or t[0].is_contiguous(), f"{name}: each replica's part has to be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.numel()


# ------------------------------------------------------------------------------------ embedding
def _embedding_desc(ids, d, vocab, table_stride, grad_stride, rows, scale, table_dtype, grad_dtype) -> binding.Embedding:
    M, tokens = ids.shape
    _want(rows.shape == (M, tokens, d), f"rows: shape {(M, tokens, d)} wanted, got {tuple(rows.shape)}")
    row = rows.stride(1) if tokens > 1 else rows.stride(0) if M > 1 else d
    _want(d == 1 or rows.stride(2) == 1, "rows: the last axis has to be contiguous")
    _want(M == 1 or tokens == 0 or rows.stride(0) == tokens * row, "rows: replicas have to follow one another at the tokens' stride")
    return binding.Embedding(M, d, tokens, vocab, table_stride, grad_stride, max(row, d), scale, _IDS[ids.dtype], table_dtype,
                             _dtype(rows, "rows"), grad_dtype)


def _check_ids(ids: torch.Tensor) -> torch.Tensor:
    if ids.dtype not in _IDS:
        raise TypeError(f"ids: int32 or int64 wanted, got {ids.dtype}")
    _want(ids.dim() == 2, f"ids: [M, tokens] wanted, got shape {tuple(ids.shape)}")
    return ids.contiguous()


def embedding_forward(ids: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """diloco_embedding_forward: ids [M, tokens], table [M, vocab, d] -> [M, tokens, d]."""
    ids = _check_ids(ids)
    _want(table.dim() == 3 and table.shape[0] == ids.shape[0], f"table: [M, vocab, d] with M = {ids.shape[0]} wanted, got {tuple(table.shape)}")
    _same_device(("ids", ids), ("table", table), ("out", out))
    M, V, d = table.shape
    stride = _replica_rows(table, "table", (M, V, d))
    with _On(table, stream) as s:
        if out is None:
            out = torch.empty((M, ids.shape[1], d), dtype=out_dtype or table.dtype, device=table.device)
        e = _embedding_desc(ids, d, V, stride, 0, out, scale, _dtype(table, "table"), 0)
        _check(binding.load_library().diloco_embedding_forward(ctypes.byref(e), _ptr(ids), _ptr(table), _ptr(out), s), "diloco_embedding_forward")
    return out


def embedding_backward(ids: torch.Tensor, dout: torch.Tensor, dtable: torch.Tensor, *, scale: float = 1.0, accumulate: bool = False,
                       stream=None) -> torch.Tensor:
    """diloco_embedding_backward: dout [M, tokens, d] summed by token into dtable [M, vocab, d], which is returned.
    accumulate: dtable keeps what it holds (a table that is also the output projection) and only rows of present ids change."""
    ids = _check_ids(ids)
    _want(dtable.dim() == 3 and dtable.shape[0] == ids.shape[0], f"dtable: [M, vocab, d] with M = {ids.shape[0]} wanted, got {tuple(dtable.shape)}")
    _same_device(("ids", ids), ("dout", dout), ("dtable", dtable))
    M, V, d = dtable.shape
    stride = _replica_rows(dtable, "dtable", (M, V, d))
    lib = binding.load_library()
    with _On(dtable, stream) as s:
        e = _embedding_desc(ids, d, V, V * d, stride, dout, scale, 0, _dtype(dtable, "dtable"))
        ws, n = _workspace(lib.diloco_embedding_workspace_bytes(ctypes.byref(e)), "diloco_embedding_workspace_bytes", dtable.device)
        _check(lib.diloco_embedding_backward(ctypes.byref(e), _ptr(ids), _ptr(dout), _ptr(dtable), int(accumulate), _ptr(ws), n, s),
               "diloco_embedding_backward")
    return dtable


# ----------------------------------------------------------------------------------- layer norm
def _norm_rows(t: torch.Tensor, name: str, shape) -> Tuple[int, int]:
    """[M, rows, groups, d] (or [M, rows, d]) with one row stride over all replicas: (row stride, group stride)."""
    _want(tuple(t.shape) == tuple(shape), f"{name}: shape {tuple(shape)} wanted, got {tuple(t.shape)}")
    M, N = shape[:2]
    _want(shape[-1] == 1 or t.stride(-1) == 1, f"{name}: the last axis has to be contiguous")
    row = t.stride(1) if N > 1 else t.stride(0) if M > 1 else 0
    _want(M == 1 or N <= 1 or t.stride(0) == N * row, f"{name}: replicas have to follow one another at the rows' stride")
    return row, t.stride(2) if t.dim() == 4 and t.shape[2] > 1 else 0


def _norm_desc(x, weight, eps) -> binding.LayerNorm:
    _want(x.dim() in (3, 4), f"x: [M, rows, d] or [M, rows, groups, d] wanted, got shape {tuple(x.shape)}")
    M, N, d = x.shape[0], x.shape[1], x.shape[-1]
    n = binding.LayerNorm(M=M, d=d, groups=x.shape[2] if x.dim() == 4 else 1, rows=N, eps=eps, act_dtype=_dtype(x, "x"),
                          param_dtype=_dtype(weight, "weight"))
    n.x_row_stride, n.x_group_stride = _norm_rows(x, "x", x.shape)
    n.param_stride = _replica_rows(weight, "weight", (M, d))
    return n


def layer_norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, eps: float = 1e-5,
                       out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """diloco_layernorm_forward: x [M, rows, d] or [M, rows, groups, d], weight and bias [M, d] -> (y, mean, rstd).
    out may be x."""
    _same_device(("x", x), ("weight", weight), ("bias", bias), ("out", out))
    n = _norm_desc(x, weight, eps)
    if bias is not None:
        _want(bias.dtype == weight.dtype, "bias: the weight's type wanted")
        _want(_replica_rows(bias, "bias", weight.shape) == n.param_stride, "bias: the weight's stride between replicas wanted")
    with _On(x, stream) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _want(out.dtype == x.dtype, "out: the type of x wanted")
        n.y_row_stride, n.y_group_stride = _norm_rows(out, "out", x.shape)
        stats = torch.empty((2,) + tuple(x.shape[:-1]), dtype=torch.float32, device=x.device)
        mean, rstd = stats[0], stats[1]
        _check(binding.load_library().diloco_layernorm_forward(ctypes.byref(n), _ptr(x), _ptr(weight), _ptr(bias), _ptr(out), _ptr(mean),
                                                               _ptr(rstd), s), "diloco_layernorm_forward")
    return out, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, *, accumulate: bool = False,
                        dx: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """diloco_layernorm_backward: returns dx and writes dweight and dbias ([M, d], where given; accumulate: adds to them).
    dx may be dy."""
    _same_device(("dy", dy), ("x", x), ("weight", weight), ("mean", mean), ("rstd", rstd), ("dweight", dweight), ("dbias", dbias), ("dx", dx))
    n = _norm_desc(x, weight, 0.0)
    _want(dy.dtype == x.dtype, "dy: the type of x wanted")
    n.y_row_stride, n.y_group_stride = _norm_rows(dy, "dy", x.shape)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _want(t.dtype == torch.float32 and t.shape == x.shape[:-1] and t.is_contiguous(), f"{name}: contiguous float32 {tuple(x.shape[:-1])} wanted")
    grads = [(name, t) for name, t in (("dweight", dweight), ("dbias", dbias)) if t is not None]
    if grads:
        n.grad_dtype = _dtype(grads[0][1], grads[0][0])
        n.grad_stride = _replica_rows(grads[0][1], grads[0][0], weight.shape)
        for name, t in grads[1:]:
            _want(t.dtype == grads[0][1].dtype and _replica_rows(t, name, weight.shape) == n.grad_stride, "dbias: the type and stride of dweight wanted")
    lib = binding.load_library()
    with _On(x, stream) as s:
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _want(dx.dtype == x.dtype, "dx: the type of x wanted")
        n.dx_row_stride, n.dx_group_stride = _norm_rows(dx, "dx", x.shape)
        ws, nbytes = None, 0
        if grads:
            ws, nbytes = _workspace(lib.diloco_layernorm_workspace_bytes(ctypes.byref(n)), "diloco_layernorm_workspace_bytes", x.device)
        _check(lib.diloco_layernorm_backward(ctypes.byref(n), _ptr(dy), _ptr(x), _ptr(weight), _ptr(mean), _ptr(rstd), _ptr(dx), _ptr(dweight),
                                             _ptr(dbias), int(accumulate), _ptr(ws), nbytes, s), "diloco_layernorm_backward")
    return dx


# ------------------------------------------------------------------------------------ attention
_status_words = {}


def device_status(device) -> torch.Tensor:
    """The word in which the attention kernels of a device report a wait that ran out (see check_device_status)."""
    device = torch.device(device)
    key = torch.cuda.current_device() if device.index is None else device.index
    if key not in _status_words:
        _status_words[key] = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", key))
    return _status_words[key]


def check_device_status(device=None, stream=None) -> None:
    """Raises DilocoError if an attention call on the device gave up a wait (its results are invalid); synchronises."""
    word = device_status("cuda" if device is None else device)
    with _On(word, stream) as s:
        _check(binding.load_library().diloco_check_status_word(_ptr(word), s), "diloco_check_status_word")


def _heads(t: torch.Tensor, name: str, tokens: int, heads: int, d: int) -> Tuple[int, int]:
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name}: bfloat16 wanted, got {t.dtype}")
    _want(tuple(t.shape) == (tokens, heads, d), f"{name}: shape {(tokens, heads, d)} wanted, got {tuple(t.shape)}")
    _want(t.stride(2) == 1, f"{name}: the last axis has to be contiguous")
    # an axis of one element may carry any stride; a contiguous one is passed in its place
    return t.stride(0) if tokens > 1 else heads * d, t.stride(1) if heads > 1 else d


def _attention_desc(q, k, v, cu_seqlens, scale) -> binding.Attention:
    _want(q.dim() == 3 and k.dim() == 3, "q, k, v: [tokens, heads, head_dim] wanted")
    T, H, D = q.shape
    K = k.shape[1]
    if cu_seqlens.dtype != torch.int32:
        raise TypeError(f"cu_seqlens: int32 wanted, got {cu_seqlens.dtype}")
    _want(cu_seqlens.dim() == 1 and cu_seqlens.numel() >= 1 and cu_seqlens.is_contiguous(), "cu_seqlens: a contiguous vector of sequences + 1 wanted")
    a = binding.Attention(heads=H, kv_heads=K, head_dim=D, sequences=cu_seqlens.numel() - 1, tokens=T,
                          scale=D ** -0.5 if scale is None else scale, device_status=_ptr(device_status(q.device)))
    a.q_row_stride, a.q_head_stride = _heads(q, "q", T, H, D)
    a.k_row_stride, a.k_head_stride = _heads(k, "k", T, K, D)
    a.v_row_stride, a.v_head_stride = _heads(v, "v", T, K, D)
    return a


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, *, scale: Optional[float] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """diloco_attention_forward: q [tokens, heads, D], k and v [tokens, kv_heads, D] bf16, cu_seqlens int32 [sequences + 1]
    -> (out [tokens, heads, D], lse [heads, tokens]).  scale: 1 / sqrt(D) unless given."""
    _same_device(("q", q), ("k", k), ("v", v), ("cu_seqlens", cu_seqlens), ("out", out))
    a = _attention_desc(q, k, v, cu_seqlens, scale)
    with _On(q, stream) as s:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        a.o_row_stride, a.o_head_stride = _heads(out, "out", *q.shape)
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
        _check(binding.load_library().diloco_attention_forward(ctypes.byref(a), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), _ptr(out),
                                                               _ptr(lse), s), "diloco_attention_forward")
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                       cu_seqlens: torch.Tensor, *, scale: Optional[float] = None, dq: Optional[torch.Tensor] = None,
                       dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                       stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """diloco_attention_backward: (dq, dk, dv) of the forward call that returned out and lse."""
    _same_device(("dout", dout), ("q", q), ("k", k), ("v", v), ("out", out), ("lse", lse), ("cu_seqlens", cu_seqlens), ("dq", dq), ("dk", dk), ("dv", dv))
    a = _attention_desc(q, k, v, cu_seqlens, scale)
    T, H, D = q.shape
    _want(lse.dtype == torch.float32 and lse.shape == (H, T) and lse.is_contiguous(), f"lse: contiguous float32 {(H, T)} wanted")
    a.o_row_stride, a.o_head_stride = _heads(out, "out", T, H, D)
    a.do_row_stride, a.do_head_stride = _heads(dout, "dout", T, H, D)
    lib = binding.load_library()
    with _On(q, stream) as s:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
        a.dq_row_stride, a.dq_head_stride = _heads(dq, "dq", T, H, D)
        a.dk_row_stride, a.dk_head_stride = _heads(dk, "dk", *k.shape)
        a.dv_row_stride, a.dv_head_stride = _heads(dv, "dv", *v.shape)
        ws, n = _workspace(lib.diloco_attention_workspace_bytes(ctypes.byref(a)), "diloco_attention_workspace_bytes", q.device)
        _check(lib.diloco_attention_backward(ctypes.byref(a), _ptr(dout), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(cu_seqlens),
                                             _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), n, s), "diloco_attention_backward")
    return dq, dk, dv


# ----------------------------------------------------------------------------------------- loss
def distill_loss(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor, *, temperature: float = 1.0,
                 z_coef: float = 0.0, row_weight: Optional[torch.Tensor] = None, grad_scale: float = 1.0, grad: bool = False,
                 dlogits: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """diloco_distill_loss: logits [rows, vocab], teacher entries [rows, k] -> (loss [rows], lse [rows], dlogits or None).
    grad: also form the gradient, into dlogits where given (it may be logits).  k = 1: cross-entropy of the target ids."""
    _same_device(("logits", logits), ("teacher_ids", teacher_ids), ("teacher_logits", teacher_logits), ("row_weight", row_weight), ("dlogits", dlogits))
    _want(logits.dim() == 2 and teacher_ids.dim() == 2, "logits: [rows, vocab], teacher_ids: [rows, k] wanted")
    N, V = logits.shape
    k = teacher_ids.shape[1]
    if teacher_ids.dtype not in _IDS:
        raise TypeError(f"teacher_ids: int32 or int64 wanted, got {teacher_ids.dtype}")
    _want(teacher_ids.shape[0] == N and teacher_logits.shape == teacher_ids.shape, f"teacher entries: shape ({N}, k) wanted for both")
    _want(V <= 1 or logits.stride(1) == 1, "logits: the last axis has to be contiguous")
    teacher_ids, teacher_logits = teacher_ids.contiguous(), teacher_logits.contiguous()
    if row_weight is not None:
        _want(row_weight.dtype == torch.float32 and row_weight.shape == (N,) and row_weight.is_contiguous(), f"row_weight: contiguous float32 ({N},) wanted")
    l = binding.Distill(rows=N, vocab=V, logits_stride=logits.stride(0) if N > 1 else V, k=k, ids_int64=_IDS[teacher_ids.dtype],
                        dtype=_dtype(logits, "logits"), teacher_dtype=_dtype(teacher_logits, "teacher_logits"), temperature=temperature,
                        z_coef=z_coef, grad_scale=grad_scale)
    with _On(logits, stream) as s:
        both = torch.empty((2, N), dtype=torch.float32, device=logits.device)
        loss, lse = both[0], both[1]
        if grad and dlogits is None:
            dlogits = torch.empty((N, V), dtype=logits.dtype, device=logits.device)
        if dlogits is not None:
            _want(dlogits.shape == logits.shape and dlogits.dtype == logits.dtype and (V <= 1 or dlogits.stride(1) == 1),
                  "dlogits: shape and type of logits wanted, the last axis contiguous")
            l.grad_stride = dlogits.stride(0) if N > 1 else V
        _check(binding.load_library().diloco_distill_loss(ctypes.byref(l), _ptr(logits), _ptr(teacher_ids), _ptr(teacher_logits),
                                                          _ptr(row_weight), _ptr(loss), _ptr(lse), _ptr(dlogits), s), "diloco_distill_loss")
    return loss, lse, dlogits


# ------------------------------------------------------------------------------------- autograd
class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, table, scale, out_dtype):
        ctx.save_for_backward(ids)
        ctx.scale, ctx.table = scale, (table.shape, table.dtype)
        return embedding_forward(ids, table, scale=scale, out_dtype=out_dtype)

    @staticmethod
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        shape, dtype = ctx.table
        dtable = torch.empty(shape, dtype=dtype, device=dout.device)
        return None, embedding_backward(ids, dout.contiguous(), dtable, scale=ctx.scale), None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps=eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias = bias is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dw = torch.empty(weight.shape, dtype=weight.dtype, device=x.device) if ctx.needs_input_grad[1] else None
        db = torch.empty(weight.shape, dtype=weight.dtype, device=x.device) if ctx.bias and ctx.needs_input_grad[2] else None
        return layer_norm_backward(dy.contiguous(), x, weight, mean, rstd, dw, db), dw, db, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_seqlens, scale):
        out, lse = attention_forward(q, k, v, cu_seqlens, scale=scale)
        ctx.save_for_backward(q, k, v, out, lse, cu_seqlens)
        ctx.scale = scale
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, cu_seqlens = ctx.saved_tensors
        return attention_backward(dout.contiguous(), q, k, v, out, lse, cu_seqlens, scale=ctx.scale) + (None, None)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, temperature, z_coef, row_weight):
        ctx.save_for_backward(logits, teacher_ids, teacher_logits, row_weight)
        ctx.how = dict(temperature=temperature, z_coef=z_coef)
        return distill_loss(logits, teacher_ids, teacher_logits, row_weight=row_weight, **ctx.how)[0]

    @staticmethod
    def backward(ctx, dloss):
        logits, ids, teacher, row_weight = ctx.saved_tensors
        weight = dloss.float().contiguous() if row_weight is None else dloss.float() * row_weight
        return distill_loss(logits, ids, teacher, row_weight=weight, grad=True, **ctx.how)[2], None, None, None, None, None


def embedding(ids, table, *, scale: float = 1.0, out_dtype=None) -> torch.Tensor:
    """embedding_forward, differentiable in table."""
    return _Embedding.apply(ids, table, scale, out_dtype)


def layer_norm(x, weight, bias=None, *, eps: float = 1e-5) -> torch.Tensor:
    """layer_norm_forward, differentiable in x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


def attention(q, k, v, cu_seqlens, *, scale=None) -> torch.Tensor:
    """attention_forward, differentiable in q, k and v."""
    return _Attention.apply(q, k, v, cu_seqlens, scale)


def distill(logits, teacher_ids, teacher_logits, *, temperature: float = 1.0, z_coef: float = 0.0, row_weight=None) -> torch.Tensor:
    """distill_loss, the loss of each row, differentiable in logits."""
    return _Distill.apply(logits, teacher_ids, teacher_logits, temperature, z_coef, row_weight)
