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
from functools import lru_cache
from typing import Optional, Tuple

import torch

from . import binding
from .binding import _check

_DTYPES = {torch.float32: binding.DTYPE_F32, torch.bfloat16: binding.DTYPE_BF16}
_IDS = {torch.int32: 0, torch.int64: 1}

# A call's checks and its descriptor depend on shapes, strides and types alone, so they are made once for each
# combination: the *_plan functions below take those and return the descriptor (never changed afterwards) with what
# else the call needs.  What is left for every call is a lookup, the outputs and the launch.
_PLANS = 4096


def _dtype(dtype: torch.dtype, name: str) -> int:
    try:
        return _DTYPES[dtype]
    except KeyError:
        raise TypeError(f"{name}: float32 or bfloat16 wanted, got {dtype}") from None


def _ids_kind(dtype: torch.dtype, name: str) -> int:
    if dtype not in _IDS:
        raise TypeError(f"{name}: int32 or int64 wanted, got {dtype}")
    return _IDS[dtype]


def _want(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _sig(t: Optional[torch.Tensor]):
    """What a plan may depend on."""
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _device(first: torch.Tensor, *others) -> int:
    """The one CUDA device of a call's tensors."""
    dev = first.get_device()
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError("all tensors of a call have to be on one CUDA device")
    if dev < 0:
        raise ValueError(f"CUDA tensors are wanted, got one on {first.device}")
    return dev


def _elsewhere(dev: int, stream):
    """None where a call may go ahead on the current device's current stream, else the context to make it in: what is
    allocated inside belongs to the stream that the kernels run on."""
    if stream is not None:
        return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=dev) if isinstance(stream, int) else stream)
    return None if dev == torch.cuda.current_device() else torch.cuda.device(dev)


def _raw_stream(dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _size(nbytes: int, where: str) -> int:
    if nbytes < 0:
        raise binding.DilocoError(int(nbytes), where)
    return int(nbytes)


def _workspace(nbytes: int, dev: int) -> torch.Tensor:
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)


def _contiguous(shape) -> Tuple[int, ...]:
    strides, n = [], 1
    for s in reversed(shape):
        strides.append(n)
        n *= max(s, 1)
    return tuple(reversed(strides))


def _is_contiguous(shape, strides) -> bool:
    """Axes of one element may carry any stride."""
    return 0 in shape or all(n == 1 or a == b for n, a, b in zip(shape, strides, _contiguous(shape)))


def _replica_rows(sig, name: str, shape) -> int:
    """A parameter or its gradient, [M, ...] with each replica's part contiguous: the distance between replicas."""
    _want(tuple(sig[0]) == tuple(shape), f"{name}: shape {tuple(shape)} wanted, got {tuple(sig[0])}")
    _want(_is_contiguous(sig[0][1:], sig[1][1:]), f"{name}: each replica's part has to be contiguous")
    return sig[1][0] if shape[0] > 1 else _contiguous(shape)[0]


# ------------------------------------------------------------------------------------ embedding
def _embedding_desc(ids, table, rows, scale, what) -> binding.Embedding:
    """table: the table of a forward call or the gradient of a backward call (`what`)."""
    kind = _ids_kind(ids[2], "ids")
    _want(len(ids[0]) == 2, f"ids: [M, tokens] wanted, got shape {tuple(ids[0])}")
    M, tokens = ids[0]
    _want(len(table[0]) == 3 and table[0][0] == M, f"{what}: [M, vocab, d] with M = {M} wanted, got {tuple(table[0])}")
    _, V, d = table[0]
    stride = _replica_rows(table, what, (M, V, d))
    shape, strides, dtype = rows
    _want(tuple(shape) == (M, tokens, d), f"rows: shape {(M, tokens, d)} wanted, got {tuple(shape)}")
    row = strides[1] if tokens > 1 else strides[0] if M > 1 else d
    _want(d == 1 or strides[2] == 1, "rows: the last axis has to be contiguous")
    _want(M == 1 or tokens == 0 or strides[0] == tokens * row, "rows: replicas have to follow one another at the tokens' stride")
    kinds = _dtype(table[2], what)
    return binding.Embedding(M, d, tokens, V, stride, stride, max(row, d), scale, kind, kinds, _dtype(dtype, "rows"), kinds)


@lru_cache(_PLANS)
def _embedding_plan(ids, table, rows, scale, what):
    e = _embedding_desc(ids, table, rows, scale, what)
    nbytes = 0
    if what == "dtable":
        nbytes = _size(binding.load_library().diloco_embedding_workspace_bytes(ctypes.byref(e)), "diloco_embedding_workspace_bytes")
    return ctypes.byref(e), nbytes


def embedding_forward(ids: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """diloco_embedding_forward: ids [M, tokens], table [M, vocab, d] -> [M, tokens, d]."""
    dev = _device(table, ids, out)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return embedding_forward(ids, table, scale=scale, out_dtype=out_dtype, out=out)
    if not ids.is_contiguous():
        ids = ids.contiguous()
    if out is None:
        _want(ids.dim() == 2 and table.dim() == 3, "ids: [M, tokens], table: [M, vocab, d] wanted")
        _dtype(out_dtype or table.dtype, "out")
        out = torch.empty((*ids.shape, table.shape[2]), dtype=out_dtype or table.dtype, device=dev)
    e, _ = _embedding_plan(_sig(ids), _sig(table), _sig(out), scale, "table")
    _check(binding.load_library().diloco_embedding_forward(e, ids.data_ptr(), table.data_ptr(), out.data_ptr(), _raw_stream(dev)),
           "diloco_embedding_forward")
    return out


def embedding_backward(ids: torch.Tensor, dout: torch.Tensor, dtable: torch.Tensor, *, scale: float = 1.0, accumulate: bool = False,
                       stream=None) -> torch.Tensor:
    """diloco_embedding_backward: dout [M, tokens, d] summed by token into dtable [M, vocab, d], which is returned.
    accumulate: dtable keeps what it holds (a table that is also the output projection) and only rows of present ids change."""
    dev = _device(dtable, ids, dout)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return embedding_backward(ids, dout, dtable, scale=scale, accumulate=accumulate)
    if not ids.is_contiguous():
        ids = ids.contiguous()
    e, nbytes = _embedding_plan(_sig(ids), _sig(dtable), _sig(dout), scale, "dtable")
    ws = _workspace(nbytes, dev)
    _check(binding.load_library().diloco_embedding_backward(e, ids.data_ptr(), dout.data_ptr(), dtable.data_ptr(), int(accumulate),
                                                            ws.data_ptr(), nbytes, _raw_stream(dev)), "diloco_embedding_backward")
    return dtable


# ----------------------------------------------------------------------------------- layer norm
def _norm_rows(sig, name: str, shape) -> Tuple[int, int]:
    """[M, rows, groups, d] (or [M, rows, d]) with one row stride over all replicas: (row stride, group stride)."""
    _want(tuple(sig[0]) == tuple(shape), f"{name}: shape {tuple(shape)} wanted, got {tuple(sig[0])}")
    M, N = shape[:2]
    st = sig[1]
    _want(shape[-1] == 1 or st[-1] == 1, f"{name}: the last axis has to be contiguous")
    row = st[1] if N > 1 else st[0] if M > 1 else 0
    _want(M == 1 or N <= 1 or st[0] == N * row, f"{name}: replicas have to follow one another at the rows' stride")
    return row, st[2] if len(shape) == 4 and shape[2] > 1 else 0


def _norm_desc(x, weight, eps) -> binding.LayerNorm:
    shape = x[0]
    _want(len(shape) in (3, 4), f"x: [M, rows, d] or [M, rows, groups, d] wanted, got shape {tuple(shape)}")
    M, N, d = shape[0], shape[1], shape[-1]
    n = binding.LayerNorm(M=M, d=d, groups=shape[2] if len(shape) == 4 else 1, rows=N, eps=eps, act_dtype=_dtype(x[2], "x"),
                          param_dtype=_dtype(weight[2], "weight"))
    n.x_row_stride, n.x_group_stride = _norm_rows(x, "x", shape)
    n.param_stride = _replica_rows(weight, "weight", (M, d))
    return n


@lru_cache(_PLANS)
def _norm_forward_plan(x, weight, bias, out, eps):
    n = _norm_desc(x, weight, eps)
    if bias is not None:
        _want(bias[2] == weight[2], "bias: the weight's type wanted")
        _want(_replica_rows(bias, "bias", weight[0]) == n.param_stride, "bias: the weight's stride between replicas wanted")
    _want(out[2] == x[2], "out: the type of x wanted")
    n.y_row_stride, n.y_group_stride = _norm_rows(out, "out", x[0])
    return ctypes.byref(n), (2, *x[0][:-1])


@lru_cache(_PLANS)
def _norm_backward_plan(x, weight, dy, dx, mean, rstd, dweight, dbias):
    n = _norm_desc(x, weight, 0.0)
    for name, t in (("dy", dy), ("dx", dx)):
        _want(t[2] == x[2], f"{name}: the type of x wanted")
    n.y_row_stride, n.y_group_stride = _norm_rows(dy, "dy", x[0])
    n.dx_row_stride, n.dx_group_stride = _norm_rows(dx, "dx", x[0])
    for name, t in (("mean", mean), ("rstd", rstd)):
        _want(t[2] == torch.float32 and t[0] == x[0][:-1] and _is_contiguous(*t[:2]), f"{name}: contiguous float32 {tuple(x[0][:-1])} wanted")
    grads = [(name, t) for name, t in (("dweight", dweight), ("dbias", dbias)) if t is not None]
    nbytes = 0
    if grads:
        n.grad_dtype = _dtype(grads[0][1][2], grads[0][0])
        n.grad_stride = _replica_rows(grads[0][1], grads[0][0], weight[0])
        for name, t in grads[1:]:
            _want(t[2] == grads[0][1][2] and _replica_rows(t, name, weight[0]) == n.grad_stride, "dbias: the type and stride of dweight wanted")
        nbytes = _size(binding.load_library().diloco_layernorm_workspace_bytes(ctypes.byref(n)), "diloco_layernorm_workspace_bytes")
    return ctypes.byref(n), nbytes


def _empty_like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def layer_norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, eps: float = 1e-5,
                       out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """diloco_layernorm_forward: x [M, rows, d] or [M, rows, groups, d], weight and bias [M, d] -> (y, mean, rstd).
    out may be x."""
    dev = _device(x, weight, bias, out)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return layer_norm_forward(x, weight, bias, eps=eps, out=out)
    if out is None:
        out = _empty_like(x)
    n, shape = _norm_forward_plan(_sig(x), _sig(weight), _sig(bias), _sig(out), eps)
    mean, rstd = torch.empty(shape, dtype=torch.float32, device=dev).unbind(0)
    _check(binding.load_library().diloco_layernorm_forward(n, x.data_ptr(), weight.data_ptr(), _ptr(bias), out.data_ptr(), mean.data_ptr(),
                                                           rstd.data_ptr(), _raw_stream(dev)), "diloco_layernorm_forward")
    return out, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None, *, accumulate: bool = False,
                        dx: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """diloco_layernorm_backward: returns dx and writes dweight and dbias ([M, d], where given; accumulate: adds to them).
    dx may be dy."""
    dev = _device(x, dy, weight, mean, rstd, dweight, dbias, dx)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return layer_norm_backward(dy, x, weight, mean, rstd, dweight, dbias, accumulate=accumulate, dx=dx)
    if dx is None:
        dx = _empty_like(x)
    n, nbytes = _norm_backward_plan(_sig(x), _sig(weight), _sig(dy), _sig(dx), _sig(mean), _sig(rstd), _sig(dweight), _sig(dbias))
    ws = _workspace(nbytes, dev) if nbytes else None
    _check(binding.load_library().diloco_layernorm_backward(n, dy.data_ptr(), x.data_ptr(), weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                                            dx.data_ptr(), _ptr(dweight), _ptr(dbias), int(accumulate), _ptr(ws), nbytes,
                                                            _raw_stream(dev)), "diloco_layernorm_backward")
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
    if (ctx := _elsewhere(word.get_device(), stream)) is not None:
        with ctx:
            return check_device_status(word.device)
    _check(binding.load_library().diloco_check_status_word(word.data_ptr(), _raw_stream(word.get_device())), "diloco_check_status_word")


def _heads(sig, name: str, tokens: int, heads: int, d: int) -> Tuple[int, int]:
    shape, strides, dtype = sig
    if dtype != torch.bfloat16:
        raise TypeError(f"{name}: bfloat16 wanted, got {dtype}")
    _want(tuple(shape) == (tokens, heads, d), f"{name}: shape {(tokens, heads, d)} wanted, got {tuple(shape)}")
    _want(d == 1 or strides[2] == 1, f"{name}: the last axis has to be contiguous")
    # an axis of one element may carry any stride; a contiguous one is passed in its place
    return strides[0] if tokens > 1 else heads * d, strides[1] if heads > 1 else d


@lru_cache(_PLANS)
def _attention_plan(q, k, v, cu, scale, dev, out, lse, dout, dq, dk, dv):
    """out ... dv: None for what the call does not have."""
    _want(len(q[0]) == 3 and len(k[0]) == 3, "q, k, v: [tokens, heads, head_dim] wanted")
    T, H, D = q[0]
    K = k[0][1]
    if cu[2] != torch.int32:
        raise TypeError(f"cu_seqlens: int32 wanted, got {cu[2]}")
    _want(len(cu[0]) == 1 and cu[0][0] >= 1 and (cu[0][0] == 1 or cu[1][0] == 1), "cu_seqlens: a contiguous vector of sequences + 1 wanted")
    a = binding.Attention(heads=H, kv_heads=K, head_dim=D, sequences=cu[0][0] - 1, tokens=T, scale=D ** -0.5 if scale is None else scale,
                          device_status=device_status(torch.device("cuda", dev)).data_ptr())
    _want(lse is None or (lse[2] == torch.float32 and tuple(lse[0]) == (H, T) and _is_contiguous(*lse[:2])), f"lse: contiguous float32 {(H, T)} wanted")
    for name, field, t, heads in (("q", "q", q, H), ("k", "k", k, K), ("v", "v", v, K), ("out", "o", out, H), ("dout", "do", dout, H), ("dq", "dq", dq, H),
                                  ("dk", "dk", dk, K), ("dv", "dv", dv, K)):
        if t is not None:
            row, head = _heads(t, name, T, heads, D)
            setattr(a, field + "_row_stride", row)
            setattr(a, field + "_head_stride", head)
    nbytes = 0
    if dout is not None:
        nbytes = _size(binding.load_library().diloco_attention_workspace_bytes(ctypes.byref(a)), "diloco_attention_workspace_bytes")
    return ctypes.byref(a), nbytes, (H, T)


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_seqlens: torch.Tensor, *, scale: Optional[float] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """diloco_attention_forward: q [tokens, heads, D], k and v [tokens, kv_heads, D] bf16, cu_seqlens int32 [sequences + 1]
    -> (out [tokens, heads, D], lse [heads, tokens]).  scale: 1 / sqrt(D) unless given."""
    dev = _device(q, k, v, cu_seqlens, out)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return attention_forward(q, k, v, cu_seqlens, scale=scale, out=out)
    if out is None:
        out = _empty_like(q)
    a, _, shape = _attention_plan(_sig(q), _sig(k), _sig(v), _sig(cu_seqlens), scale, dev, _sig(out), None, None, None, None, None)
    lse = torch.empty(shape, dtype=torch.float32, device=dev)
    _check(binding.load_library().diloco_attention_forward(a, q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), out.data_ptr(),
                                                           lse.data_ptr(), _raw_stream(dev)), "diloco_attention_forward")
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                       cu_seqlens: torch.Tensor, *, scale: Optional[float] = None, dq: Optional[torch.Tensor] = None,
                       dk: Optional[torch.Tensor] = None, dv: Optional[torch.Tensor] = None,
                       stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """diloco_attention_backward: (dq, dk, dv) of the forward call that returned out and lse."""
    dev = _device(q, k, v, out, lse, cu_seqlens, dout, dq, dk, dv)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return attention_backward(dout, q, k, v, out, lse, cu_seqlens, scale=scale, dq=dq, dk=dk, dv=dv)
    dq = _empty_like(q) if dq is None else dq
    dk = _empty_like(k) if dk is None else dk
    dv = _empty_like(v) if dv is None else dv
    a, nbytes, _ = _attention_plan(_sig(q), _sig(k), _sig(v), _sig(cu_seqlens), scale, dev, _sig(out), _sig(lse), _sig(dout), _sig(dq), _sig(dk), _sig(dv))
    ws = _workspace(nbytes, dev)
    _check(binding.load_library().diloco_attention_backward(a, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                                            cu_seqlens.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), nbytes,
                                                            _raw_stream(dev)), "diloco_attention_backward")
    return dq, dk, dv


# ----------------------------------------------------------------------------------------- loss
@lru_cache(_PLANS)
def _distill_plan(logits, ids, teacher, row_weight, dlogits, temperature, z_coef, grad_scale):
    _want(len(logits[0]) == 2 and len(ids[0]) == 2, "logits: [rows, vocab], teacher_ids: [rows, k] wanted")
    N, V = logits[0]
    kind = _ids_kind(ids[2], "teacher_ids")
    _want(ids[0][0] == N and teacher[0] == ids[0], f"teacher entries: shape ({N}, k) wanted for both")
    _want(V <= 1 or logits[1][1] == 1, "logits: the last axis has to be contiguous")
    _want(row_weight is None or (row_weight[2] == torch.float32 and tuple(row_weight[0]) == (N,) and _is_contiguous(*row_weight[:2])),
          f"row_weight: contiguous float32 ({N},) wanted")
    l = binding.Distill(rows=N, vocab=V, logits_stride=logits[1][0] if N > 1 else V, k=ids[0][1], ids_int64=kind, dtype=_dtype(logits[2], "logits"),
                        teacher_dtype=_dtype(teacher[2], "teacher_logits"), temperature=temperature, z_coef=z_coef, grad_scale=grad_scale)
    if dlogits is not None:
        _want(dlogits[0] == logits[0] and dlogits[2] == logits[2] and (V <= 1 or dlogits[1][1] == 1),
              "dlogits: shape and type of logits wanted, the last axis contiguous")
        l.grad_stride = dlogits[1][0] if N > 1 else V
    return ctypes.byref(l), (2, N)


def distill_loss(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor, *, temperature: float = 1.0,
                 z_coef: float = 0.0, row_weight: Optional[torch.Tensor] = None, grad_scale: float = 1.0, grad: bool = False,
                 dlogits: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """diloco_distill_loss: logits [rows, vocab], teacher entries [rows, k] -> (loss [rows], lse [rows], dlogits or None).
    grad: also form the gradient, into dlogits where given (it may be logits).  k = 1: cross-entropy of the target ids."""
    dev = _device(logits, teacher_ids, teacher_logits, row_weight, dlogits)
    if (ctx := _elsewhere(dev, stream)) is not None:
        with ctx:
            return distill_loss(logits, teacher_ids, teacher_logits, temperature=temperature, z_coef=z_coef, row_weight=row_weight,
                                grad_scale=grad_scale, grad=grad, dlogits=dlogits)
    if not teacher_ids.is_contiguous():
        teacher_ids = teacher_ids.contiguous()
    if not teacher_logits.is_contiguous():
        teacher_logits = teacher_logits.contiguous()
    if grad and dlogits is None:
        dlogits = _empty_like(logits)
    l, shape = _distill_plan(_sig(logits), _sig(teacher_ids), _sig(teacher_logits), _sig(row_weight), _sig(dlogits), temperature, z_coef, grad_scale)
    loss, lse = torch.empty(shape, dtype=torch.float32, device=dev).unbind(0)
    _check(binding.load_library().diloco_distill_loss(l, logits.data_ptr(), teacher_ids.data_ptr(), teacher_logits.data_ptr(), _ptr(row_weight),
                                                      loss.data_ptr(), lse.data_ptr(), _ptr(dlogits), _raw_stream(dev)), "diloco_distill_loss")
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
