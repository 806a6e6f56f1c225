"""Python binding of the layer operators (``include/dqgan_layers.h``): an
embedding, layer norm and distillation from a teacher's top logits for the M
workers of a plan, whose parameters lie in the rows of the evaluation points
and whose parameter gradients go into the rows of the gradients.

As in ``dqgan``, torch tensors supply device memory and the stream, and every
tensor is checked against the plan and the other tensors before the call;
outputs and workspaces are the caller's.  The calls leave no autograd graph: each
operator's gradient is a call of its own.  Activations are float32, bfloat16 or
float16, ``[M][tokens][width]`` and contiguous.
"""
import ctypes

import torch

from . import dqgan
from .dqgan import F32, U32, _check, _ptr

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
INDEX_TYPES = {torch.int32: 0, torch.int64: 1}

EXPORTS = ("dqgan_embed_forward", "dqgan_embed_bytes", "dqgan_embed_backward", "dqgan_norm_forward",
           "dqgan_norm_bytes", "dqgan_norm_backward", "dqgan_distill_forward", "dqgan_distill_backward",
           "dqgan_distill_fused", "dqgan_distill_bytes")


class EmbedDesc(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("vocab", ctypes.c_int64), ("width", ctypes.c_int64),
                ("tokens", ctypes.c_int64), ("scale", ctypes.c_float), ("type", ctypes.c_int32),
                ("index_type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("gamma", ctypes.c_int64), ("beta", ctypes.c_int64), ("width", ctypes.c_int64),
                ("tokens", ctypes.c_int64), ("eps", ctypes.c_float), ("type", ctypes.c_int32),
                ("reserved", ctypes.c_int64)]


class DistillDesc(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int64), ("ld", ctypes.c_int64), ("tokens", ctypes.c_int64), ("k", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_lib = None


def load():
    """The built library, with the layer operators' argument types."""
    global _lib
    if _lib is not None:
        return _lib
    L = dqgan.load()
    P, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    size = ctypes.POINTER(ctypes.c_size_t)
    E, N, D = (ctypes.POINTER(x) for x in (EmbedDesc, NormDesc, DistillDesc))
    L.dqgan_embed_forward.argtypes = [P, E, P, P, i64, P, P]
    L.dqgan_embed_bytes.argtypes = [P, E, size]
    L.dqgan_embed_backward.argtypes = [P, E, P, P, P, i32, P, P]
    L.dqgan_norm_forward.argtypes = [P, N, P, P, i64, P, P, P]
    L.dqgan_norm_bytes.argtypes = [P, N, size]
    L.dqgan_norm_backward.argtypes = [P, N, P, P, P, i64, P, P, P, i32, P, P]
    L.dqgan_distill_forward.argtypes = [P, D, P, P, P, P, P, P, P, P]
    L.dqgan_distill_backward.argtypes = [P, D, P, P, P, P, P, P, P]
    L.dqgan_distill_fused.argtypes = [P, D, P, P, P, P, P, P, P, P]
    L.dqgan_distill_bytes.argtypes = [P, D, size]
    for name in EXPORTS:
        getattr(L, name).restype = i32
    _lib = L
    return L


def _type(dtype, name, types=TYPES):
    t = types.get(dtype)
    if t is None:
        raise TypeError("%s: dtype %s, expected one of %s" % (name, dtype, ", ".join(str(t) for t in types)))
    return t


# descriptors by their values and the plan's sizes, with the workspace that the
# library asks for: neither depends on anything else (-0.0 as a scale is 0.0, its
# equal as a key)
_descs = {}


def _desc(plan, cls, fn, *fields):
    """(reference to the descriptor, bytes of workspace)."""
    key = (cls, plan.M, plan.d, plan.ld, fields)
    hit = _descs.get(key)
    if hit is None:
        d, n = cls(*fields), ctypes.c_size_t()
        _check(fn, getattr(load(), fn)(plan.handle, ctypes.byref(d), ctypes.byref(n)))
        if len(_descs) >= 4096:
            _descs.clear()
        hit = _descs[key] = (ctypes.byref(d), n.value)
    return hit


def _sizes(plan, t, name):
    """Device pointer, shape and dtype of the tensor that says what sizes a call has."""
    if isinstance(t, torch.Tensor):
        shape = t.shape
        if len(shape) == 3 and shape[0] == plan.M:
            dtype = t.dtype
            if dtype in TYPES and t.get_device() == plan.device and t.is_contiguous():
                return t.data_ptr() or None, shape, dtype
            _ptr(t, name, 0, TYPES, plan.device)
    raise ValueError("%s: expected a tensor of [%d][tokens][width]" % (name, plan.M))


def _like(plan, t, name, shape, dtypes):
    """Device pointer of a tensor that has to have this shape (None: NULL)."""
    if t is None:
        return None
    # the usual case by the fewest attribute reads; what fails here is named below
    if (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype in dtypes and t.get_device() == plan.device
            and t.is_contiguous()):
        return t.data_ptr() or None
    _ptr(t, name, 0, dtypes, plan.device)
    raise ValueError("%s: shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))


def _params(plan, P):
    """Pointer and row stride of parameters: [M][ld], one row per worker, or
    one vector of ld that all workers read."""
    if P is None:
        return None, plan.ld
    # the usual case by the fewest attribute reads; what fails here is named below
    if (isinstance(P, torch.Tensor) and P.dtype == torch.float32 and P.dim() == 2 and P.get_device() == plan.device
            and P.is_contiguous() and P.nbytes >= 4 * plan.M * plan.ld):
        return P.data_ptr(), plan.ld
    if isinstance(P, torch.Tensor) and P.dim() == 1 and plan.M > 1:
        return plan._vec(P, "P"), 0
    return plan._mat(P, "P"), plan.ld


def _workspace(plan, t, need):
    """Pointer of the caller's workspace: any contiguous tensor of enough bytes."""
    if t is None:
        if need:
            raise ValueError("workspace: the call needs %d bytes" % need)
        return None
    return _ptr(t, "workspace", need, None, plan.device) or None


def _on(plan, stream):
    if stream is None:  # the plan's device is the current one, or the library refuses the call
        return torch._C._cuda_getCurrentRawStream(plan.device)
    return stream.cuda_stream


def _new(plan, n):
    return torch.empty(n, dtype=torch.uint8, device="cuda:%d" % plan.device) if n else None


# ---------------------------------------------------------------------------
# embedding


def _embed(plan, tokens, x, name, vocab, offset, scale):
    """Descriptor, workspace, pointers of the tokens and of the activations x."""
    at, shape, dtype = _sizes(plan, x, name)
    tok = _like(plan, tokens, "tokens", shape[:2], INDEX_TYPES)
    d, need = _desc(plan, EmbedDesc, "dqgan_embed_bytes", offset, vocab, shape[2], shape[1], scale + 0.0, TYPES[dtype],
                    0 if tokens is None else INDEX_TYPES[tokens.dtype], 0)
    return d, need, tok, at


def embed_forward(plan, tokens, P, out, vocab, offset=0, scale=1.0, stream=None):
    """out[m][n] = scale * row tokens[m][n] of worker m's table, which lies at
    `offset` of its row of P ([vocab][width]); 0 where the token is below 0 or
    at or beyond vocab.  tokens int32 or int64 [M][tokens]; P [M][ld], or [ld]
    for all workers; out [M][tokens][width]."""
    d, _, tok, to = _embed(plan, tokens, out, "out", vocab, offset, scale)
    p, ldp = _params(plan, P)
    _check("dqgan_embed_forward", load().dqgan_embed_forward(plan.handle, d, tok, p, ldp, to, _on(plan, stream)))


def embed_workspace(plan, tokens, vocab, width, dtype, index_dtype=torch.int64, offset=0):
    """A workspace for embed_backward with `tokens` tokens per worker."""
    return _new(plan, _desc(plan, EmbedDesc, "dqgan_embed_bytes", offset, vocab, width, tokens, 1.0,
                            _type(dtype, "dtype"), _type(index_dtype, "index_dtype", INDEX_TYPES), 0)[1])


def embed_backward(plan, tokens, dout, G, vocab, workspace, offset=0, scale=1.0, add=False, stream=None):
    """The table's part of G [M][ld]: row v is scale * the sum of dout over the
    tokens that are v, 0 for those that do not occur; with `add` the sums are
    added to what is there."""
    d, need, tok, at = _embed(plan, tokens, dout, "dout", vocab, offset, scale)
    _check("dqgan_embed_backward", load().dqgan_embed_backward(plan.handle, d, tok, at, plan._mat(G, "G"), int(add),
                                                               _workspace(plan, workspace, need), _on(plan, stream)))


# ---------------------------------------------------------------------------
# layer norm


def _norm(plan, tokens, width, type, gamma, beta, eps):
    return _desc(plan, NormDesc, "dqgan_norm_bytes", -1 if gamma is None else gamma, -1 if beta is None else beta, width,
                 tokens, eps, type, 0)


def norm_forward(plan, x, P, y, stats=None, gamma=0, beta=None, eps=1e-5, stream=None):
    """y = (x - mean) * rstd * weight + bias over the last dimension; weight and
    bias at `gamma` and `beta` of each worker's row of P (None: without).
    stats [M][tokens][2] float32 takes mean and rstd for norm_backward; y may
    be x."""
    at, shape, dtype = _sizes(plan, x, "x")
    d, _ = _norm(plan, shape[1], shape[2], TYPES[dtype], gamma, beta, eps)
    p, ldp = _params(plan, P)
    _check("dqgan_norm_forward",
           load().dqgan_norm_forward(plan.handle, d, at, p, ldp, _like(plan, y, "y", shape, (dtype,)),
                                     _like(plan, stats, "stats", (shape[0], shape[1], 2), F32), _on(plan, stream)))


def norm_workspace(plan, tokens, width, dtype, gamma=0, beta=None):
    """A workspace for norm_backward of these sizes (None if it needs none)."""
    return _new(plan, _norm(plan, tokens, width, _type(dtype, "dtype"), gamma, beta, 0.0)[1])


def norm_backward(plan, x, dy, P, stats, dx, G, workspace, gamma=0, beta=None, add=False, stream=None):
    """dx (None: not wanted; it may be dy), and the sums over a worker's tokens
    of dy * (x - mean) * rstd and of dy into its row of G at `gamma` and
    `beta`; with `add` added to what is there."""
    at, shape, dtype = _sizes(plan, x, "x")
    d, need = _norm(plan, shape[1], shape[2], TYPES[dtype], gamma, beta, 0.0)
    p, ldp = _params(plan, P)
    same = (dtype,)
    _check("dqgan_norm_backward",
           load().dqgan_norm_backward(plan.handle, d, at, _like(plan, dy, "dy", shape, same), p, ldp,
                                      _like(plan, stats, "stats", (shape[0], shape[1], 2), F32),
                                      _like(plan, dx, "dx", shape, same), plan._mat(G, "G"), int(add),
                                      _workspace(plan, workspace, need), _on(plan, stream)))


# ---------------------------------------------------------------------------
# distillation


def _distill(plan, z, val, idx, weight, vocab, temperature):
    """Descriptor, workspace, the pointers that every form of the loss takes,
    and [M][tokens]."""
    at, shape, dtype = _sizes(plan, z, "z")
    rows = shape[:2]
    if not isinstance(val, torch.Tensor) or val.dim() != 3:
        raise ValueError("val: expected a tensor of [%d][%d][k]" % rows)
    sent = (rows[0], rows[1], val.shape[2])
    d, need = _desc(plan, DistillDesc, "dqgan_distill_bytes", shape[2] if vocab is None else vocab, shape[2], rows[1],
                    sent[2], temperature, TYPES[dtype], 0)
    return d, need, (at, _like(plan, val, "val", sent, F32),
                     _like(plan, idx, "idx", sent, U32), _like(plan, weight, "weight", rows, F32)), rows


def distill_workspace(plan, tokens, vocab, k, dtype, ld=None):
    """A workspace for distill_forward and distill_fused of these sizes (None
    if they need none)."""
    return _new(plan, _desc(plan, DistillDesc, "dqgan_distill_bytes", vocab, vocab if ld is None else ld, tokens, k, 1.0,
                            _type(dtype, "dtype"), 0)[1])


def distill_forward(plan, z, val, idx, weight, loss, stats, vocab=None, workspace=None, temperature=1.0, stream=None):
    """loss [M][tokens] of student logits z [M][tokens][ld] (columns from vocab
    on are padding) against softmax(val / T) over the teacher's entries val,
    idx [M][tokens][k] (indices at or beyond vocab, as -1, are skipped):
    weight * T^2 * KL; weight [M][tokens] or None.  stats [M][tokens][2] is
    what distill_backward takes."""
    d, need, args, rows = _distill(plan, z, val, idx, weight, vocab, temperature)
    _check("dqgan_distill_forward",
           load().dqgan_distill_forward(plan.handle, d, *args, _like(plan, loss, "loss", rows, F32),
                                        _like(plan, stats, "stats", (rows[0], rows[1], 2), F32),
                                        _workspace(plan, workspace, need), _on(plan, stream)))


def distill_backward(plan, z, val, idx, weight, stats, dz, vocab=None, temperature=1.0, stream=None):
    """dz of distill_forward's loss; `weight` times the gradient that each loss
    receives takes its place as `weight`.  dz may be z."""
    d, _, args, rows = _distill(plan, z, val, idx, weight, vocab, temperature)
    _check("dqgan_distill_backward",
           load().dqgan_distill_backward(plan.handle, d, *args,
                                         _like(plan, stats, "stats", (rows[0], rows[1], 2), F32),
                                         _like(plan, dz, "dz", z.shape, (z.dtype,)), _on(plan, stream)))


def distill_fused(plan, z, val, idx, weight, loss, dz, vocab=None, workspace=None, temperature=1.0, stream=None):
    """distill_forward and distill_backward in one call, the same bits; dz may
    be z."""
    d, need, args, rows = _distill(plan, z, val, idx, weight, vocab, temperature)
    _check("dqgan_distill_fused",
           load().dqgan_distill_fused(plan.handle, d, *args, _like(plan, loss, "loss", rows, F32),
                                      _like(plan, dz, "dz", z.shape, (z.dtype,)), _workspace(plan, workspace, need),
                                      _on(plan, stream)))
