"""ctypes binding of ``include/cnr_loss.h``: argument marshalling only, as in :mod:`lm_binding`, whose manner it has: sizes, strides and element types are
read off the tensors, everything else has the name and the order of the C declaration.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B
from . import lm_binding as L
from .binding import U32, F32, _check, _stream

CNR_LOSS_MAX_TOP, CNR_LOSS_MAX_ROWS, CNR_LOSS_MAX_VOCABULARY, CNR_LOSS_MAX_DIM = 1024, 1048576, 134217728, 1048576

# Every symbol include/cnr_loss.h declares.
LOSS_EXPORTS = ("cnr_loss_state_floats", "cnr_loss_workspace_bytes", "cnr_vocabulary_loss", "cnr_vocabulary_loss_backward", "cnr_top_logits")

__all__ = [*LOSS_EXPORTS, "cnr_vocabulary", "cnr_targets", "LOSS_EXPORTS", "CNR_LOSS_MAX_TOP", "CNR_LOSS_MAX_ROWS", "CNR_LOSS_MAX_VOCABULARY", "CNR_LOSS_MAX_DIM"]


class cnr_vocabulary(ctypes.Structure):
    """Field for field the C struct."""
    _fields_ = [("hidden", ctypes.c_void_p), ("hidden_stride", ctypes.c_uint64), ("weight", ctypes.c_void_p), ("weight_stride", ctypes.c_uint64),
                ("type", ctypes.c_int), ("n", ctypes.c_uint64), ("vocab", ctypes.c_uint64), ("dim", ctypes.c_uint64)]


class cnr_targets(ctypes.Structure):
    """Field for field the C struct."""
    _fields_ = [("tokens", ctypes.c_void_p), ("token_type", ctypes.c_int), ("token_stride", ctypes.c_uint64), ("top", ctypes.c_uint64),
                ("logits", ctypes.c_void_p), ("logit_type", ctypes.c_int), ("logit_stride", ctypes.c_uint64), ("temperature", ctypes.c_float)]


_lib = None


def load() -> ctypes.CDLL:
    """The library of :func:`binding.load`, with this header's functions bound."""
    global _lib
    if _lib is None:
        lib = L.load()
        vp, u64, i32, sz = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_size_t
        sig = {
            "cnr_loss_state_floats": (sz, [u64, u64]),
            "cnr_loss_workspace_bytes": (sz, [u64, u64, u64, i32, i32, i32]),
            "cnr_vocabulary_loss": (i32, [vp, ctypes.POINTER(cnr_vocabulary), ctypes.POINTER(cnr_targets), vp, vp, vp, sz, vp]),
            "cnr_vocabulary_loss_backward": (i32, [vp, ctypes.POINTER(cnr_vocabulary), ctypes.POINTER(cnr_targets), vp, vp, vp, u64, vp, i32, u64, i32, vp, sz,
                                                   vp]),
            "cnr_top_logits": (i32, [vp, vp, u64, i32, u64, u64, u64, vp, vp, vp, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def cnr_loss_state_floats(n: int, top: int) -> int:
    return int(load().cnr_loss_state_floats(n, top))


def cnr_loss_workspace_bytes(n: int, vocab: int, dim: int, type: int, training: bool, dweight_type: int) -> int:
    return int(load().cnr_loss_workspace_bytes(n, vocab, dim, type, int(training), dweight_type))


def _loss_arguments(hidden, weight, tokens, logits, temperature: float):
    """The two structs of a loss, and the places (see _share) of the matrices in them."""
    at, n, dim, stride = L._rows(hidden, "hidden")
    weight_at, vocab, weight_dim, weight_stride = L._rows(weight, "weight")
    if weight_dim != dim:
        raise ValueError("hidden states of %d columns, a weight of %d" % (dim, weight_dim))
    kind = L._float(hidden, "hidden")
    if weight.dtype != hidden.dtype:
        raise TypeError("weight must be of hidden's type, got %s and %s" % (weight.dtype, hidden.dtype))
    if logits is None and isinstance(tokens, torch.Tensor) and tokens.dim() == 1:
        tokens = tokens.unsqueeze(1)
    tokens_at, rows, top, token_stride = L._rows(tokens, "tokens")
    if rows != n or (logits is None and top != 1):
        raise ValueError("tokens must hold %s for each of the %d rows" % ("a target" if logits is None else "a list", n))
    token_type = L._kind(L._INDICES, tokens, "tokens", "int32 or int64")
    logits_at, logit_type, logit_stride = 0, 0, 0
    size, token_size = hidden.element_size(), tokens.element_size()
    places = [(at, n, dim * size, stride * size), (weight_at, vocab, dim * size, weight_stride * size), (tokens_at, n, top * token_size, token_stride * token_size)]
    if logits is not None:
        logits_at, rows, columns, logit_stride = L._rows(logits, "logits")
        if rows != n or columns != top:
            raise ValueError("logits must have the shape of tokens")
        logit_type = L._float(logits, "logits")
        if not 2.0 ** -126 <= temperature < 3e38:
            raise ValueError("the temperature must be positive, from 2^-126 to 3e38")
        size = logits.element_size()
        places.append((logits_at, n, top * size, logit_stride * size))
        logits_at = logits_at or 16  # an empty matrix is none that is missing
    return (cnr_vocabulary(at, stride, weight_at, weight_stride, kind, n, vocab, dim),
            cnr_targets(tokens_at, token_type, token_stride, top, logits_at, logit_type, logit_stride, temperature), places)


def _share(a, b) -> bool:
    """Whether two places, (address, rows, bytes of a row, bytes from one row to the next), have a byte in common.  Column ranges of one matrix have none, though
    either's rows lie among the other's."""
    (at, n, width, step), (at_b, n_b, width_b, step_b) = a, b
    by = at_b - at
    if not (n and width and n_b and width_b) or by >= (n - 1) * step + width or -by >= (n_b - 1) * step_b + width_b:
        return False
    if n > n_b:
        return _share(b, a)
    if n > 1 and step != step_b:
        # each of the fewer rows among the other's
        return any(_share((at + i * step, 1, width, 0), b) for i in range(n))
    # rows i of a and j of b share bytes where -width_b < by + (j - i) step_b < width: the whole numbers k = j - i for which that holds
    if n_b == 1:
        return True
    first, last = (-width_b - by) // step_b + 1, -((by - width) // step_b) - 1
    return max(first, 1 - n) <= min(last, n_b - 1)


def _check_apart(results, operands) -> None:
    """Results' places share no byte with operands' or each other; operands may."""
    last = 0
    for at, n, width, step in sorted(results + operands):
        if at < last:
            break
        last = at + (n - 1) * step + width
    else:
        return
    if any(_share(a, b) for i, a in enumerate(results) for b in results[i + 1:] + operands):
        raise ValueError("a result overlaps an operand or another result")


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def cnr_vocabulary_loss(ctx, hidden, weight, tokens, logits, temperature: float, loss, state, workspace, stream=None) -> None:
    """``tokens``: a list of targets with ``logits`` None, else a matrix as ``logits`` is; ``state`` may be None for targets that no backward pass follows."""
    v, t, operands = _loss_arguments(hidden, weight, tokens, logits, temperature)
    n, top = v.n, t.top
    if top > CNR_LOSS_MAX_TOP:
        raise ValueError("at most %d entries a row" % CNR_LOSS_MAX_TOP)
    if loss is None or loss.numel() < n:
        raise ValueError("loss shorter than %d" % n)
    if state is None and logits is not None:
        raise ValueError("a teacher's entries need a state")
    if state is not None and state.numel() < n * (1 + 3 * top):
        raise ValueError("state shorter than cnr_loss_state_floats")
    room = _bytes(workspace)
    if room < cnr_loss_workspace_bytes(n, v.vocab, v.dim, v.type, False, v.type):
        raise ValueError("workspace smaller than cnr_loss_workspace_bytes")
    loss_at, state_at, workspace_at = B._dev(loss, F32, "loss"), B._dev(state, F32, "state") or 0, B._dev(workspace, None, "workspace") or 0
    _check_apart([(loss_at, 1, 4 * n, 0), (state_at, 1, 4 * n * (1 + 3 * top) if state_at else 0, 0), (workspace_at, 1, room, 0)], operands)
    _check((_lib or load()).cnr_vocabulary_loss(ctx, ctypes.byref(v), ctypes.byref(t), loss_at, state_at, workspace_at, room, _stream(stream)), "cnr_vocabulary_loss")
    L._written(loss, state)


def cnr_vocabulary_loss_backward(ctx, hidden, weight, tokens, logits, temperature: float, state, dloss, dhidden, dweight, accumulate: bool, workspace,
                                 stream=None) -> None:
    """``dhidden`` and ``dweight``: matrices of the shapes of ``hidden`` and ``weight``, or None."""
    v, t, operands = _loss_arguments(hidden, weight, tokens, logits, temperature)
    n, top = v.n, t.top
    if top > CNR_LOSS_MAX_TOP:
        raise ValueError("at most %d entries a row" % CNR_LOSS_MAX_TOP)
    if state is None or state.numel() < n * (1 + 3 * top):
        raise ValueError("state missing or shorter than cnr_loss_state_floats")
    if dloss is None or dloss.numel() < n:
        raise ValueError("dloss shorter than %d" % n)
    to_hidden, to_weight, kind, results = (0, 0, 0, 0), (0, 0, 0, 0), v.type, []
    if dhidden is not None:
        to_hidden = L._rows(dhidden, "dhidden")
        if dhidden.shape != hidden.shape or dhidden.dtype != hidden.dtype:
            raise ValueError("dhidden must have the shape and type of hidden")
        size = hidden.element_size()
        results.append((to_hidden[0], n, v.dim * size, to_hidden[3] * size))
    if dweight is not None:
        to_weight, kind = L._rows(dweight, "dweight"), L._float(dweight, "dweight")
        if dweight.shape != weight.shape or kind not in (v.type, L.CNR_FLOAT_F32):
            raise ValueError("dweight must have the shape of weight and its type, or float32")
        size = dweight.element_size()
        results.append((to_weight[0], v.vocab, v.dim * size, to_weight[3] * size))
    room = _bytes(workspace)
    if room < cnr_loss_workspace_bytes(n, v.vocab, v.dim, v.type, True, kind):
        raise ValueError("workspace smaller than cnr_loss_workspace_bytes")
    state_at, dloss_at, workspace_at = B._dev(state, F32, "state"), B._dev(dloss, F32, "dloss"), B._dev(workspace, None, "workspace") or 0
    results.append((workspace_at, 1, room, 0))
    _check_apart(results, operands + [(state_at, 1, 4 * n * (1 + 3 * top), 0), (dloss_at, 1, 4 * n, 0)])
    _check((_lib or load()).cnr_vocabulary_loss_backward(
        ctx, ctypes.byref(v), ctypes.byref(t), state_at, dloss_at, to_hidden[0], to_hidden[3], to_weight[0], kind, to_weight[3], int(accumulate), workspace_at, room,
        _stream(stream)), "cnr_vocabulary_loss_backward")
    L._written(dhidden, dweight)


def cnr_top_logits(ctx, logits, top: int, tokens=None, values=None, lse=None, stream=None) -> None:
    """``logits``: a matrix; ``tokens`` and ``values``: room for ``top`` entries of each row, or None."""
    at, n, vocab, stride = L._rows(logits, "logits")
    kind = L._float(logits, "logits")
    if not 0 <= top <= CNR_LOSS_MAX_TOP:
        raise ValueError("at most %d entries a row" % CNR_LOSS_MAX_TOP)
    tokens_at, values_at, lse_at = L._listed(tokens, n * top, U32, "tokens") or 0, L._listed(values, n * top, logits.dtype, "values") or 0, L._listed(lse, n, F32, "lse") or 0
    size = 4 if kind == L.CNR_FLOAT_F32 else 2
    _check_apart([(tokens_at, 1, 4 * n * top if tokens_at else 0, 0), (values_at, 1, size * n * top if values_at else 0, 0), (lse_at, 1, 4 * n if lse_at else 0, 0)],
                 [(at, n, vocab * size, stride * size)])
    _check((_lib or load()).cnr_top_logits(ctx, at, stride, kind, n, vocab, top, tokens_at, values_at, lse_at, _stream(stream)), "cnr_top_logits")
    L._written(tokens, values, lse)
