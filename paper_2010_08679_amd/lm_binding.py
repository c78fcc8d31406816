"""ctypes binding of ``include/cnr_lm.h``: argument marshalling only, as in :mod:`binding`.

The calls themselves go through the extension of :mod:`binding` where everything is in order; where it is missing, or
leaves a call to the general way below, the checks are made and refused here.

Matrices are two-dimensional tensors whose rows may lie further apart than they are long; the sizes, the strides and the
element type that the C side takes are read off the tensors, everything else has the name and the
order of the C declaration.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B
from .binding import CNR_IDX_I32, CNR_IDX_I64, U8, U32, U64, F32, _check, _stream

CNR_FLOAT_F32, CNR_FLOAT_BF16, CNR_FLOAT_F16 = 0, 1, 2
CNR_SCALE_E8M0, CNR_SCALE_F32 = 0, 1
CNR_BLOCK_ROW, CNR_BLOCK_TILE = 0, 1
CNR_BLOCK = 128
CNR_LM_MAX_SIZE = 2147483647

# Every symbol include/cnr_lm.h declares.
LM_EXPORTS = (
    "cnr_block_row_bytes", "cnr_block_scale_stride", "cnr_block_scale_count", "cnr_quantize_blocks",
    "cnr_block_product_workspace_bytes", "cnr_block_product", "cnr_count_tokens", "cnr_adjust_logits",
)

__all__ = [*LM_EXPORTS, "cnr_adjustments", "LM_EXPORTS", "CNR_FLOAT_F32", "CNR_FLOAT_BF16", "CNR_FLOAT_F16", "CNR_SCALE_E8M0", "CNR_SCALE_F32",
           "CNR_BLOCK_ROW", "CNR_BLOCK_TILE", "CNR_BLOCK", "CNR_LM_MAX_SIZE"]

_FLOATS = {torch.float32: CNR_FLOAT_F32, torch.bfloat16: CNR_FLOAT_BF16, torch.float16: CNR_FLOAT_F16}
_SCALES = {torch.uint8: CNR_SCALE_E8M0, torch.float32: CNR_SCALE_F32}
_INDICES = {torch.int32: CNR_IDX_I32, torch.int64: CNR_IDX_I64}


class cnr_adjustments(ctypes.Structure):
    """Field for field the C struct."""
    _fields_ = [("seen", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("n_slots", ctypes.c_uint64), ("slots", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p), ("presence", ctypes.c_void_p),
                ("bias_offsets", ctypes.c_void_p), ("bias_tokens", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("n_bias", ctypes.c_uint64), ("masks", ctypes.c_void_p), ("n_masks", ctypes.c_uint64), ("mask_of", ctypes.c_void_p)]


_lib = None


def _no_call(*args):
    """In place of the extension's calls: the general way has to look."""


_quantize = _product = _count = _adjust = _no_call


def load() -> ctypes.CDLL:
    """The library of :func:`binding.load`, with this header's functions bound."""
    global _lib, _quantize, _product, _count, _adjust
    if _lib is None:
        lib = B.load()
        vp, u64, i32, sz = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int, ctypes.c_size_t
        sig = {
            "cnr_block_row_bytes": (sz, [u64]),
            "cnr_block_scale_stride": (sz, [u64, i32]),
            "cnr_block_scale_count": (sz, [u64, u64, i32]),
            "cnr_quantize_blocks": (i32, [vp, vp, i32, u64, u64, u64, i32, i32, vp, vp, vp, vp, vp]),
            "cnr_block_product_workspace_bytes": (sz, [vp, u64, u64, u64]),
            "cnr_block_product": (i32, [vp, vp, vp, i32, u64, vp, vp, i32, u64, u64, i32, vp, i32, u64, i32, vp, vp]),
            "cnr_count_tokens": (i32, [vp, vp, vp, u64, u64, vp, u64, i32, vp, vp, u64, i32, i32, vp]),
            "cnr_adjust_logits": (i32, [vp, vp, u64, vp, u64, i32, u64, u64, ctypes.POINTER(cnr_adjustments), vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        if B._extension is not None:
            m = B._extension
            m.set_lm(*(ctypes.cast(getattr(lib, name), vp).value for name in (
                "cnr_quantize_blocks", "cnr_block_product_workspace_bytes", "cnr_block_product", "cnr_count_tokens", "cnr_adjust_logits")), _stream)
            _quantize, _product, _count, _adjust = m.quantize_blocks, m.block_product, m.count_tokens, m.adjust_logits
        _lib = lib
    return _lib


def cnr_block_row_bytes(dim: int) -> int:
    return int(load().cnr_block_row_bytes(dim))


def cnr_block_scale_stride(n_rows: int, kind: int) -> int:
    return int(load().cnr_block_scale_stride(n_rows, kind))


def cnr_block_scale_count(n_rows: int, dim: int, kind: int) -> int:
    return int(load().cnr_block_scale_count(n_rows, dim, kind))


def _rows(t, name: str):
    """(address, rows, columns, elements from one row to the next) of a matrix on the GPU whose rows are contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a tensor on the GPU" % name)
    if t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    rows, cols = t.shape
    step, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError("the rows of %s must be contiguous" % name)
    if rows <= 1:
        step = cols
    elif step < cols:
        raise ValueError("the rows of %s overlap" % name)
    return t.data_ptr(), rows, cols, step


def _kind(table, t, name: str, names: str) -> int:
    try:
        return table[t.dtype]
    except KeyError:
        raise TypeError("%s must be %s, got %s" % (name, names, t.dtype)) from None


def _float(t, name: str) -> int:
    return _kind(_FLOATS, t, name, "float32, bfloat16 or float16")


def _written(*tensors) -> None:
    """Autograd learns that these were written, as of torch's operations in place: what a graph has saved of them is not taken for unchanged."""
    torch.autograd.graph.increment_version([t for t in tensors if t is not None])


def _listed(t, n: int, dtype, name: str) -> int:
    """Address of a list with room for n entries; 0 for None."""
    if t is not None and t.numel() < n:
        raise ValueError("%s shorter than %d" % (name, n))
    return B._dev(t, dtype, name)


def _blocked(codes, scale, n_rows: int, dim: int, kind: int, scale_type: int, name: str):
    """Addresses of a blocked matrix's two buffers."""
    across, stride = (dim + 127) // CNR_BLOCK, (n_rows + 127) // CNR_BLOCK
    if kind == CNR_BLOCK_ROW:
        stride *= CNR_BLOCK
    elif kind != CNR_BLOCK_TILE:
        raise ValueError("the kind of %s must be CNR_BLOCK_ROW or CNR_BLOCK_TILE" % name)
    if codes is None or scale is None or codes.numel() < n_rows * across * CNR_BLOCK or scale.numel() < across * stride:
        raise ValueError("codes or scale of %s missing or shorter than its size" % name)
    return B._dev(codes, U8, "the codes of " + name), B._dev(scale, F32 if scale_type else U8, "the scale of " + name)


def cnr_quantize_blocks(ctx, x, kind: int, scale_type: int, codes, scale, codes_t=None, scale_t=None, stream=None) -> None:
    """``x``: a matrix of float32, bfloat16 or float16."""
    status = _quantize(ctx, x, kind, scale_type, codes, scale, codes_t, scale_t, stream)
    if status is not None:
        return _check(status, "cnr_quantize_blocks")
    at, n_rows, dim, stride = _rows(x, "x")
    direct = _blocked(codes, scale, n_rows, dim, kind, scale_type, "the quantized x") if codes is not None or scale is not None else (0, 0)
    turned = _blocked(codes_t, scale_t, dim, n_rows, kind, scale_type, "x's transpose") if codes_t is not None or scale_t is not None else (0, 0)
    _check((_lib or load()).cnr_quantize_blocks(ctx, at, _float(x, "x"), n_rows, dim, stride, kind, scale_type, *direct, *turned, _stream(stream)),
           "cnr_quantize_blocks")
    _written(codes, scale, codes_t, scale_t)


def cnr_block_product_workspace_bytes(ctx, m: int, n: int, k: int) -> int:
    return int(load().cnr_block_product_workspace_bytes(ctx, m, n, k))


def cnr_block_product(ctx, a_codes, a_scale, a_kind: int, m: int, b_codes, b_scale, b_kind: int, n: int, k: int, out,
                      accumulate: bool = False, workspace=None, stream=None) -> None:
    """``out``: a matrix of at least m x n, float32, bfloat16 or float16."""
    status = _product(ctx, a_codes, a_scale, a_kind, m, b_codes, b_scale, b_kind, n, k, out, accumulate, workspace, stream)
    if status is not None:
        return _check(status, "cnr_block_product")
    scale_type = _kind(_SCALES, a_scale, "a_scale", "uint8 or float32")
    a = _blocked(a_codes, a_scale, m, k, a_kind, scale_type, "A")
    b = _blocked(b_codes, b_scale, n, k, b_kind, scale_type, "B")
    to, rows, columns, stride = _rows(out, "out")
    if rows < m or columns < n:
        raise ValueError("out smaller than m x n")
    if workspace is not None and workspace.numel() * workspace.element_size() < cnr_block_product_workspace_bytes(ctx, m, n, k):
        raise ValueError("workspace smaller than cnr_block_product_workspace_bytes")
    _check((_lib or load()).cnr_block_product(ctx, *a, a_kind, m, *b, b_kind, n, k, scale_type, to, _float(out, "out"), stride,
                                    int(accumulate), B._dev(workspace, None, "workspace"), _stream(stream)), "cnr_block_product")
    _written(out)


def cnr_count_tokens(ctx, seen, counts, n_slots: int, vocab: int, tokens, offsets=None, slots=None, prompt: bool = False,
                     restart: bool = False, stream=None) -> None:
    """The sequences are as many as ``offsets`` has entries, less one; without it, as there are tokens."""
    status = _count(ctx, seen, counts, n_slots, vocab, tokens, offsets, slots, prompt, restart, stream)
    if status is not None:
        return _check(status, "cnr_count_tokens")
    n = tokens.numel() if offsets is None else offsets.numel() - 1
    if n < 0:
        raise ValueError("offsets must hold at least one entry")
    _check((_lib or load()).cnr_count_tokens(ctx, _listed(seen, n_slots * ((vocab + 31) // 32), U32, "seen"), _listed(counts, n_slots * vocab, U32, "counts"),
                                   n_slots, vocab, B._dev(tokens, None, "tokens"), tokens.numel(),
                                   _kind(_INDICES, tokens, "tokens", "int32 or int64"), B._dev(offsets, U64, "offsets"),
                                   _listed(slots, n, U32, "slots"), n, int(prompt), int(restart), _stream(stream)), "cnr_count_tokens")
    _written(seen, counts)


def cnr_adjust_logits(ctx, logits, out, seen=None, counts=None, n_slots: int = 0, slots=None, repetition=None, frequency=None, presence=None,
                      bias_offsets=None, bias_tokens=None, bias_values=None, masks=None, n_masks: int = 0, mask_of=None,
                      stream=None) -> None:
    """``logits`` and ``out``: matrices of one type and size, or one and the same."""
    status = _adjust(ctx, logits, out, seen, counts, n_slots, slots, repetition, frequency, presence, bias_offsets, bias_tokens, bias_values, masks, n_masks,
                     mask_of, stream)
    if status is not None:
        return _check(status, "cnr_adjust_logits")
    at, n, vocab, stride = _rows(logits, "logits")
    to, rows, columns, out_stride = _rows(out, "out")
    if rows != n or columns != vocab or out.dtype != logits.dtype:
        raise ValueError("out must have the shape and type of logits")
    if to != at and to < at + ((n - 1) * stride + vocab) * logits.element_size() and at < to + ((n - 1) * out_stride + vocab) * out.element_size():
        raise ValueError("out overlaps logits without being the same")
    words = (vocab + 31) // 32
    n_bias = 0
    if bias_offsets is not None:
        if bias_tokens is None or bias_values is None or bias_tokens.numel() != bias_values.numel():
            raise ValueError("biases need as many values as tokens")
        n_bias = bias_tokens.numel()
    given = cnr_adjustments(
        _listed(seen, n_slots * words, U32, "seen"), _listed(counts, n_slots * vocab, U32, "counts"), n_slots, _listed(slots, n, U32, "slots"),
        _listed(repetition, n, F32, "repetition"), _listed(frequency, n, F32, "frequency"), _listed(presence, n, F32, "presence"),
        _listed(bias_offsets, n + 1, U64, "bias_offsets"), B._dev(bias_tokens, U32, "bias_tokens"), B._dev(bias_values, F32, "bias_values"), n_bias,
        _listed(masks, n_masks * words, U32, "masks"), n_masks, _listed(mask_of, n, U32, "mask_of"))
    _check((_lib or load()).cnr_adjust_logits(ctx, at, stride, to, out_stride, _float(logits, "logits"), n, vocab, ctypes.byref(given), _stream(stream)),
           "cnr_adjust_logits")
    _written(out)
