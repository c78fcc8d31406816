"""Operators for language models over the library's calls (``include/cnr_lm.h``): matrices in 8-bit floating point with
a scale for each block of 128, a linear layer trained and served in them, and the tokens that sequences hold with
what follows from them for their logits.

Plumbing only, as in :mod:`checkpoint`: torch allocates the memory and provides the stream, every step runs in libcnr's
kernels.  A call with ``stream`` is one under ``torch.cuda.stream(stream)``: what it allocates belongs to that stream, what it is
given has to be ready there.
"""
from __future__ import annotations

from contextlib import nullcontext
from dataclasses import dataclass

import torch

from . import lm_binding as L
from . import loss_binding as S


def _on(stream):
    """Memory that a call allocates comes from the stream that it works on: of the current one's it would be handed out while work queued
    there still uses it, and again before `stream` is done."""
    return nullcontext() if stream is None else torch.cuda.stream(stream)


class _Holder:
    """What keeps device memory from one call to the next, made on the current stream and used on the streams that calls name."""

    def _holds(self, tensors) -> None:
        self._held, self._used_on = list(tensors), set()
        self._made_on = next((torch.cuda.current_stream(t.device) for t in self._held if t.is_cuda), None)

    def _hold(self, tensor):
        """One more, allocated by a call."""
        self._held.append(tensor)
        for s in self._used_on:
            tensor.record_stream(s)
        return tensor

    def _use(self, stream) -> None:
        """The first call on a stream lets it wait for what is queued where the memory came from, which that work may still use; freed
        memory is not handed on before that stream is done with it.  (torch begins a capture on an idle GPU; a stream under capture cannot wait for others.)"""
        if stream is None or stream in self._used_on or self._made_on is None:
            return
        with torch.cuda.stream(stream):
            if not torch.cuda.is_current_stream_capturing():
                stream.wait_stream(self._made_on)
        self._used_on.add(stream)
        for t in self._held:
            t.record_stream(stream)


@dataclass
class BlockMatrix:
    """A matrix of n_rows x dim as e4m3 codes and the scales of its blocks (layout in ``include/cnr_lm.h``)."""
    codes: torch.Tensor   # uint8 [n_rows, dim rounded up to a multiple of 128]
    scale: torch.Tensor   # uint8 (powers of two, e8m0) or float32 [ceil(dim / 128), cnr_block_scale_stride(n_rows, kind)]
    n_rows: int
    dim: int
    kind: int = L.CNR_BLOCK_ROW

    @property
    def scale_type(self) -> int:
        return L._kind(L._SCALES, self.scale, "scale", "uint8 or float32")

    @staticmethod
    def empty(n_rows: int, dim: int, kind: int = L.CNR_BLOCK_ROW, scale_type: int = L.CNR_SCALE_E8M0, device="cuda:0") -> "BlockMatrix":
        across, down = -(-dim // L.CNR_BLOCK), -(-n_rows // L.CNR_BLOCK)
        return BlockMatrix(torch.empty(n_rows, across * L.CNR_BLOCK, dtype=torch.uint8, device=device),
                           torch.empty(across, down if kind == L.CNR_BLOCK_TILE else down * L.CNR_BLOCK,
                                       dtype=torch.uint8 if scale_type == L.CNR_SCALE_E8M0 else torch.float32, device=device),
                           n_rows, dim, kind)


def quantize_blocks(ctx, x: torch.Tensor, out: BlockMatrix | None = None, out_t: BlockMatrix | None = None, stream=None) -> BlockMatrix | None:
    """Quantizes the matrix ``x`` into ``out`` and its transpose into ``out_t`` (either may be None; a new matrix of rows' blocks
    with scales of powers of two where both are)."""
    if out is None and out_t is None:
        with _on(stream):
            out = BlockMatrix.empty(*x.shape, device=x.device)
    like = out if out is not None else out_t
    n_rows, dim = x.shape
    if ((out is not None and (out.n_rows != n_rows or out.dim != dim))
            or (out_t is not None and (out_t.n_rows != dim or out_t.dim != n_rows or out_t.kind != like.kind or out_t.scale.dtype != like.scale.dtype))):
        raise ValueError("a blocked matrix of another size, kind or scale type")
    codes, scale = (out.codes, out.scale) if out is not None else (None, None)
    codes_t, scale_t = (out_t.codes, out_t.scale) if out_t is not None else (None, None)
    L.cnr_quantize_blocks(ctx, x, like.kind, like.scale_type, codes, scale, codes_t, scale_t, stream)
    return out


def block_workspace(ctx, m: int, n: int, k: int, device="cuda:0") -> torch.Tensor | None:
    """What :func:`block_product` may use for a product of these sizes; None where it has no use for any."""
    size = L.cnr_block_product_workspace_bytes(ctx, m, n, k)
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


def block_product(ctx, a: BlockMatrix, b: BlockMatrix, out: torch.Tensor | None = None, accumulate: bool = False,
                  workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """``a`` times the transpose of ``b``, written to or added to ``out`` (a new bfloat16 matrix when None).

    A float32 ``out`` holds sums added up in fp32.  16-bit ones are added up by the 8-bit matrix instructions: off by up to 2^-10 of the sum of the
    products' magnitudes, which is below their rounding unless products cancel."""
    if a.dim != b.dim:
        raise ValueError("rows of %d and of %d columns" % (a.dim, b.dim))
    if out is None:
        if accumulate:
            raise ValueError("nothing to add to")
        with _on(stream):
            out = torch.empty(a.n_rows, b.n_rows, dtype=torch.bfloat16, device=a.codes.device)
    elif out.shape != (a.n_rows, b.n_rows):
        raise ValueError("out must be %d x %d" % (a.n_rows, b.n_rows))
    L.cnr_block_product(ctx, a.codes, a.scale, a.kind, a.n_rows, b.codes, b.scale, b.kind, b.n_rows, a.dim, out, accumulate, workspace, stream)
    return out


class BlockLinear(_Holder):
    """y = x W^T in 8 bits, forward and backward, for up to max_tokens rows of x at a time.

    The layer keeps the weight in tiles in both directions (:meth:`load`, after every change of the weight) and, from :meth:`forward` to
    :meth:`backward`, the transpose of its input.  Outputs and input gradients of 16 bits and float32 ones differ in how they are added up, see
    :func:`block_product`; the weight's gradient is float32 unless given otherwise.  It is no autograd function: its results have no history,
    gradients are what :meth:`backward` returns.  A second :meth:`forward` takes the place of the first.  Calls of one layer belong on one stream."""

    def __init__(self, ctx, n_out: int, n_in: int, max_tokens: int, scale_type: int = L.CNR_SCALE_E8M0, device="cuda:0"):
        self.ctx, self.n_out, self.n_in, self.max_tokens, self.scale_type = ctx, int(n_out), int(n_in), int(max_tokens), scale_type
        self.device = torch.device(device)
        self.weight = BlockMatrix.empty(n_out, n_in, L.CNR_BLOCK_TILE, scale_type, device)
        self.weight_t = BlockMatrix.empty(n_in, n_out, L.CNR_BLOCK_TILE, scale_type, device)
        self._x, self._x_t = self._buffers(max_tokens, n_in), self._buffers(n_in, max_tokens)
        self._dy, self._dy_t = self._buffers(max_tokens, n_out), self._buffers(n_out, max_tokens)
        self._input_t = None
        self._sized = {}
        self._spaces = []  # workspaces, the last one the largest; earlier ones stay, since captured graphs may hold them
        self._holds((self.weight.codes, self.weight.scale, self.weight_t.codes, self.weight_t.scale, *self._x, *self._x_t, *self._dy, *self._dy_t))

    def _buffers(self, n_rows: int, dim: int):
        m = BlockMatrix.empty(n_rows, dim, L.CNR_BLOCK_ROW, self.scale_type, self.device)
        return m.codes.view(-1), m.scale.view(-1)

    def _of(self, buffers, n_rows: int, dim: int) -> BlockMatrix:
        across, stride = -(-dim // L.CNR_BLOCK), -(-n_rows // L.CNR_BLOCK) * L.CNR_BLOCK
        codes, scale = buffers
        return BlockMatrix(codes[: n_rows * across * L.CNR_BLOCK].view(n_rows, across * L.CNR_BLOCK), scale[: across * stride].view(across, stride),
                           n_rows, dim, L.CNR_BLOCK_ROW)

    def _for(self, tokens: int, stream=None):
        """Input and output gradient of that many tokens within the layer's buffers, and a workspace for their products."""
        if tokens > self.max_tokens:
            raise ValueError("%d tokens, the layer was made for %d" % (tokens, self.max_tokens))
        if tokens not in self._sized:
            space = max(L.cnr_block_product_workspace_bytes(self.ctx, *s) for s in (
                (tokens, self.n_out, self.n_in), (tokens, self.n_in, self.n_out), (self.n_out, self.n_in, tokens)))
            had = self._spaces[-1].numel() if self._spaces else 0
            if space > had:
                with _on(stream):
                    self._spaces.append(self._hold(torch.empty(max(space, 2 * had), dtype=torch.uint8, device=self.device)))
            self._sized = {tokens: (self._of(self._x, tokens, self.n_in), self._of(self._x_t, self.n_in, tokens),
                                    self._of(self._dy, tokens, self.n_out), self._of(self._dy_t, self.n_out, tokens),
                                    self._spaces[-1] if space else None)}
        return self._sized[tokens]

    def load(self, weight: torch.Tensor, stream=None) -> None:
        """Takes the weight [n_out, n_in] as it is now."""
        self._use(stream)
        quantize_blocks(self.ctx, weight, self.weight, self.weight_t, stream)

    def forward(self, x: torch.Tensor, out: torch.Tensor | None = None, training: bool = True, stream=None) -> torch.Tensor:
        """x [tokens, n_in] -> [tokens, n_out], of x's type when ``out`` is None; ``training``: :meth:`backward` follows."""
        self._use(stream)
        qx, qx_t, _, _, space = self._for(x.shape[0], stream)
        quantize_blocks(self.ctx, x, qx, qx_t if training else None, stream)
        self._input_t = qx_t if training else None
        if out is None:
            with _on(stream):
                out = torch.empty(x.shape[0], self.n_out, dtype=x.dtype, device=self.device)
        return block_product(self.ctx, qx, self.weight, out, workspace=space, stream=stream)

    def backward(self, dy: torch.Tensor, dx: torch.Tensor | None = None, dw: torch.Tensor | None = None, accumulate: bool = False, stream=None):
        """The gradients (dx of dy's type, dw in float32 unless given) of the last :meth:`forward`'s input and of the weight, the latter
        added to ``dw`` where ``accumulate`` is set."""
        if self._input_t is None or self._input_t.dim != dy.shape[0]:
            raise ValueError("no forward pass of %d tokens in training precedes" % dy.shape[0])
        if dw is None and accumulate:
            raise ValueError("nothing to add to")
        self._use(stream)
        _, _, qdy, qdy_t, space = self._for(dy.shape[0], stream)
        quantize_blocks(self.ctx, dy, qdy, qdy_t, stream)
        with _on(stream):
            if dx is None:
                dx = torch.empty(dy.shape[0], self.n_in, dtype=dy.dtype, device=self.device)
            if dw is None:
                dw = torch.empty(self.n_out, self.n_in, dtype=torch.float32, device=self.device)
        block_product(self.ctx, qdy, self.weight_t, dx, workspace=space, stream=stream)
        block_product(self.ctx, qdy_t, self._input_t, dw, accumulate, space, stream)
        return dx, dw


class TokenLedger(_Holder):
    """The tokens of up to n_slots sequences: which of the vocabulary each has seen (a bitmap, as a table's tracking bitmap) and
    how often the model wrote each."""

    def __init__(self, ctx, n_slots: int, vocab: int, seen: torch.Tensor | None = None, counts: torch.Tensor | None = None, device="cuda:0"):
        self.ctx, self.n_slots, self.vocab = ctx, int(n_slots), int(vocab)
        words = (self.vocab + 31) // 32
        self.seen = torch.zeros(n_slots, words, dtype=torch.int32, device=device) if seen is None else seen
        self.counts = torch.zeros(n_slots, vocab, dtype=torch.int32, device=device) if counts is None and seen is None else counts
        for t, width, name in ((self.seen, words, "seen"), (self.counts, self.vocab, "counts")):
            if t is not None and t.dim() > 1 and t.shape[-1] != width:
                raise ValueError("the rows of %s hold %d entries, not %d" % (name, width, t.shape[-1]))
        self._holds([t for t, given in ((self.seen, seen), (self.counts, counts)) if given is None and t is not None])

    def count(self, tokens: torch.Tensor, offsets: torch.Tensor | None = None, slots: torch.Tensor | None = None, prompt: bool = False,
              restart: bool = False, stream=None) -> None:
        """Enters one token of each sequence, or those that ``offsets`` gives each; ``restart`` empties the slots first."""
        self._use(stream)
        L.cnr_count_tokens(self.ctx, self.seen, self.counts, self.n_slots, self.vocab, tokens, offsets, slots, prompt, restart, stream)

    def adjust(self, logits: torch.Tensor, out: torch.Tensor | None = None, slots: torch.Tensor | None = None, repetition=None, frequency=None,
               presence=None, bias=None, masks: torch.Tensor | None = None, mask_of: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Applies penalties (float32 [n] each), biases (offsets, tokens, values) and masks to ``logits`` [n, vocab], in place when ``out``
        is None."""
        if logits.shape[1] != self.vocab:
            raise ValueError("logits of %d tokens, a vocabulary of %d" % (logits.shape[1], self.vocab))
        if masks is not None and (masks.dim() != 2 or masks.shape[1] != (self.vocab + 31) // 32):
            raise ValueError("masks must be [n_masks, %d]" % ((self.vocab + 31) // 32))
        self._use(stream)
        out = logits if out is None else out
        penalties = repetition is not None or frequency is not None or presence is not None
        seen, counts = (self.seen, self.counts) if penalties else (None, None)
        L.cnr_adjust_logits(self.ctx, logits, out, seen, counts, self.n_slots if penalties else 0, slots, repetition, frequency, presence,
                            *(bias if bias is not None else (None, None, None)), masks, 0 if masks is None else masks.shape[0], mask_of, stream)
        return out


class VocabularyLoss(_Holder):
    """Losses of the matrix that gives the logits, ``hidden`` [n, dim] times the transpose of ``weight`` [vocab, dim], for up to max_tokens rows at a time
    and without all logits in memory: softmax cross entropy, and distillation from up to ``top`` logits a row of a teacher.

    The object keeps a workspace and, from a loss in training to :meth:`backward`, what that loss was made of: its tensors must stay as they are until then.
    ``gradient_dtype``: the type of the weight's gradient, ``dtype`` or float32 (which costs a second product where ``dtype`` has 16 bits, a third for up to 128 rows of bfloat16).
    It is no autograd function: results have no history, gradients are what :meth:`backward` returns.  A second loss in training, or any distillation, takes the
    place of the first; a call that is refused does not.
    Calls of one object belong on one stream."""

    def __init__(self, ctx, vocab: int, dim: int, max_tokens: int, dtype=torch.bfloat16, top: int = 1, training: bool = True, gradient_dtype=None, device="cuda:0"):
        self.ctx, self.vocab, self.dim, self.max_tokens, self.top = ctx, int(vocab), int(dim), int(max_tokens), int(top)
        self.dtype, self.gradient_dtype, self.device = dtype, dtype if gradient_dtype is None else gradient_dtype, torch.device(device)
        if dtype not in L._FLOATS or self.gradient_dtype not in (dtype, torch.float32):
            raise TypeError("losses of float32, bfloat16 or float16, gradients of the weight in that type or float32")
        if not 1 <= self.top <= S.CNR_LOSS_MAX_TOP:
            raise ValueError("1 to %d entries a row" % S.CNR_LOSS_MAX_TOP)
        for size, most, name in ((self.max_tokens, S.CNR_LOSS_MAX_ROWS, "max_tokens"), (self.vocab, S.CNR_LOSS_MAX_VOCABULARY, "vocab"), (self.dim, S.CNR_LOSS_MAX_DIM, "dim")):
            if not 0 <= size <= most:
                raise ValueError("%s must be 0 to %d" % (name, most))
        space = S.cnr_loss_workspace_bytes(self.max_tokens, self.vocab, self.dim, L._FLOATS[dtype], training, L._FLOATS[self.gradient_dtype])
        self._space = torch.empty(space, dtype=torch.uint8, device=self.device)
        self._state = torch.empty(S.cnr_loss_state_floats(self.max_tokens, self.top), dtype=torch.float32, device=self.device)
        self.training = bool(training)
        self._last = None
        self._holds((self._space, self._state))

    def _loss(self, hidden, weight, tokens, logits, temperature, out, training, stream):
        if hidden.dim() != 2 or hidden.shape[1] != self.dim or tuple(weight.shape) != (self.vocab, self.dim):
            raise ValueError("hidden states of %d columns and a weight of %d x %d" % (self.dim, self.vocab, self.dim))
        if hidden.dtype != self.dtype:
            raise TypeError("hidden must be %s, got %s" % (self.dtype, hidden.dtype))
        if hidden.shape[0] > self.max_tokens:
            raise ValueError("%d tokens, made for %d" % (hidden.shape[0], self.max_tokens))
        if training and not self.training:
            raise ValueError("made without training")
        self._use(stream)
        if out is None:
            with _on(stream):
                out = torch.empty(hidden.shape[0], dtype=torch.float32, device=hidden.device)
        state, last = self._state if training or logits is not None else None, self._last
        if state is not None:  # another's from here on
            self._last = None
        try:
            S.cnr_vocabulary_loss(self.ctx, hidden, weight, tokens, logits, temperature, out, state, self._space, stream)
        except (TypeError, ValueError):  # refused: nothing was written
            self._last = last
            raise
        if training:
            self._last = (hidden, weight, tokens, logits, temperature)
        return out

    def cross_entropy(self, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, out: torch.Tensor | None = None, training: bool = True,
                      stream=None) -> torch.Tensor:
        """Each row's loss (float32 [n]) for its target; 0 for negative ones, which are padding.  ``training``: :meth:`backward` follows."""
        return self._loss(hidden, weight, targets, None, 1.0, out, training, stream)

    def distill(self, hidden: torch.Tensor, weight: torch.Tensor, tokens: torch.Tensor, logits: torch.Tensor, temperature: float = 1.0,
                out: torch.Tensor | None = None, training: bool = True, stream=None) -> torch.Tensor:
        """Each row's divergence from a teacher whose top logits are ``logits`` [n, k] of ``tokens`` [n, k] (negative: none), both divided by
        the temperature.  Gradients shrink with the temperature's square, which ``backward``'s argument can make up for."""
        if tokens.dim() != 2 or tokens.shape[1] > self.top:
            raise ValueError("tokens must be a matrix of up to %d columns" % self.top)
        return self._loss(hidden, weight, tokens, logits, temperature, out, training, stream)

    def backward(self, dloss: torch.Tensor, dhidden: torch.Tensor | None = None, dweight: torch.Tensor | None = None, accumulate: bool = False,
                 hidden: bool = True, weight: bool = True, stream=None):
        """The gradients (dhidden, dweight) of the last loss in training, dloss (float32 [n]) times each row's, the weight's added to ``dweight`` where
        ``accumulate`` is set; None in the place of one that is not wanted."""
        if self._last is None:
            raise ValueError("no loss in training precedes")
        x, w = self._last[:2]
        if accumulate and (dweight is None or not weight):
            raise ValueError("nothing to add to")
        if weight and dweight is not None and dweight.dtype != self.gradient_dtype:
            raise TypeError("dweight must be %s, got %s" % (self.gradient_dtype, dweight.dtype))
        self._use(stream)
        with _on(stream):
            if hidden and dhidden is None:
                dhidden = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            if weight and dweight is None:
                dweight = torch.empty(w.shape, dtype=self.gradient_dtype, device=w.device)
        dhidden, dweight = dhidden if hidden else None, dweight if weight else None
        S.cnr_vocabulary_loss_backward(self.ctx, *self._last, self._state, dloss, dhidden, dweight, accumulate, self._space, stream)
        return dhidden, dweight


def top_logits(ctx, logits: torch.Tensor, top: int, tokens: torch.Tensor | None = None, values: torch.Tensor | None = None, lse: torch.Tensor | None = None, stream=None):
    """The ``top`` largest of each row of ``logits`` [n, vocab], largest first and the lower token first of equal ones: (tokens int32 [n, top], their logits,
    float32 [n] the logarithm of the sum of all exponentials).  What they are written to may be given."""
    n = logits.shape[0]
    with _on(stream):
        tokens = torch.empty(n, top, dtype=torch.int32, device=logits.device) if tokens is None else tokens
        values = torch.empty(n, top, dtype=logits.dtype, device=logits.device) if values is None else values
        lse = torch.empty(n, dtype=torch.float32, device=logits.device) if lse is None else lse
    S.cnr_top_logits(ctx, logits, top, tokens, values, lse, stream)
    return tokens, values, lse
