"""Operators of a recurrent language model on one MI355X (C ABI in include/gs.h), and a small
model made of them.

Three operators, which one training step of such a model runs between its matrix products:

* the gated linear recurrence ``h_t = a_t h_(t-1) + (1 - a_t) x_t``, ``a = sigmoid(f)``,
  ``y_t = sigmoid(o_t) h_t``: ``recurrence_forward`` / ``recurrence_backward``, or
  ``gated_recurrence`` and ``gated_recurrence_packed`` under autograd. With T = 1 and the state of the
  call before as ``h0`` it serves single tokens;
* dropout whose mask is drawn from a counter and never stored, with the residual sum:
  ``dropout_forward`` / ``dropout_backward``, or ``dropout`` under autograd;
* softmax cross-entropy over a vocabulary: ``cross_entropy_forward`` gives the losses and, in the same pass
  over the logits, their gradient; ``cross_entropy`` under autograd.

Tensors are fp32, bf16 or fp16 CUDA (ROCm) tensors of the current device (states, losses and
statistics fp32); calls run on torch's current stream and do not wait. An output that the caller gives
counts for autograd as changed in place. ``RecurrentLM`` is a language model of these operators; with
``train.GlobalSketchOptimizer`` its P workers' gradients go through the compression step.
"""
from __future__ import annotations

import ctypes

import torch

from . import (GS_BF16, GS_F16, GS_F32, GS_RECURRENCE_BLOCK, GS_RECURRENCE_MAX_STRIDE, GS_RECURRENCE_WHOLE, _check,
               gs_recurrence, gs_rows, gs_xent, load_library)

DTYPES = {torch.float32: GS_F32, torch.bfloat16: GS_BF16, torch.float16: GS_F16}
U64 = (1 << 64) - 1


def _current_stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# the stream's handle without a Stream object around it (2.7 us a call less), where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else _current_stream()


def _activation(t, name: str, dim: int | None = None) -> tuple[int, int]:
    """(the C ABI's type code, the device) of an activation tensor, after its checks."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    code = DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current device")
    if dim is not None and t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions, got {t.dim()}")
    return code, device


def _rows(t, like, device: int, name: str) -> gs_rows:
    """A [B][T][C] tensor whose channels are contiguous, as the C ABI takes it."""
    if t is None:
        return gs_rows(None, 0, 0)
    if not isinstance(t, torch.Tensor) or t.dtype is not like.dtype or t.get_device() != device:
        raise TypeError(f"{name} must be a {like.dtype} tensor on {like.device}")
    shape = t.shape
    if shape != like.shape:
        raise ValueError(f"{name} must have shape {tuple(like.shape)}, got {tuple(shape)}")
    sb, st, sc = t.stride()
    if sc != 1 and shape[2] > 1:
        raise ValueError(f"{name}: channels must be contiguous")
    return gs_rows(t.data_ptr(), sb, st)


def _made(t, like, device: int, name: str):
    """(the tensor, its rows) of an output: the given one, or a new contiguous one."""
    if t is not None:
        _written(t, name)
        return t, _rows(t, like, device, name)
    t = torch.empty_like(like, memory_format=torch.contiguous_format)
    _, T, C = like.shape
    return t, gs_rows(t.data_ptr(), T * C, C)


def _written(t, name: str) -> None:
    """Refuse an output tensor in which two elements share an address (an expanded one)."""
    for n, s in zip(t.shape, t.stride()):
        if n > 1 and s == 0:
            raise ValueError(f"{name} must not be an expanded tensor")


def _wrote(*given) -> None:
    """Count the given outputs as changed in place, as torch's own operations do: a backward pass that needs what a
    tensor held before is then an error."""
    for t in given:
        if t is not None:
            torch.autograd.graph.increment_version(t)


def _side(t, dtype, shape, device: int, name: str):
    """The pointer of a contiguous tensor of the given type and shape on `device` (None: NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype is not dtype:
        raise TypeError(f"{name} must be a {dtype} tensor on cuda:{device}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of shape {shape}, got {tuple(t.shape)}")
    return t.data_ptr()


def _recurrence(x, f, o, h0, lengths):
    code, device = _activation(x, "x", 3)
    B, T, C = x.shape
    r = gs_recurrence(B, T, C, code, _rows(x, x, device, "x"), _rows(f, x, device, "f"), _rows(o, x, device, "o"),
                      _side(lengths, torch.int32, (B,), device, "lengths"),
                      _side(h0, torch.float32, (B, C), device, "h0"))
    work = None
    if T > GS_RECURRENCE_WHOLE:
        n = load_library().gs_recurrence_work(B, T, C, code)
        work = torch.empty(n, dtype=torch.uint8, device=x.device) if n > 0 else None
    return r, device, work


def recurrence_forward(x, f, o=None, h0=None, lengths=None, save: bool = False, y=None, h_last=None):
    """The gated linear recurrence over [B][T][C] tensors: ``(y, h_last, saved)``.

    x, f, o: candidates, forget-gate and output-gate pre-activations, channels contiguous (o may be
    None: y is the state). h0: [B][C] fp32 or None (zero). lengths: int32 [B] or None; positions from
    a sequence's length on are padding: they keep its state and give y = 0. y and h_last ([B][C] fp32, h0
    itself for a step in place) are made unless given and overlap no other input. Strides are free, but with T > 1 a time
    stride is at most GS_RECURRENCE_MAX_STRIDE elements. save: also the states that ``recurrence_backward`` needs."""
    r, device, work = _recurrence(x, f, o, h0, lengths)
    B, T, C = x.shape
    given = (y, h_last)
    y, to = _made(y, x, device, "y")
    if h_last is None:
        h_last = x.new_empty((B, C), dtype=torch.float32)
        last = h_last.data_ptr()
    else:
        last = _side(h_last, torch.float32, (B, C), device, "h_last")
    saved = None
    if save:
        saved = x.new_empty((B, -(-T // GS_RECURRENCE_BLOCK), C), dtype=torch.float32)
    _check(load_library().gs_recurrence_forward(ctypes.byref(r), _stream(device), to, last,
                                                saved.data_ptr() if save else None,
                                                work.data_ptr() if work is not None else None),
           None, "gs_recurrence_forward")
    _wrote(*given)
    return y, h_last, saved


def recurrence_backward(gy, x, f, o, saved, lengths=None, gh=None, dx=None, df=None, do=None):
    """The gradients ``(dx, df, do, dh0)`` of the recurrence. gy: [B][T][C], the gradient of y; gh:
    [B][C] fp32, that of h_last, or None; saved: the forward call's, on the same inputs. dx, df and do are
    made unless given (do is None without o) and overlap no input."""
    r, device, work = _recurrence(x, f, o, None, lengths)
    B, T, C = x.shape

    if o is None and do is not None:
        raise ValueError("do is given but o is not")
    given = (dx, df, do)
    dx, to_x = _made(dx, x, device, "dx")
    df, to_f = _made(df, x, device, "df")
    do, to_o = _made(do, x, device, "do") if o is not None else (None, gs_rows(None, 0, 0))
    dh0 = x.new_empty((B, C), dtype=torch.float32)
    blocks = -(-T // GS_RECURRENCE_BLOCK)
    _check(load_library().gs_recurrence_backward(ctypes.byref(r), _stream(device), _rows(gy, x, device, "gy"),
                                                 _side(gh, torch.float32, (B, C), device, "gh"),
                                                 _side(saved, torch.float32, (B, blocks, C), device, "saved"), to_x,
                                                 to_f, to_o, dh0.data_ptr(),
                                                 work.data_ptr() if work is not None else None),
           None, "gs_recurrence_backward")
    _wrote(*given)
    return dx, df, do, dh0


def _taken(gy):
    """A gradient as autograd hands it over, in a layout that the recurrence takes."""
    _, T, C = gy.shape
    _, st, sc = gy.stride()
    return gy if (sc == 1 or C == 1) and (st <= GS_RECURRENCE_MAX_STRIDE or T == 1) else gy.contiguous()


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, o, h0, lengths):
        y, h_last, saved = recurrence_forward(x, f, o, h0, lengths, save=any(ctx.needs_input_grad))
        ctx.save_for_backward(x, f, o, lengths, saved)
        ctx.set_materialize_grads(False)
        return y, h_last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy, gh):
        x, f, o, lengths, saved = ctx.saved_tensors
        gy = torch.zeros_like(x) if gy is None else gy
        gy = _taken(gy)
        gh = gh.contiguous() if gh is not None else None
        dx, df, do, dh0 = recurrence_backward(gy, x, f, o, saved, lengths, gh)
        return dx, df, do, dh0 if ctx.needs_input_grad[3] else None, None


def _parts(xfo, channels: int):
    """x, f and o (or x and f) of a projection; three of no channels where it has none."""
    return xfo.split(channels, -1) if channels else (xfo, xfo, xfo)


class _PackedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, xfo, channels, h0, lengths):
        parts = _parts(xfo, channels)
        y, h_last, saved = recurrence_forward(parts[0], parts[1], parts[2] if len(parts) == 3 else None, h0, lengths,
                                              save=any(ctx.needs_input_grad))
        ctx.save_for_backward(xfo, lengths, saved)
        ctx.channels = channels
        ctx.set_materialize_grads(False)
        return y, h_last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy, gh):
        xfo, lengths, saved = ctx.saved_tensors
        parts = _parts(xfo, ctx.channels)
        gy = torch.zeros(parts[0].shape, dtype=xfo.dtype, device=xfo.device) if gy is None else gy
        gy = _taken(gy)
        gh = gh.contiguous() if gh is not None else None
        grad = torch.empty(xfo.shape, dtype=xfo.dtype, device=xfo.device)
        to = _parts(grad, ctx.channels)
        gate = len(parts) == 3
        _, _, _, dh0 = recurrence_backward(gy, parts[0], parts[1], parts[2] if gate else None, saved, lengths, gh,
                                           dx=to[0], df=to[1], do=to[2] if gate else None)
        return grad, None, dh0 if ctx.needs_input_grad[2] else None, None


def gated_recurrence(x, f, o=None, h0=None, lengths=None):
    """``recurrence_forward`` under autograd: ``(y, h_last)``."""
    return _Recurrence.apply(x, f, o, h0, lengths)


def gated_recurrence_packed(xfo, channels: int, h0=None, lengths=None):
    """``gated_recurrence`` of a projection [B][T][3 channels] that holds x, f and o side by side (or
    [B][T][2 channels]: no output gate); its gradient is written as one such tensor. ``(y, h_last)``."""
    if xfo.dim() != 3 or xfo.shape[2] not in (2 * channels, 3 * channels):
        raise ValueError(f"xfo must be [B][T][{3 * channels}] or [B][T][{2 * channels}], got {tuple(xfo.shape)}")
    return _PackedRecurrence.apply(xfo, channels, h0, lengths)


def _like(t, x, name: str) -> None:
    if not isinstance(t, torch.Tensor) or t.dtype != x.dtype or t.shape != x.shape or t.device != x.device:
        raise ValueError(f"{name} must be like x in type, shape and device")


def _dropout(x, p, seed, site, step, residual, y):
    code, device = _activation(x, "x")
    if residual is not None:
        _like(residual, x, "residual")
    given = y
    if y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        _like(y, x, "y")
        _written(y, "y")
    if x.is_contiguous() and y.is_contiguous() and (residual is None or residual.is_contiguous()):
        rows, cols = 1, x.numel()
        xs = rs = ys = cols
    else:
        if x.dim() != 2 or any(t.stride(1) != 1 and t.shape[1] > 1 for t in (x, residual, y) if t is not None):
            raise ValueError("x, residual and y must be contiguous, or two-dimensional with contiguous rows")
        rows, cols = x.shape
        xs, ys, rs = x.stride(0), y.stride(0), residual.stride(0) if residual is not None else 0
    _check(load_library().gs_dropout(_stream(device), code, rows, cols, x.data_ptr(), xs,
                                     residual.data_ptr() if residual is not None else None, rs, y.data_ptr(), ys, p,
                                     seed & U64, site & U64, _side(step, torch.int64, (1,), device, "step")),
           None, "gs_dropout")
    _wrote(given)
    return y


def dropout_forward(x, p: float, seed: int, site: int = 0, step=None, residual=None, y=None):
    """``residual + dropout(x)`` (``dropout(x)`` without one), each element kept with probability
    1 - p and scaled by its inverse. The mask is a function of (seed, step, site, element index):
    seed is the program's, site tells its dropouts (and simulated workers) apart, step is an int64 tensor of one element
    on the device (or None: 0) that the program counts up, so a captured graph draws anew on each replay. x is
    contiguous, or two-dimensional with contiguous rows; y is made unless given and may be x or residual."""
    return _dropout(x, p, seed, site, step, residual, y)


def dropout_backward(gy, p: float, seed: int, site: int = 0, step=None, dx=None):
    """The gradient of x: the same mask and factor on gy (the residual's gradient is gy itself)."""
    return _dropout(gy, p, seed, site, step, None, dx)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, site, step, residual):
        ctx.drawn = (p, seed, site)
        ctx.save_for_backward(step)  # a step counted up before the backward pass is an error there
        return dropout_forward(x, p, seed, site, step, residual)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, gy):
        p, seed, site = ctx.drawn
        (step,) = ctx.saved_tensors
        dx = dropout_backward(gy.contiguous(), p, seed, site, step) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, None, gy if ctx.needs_input_grad[5] else None


def dropout(x, p: float, seed: int, site: int = 0, step=None, residual=None):
    """``dropout_forward`` under autograd. step may be counted up only after the backward pass."""
    return _Dropout.apply(x, p, seed, site, step, residual)


def _cross_entropy(logits, targets, ignore_index, losses, mean_loss, grad, factor=1.0, scale=None, mean=False):
    lib = load_library()
    code, device = _activation(logits, "logits", 2)
    N, V = logits.shape
    if logits.stride(1) != 1 and V > 1:
        raise ValueError("logits: rows must be contiguous")
    grad_stride = V
    if grad is not None:
        _like(grad, logits, "grad")
        grad_stride = grad.stride(0)
        if grad.stride(1) != 1 and V > 1:
            raise ValueError("grad: rows must be contiguous")
    n = lib.gs_cross_entropy_work(N, V, code)
    work = torch.empty(n // 8, dtype=torch.int64, device=logits.device) if n > 0 else None
    per_row = int(scale is not None and scale.dim() == 1)
    x = gs_xent(N, V, code, mean, logits.data_ptr(), logits.stride(0),
                _side(targets, torch.int64, (N,), device, "targets"), ignore_index, factor,
                _side(scale, torch.float32, (N,) if per_row else (), device, "scale"), per_row,
                losses.data_ptr() if losses is not None else None,
                mean_loss.data_ptr() if mean_loss is not None else None,
                grad.data_ptr() if grad is not None else None, grad_stride,
                work.data_ptr() if work is not None else None)
    _check(lib.gs_cross_entropy(ctypes.byref(x), _stream(device)), None, "gs_cross_entropy")


def cross_entropy_forward(logits, targets, ignore_index: int = -100, grad=False, factor: float = 1.0):
    """``(mean, losses, dlogits)`` of softmax cross-entropy in one pass over the logits. logits: [N][V], rows
    contiguous; targets: int64 [N], contiguous. mean: fp32 scalar, over the rows whose target is not ignore_index (0 when there is
    none); losses: fp32 [N]. grad: False (dlogits is None), True, or a tensor to write, the logits themselves
    included: the gradient of factor * mean (the factor scales a loss of 16-bit gradients)."""
    out = logits.new_empty(logits.shape[:1], dtype=torch.float32)
    mean = logits.new_empty((), dtype=torch.float32)
    given = None
    if grad is True:
        grad = torch.empty_like(logits, memory_format=torch.contiguous_format)
    elif grad is False:
        grad = None
    else:
        given = grad
    _cross_entropy(logits, targets, ignore_index, out, mean, grad, factor=factor, mean=True)
    _wrote(given)
    return mean, out, grad


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, ignore_index, reduction):
        f32 = dict(dtype=torch.float32, device=logits.device)
        losses = torch.empty((logits.shape[0],), **f32)
        mean = torch.empty((), **f32) if reduction == "mean" else None
        _cross_entropy(logits, targets, ignore_index, losses, mean, None)
        ctx.save_for_backward(logits, targets)
        ctx.how = (ignore_index, reduction)
        return mean if reduction == "mean" else losses

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        logits, targets = ctx.saved_tensors
        ignore_index, reduction = ctx.how
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _cross_entropy(logits, targets, ignore_index, None, None, grad, scale=g.contiguous(),
                       mean=reduction == "mean")
        return grad, None, None, None


def cross_entropy(logits, targets, ignore_index: int = -100, reduction: str = "mean"):
    """Softmax cross-entropy under autograd: the mean over the rows that count ("mean"), or each row's loss
    ("none"). Its backward pass reads the logits again; a program whose loss this is saves that pass with
    ``cross_entropy_forward(..., grad=True)`` and ``logits.backward(dlogits)``."""
    if reduction not in ("mean", "none"):
        raise ValueError("reduction must be 'mean' or 'none'")
    return _CrossEntropy.apply(logits, targets, ignore_index, reduction)


# With fp16 activations RecurrentLM.loss_backward multiplies the loss by a power of two up to the number of tokens, this at
# most: a mean's gradient of the logits, probability / tokens, falls below fp16's smallest number (6e-8) otherwise (2,048
# tokens of 20,000 words: the embedding's gradient 7% off, the biases of words that do not occur 0). The output projection's
# gradients, sums over the tokens, are at most this times the largest activation, against fp16's largest number of 65,504.
HALF_FACTOR = 4096


class _Scaled(torch.autograd.Function):
    """A tensor in another type; its gradient multiplied by a factor, in the tensor's own type."""

    @staticmethod
    def forward(ctx, t, dtype, factor):
        ctx.to = (t.dtype, factor)
        return t.to(dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        dtype, factor = ctx.to
        return g.to(dtype) * factor, None, None


def _scaled(t, factor: float, dtype=None):
    if t is None or (factor == 1.0 and dtype is None):
        return t
    dtype = t.dtype if dtype is None else dtype
    return t.to(dtype) if factor == 1.0 else _Scaled.apply(t, dtype, factor)


class RecurrentLM(torch.nn.Module):
    """A language model of these operators: an embedding, layers of projection, gated recurrence and dropout
    onto a residual stream, and an output projection. Parameters are fp32; activations have type ``dtype``.

    ``step`` (a device buffer) is the dropouts' step: count it up once per optimizer step. ``worker`` tells the
    simulated workers' masks apart. A state is the list of the layers' [B][C] fp32 states."""

    def __init__(self, vocab: int, width: int, layers: int = 1, p: float = 0.1, seed: int = 0,
                 dtype: torch.dtype = torch.float32):
        super().__init__()
        if dtype not in DTYPES:
            raise TypeError("dtype must be float32, bfloat16 or float16")
        self.vocab, self.width, self.p, self.seed, self.dtype = vocab, width, float(p), int(seed), dtype
        self.worker = 0
        self.embedding = torch.nn.Embedding(vocab, width)
        self.inner = torch.nn.ModuleList([torch.nn.Linear(width, 3 * width) for _ in range(layers)])
        self.outer = torch.nn.Linear(width, vocab)
        with torch.no_grad():
            for layer in self.inner:
                layer.bias[width:2 * width] = 1.0  # forget gates start by remembering
        self.register_buffer("step", torch.zeros(1, dtype=torch.int64))

    def _linear(self, layer, u, factor):
        return torch.nn.functional.linear(u, _scaled(layer.weight, 1 / factor, self.dtype),
                                          _scaled(layer.bias, 1 / factor, self.dtype))

    def forward(self, tokens, state=None, lengths=None, factor: float = 1.0):
        """tokens: int64 [B][T]. Returns (logits [B][T][vocab], the state after the tokens). factor: what the logits' gradient
        will come multiplied by (``cross_entropy_forward``'s factor; a power of two costs no rounding). Activations'
        gradients then hold it, those of parameters and states, which are fp32, do not."""
        u = _scaled(self.embedding(tokens), 1 / factor, self.dtype)
        after = []
        for j, layer in enumerate(self.inner):
            before = _scaled(state[j], 1 / factor) if state is not None else None
            y, h = gated_recurrence_packed(self._linear(layer, u, factor), self.width, before, lengths)
            after.append(_scaled(h, factor))
            if self.training and self.p > 0:
                u = dropout(y, self.p, self.seed, self.worker * len(self.inner) + j, self.step, residual=u)
            else:
                u = u + y
        return self._linear(self.outer, u, factor), after

    def loss_backward(self, tokens, targets, ignore_index: int = -100):
        """The mean loss (a detached scalar) of predicting targets ([B][T]); adds its gradient to the parameters. With
        fp16 activations the gradient is held at a power of two times itself (``HALF_FACTOR``) on its way to them."""
        factor = 1.0
        if self.dtype is torch.float16:
            factor = float(min(HALF_FACTOR, 1 << max(0, targets.numel().bit_length() - 1)))
        logits, _ = self(tokens) if factor == 1.0 else self(tokens, factor=factor)
        flat = logits.view(-1, self.vocab)
        mean, _, grad = cross_entropy_forward(flat.detach(), targets.reshape(-1), ignore_index, grad=True, factor=factor)
        flat.backward(grad)
        return mean

    @torch.no_grad()
    def generate(self, tokens, count: int):
        """The `count` likeliest next tokens, one at a time, after tokens ([B][T], T >= 1): int64 [B][count]."""
        was, out = self.training, []
        self.eval()
        try:
            logits, state = self(tokens)
            for _ in range(count):
                out.append(logits[:, -1].argmax(-1))
                logits, state = self(out[-1][:, None], state)
        finally:
            self.train(was)
        return torch.stack(out, 1) if out else tokens[:, :0]
