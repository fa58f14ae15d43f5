"""Operators of the training steps between two synchronisations.

Holders of the device tensors (torch) that the library's training-operator
contexts borrow, in the manner of :class:`binding.Swarm`: they check arguments,
allocate workspaces and outputs, and forward to the C entry points; every
computation runs in the CUDA library.

  LinearXent   softmax cross entropy of a linear head without keeping the logits,
               with its gradients; its loss alone is a worker's fitness
  Attention    causal attention over packed sequences, with grouped heads and a learned
               bias by buckets of the distance, with its gradients
  Keep8        activations kept in 8 bits for the backward pass, and the (gated) activation
               whose backward pass reads them
  AdamW        one AdamW step over many tensors, moments in 32 or in 8 bits
  GradNorm     2-norm of many gradients and the factor that clips it

Calls enqueue on the current stream of the holder's GPU, or always on the one
given when it is made; a call on another stream than the one before comes after
it.  A given stream waits in each call for what the current one has been given
so far, and tensors that are let go of meanwhile are kept from other uses until
it is done with them; its results are the caller's to wait for, but for the
differentiable call, whose results the current stream waits for.  Inside a stream
capture nothing of this is recorded: there the caller orders the two.  Tensors that
were produced on yet another stream have to be ordered before the call by the
caller, as for any kernel.
"""
from __future__ import annotations

import ctypes
import math
import threading
import weakref

import torch
from torch.multiprocessing.reductions import StorageWeakRef

from . import binding
from .binding import (PSOPS_ATTENTION_GRADS, PSOPS_BF16, PSOPS_GELU, PSOPS_RELU, PSOPS_SILU, PSOPS_EINVAL, PSOPS_ESTATE, PSOPS_F16, PSOPS_F32, PSOPS_MEAN, PSOPS_NONE,
                      PSOPS_PER_TOKEN, PSOPS_SUM, PSOPS_XENT_GRADS, PSOPS_XENT_STAGED, PsopsError)

_TYPES = {torch.float32: PSOPS_F32, torch.float16: PSOPS_F16, torch.bfloat16: PSOPS_BF16}
_REDUCTIONS = {"mean": PSOPS_MEAN, "sum": PSOPS_SUM, "none": PSOPS_PER_TOKEN}
_KINDS = {"relu": PSOPS_RELU, "silu": PSOPS_SILU, "gelu": PSOPS_GELU}
KEPT_BLOCK = 128                 # elements of a row that share one scale of a kept activation
MOMENT_BLOCK = 256               # elements that share one scale of an 8-bit moment

# The kernels write through addresses, which autograd does not see: what they change in a caller's tensor is told
# it here, so that a backward pass that had saved the tensor raises an error as it does after torch's own operations.
_changed = torch.autograd.graph.increment_version


def _refuse(where: str, why: str):
    raise PsopsError(PSOPS_EINVAL, where, why)


def _flat_list(where, what, tensors, dtypes, device, count=None, sizes=None):
    """A list of contiguous device tensors of one of `dtypes`."""
    tensors = list(tensors)
    if count is not None and len(tensors) != count:
        _refuse(where, f"{len(tensors)} tensors in `{what}`, {count} parameters")
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor) or t.device != device:
            _refuse(where, f"{what}[{i}] is not a tensor on {device}")
        if t.dtype not in dtypes:
            _refuse(where, f"{what}[{i}] is {t.dtype}, not one of {[str(d) for d in dtypes]}")
        if not t.is_contiguous():
            _refuse(where, f"{what}[{i}] is not contiguous")
        if sizes is not None and t.numel() != sizes[i]:
            _refuse(where, f"{what}[{i}] has {t.numel()} elements, not {sizes[i]}")
    return tensors


def _device_of(where, tensors):
    if not tensors:
        _refuse(where, "no tensors")
    t = tensors[0]
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(where, "the tensors have to be on a GPU")
    return t.device


def _is_capturing(stream):
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Exactly(threading.local):
    """Around an operation that saves statistics of its inputs beside them: Keep8.hooks leaves these inputs alone, since
    with others the statistics would be wrong (probabilities that do not sum to 1, beyond a 16-bit type's range even)."""

    depth = 0

    def __enter__(self):
        self.depth += 1

    def __exit__(self, *error):
        self.depth -= 1


_exactly = _Exactly()


class _Holder:
    """What the holders have in common: a context, its GPU and the stream its work goes to."""

    ctx = None

    def _on(self, device, stream):
        self.device = device
        self._follows = stream is None
        self.stream = torch.cuda.current_stream(device).cuda_stream if stream is None else int(stream)
        return self.stream

    def _follow(self, *tensors):
        """Moves the context to the current stream; one that was given its stream lets that wait for the current one, and
        has `tensors`, the ones of the call that the holder does not keep, not used for anything else before it is done."""
        now = torch._C._cuda_getCurrentRawStream(self.device.index)
        if now == self.stream:
            return
        if self._follows:
            if self.ctx is not None:
                self._move(now)
            self.stream = now
            return
        self._order(to_own=True)
        own = self._own()
        for t in tensors:
            if t is not None:
                t.record_stream(own)

    def _move(self, stream):
        self._set_stream(self.ctx, stream)

    def _own(self):
        return torch.cuda.ExternalStream(self.stream, self.device)

    def _order(self, to_own):
        """A given stream behind the current one, or the other way round (unless one of them is being captured)."""
        now, own = torch.cuda.current_stream(self.device), self._own()
        if now.cuda_stream != own.cuda_stream and not any(map(_is_capturing, (now, own))):
            own.wait_stream(now) if to_own else now.wait_stream(own)

    def _capturing(self):
        """Whether the stream of the next call is being captured."""
        return _is_capturing(torch.cuda.current_stream(self.device) if self._follows else self._own())

    @property
    def launches(self) -> int:
        return self._launch_count(self.ctx) if self.ctx is not None else 0

    def close(self):
        ctx, self.ctx = self.ctx, None             # it is freed even where the entry reports an error
        if ctx is not None:
            self._destroy(ctx)

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def _workspace(nbytes, device, where):
    if nbytes == 0:
        _refuse(where, "sizes out of range")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


class LinearXent(_Holder):
    """Cross entropy of logits = h w^T against one label per token.

    tokens, dim, vocab   the most tokens of a call, and the sizes of w (vocab x dim)
    dtype                torch.bfloat16 or torch.float16, the type of h and w
    gradients            False: no workspace for backward (the loss alone)

    h may have any leading dimensions, with rows of `dim` consecutive elements; `targets`
    (int64) has those leading dimensions.  A label outside [0, vocab) leaves its token out.
    A w or dw whose rows are not 16-byte aligned although dim is a multiple of 8 passes through
    a second context with a larger workspace.  It is made when such rows are first met, which
    cannot be inside a stream capture, and the first context stays as it is: CUDA graphs that
    were captured through this object keep their workspace as long as the object lives.
    Calling the object gives the loss as a torch value with gradients (of the first order)::

        loss = xent(h, w, targets)            # reduction="mean", "sum" or "none"
        loss.backward()
    """

    _set_stream = staticmethod(binding.psops_xent_set_stream)
    _launch_count = staticmethod(binding.psops_xent_launch_count)
    _destroy = staticmethod(binding.psops_xent_destroy)
    _launched = 0                   # by contexts that are closed
    _staged = None                  # the second context

    def __init__(self, tokens, dim, vocab, *, dtype=torch.bfloat16, device="cuda", gradients=True, stream=None):
        device = torch.device(device)
        if device.type != "cuda":
            _refuse("LinearXent", "needs a GPU")
        if dtype not in (torch.float16, torch.bfloat16):
            _refuse("LinearXent", f"h and w of {dtype}: torch.bfloat16 or torch.float16")
        self.device = torch.device("cuda", torch.cuda.current_device()) if device.index is None else device
        self.tokens, self.dim, self.vocab, self.dtype = int(tokens), int(dim), int(vocab), dtype
        self._w_shape = torch.Size((self.vocab, self.dim)) if min(self.vocab, self.dim) >= 0 else None
        self._flags = PSOPS_XENT_GRADS if gradients else 0
        self._on(self.device, stream)
        self._workspace, self.ctx = self._open(self._flags)

    def _open(self, flags):
        cfg = binding.psops_xent_config(self.tokens, self.dim, self.vocab, _TYPES[self.dtype], flags)
        with torch.cuda.device(self.device):
            workspace = _workspace(binding.psops_xent_workspace_bytes(cfg), self.device, "LinearXent")
            self._follow()
            return workspace, binding.psops_xent_create(cfg, workspace, None, self.stream)

    def _rows(self, where, name, t):
        """Stride of a matrix that has consecutive elements in each row, its leading dimensions seen as one."""
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.dtype is not self.dtype:
            _refuse(where, f"{name} is not a {self.dtype} tensor on {self.device}")
        shape = t.shape
        if len(shape) < 1 or shape[-1] != self.dim:
            _refuse(where, f"{name} has no last dimension of {self.dim}")
        if t.is_contiguous():
            return self.dim
        if len(shape) != 2:
            try:
                t = t.view(-1, self.dim)
            except RuntimeError:
                _refuse(where, f"{name}: its leading dimensions cannot be seen as one")
        if self.dim > 1 and t.stride(1) != 1:
            _refuse(where, f"{name}: the elements of a row are not consecutive")
        ld = t.stride(0) if t.shape[0] > 1 else self.dim
        if ld < self.dim:
            _refuse(where, f"{name}: rows overlap")
        return ld

    def _arguments(self, where, h, w, targets):
        """(tokens, strides of h and w)."""
        h_ld, w_ld = self._rows(where, "h", h), self._rows(where, "w", w)
        if w.shape != self._w_shape:
            _refuse(where, f"w is not {self.vocab} x {self.dim}")
        if not isinstance(targets, torch.Tensor) or targets.get_device() != self.device.index or \
                targets.dtype is not torch.int64:
            _refuse(where, f"targets is not an int64 tensor on {self.device}")
        if targets.shape != h.shape[:-1] or not targets.is_contiguous():
            _refuse(where, f"targets has to be contiguous and of shape {tuple(h.shape[:-1])}")
        tokens = targets.numel()
        if tokens > self.tokens:
            _refuse(where, f"{tokens} tokens, made for {self.tokens}")
        return tokens, h_ld, w_ld

    def _context(self, where, tensors, w, w_ld, dw=None, dw_ld=0):
        """The context for these rows, ready for a call with `tensors`."""
        if self.dim % 8 == 0 and self.ctx is not None and (
                w.data_ptr() % 16 or w_ld % 8 or dw is not None and (dw.data_ptr() % 16 or dw_ld % 8)):
            if self._staged is None and self._capturing():
                raise PsopsError(PSOPS_ESTATE, where, "rows that are not 16-byte aligned, met for the first time inside a "
                                                      "stream capture: make one such call before it")
            self._follow(*tensors)
            if self._staged is None:
                self._staged_workspace, self._staged = self._open(self._flags | PSOPS_XENT_STAGED)
            return self._staged
        self._follow(*tensors)
        return self.ctx

    def _move(self, stream):
        super()._move(stream)
        if self._staged is not None:
            self._set_stream(self._staged, stream)

    def forward(self, h, w, targets, reduction="mean", *, loss=None):
        """(loss, rows, lse): the loss of all tokens ("mean" or "sum"), and each token's loss and log-sum-exp.
        `loss`: one fp32 number to hold it, such as an element of the loss vector a swarm reads."""
        if reduction != "mean" and reduction != "sum":
            _refuse("LinearXent.forward", f"reduction {reduction!r}")
        tokens, h_ld, w_ld = self._arguments("LinearXent.forward", h, w, targets)
        given = [] if loss is None else [loss]
        if loss is None:
            loss = torch.empty((), dtype=torch.float32, device=self.device)
        else:
            self._numbers("LinearXent.forward", "loss", loss, None)
        rows = torch.empty(targets.shape, dtype=torch.float32, device=self.device)
        lse = torch.empty_like(rows)
        ctx = self._context("LinearXent.forward", (h, w, targets, loss, rows, lse), w, w_ld)
        binding.psops_xent_forward(ctx, h, h_ld, w, w_ld, targets, tokens, _REDUCTIONS[reduction], loss, rows, lse)
        if given:
            _changed(given)
        return loss, rows, lse

    def backward(self, h, w, targets, lse, grad, reduction="mean", *, rows=None, dh=None, dw=None, want=(True, True)):
        """(dh, dw) from the upstream gradient: one fp32 number, or one per token for reduction "none".
        rows: forward's, which keep the digits of the gradients of confident tokens; dh, dw: tensors to hold the
        result; want: which of the two is computed."""
        where = "LinearXent.backward"
        code = _REDUCTIONS.get(reduction)
        if code is None:
            _refuse(where, f"reduction {reduction!r}")
        tokens, h_ld, w_ld = self._arguments(where, h, w, targets)
        self._numbers(where, "lse", lse, targets.shape)
        if rows is not None:
            self._numbers(where, "rows", rows, targets.shape)
        self._numbers(where, "grad", grad, targets.shape if code == PSOPS_PER_TOKEN else None)
        given = [t for t, wanted in ((dh, want[0]), (dw, want[1])) if wanted and t is not None]
        dh, dh_ld = self._gradient(where, "dh", dh, h) if want[0] else (None, 0)
        dw, dw_ld = self._gradient(where, "dw", dw, w) if want[1] else (None, 0)
        ctx = self._context(where, (h, w, targets, lse, rows, grad, dh, dw), w, w_ld, dw, dw_ld)
        binding.psops_xent_backward(ctx, h, h_ld, w, w_ld, targets, tokens, lse, rows, grad, code, dh, dh_ld, dw, dw_ld)
        if given:
            _changed(given)
        return dh, dw

    def _join(self):
        """The current stream behind a given one: autograd's own operations follow there."""
        if not self._follows:
            self._order(to_own=False)

    def _numbers(self, where, name, t, shape):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.dtype is not torch.float32 or \
                not t.is_contiguous() or (t.shape != shape if shape is not None else t.numel() != 1):
            _refuse(where, f"{name} has to be contiguous, fp32, on {self.device}, of shape "
                           f"{tuple(shape) if shape is not None else ()}")

    def _gradient(self, where, name, t, like):
        if t is None:
            return torch.empty(like.shape, dtype=self.dtype, device=self.device), self.dim
        ld = self._rows(where, name, t)
        if t.shape != like.shape:
            _refuse(where, f"{name} is not of shape {tuple(like.shape)}")
        return t, ld

    def __call__(self, h, w, targets, reduction="mean"):
        """The loss with gradients.  Here h, w and targets may have any strides (a slice of a sequence, say)."""
        if isinstance(h, torch.Tensor) and h.dim() > 2:
            h = h.contiguous()
        elif isinstance(h, torch.Tensor) and h.dim() == 2 and h.shape[1] > 1 and (h.stride(1) != 1 or h.stride(0) < h.shape[1]):
            h = h.contiguous()
        if isinstance(w, torch.Tensor) and w.dim() == 2 and w.shape[1] > 1 and (w.stride(1) != 1 or w.stride(0) < w.shape[1]):
            w = w.contiguous()
        if isinstance(targets, torch.Tensor):
            targets = targets.contiguous()
        with _exactly:
            return _LinearXentFunction.apply(h, w, targets, self, reduction)

    @property
    def launches(self) -> int:
        return self._launched + super().launches + (self._launch_count(self._staged) if self._staged is not None else 0)

    def close(self):
        self._launched = self.launches
        staged, self._staged = self._staged, None
        try:
            if staged is not None:
                self._destroy(staged)
        finally:
            super().close()


class _LinearXentFunction(torch.autograd.Function):
    """LinearXent.forward and .backward as one differentiable step; a second derivative raises an error."""

    @staticmethod
    def forward(ctx, h, w, targets, op, reduction):
        if reduction not in ("mean", "sum", "none"):
            _refuse("LinearXent", f"reduction {reduction!r}")
        loss, rows, lse = op.forward(h, w, targets, "mean" if reduction == "mean" else "sum")
        op._join()
        ctx.save_for_backward(h, w, targets, rows, lse)
        ctx.op, ctx.reduction = op, reduction
        return rows if reduction == "none" else loss

    @staticmethod
    def backward(ctx, grad):
        h, w, targets, rows, lse = ctx.saved_tensors
        with torch.no_grad():
            dh, dw = ctx.op.backward(h, w, targets, lse, grad.float().contiguous(), ctx.reduction, rows=rows,
                                     want=(ctx.needs_input_grad[0], ctx.needs_input_grad[1]))
            ctx.op._join()
        if torch.is_grad_enabled():                # create_graph: what is done with the gradients is recorded
            dh, dw = (None if d is None else _FirstOrderOnly.apply(d, h, w, grad) for d in (dh, dw))
        return dh, dw, None, None, None


class _FirstOrderOnly(torch.autograd.Function):
    """A gradient as it is, dependent on all that it came from, with an error in place of its derivative."""

    @staticmethod
    def forward(ctx, gradient, *came_from):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError("LinearXent, Attention, Keep8: gradients are of the first order only (once_differentiable); a function of them "
                           "cannot be differentiated")


def distance_buckets(count, far):
    """The first distance of each of `count` buckets: the lower half holds one distance each, the others grow by a
    common ratio up to `far`, and the last holds all that is farther."""
    count, far = int(count), int(far)
    near = count // 2
    if not 1 <= count <= 64 or not count <= far <= 1024:
        _refuse("distance_buckets", f"{count} buckets up to {far}: 1 to 64, and no more than distances, 1024 at most")
    first = list(range(near))
    for k in range(count - near):
        # the smallest d with (d / near)^(count - near) >= (far / near)^k, in whole numbers
        d = near
        if near:
            low, high, n = near, far, count - near
            while low < high:
                mid = (low + high) // 2
                if mid ** n * near ** k >= far ** k * near ** n:
                    high = mid
                else:
                    low = mid + 1
            d = low
        first.append(max(d, first[-1] + 1) if first else 0)
    return first


class Attention(_Holder):
    """Causal attention over packed sequences.

    tokens, sequences       the most of a call
    heads, kv_heads, dim    query heads, key heads (a divisor of them) and elements of a head (a multiple of 8, to 128)
    dtype                   torch.bfloat16 or torch.float16, the type of q, k and v
    buckets                 None, or the first distance of each bucket of a learned bias, ascending from 0 (such as
                            :func:`distance_buckets` gives)
    scale                   of the products of q and k, 1 / sqrt(dim) if not given
    gradients               False: no workspace for backward

    q is tokens x heads x dim, k and v are tokens x kv_heads x dim, with consecutive elements in each head and rows on
    multiples of 16 bytes (views of one projection's output, for instance); `offsets` (int32, on the GPU, one more than
    there are sequences) has each sequence's first token, and behind the last one its end; `bias` is buckets x heads, fp32
    or of q's type, of any finite size, and -inf takes its pairs out.  Rows of no sequence are zeros in results that a call makes, and left as they were in given ones.
    Calling the object gives the output as a torch value with gradients (of the first order)::

        out = attention(q, k, v, offsets, bias)
    """

    _set_stream = staticmethod(binding.psops_attention_set_stream)
    _launch_count = staticmethod(binding.psops_attention_launch_count)
    _destroy = staticmethod(binding.psops_attention_destroy)

    def __init__(self, tokens, sequences, heads, kv_heads, dim, *, dtype=torch.bfloat16, buckets=None, scale=None,
                 device="cuda", gradients=True, stream=None):
        device = torch.device(device)
        if device.type != "cuda":
            _refuse("Attention", "needs a GPU")
        if dtype not in (torch.float16, torch.bfloat16):
            _refuse("Attention", f"q, k and v of {dtype}: torch.bfloat16 or torch.float16")
        self.device = torch.device("cuda", torch.cuda.current_device()) if device.index is None else device
        self.tokens, self.sequences, self.dtype = int(tokens), int(sequences), dtype
        self.heads, self.kv_heads, self.dim = int(heads), int(kv_heads), int(dim)
        self.buckets = [] if buckets is None else [int(b) for b in buckets]
        self.scale = self.dim ** -0.5 if scale is None and self.dim > 0 else float(scale or 0.0)
        first = (ctypes.c_int32 * len(self.buckets))(*self.buckets) if self.buckets else None
        cfg = binding.psops_attention_config(self.tokens, self.sequences, self.heads, self.kv_heads, self.dim,
                                             _TYPES[dtype], len(self.buckets), first, self.scale,
                                             PSOPS_ATTENTION_GRADS if gradients else 0)
        self._on(self.device, stream)
        with torch.cuda.device(self.device):
            self._workspace = _workspace(binding.psops_attention_workspace_bytes(cfg), self.device, "Attention")
            self._follow()
            self.ctx = binding.psops_attention_create(cfg, self._workspace, None, self.stream)

    def _tensor(self, where, name, t, heads, tokens=None):
        """The tensor as the library takes it."""
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.dtype is not self.dtype:
            _refuse(where, f"{name} is not a {self.dtype} tensor on {self.device}")
        shape = t.shape
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.dim or tokens is not None and shape[0] != tokens:
            _refuse(where, f"{name} is not {'tokens' if tokens is None else tokens} x {heads} x {self.dim}")
        stride = t.stride()
        if stride[2] != 1:
            _refuse(where, f"{name}: the elements of a head are not consecutive")
        return binding.psops_heads(t.data_ptr() or None, stride[0], stride[1])

    def _result(self, like):
        """A new tensor of this shape, and as the library takes it."""
        t = torch.empty_like(like, memory_format=torch.contiguous_format)
        return t, binding.psops_heads(t.data_ptr() or None, like.shape[1] * self.dim, self.dim)

    def _arguments(self, where, q, k, v, offsets, bias):
        Q = self._tensor(where, "q", q, self.heads)
        tokens = q.shape[0]
        if tokens > self.tokens:
            _refuse(where, f"{tokens} tokens, made for {self.tokens}")
        K, V = self._tensor(where, "k", k, self.kv_heads, tokens), self._tensor(where, "v", v, self.kv_heads, tokens)
        if not isinstance(offsets, torch.Tensor) or offsets.get_device() != self.device.index or \
                offsets.dtype is not torch.int32 or offsets.dim() != 1 or not offsets.is_contiguous() or offsets.numel() < 1:
            _refuse(where, f"offsets has to be contiguous, int32, of one axis, on {self.device}")
        sequences = offsets.numel() - 1
        if sequences > self.sequences:
            _refuse(where, f"{sequences} sequences, made for {self.sequences}")
        if bool(self.buckets) != (bias is not None):
            _refuse(where, "a bias goes with buckets")
        if bias is not None:
            self._bias(where, "bias", bias, (self.dtype, torch.float32))
        return Q, K, V, tokens, sequences, _TYPES[bias.dtype] if bias is not None else PSOPS_NONE

    def _bias(self, where, name, t, types):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.dtype not in types or \
                t.shape != (len(self.buckets), self.heads) or not t.is_contiguous():
            _refuse(where, f"{name} has to be contiguous, {len(self.buckets)} x {self.heads}, of "
                           f"{' or '.join(map(str, types))}, on {self.device}")

    def _lse(self, where, t, tokens):
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.dtype is not torch.float32 or \
                t.shape != (self.heads, tokens) or not t.is_contiguous():
            _refuse(where, f"lse has to be contiguous, fp32, {self.heads} x {tokens}, on {self.device}")

    def forward(self, q, k, v, offsets, bias=None, *, out=None):
        """(out, lse): the output, and heads x tokens log-sum-exps.  `out`: a tensor to hold the output."""
        where = "Attention.forward"
        Q, K, V, tokens, sequences, bias_type = self._arguments(where, q, k, v, offsets, bias)
        given = out is not None
        if given:
            O = self._tensor(where, "out", out, self.heads, tokens)
        else:
            out, O = self._result(q)
        lse = (q.new_zeros if given else q.new_empty)((self.heads, tokens), dtype=torch.float32)
        self._follow(q, k, v, offsets, bias, out, lse)
        binding.psops_attention_forward(self.ctx, Q, K, V, offsets, sequences, tokens, bias, bias_type, O, lse, not given)
        if given:
            _changed([out])
        return out, lse

    def backward(self, q, k, v, offsets, out, lse, grad, bias=None, *, dq=None, dk=None, dv=None, dbias=None,
                 want=(True, True, True, True)):
        """(dq, dk, dv, dbias) from forward's inputs and results and the gradient of its output.
        dq, dk, dv, dbias: tensors to hold the results; want: which of them are computed."""
        where = "Attention.backward"
        Q, K, V, tokens, sequences, bias_type = self._arguments(where, q, k, v, offsets, bias)
        O, G = self._tensor(where, "out", out, self.heads, tokens), self._tensor(where, "grad", grad, self.heads, tokens)
        self._lse(where, lse, tokens)
        held, results, given = [], [], []
        mine = dq is None and dk is None and dv is None
        for name, t, like, heads, wanted in (("dq", dq, q, self.heads, want[0]), ("dk", dk, k, self.kv_heads, want[1]),
                                             ("dv", dv, v, self.kv_heads, want[2])):
            if not wanted:
                t = as_taken = None
            elif t is None:
                t, as_taken = self._result(like)
                if not mine:               # what is given keeps its rows of no sequence, what is made here has zeros there
                    t.zero_()
            else:
                as_taken = self._tensor(where, name, t, heads, tokens)
                given.append(t)
            results.append(t)
            held.append(as_taken)
        if not want[3] or bias is None:
            dbias = None
        elif dbias is None:
            dbias = torch.empty_like(bias)
        else:
            self._bias(where, "dbias", dbias, (bias.dtype,))
            given.append(dbias)
        self._follow(q, k, v, offsets, bias, out, lse, grad, *results, dbias)
        binding.psops_attention_backward(self.ctx, Q, K, V, offsets, sequences, tokens, bias, bias_type, O, lse, G, *held,
                                         dbias, mine)
        if given:
            _changed(given)
        return (*results, dbias)

    def _fitting(self, t):
        """The tensor, or a copy of it where its rows do not lie as the library reads them."""
        if not isinstance(t, torch.Tensor) or t.dim() != 3 or not t.is_cuda:
            return t
        (a, b, c), (n, h, _) = t.stride(), t.shape
        if c == 1 and t.data_ptr() % 16 == 0 and (n <= 1 or a % 8 == 0 and a >= self.dim) and \
                (h <= 1 or b % 8 == 0 and b >= self.dim):
            return t
        return t.contiguous() if not t.is_contiguous() else t.clone()

    def _join(self):
        if not self._follows:
            self._order(to_own=False)

    def __call__(self, q, k, v, offsets, bias=None):
        """The output with gradients.  Here q, k and v may have any strides."""
        q, k, v = map(self._fitting, (q, k, v))
        if isinstance(bias, torch.Tensor):
            bias = bias.contiguous()
        with _exactly:
            return _AttentionFunction.apply(q, k, v, bias, offsets, self)


class _AttentionFunction(torch.autograd.Function):
    """Attention.forward and .backward as one differentiable step; a second derivative raises an error."""

    @staticmethod
    def forward(ctx, q, k, v, bias, offsets, op):
        out, lse = op.forward(q, k, v, offsets, bias)
        op._join()
        ctx.save_for_backward(q, k, v, bias, offsets, out, lse)
        ctx.op = op
        return out

    @staticmethod
    def backward(ctx, grad):
        q, k, v, bias, offsets, out, lse = ctx.saved_tensors
        with torch.no_grad():
            results = ctx.op.backward(q, k, v, offsets, out, lse, ctx.op._fitting(grad), bias, want=ctx.needs_input_grad[:4])
            ctx.op._join()
        if torch.is_grad_enabled():                # create_graph: what is done with the gradients is recorded
            came_from = [t for t in (q, k, v, bias, grad) if t is not None]
            results = [None if d is None else _FirstOrderOnly.apply(d, *came_from) for d in results]
        return (*results, None, None)


class Keep8(_Holder):
    """Activations kept in 8 bits between the forward and the backward pass.

    A tensor of a 16-bit type becomes codes (int8, its last dimension padded to a multiple of 16) and
    scales (fp32, one for every 128 elements of a row), 1.03 bytes an element; psops.h has the rule.  Three ways:

      pack, unpack    any tensor there and back
      hooks           a context in which autograd keeps what it saves in 8 bits, whatever the operation::

          with keep.hooks():
              y = block(x)

      calling it      y = f(a) or f(a) * b with f one of "relu", "silu", "gelu" (tanh form), differentiable, the
                      inputs kept in 8 bits: keep(a, b, "silu")
    """

    _set_stream = staticmethod(binding.psops_keep_set_stream)
    _launch_count = staticmethod(binding.psops_keep_launch_count)
    _destroy = staticmethod(binding.psops_keep_destroy)

    def __init__(self, *, device="cuda", stream=None):
        device = torch.device(device)
        if device.type != "cuda":
            _refuse("Keep8", "needs a GPU")
        self.device = torch.device("cuda", torch.cuda.current_device()) if device.index is None else device
        self._on(self.device, stream)
        with torch.cuda.device(self.device):
            self._follow()
            self.ctx = binding.psops_keep_create(self.stream)

    def _rows(self, where, name, t, like=None):
        """(rows, elements of a row, stride) of a tensor with consecutive elements in each row, its leading dimensions
        seen as one."""
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or \
                t.dtype is not torch.bfloat16 and t.dtype is not torch.float16:
            _refuse(where, f"{name} is not a 16-bit floating-point tensor on {self.device}")
        shape = t.shape
        if len(shape) < 1 or shape[-1] < 1:
            _refuse(where, f"{name} has no elements in its rows")
        if like is not None and (shape != like.shape or t.dtype is not like.dtype):
            _refuse(where, f"{name} is not {like.dtype} of shape {tuple(like.shape)}")
        cols = shape[-1]
        rows = t.numel() // cols
        if t.is_contiguous():
            return rows, cols, cols
        if len(shape) != 2:
            try:
                t = t.view(-1, cols)
            except RuntimeError:
                _refuse(where, f"{name}: its leading dimensions cannot be seen as one")
        if cols > 1 and t.stride(1) != 1:
            _refuse(where, f"{name}: the elements of a row are not consecutive")
        ld = t.stride(0) if rows > 1 else cols
        if ld < cols:
            _refuse(where, f"{name}: rows overlap")
        return rows, cols, ld

    @staticmethod
    def _like(t):
        """A contiguous tensor like this one."""
        return torch.empty_like(t, memory_format=torch.contiguous_format)

    @staticmethod
    def _room(t):
        """Codes and scales for a tensor like this one."""
        *leading, cols = t.shape
        return (t.new_empty((*leading, -(-cols // 16) * 16), dtype=torch.int8),
                t.new_empty((*leading, -(-cols // KEPT_BLOCK)), dtype=torch.float32))

    def _kept(self, where, name, codes, scales, shape):
        *leading, cols = shape
        for what, t, width, dtype in (("codes", codes, -(-cols // 16) * 16, torch.int8),
                                      ("scales", scales, -(-cols // KEPT_BLOCK), torch.float32)):
            if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != self.device.index or \
                    t.shape != (*leading, width) or not t.is_contiguous():
                _refuse(where, f"{what} of {name} have to be contiguous, {dtype}, of shape {(*leading, width)}, on {self.device}")

    def pack(self, x):
        """(codes, scales)."""
        rows, cols, ld = self._rows("Keep8.pack", "x", x)
        codes, scales = self._room(x)
        self._follow(x, codes, scales)
        binding.psops_keep_pack(self.ctx, _TYPES[x.dtype], rows, cols, x, ld, codes, scales)
        return codes, scales

    def unpack(self, codes, scales, shape, dtype, *, out=None):
        """The tensor of this shape and type that pack was given, each element half a scale off at most.
        `out`: a tensor to hold it."""
        where = "Keep8.unpack"
        shape = torch.Size(shape)
        if dtype not in (torch.float16, torch.bfloat16) or len(shape) < 1 or shape[-1] < 1:
            _refuse(where, f"{dtype} of shape {tuple(shape)}")
        self._kept(where, "x", codes, scales, shape)
        given = out is not None
        if given:
            rows, cols, ld = self._rows(where, "out", out)
            if out.shape != shape or out.dtype is not dtype:
                _refuse(where, f"out is not {dtype} of shape {tuple(shape)}")
        else:
            out, cols = scales.new_empty(shape, dtype=dtype), shape[-1]
            rows, ld = shape.numel() // cols, cols
        self._follow(codes, scales, out)
        binding.psops_keep_unpack(self.ctx, _TYPES[dtype], rows, cols, codes, scales, out, ld)
        if given:
            _changed([out])
        return out

    def _kind(self, where, kind):
        code = _KINDS.get(kind)
        if code is None:
            _refuse(where, f"activation {kind!r}: one of {', '.join(_KINDS)}")
        return code

    def activate(self, a, b=None, kind="silu", *, out=None):
        """(y, kept): f(a), or f(a) * b, and (codes, scales) of a, or (codes, scales, codes, scales) of a and b, for the
        backward pass.  `out`: a tensor to hold y."""
        where = "Keep8.activate"
        code = self._kind(where, kind)
        rows, cols, a_ld = self._rows(where, "a", a)
        b_ld = self._rows(where, "b", b, a)[2] if b is not None else 0
        given = out is not None
        if given:
            y_ld = self._rows(where, "out", out, a)[2]
        else:
            out, y_ld = self._like(a), cols
        kept = self._room(a) + (self._room(a) if b is not None else ())
        self._follow(a, b, out, *kept)
        binding.psops_keep_activate(self.ctx, code, _TYPES[a.dtype], rows, cols, a, a_ld, b, b_ld, out, y_ld,
                                     *kept, *((None, None) if b is None else ()))
        if given:
            _changed([out])
        return out, kept

    def activate_backward(self, kept, grad, kind="silu", *, again=False, da=None, db=None, want=(True, True)):
        """(da, db) from what activate kept and the gradient of y, or (da, db, y) with `again`: y from the kept inputs,
        for a product's gradient that needs it.  da, db: tensors to hold the results (views of one gradient, for
        instance); want: which of the two are computed.  db is None without b."""
        where = "Keep8.activate_backward"
        code = self._kind(where, kind)
        rows, cols, ld = self._rows(where, "grad", grad)
        if len(kept) not in (2, 4):
            _refuse(where, "`kept` is (codes, scales) of a, or of a and b")
        gated = len(kept) == 4
        for i in range(0, len(kept), 2):
            self._kept(where, "ab"[i // 2], kept[i], kept[i + 1], grad.shape)
        results, strides, given = [], [], []
        for name, t, wanted in (("da", da, want[0]), ("db", db, want[1] and gated), ("y", None, again)):
            ld_of = cols
            if not wanted:
                t = None
            elif t is None:
                t = self._like(grad)
            else:
                ld_of = self._rows(where, name, t, grad)[2]
                given.append(t)
            results.append(t)
            strides.append(ld_of)
        self._follow(grad, *kept, *results)
        binding.psops_keep_activate_backward(self.ctx, code, _TYPES[grad.dtype], rows, cols, *kept,
                                              *(() if gated else (None, None)), grad, ld, results[0], strides[0],
                                              results[1], strides[1], results[2], strides[2])
        if given:
            _changed(given)
        return tuple(results) if again else tuple(results[:2])

    def _join(self):
        if not self._follows:
            self._order(to_own=False)

    @staticmethod
    def _fitting(t):
        """The tensor, or a copy of it where the elements of its rows are not consecutive or its rows overlap."""
        if not isinstance(t, torch.Tensor) or t.dim() < 1 or t.is_contiguous() or \
                t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]):
            return t
        return t.contiguous()

    def __call__(self, a, b=None, kind="silu"):
        """f(a), or f(a) * b, with gradients.  Here a and b may have any strides.  The result is kept by what uses it, as
        any tensor is (in 8 bits under hooks()); activate and activate_backward with `again` do without that."""
        return _Keep8Function.apply(self._fitting(a), self._fitting(b), kind, self)

    def hooks(self, least=4096):
        """A context in which autograd keeps the 16-bit tensors that it saves in 8 bits, those of `least` elements or
        more on this GPU.  Left alone are leaves that have gradients (weights), views of them, which are there anyway,
        and casts of them, which are weights all the same; broadcast tensors, which take less room as they are; and
        what Attention and LinearXent save, whose statistics belong to the numbers as they are.  A tensor that several
        operations save is kept once, as long as nothing writes to it in between that autograd does not see (through
        .data, say)."""
        kept_now = weakref.WeakValueDictionary()       # what graphs hold, by where it came from

        def pack(t):
            if _exactly.depth or t.get_device() != self.device.index or t.dtype not in (torch.float16, torch.bfloat16) or \
                    t.numel() < max(1, least) or t.dim() < 1 or _is_of_a_leaf(t) or \
                    any(n > 1 and ld == 0 for n, ld in zip(t.shape, t.stride())):
                return _AsItIs(t)
            # a weak reference: no other storage is known by its number as long as there is one
            source = StorageWeakRef(t.untyped_storage())
            now = None if t.get_device() < 0 else (torch._C._cuda_getCurrentRawStream(t.get_device()), torch.cuda.is_current_stream_capturing())
            key = source.cdata, t.storage_offset(), t.shape, t.stride(), t.dtype, t._version, now
            kept = kept_now.get(key)
            if kept is None:
                with torch.no_grad():
                    codes, scales = self.pack(self._fitting(t.detach()))
                    self._join()
                kept = kept_now[key] = _InCodes(codes, scales, t.shape, t.dtype, source)
            return kept

        def unpack(kept):
            if isinstance(kept, _AsItIs):
                return kept.get()
            with torch.no_grad():
                x = self.unpack(kept.codes, kept.scales, kept.shape, kept.dtype)
                self._join()
            return x

        return torch.autograd.graph.saved_tensors_hooks(pack, unpack)


# Operations whose result is their input in another type or seen in another way.
_SAME_NUMBERS = frozenset(f"{name}Backward0" for name in (
    "ToCopy", "View", "UnsafeView", "ReshapeAlias", "AsStrided", "T", "Transpose", "Permute", "Select", "Slice", "Split", "SplitWithSizes", "Unbind",
    "Squeeze", "Unsqueeze", "Alias"))


def _is_of_a_leaf(t):
    """Whether this is a leaf that has gradients, a view or a cast of one."""
    base = t._base if t._is_view() else t
    if base.is_leaf:
        return base.requires_grad
    node = t.grad_fn
    while node is not None and node.name() in _SAME_NUMBERS:
        node = node.next_functions[0][0]
    return node is not None and node.name() == "torch::autograd::AccumulateGrad"


class _InCodes:
    """A tensor that Keep8.hooks keeps in 8 bits."""

    def __init__(self, codes, scales, shape, dtype, source):
        self.codes, self.scales, self.shape, self.dtype, self.source = codes, scales, shape, dtype, source


class _AsItIs:
    """A tensor that Keep8.hooks leaves alone.  Autograd does not look at versions where there are hooks, and an operation's
    own result would hold the graph that holds it, so that neither were ever freed."""

    def __init__(self, t):
        self.tensor, self.version = t.detach(), t._version

    def get(self):
        if self.tensor._version != self.version:
            raise RuntimeError(f"one of the variables needed for gradient computation has been modified by an inplace operation: "
                               f"{tuple(self.tensor.shape)} {self.tensor.dtype}, at version {self.tensor._version}, saved at version "
                               f"{self.version} (kept as it is by Keep8.hooks)")
        return self.tensor


class _Keep8Function(torch.autograd.Function):
    """Keep8.activate and .activate_backward as one differentiable step; a second derivative raises an error."""

    @staticmethod
    def forward(ctx, a, b, kind, op):
        y, kept = op.activate(a, b, kind)
        op._join()
        ctx.save_for_backward(*kept)
        ctx.op, ctx.kind = op, kind
        return y

    @staticmethod
    def backward(ctx, grad):
        kept = ctx.saved_tensors
        with torch.no_grad():
            da, db = ctx.op.activate_backward(kept, ctx.op._fitting(grad), ctx.kind, want=ctx.needs_input_grad[:2])
            ctx.op._join()
        if torch.is_grad_enabled():                # create_graph: what is done with the gradients is recorded
            da, db = (None if d is None else _FirstOrderOnly.apply(d, grad) for d in (da, db))
        return da, db, None, None


class AdamW(_Holder):
    """AdamW over a list of parameter tensors, in one launch per step.

    params        fp32 device tensors, contiguous (views of a swarm's row, for instance)
    grads         their gradients, all fp32, all fp16 or all bf16
    bits          32: fp32 moments (m, v); 8: moments (m, sqrt v) of 8 bits with a
                  scale for every 256 elements of a tensor
    moments       state to go on with, else zeros: (m, v), lists of fp32 tensors, or for
                  8 bits (m, m_scale, root, root_scale), lists of torch.float8_e4m3fn
                  (or uint8) tensors of the parameters' sizes and of fp32 tensors of
                  ceil(n / 256) scales
    copies        16-bit tensors (None for a parameter without one) that receive the new
                  weights, rounded to nearest
    weight_decay  one number, or one for each parameter
    steps_done    steps that the given moments have already seen

    A step whose grad_scale is not finite is skipped on the device.
    """

    _set_stream = staticmethod(binding.psops_adamw_set_stream)
    _launch_count = staticmethod(binding.psops_adamw_launch_count)
    _destroy = staticmethod(binding.psops_adamw_destroy)

    def __init__(self, params, grads, *, bits=32, moments=None, copies=None, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay=0.01, steps_done=0, stream=None):
        where = "AdamW"
        params = list(params)
        device = _device_of(where, params)
        self.params = _flat_list(where, "params", params, (torch.float32,), device)
        n, sizes = len(params), [p.numel() for p in params]
        self._sizes = sizes
        self.grads = _flat_list(where, "grads", grads, tuple(_TYPES), device, n, sizes)
        if len({g.dtype for g in self.grads}) != 1:
            _refuse(where, "gradients of more than one type")
        if bits not in (8, 32):
            _refuse(where, f"moments of {bits} bits")
        blocks = [-(-s // MOMENT_BLOCK) for s in sizes]
        held = (torch.float32,) if bits == 32 else (torch.float8_e4m3fn, torch.uint8)
        if moments is None:
            zeros = lambda counts, dtype: [torch.zeros(c, dtype=torch.uint8 if dtype != torch.float32 else dtype,
                                                       device=device).view(dtype) for c in counts]
            moments = (zeros(sizes, held[0]), zeros(sizes, held[0])) if bits == 32 else \
                (zeros(sizes, held[0]), zeros(blocks, torch.float32), zeros(sizes, held[0]), zeros(blocks, torch.float32))
        if len(moments) != (2 if bits == 32 else 4):
            _refuse(where, "`moments` is (m, v), or (m, m_scale, root, root_scale) for 8 bits")
        if bits == 32:
            self.moments = tuple(_flat_list(where, k, x, held, device, n, sizes) for k, x in zip(("m", "v"), moments))
            m, v, ms, vs = self.moments[0], self.moments[1], [None] * n, [None] * n
        else:
            names = (("m", held, sizes), ("m_scale", (torch.float32,), blocks), ("root", held, sizes),
                     ("root_scale", (torch.float32,), blocks))
            self.moments = tuple(_flat_list(where, k, x, d, device, n, s) for (k, d, s), x in zip(names, moments))
            m, ms, v, vs = self.moments
        copy_type = PSOPS_NONE
        if copies is not None:
            copies = list(copies)
            if len(copies) != n:
                _refuse(where, f"{len(copies)} copies, {n} parameters")
            there = [i for i, c in enumerate(copies) if c is not None]
            _flat_list(where, "copies", [copies[i] for i in there], (torch.float16, torch.bfloat16), device,
                       len(there), [sizes[i] for i in there])
            kinds = {copies[i].dtype for i in there}
            if len(kinds) > 1:
                _refuse(where, "copies of more than one type")
            copy_type = _TYPES[kinds.pop()] if kinds else PSOPS_NONE
        self.copies = copies
        decay = [float(weight_decay)] * n if not isinstance(weight_decay, (list, tuple)) else [float(d) for d in weight_decay]
        if len(decay) != n:
            _refuse(where, f"{len(decay)} weight decays, {n} parameters")
        self.bits = bits
        cfg = binding.psops_adamw_config(float(betas[0]), float(betas[1]), float(eps), int(steps_done), bits,
                                         _TYPES[self.grads[0].dtype], copy_type, n)
        at = lambda t: t.data_ptr() if t is not None and t.numel() else None
        table = (binding.psops_adamw_tensor * n)(*[
            binding.psops_adamw_tensor(at(self.params[i]), at(self.grads[i]),
                                       at(copies[i]) if copies is not None else None, at(m[i]), at(v[i]), at(ms[i]),
                                       at(vs[i]), sizes[i], decay[i]) for i in range(n)])
        with torch.cuda.device(device):
            self._workspace = _workspace(binding.psops_adamw_workspace_bytes(cfg, table), device, where)
            self._on(device, stream)
            self._follow()
            self.ctx = binding.psops_adamw_create(cfg, table, self._workspace, None, self.stream)
        # parameters and copies as autograd counts their changes: views share the count of what they are views of
        self._written = list({id(t): t for t in (t._base if t._is_view() else t for t in (
            *self.params, *(c for c in copies or () if c is not None)))}.values())

    def set_grads(self, grads):
        """Other gradient tensors for the steps to come, of the type given at first."""
        grads = _flat_list("AdamW.set_grads", "grads", grads, (self.grads[0].dtype,), self.device, len(self._sizes),
                           self._sizes)
        self._follow(*self.grads)                  # the old ones: steps on their way still read them
        binding.psops_adamw_set_grads(self.ctx, grads)
        self.grads = grads

    def step(self, lr, grad_scale=None):
        """One step; grad_scale: a device fp32 scalar that multiplies every gradient."""
        if grad_scale is not None and not (isinstance(grad_scale, torch.Tensor)
                                           and grad_scale.get_device() == self.device.index
                                           and grad_scale.dtype is torch.float32 and grad_scale.numel() == 1):
            _refuse("AdamW.step", f"grad_scale has to be one fp32 number on {self.device}")
        self._follow(grad_scale)
        self._scale = grad_scale               # read by the kernel, and by a captured one again: keep it alive
        binding.psops_adamw_step(self.ctx, lr, grad_scale)
        _changed(self._written)

    @property
    def steps(self) -> int:
        """Steps taken so far (waits for the stream)."""
        self._follow()
        return binding.psops_adamw_steps(self.ctx)



class GradNorm(_Holder):
    """2-norm of a list of gradient tensors (all of one type) together."""

    _set_stream = staticmethod(binding.psops_gradnorm_set_stream)
    _launch_count = staticmethod(binding.psops_gradnorm_launch_count)
    _destroy = staticmethod(binding.psops_gradnorm_destroy)

    def __init__(self, grads, *, stream=None):
        where = "GradNorm"
        grads = list(grads)
        self.device = _device_of(where, grads)
        self.grads = _flat_list(where, "grads", grads, tuple(_TYPES), self.device)
        if len({g.dtype for g in grads}) != 1:
            _refuse(where, "gradients of more than one type")
        self._sizes = [g.numel() for g in grads]
        with torch.cuda.device(self.device):
            self._workspace = _workspace(binding.psops_gradnorm_workspace_bytes(self._sizes), self.device, where)
            self._on(self.device, stream)
            self._follow()
            self.ctx = binding.psops_gradnorm_create([g if g.numel() else None for g in grads], self._sizes,
                                                     _TYPES[grads[0].dtype], self._workspace, None, self.stream)

    def set_grads(self, grads):
        grads = _flat_list("GradNorm.set_grads", "grads", grads, (self.grads[0].dtype,), self.device,
                           len(self._sizes), self._sizes)
        self._follow(*self.grads)
        binding.psops_gradnorm_set_grads(self.ctx, [g if g.numel() else None for g in grads])
        self.grads = grads

    def norm(self, max_norm=math.inf, out=None):
        """(norm, factor), two device scalars: factor = min(1, max_norm / (norm + 1e-6)), NaN
        if the norm is not finite.  `out`: an fp32 device tensor of 2 elements to hold them."""
        given = out is not None
        if out is None:
            out = torch.empty(2, dtype=torch.float32, device=self.device)
        elif not isinstance(out, torch.Tensor) or out.device != self.device or out.dtype != torch.float32 or \
                out.numel() != 2 or not out.is_contiguous():
            _refuse("GradNorm.norm", f"`out` has to be 2 fp32 numbers on {self.device}")
        self._follow(out)
        binding.psops_gradnorm_run(self.ctx, max_norm, out)
        if given:
            _changed(out)
        return out.view(2).unbind(0)

