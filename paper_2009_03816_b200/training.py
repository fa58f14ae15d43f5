"""Operators of the training steps between two synchronisations.

Holders of the device tensors (torch) that the library's training-operator
contexts borrow, in the manner of :class:`binding.Swarm`: they check arguments,
allocate workspaces and outputs, and forward to the C entry points; every
computation runs in the CUDA library.

  LinearXent   softmax cross entropy of a linear head without keeping the logits,
               with its gradients; its loss alone is a worker's fitness
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

import math

import torch

from . import binding
from .binding import (PSOPS_BF16, PSOPS_EINVAL, PSOPS_ESTATE, PSOPS_F16, PSOPS_F32, PSOPS_MEAN, PSOPS_NONE,
                      PSOPS_PER_TOKEN, PSOPS_SUM, PSOPS_XENT_GRADS, PSOPS_XENT_STAGED, PsopsError)

_TYPES = {torch.float32: PSOPS_F32, torch.float16: PSOPS_F16, torch.bfloat16: PSOPS_BF16}
_REDUCTIONS = {"mean": PSOPS_MEAN, "sum": PSOPS_SUM, "none": PSOPS_PER_TOKEN}
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


class _Holder:
    """What the three have in common: a context, its GPU and the stream its work goes to."""

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
        raise RuntimeError("LinearXent: gradients are of the first order only (once_differentiable); a function of them "
                           "cannot be differentiated")


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

