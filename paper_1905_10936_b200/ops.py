"""The operators that make a worker's gradient, on torch tensors: RMS norm with the residual's
addition, 8-bit activation checkpoints, the activation that keeps its input as one, the weight
gradient from a checkpoint, and the clipped policy loss with a KL term.

Matrices are 2-D CUDA tensors with neighbouring columns (``stride(1) == 1``; rows may be strided
or start anywhere) of type float32, bfloat16 or float16.  Work is enqueued on the device's current
stream; a tensor made on another stream has to be complete there first (``Stream.wait_stream``),
and ``Tensor.record_stream`` is the caller's, as for any torch operator.

The functions are the two halves of a pass, forward and backward, and not differentiable calls: torch
records no graph through them, whether their inputs require gradients or not.  A forward function's
results go to its backward function, and gradients where the caller wants them (``policy_loss(...).grad``
into ``logits.backward(grad)``, for instance).  ``in_place`` and ``out`` refuse a leaf that requires
gradients while gradients are recorded, as torch's own in-place operators do.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Tuple, Union

import torch

from . import binding as ef

_TYPES = {torch.float32: ef.EF_TYPE_F32, torch.bfloat16: ef.EF_TYPE_BF16, torch.float16: ef.EF_TYPE_F16}
_KINDS = {"gelu": ef.EF_ACT_GELU, "swiglu": ef.EF_ACT_SWIGLU}
# the entry points that the native half calls, in the order of its table
_CALLS = ("ef_checkpoint_save", "ef_checkpoint_load", "ef_rmsnorm_forward", "ef_rmsnorm_backward_workspace_bytes",
          "ef_rmsnorm_backward", "ef_activation_forward", "ef_activation_backward",
          "ef_checkpoint_weight_grad_workspace_bytes", "ef_checkpoint_weight_grad", "ef_token_logprob", "ef_policy_loss")
_bound = _module = None


def _native():
    """The native half, bound to the library that the binding has loaded (see binding.use_library)."""
    global _bound, _module
    lib = ef._lib or ef.load_library()
    if lib is not _bound:
        try:
            from . import _ef_torch
        except ImportError as e:
            raise OSError("_ef_torch.so is missing: build it with `python -m paper_1905_10936_b200.build` "
                          "(there is no fallback path)") from e
        if _ef_torch.torch_version != torch.__version__:
            raise OSError(f"_ef_torch.so was built against torch {_ef_torch.torch_version}, this is {torch.__version__}: "
                          "build it again with `python -m paper_1905_10936_b200.build`")
        _ef_torch.bind(tuple(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALLS), ef.EFError)
        _module, _bound = _ef_torch, lib
    return _module


def checkpoint_pitch(c: int) -> int:
    """Bytes per row of a checkpoint's codes."""
    return (c + 15) // 16 * 16


def checkpoint_groups(c: int) -> int:
    """Scales per row of a checkpoint."""
    return (c + ef.EF_CHECKPOINT_GROUP - 1) // ef.EF_CHECKPOINT_GROUP


class Checkpoint:
    """An n x cols matrix kept in 8 bits: codes [n, pitch] int8 and scales [n, groups] float32,
    both contiguous (layout as in include/ef.h)."""

    __slots__ = ("rows", "cols", "_where")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: int):
        n = codes.shape[0]
        if not (codes.is_cuda and codes.dtype == torch.int8 and codes.is_contiguous() and cols >= 1
                and codes.shape == (n, checkpoint_pitch(cols)) and scales.dtype == torch.float32
                and scales.is_contiguous() and scales.shape == (n, checkpoint_groups(cols))
                and scales.get_device() == codes.get_device()):
            raise ValueError("codes and scales do not make a checkpoint of this width")
        self.rows, self.cols = n, cols
        self._where = (n, cols, codes, scales)

    @classmethod
    def _of(cls, buffer: torch.Tensor, n: int, cols: int) -> "Checkpoint":
        """The checkpoint in one buffer, codes first, as the native half allocates it."""
        self = object.__new__(cls)
        self.rows, self.cols = n, cols
        self._where = (n, cols, buffer, None)
        return self

    @property
    def codes(self) -> torch.Tensor:
        n, cols, first, scales = self._where
        return first if scales is not None else first[:n * checkpoint_pitch(cols)].view(n, checkpoint_pitch(cols))

    @property
    def scales(self) -> torch.Tensor:
        n, cols, first, scales = self._where
        if scales is not None:
            return scales
        return first[n * checkpoint_pitch(cols):].view(torch.float32).view(n, checkpoint_groups(cols))

    def nbytes(self) -> int:
        return self.rows * (checkpoint_pitch(self.cols) + 4 * checkpoint_groups(self.cols))

    def record_stream(self, stream: torch.cuda.Stream) -> None:
        """Marks the memory as used on another stream, as Tensor.record_stream."""
        for t in self._where[2:]:
            if t is not None:
                t.record_stream(stream)


_NONE = (0, 0, None, None)               # no checkpoint


def checkpoint_save(x: torch.Tensor) -> Checkpoint:
    """x in 8 bits."""
    return Checkpoint._of(_native().checkpoint_save(x), *x.shape)


def checkpoint_load(kept: Checkpoint, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """The matrix that a checkpoint stands for."""
    if dtype not in _TYPES:
        raise ValueError("dtype: float32, bfloat16 or float16")
    return _native().checkpoint_load(*kept._where, _TYPES[dtype])


class RmsNorm(NamedTuple):
    h: torch.Tensor                      # x + residual (x itself without a residual)
    y: torch.Tensor
    rstd: torch.Tensor
    checkpoint: Optional[Checkpoint]     # of y


def rmsnorm_forward(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-5,
                    residual: Optional[torch.Tensor] = None, checkpoint: bool = False) -> RmsNorm:
    """h = x + residual, y = h / rms(h) * weight; with checkpoint=True y is kept in 8 bits as well and
    holds the values that the checkpoint stands for."""
    h, y, rstd, kept = _native().rmsnorm_forward(x, weight, eps, residual, checkpoint)
    return RmsNorm(x if h is None else h, y, rstd, None if kept is None else Checkpoint._of(kept, *x.shape))


def rmsnorm_backward(dy: torch.Tensor, h: Union[torch.Tensor, Checkpoint], weight: torch.Tensor, rstd: torch.Tensor,
                     dh: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(gradient of x and of the residual, gradient of weight) from dy and, where given, the gradient dh
    that reaches h on other ways; h as a matrix or as its checkpoint."""
    if isinstance(h, Checkpoint):
        return _native().rmsnorm_backward(dy, None, *h._where, weight, rstd, dh)
    if h is None:
        raise ValueError("h: a matrix or a checkpoint is needed")
    return _native().rmsnorm_backward(dy, h, *_NONE, weight, rstd, dh)


class Activation(NamedTuple):
    a: torch.Tensor
    z: Optional[Checkpoint]              # of the input; for "swiglu" its rows are g_0, u_0, g_1, u_1, ...
    kept: Optional[Checkpoint]           # of a


def _kind(kind: str) -> int:
    if kind not in _KINDS:
        raise ValueError("kind: gelu or swiglu")
    return _KINDS[kind]


def activation_forward(z: torch.Tensor, kind: str = "gelu", checkpoint: bool = True,
                       checkpoint_out: bool = False) -> Activation:
    """a = gelu(z), or silu(g) * u for rows z = [g | u] ("swiglu").  With checkpoint=True z is kept in 8 bits and
    a is computed from the values that it stands for; with checkpoint_out=True a is kept as well and
    holds the values that its checkpoint stands for."""
    a, of_z, of_a = _native().activation_forward(z, _kind(kind), checkpoint, checkpoint_out)
    n, c = a.shape
    return Activation(a, None if of_z is None else Checkpoint._of(of_z, 2 * n if kind == "swiglu" else n, c),
                      None if of_a is None else Checkpoint._of(of_a, n, c))


def activation_backward(da: torch.Tensor, z: Checkpoint, kind: str = "gelu") -> torch.Tensor:
    """The gradient of activation_forward's input from da and the input's checkpoint."""
    return _native().activation_backward(da, _kind(kind), *z._where)


def checkpoint_weight_grad(x: Checkpoint, dy: torch.Tensor, out: Optional[torch.Tensor] = None,
                           accumulate: bool = False) -> torch.Tensor:
    """Gradient [x.cols, dy columns], float32, of a linear layer's weight from its input's checkpoint and
    the gradient of its output: into `out` where given (its rows may be strided), added to it with accumulate=True."""
    return _native().checkpoint_weight_grad(*x._where, dy, out, accumulate)


def token_logprob(logits: torch.Tensor, targets: torch.Tensor, temperature: float = 1.0) -> torch.Tensor:
    """Log-probability of each row's target."""
    return _native().token_logprob(logits, targets, temperature)


class PolicyLoss(NamedTuple):
    loss: torch.Tensor                   # scalar
    logp: torch.Tensor
    token_loss: torch.Tensor             # weights * loss of each token
    grad: Optional[torch.Tensor]         # of the logits


def policy_loss(logits: torch.Tensor, targets: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: torch.Tensor, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, beta: float = 0.0, temperature: float = 1.0, need_grad: bool = True,
                in_place: bool = False) -> PolicyLoss:
    """Clipped policy loss with a KL term towards ref_logp (where given), summed with `weights` (0 masks a
    token), and its gradient; in_place=True writes the gradient over the logits."""
    loss, logp, token, grad = _native().policy_loss(logits, targets, old_logp, advantages, weights, ref_logp, clip_low,
                                                    clip_high, beta, temperature, need_grad, in_place)
    return PolicyLoss(loss, logp, token, logits if need_grad and in_place else grad)
