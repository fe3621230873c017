"""Operators of a language model's training step on the GPU, for k worker replicas in one call: the tensor-level form of
the library's handle-free entry points (include/dw.h).

Tensors of activations are [k][rows][n] with contiguous rows (views of wider buffers do: rows of a worker n or more elements
apart, workers any number, 0 for an input that they share; rows that are written share no element), float32 or bfloat16;
parameters and their gradients are float32.  Outputs and scratch are allocated by torch on the
current stream of the tensors' device, where the work is enqueued; nothing is synchronised.  As with any torch operator,
a tensor made on another stream has to be waited for, and recorded, by the caller.  Nothing is recorded for autograd: the
backward passes are calls of their own; tensors that a call writes into count as changed in place, so that a graph which
saved one refuses its backward pass.  Wrong shapes, types or layouts raise ValueError, what the library refuses
binding.DwError; there is no CPU path.

Tensors are taken apart in a compiled module, _dw_torch (csrc/dw_torch.cpp), which calls the same C functions as
binding.py: these operators run for a few microseconds, and in Python that costs more than the work.
"""
from __future__ import annotations

import os

import torch

from . import binding as B

_MODULE = None


def _ops():
    """The compiled module, loaded once."""
    global _MODULE
    if _MODULE is None:
        B.lib()                                       # the library it calls; raises when it is missing
        if not os.path.exists(os.path.join(B.HERE, "_dw_torch.so")):
            raise RuntimeError("_dw_torch.so is missing: build it with `python -m paper_2409_09242_amd.build` "
                               "(there is no fallback path)")
        from . import _dw_torch
        _dw_torch.set_error(B.DwError)
        _MODULE = _dw_torch
    return _MODULE


# ---- layer norm ------------------------------------------------------------------------------------------------------

def layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, out=None, stats: bool = True):
    """y = (x - mean) * rstd * gamma + beta over the last axis of x [k][rows][n]; gamma, beta: float32 [k][n] with the same
    worker stride, or None.

    Returns (y, mean, rstd), the latter float32 [k][rows] for layer_norm_grad, or None both with stats=False (a served
    model).  out: a tensor like x for y."""
    return (_MODULE or _ops()).layer_norm(x, gamma, beta, eps, out, stats)


def layer_norm_grad(dy, x, gamma, mean, rstd, dx=None, dgamma=None, dbeta=None, want_dx: bool = True, want_params: bool = True):
    """(dx, dgamma, dbeta) of layer_norm from dy, its input and the statistics it returned.  dx, dgamma, dbeta: tensors to
    write into (float32 [k][n] for the latter two, such as views of the flat gradient of Handle.update_only, with the same
    worker stride where both are given); what is not wanted is returned as None."""
    return (_MODULE or _ops()).layer_norm_grad(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, want_dx, want_params)


# ---- policy loss -----------------------------------------------------------------------------------------------------

def token_logp(logits, target, out=None):
    """Log probabilities, float32 [k][rows], of the tokens target (int32 [k][rows]) under logits [k][rows][vocab]; 0 where
    the target lies outside the vocabulary."""
    return (_MODULE or _ops()).token_logp(logits, target, out)


def policy_loss(logits, target, old_logp, advantage, weight=None, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, grad=None, want_grad: bool = True):
    """(loss [k], logp [k][rows], gradient of the logits) of the clipped policy loss with a KL term; see dw_policy_loss.

    weight (float32 [k][rows], None: 1/rows): mask and average in one, the loss is the weighted sum; rows of weight 0 are
    not read.  grad: a tensor like logits to write into, the logits themselves among them; want_grad=False: None."""
    return (_MODULE or _ops()).policy_loss(logits, target, old_logp, advantage, weight, ref_logp, clip_low, clip_high, kl_coef,
                                           grad, want_grad)


# ---- gradient norm and clipping --------------------------------------------------------------------------------------

def clip_grads(grads, max_norm: float, workers: int = 1, out=None):
    """Clip every worker's gradients to a global 2-norm of at most max_norm; returns the norms before, float32 [workers].

    grads: the tensors of worker 0, then those of worker 1 in the same order and so on (contiguous, float32 or bfloat16, each
    once: none overlaps another).
    They are scaled in place, or left alone with out, float32 [workers][total]: the clipped gradients one behind the other,
    as Handle.update_only takes them."""
    return (_MODULE or _ops()).clip_grads(grads, max_norm, workers, out)


def grad_norm(grads, workers: int = 1):
    """The global 2-norm of every worker's gradients, float32 [workers]; grads as for clip_grads."""
    return (_MODULE or _ops()).clip_grads(grads, float("inf"), workers, None)


# ---- products in 8 bits ----------------------------------------------------------------------------------------------

class Fp8Matrix:
    """[k][rows] rows of n numbers in e4m3, each row padded with zeros to whole blocks of 128, and their scales.

    q: float8_e4m3fn [k][rows][padded n]; scale: uint8 [k][rows][blocks, to a multiple of 4], 2^(scale - 127)."""

    __slots__ = ("q", "scale", "n")

    def __init__(self, q, scale, n: int):
        self.q, self.scale, self.n = q, scale, n

    @property
    def shape(self):
        return (self.q.shape[0], self.q.shape[1], self.n)


def fp8_quantize(x, square: bool = False, transposed: bool = False):
    """x [k][rows][n] in 8 bits with a scale per block of 128 along its rows (square: per 128 x 128), an Fp8Matrix.
    transposed=True: (that, the same of x^T): [k][n] rows of `rows`, its blocks along those."""
    t = (_MODULE or _ops()).fp8_quantize(x, square, transposed)
    m = Fp8Matrix(t[0], t[1], x.shape[2])
    return (m, Fp8Matrix(t[2], t[3], x.shape[1])) if transposed else m


def fp8_matmul(a: Fp8Matrix, b: Fp8Matrix, bias=None, dtype=torch.bfloat16, out=None):
    """a b^T (+ bias) per worker: a [k][m] and b [k][n] rows of the same length; [k][m][n] in dtype, or into out."""
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError("dtype is %s: float32 or bfloat16 is wanted" % dtype)
    return (_MODULE or _ops()).fp8_matmul(a.q, a.scale, a.n, b.q, b.scale, b.n, bias, out, dtype is torch.bfloat16)


def fp8_linear(x, weight: Fp8Matrix, bias=None, out=None):
    """x W^T (+ bias) with x [k][rows][n] quantised on the way and W kept in 8 bits; [k][rows][W's rows] in x's type."""
    return (_MODULE or _ops()).fp8_linear(x, weight.q, weight.scale, weight.n, bias, out)
