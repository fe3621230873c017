"""Operators of a language model's training step on the GPU, for k worker replicas in one call: thin wrappers over the
library's handle-free entry points (include/dw.h).

Tensors of activations are [k][rows][n] with contiguous rows (any row and worker stride, so views of wider buffers do),
float32 or bfloat16; parameters and their gradients are float32.  Outputs and scratch are allocated by torch on the
current stream of the tensors' device, where the work is enqueued; nothing is synchronised.  As with any torch operator,
a tensor made on another stream has to be waited for, and recorded, by the caller.  Wrong shapes, types or layouts raise
ValueError, what the library refuses DwError; there is no CPU path.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Tuple

import torch

from . import binding as B

_TYPES = {torch.float32: B.DW_F32, torch.bfloat16: B.DW_BF16}
_NO_GUARD = contextlib.nullcontext()


def _check(status: int, where: str) -> None:
    if status < 0:
        raise B.DwError(int(status), where)


def _type(t: torch.Tensor, name: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError("%s has type %s: float32 or bfloat16 is wanted" % (name, t.dtype))
    return code


def _on(device: torch.device):
    """The stream to enqueue on, and a guard for the case that the tensors' device is not the current one."""
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are wanted: got %s" % device)
    stream = torch.cuda.current_stream(device).cuda_stream
    return stream, (_NO_GUARD if device.index == torch.cuda.current_device() else torch.cuda.device(device))


def _matrix(t: torch.Tensor, name: str, shape=None, dtype=None, device=None) -> Tuple[int, int, int]:
    """(address, row stride, worker stride) of a [k][rows][n] tensor."""
    if t.dim() != 3 or (shape is not None and t.shape != shape):
        raise ValueError("%s has shape %s: %s is wanted" % (name, tuple(t.shape), "[k][rows][n]" if shape is None else tuple(shape)))
    if (dtype is not None and t.dtype != dtype) or (device is not None and t.device != device):
        raise ValueError("%s is %s on %s: %s on %s is wanted" % (name, t.dtype, t.device, dtype or t.dtype, device or t.device))
    k, rows, n = t.shape
    s0, s1, s2 = t.stride()
    if s2 != 1 and n > 1:
        raise ValueError("the rows of %s are not contiguous" % name)
    if rows <= 1:
        s1 = n
    return t.data_ptr(), s1, (rows * s1 if k <= 1 else s0)


def _param(t: Optional[torch.Tensor], name: str, k: int, n: int, device) -> Tuple[Optional[int], int]:
    """(address, worker stride) of a float32 [k][n] tensor, such as a view of flat parameter vectors."""
    if t is None:
        return None, n
    if t.shape != (k, n) or t.dtype != torch.float32 or t.device != device:
        raise ValueError("%s is %s %s on %s: float32 [%d][%d] on %s is wanted" % (name, t.dtype, tuple(t.shape), t.device, k, n, device))
    if n > 1 and t.stride(1) != 1:
        raise ValueError("the rows of %s are not contiguous" % name)
    return t.data_ptr(), (n if k == 1 else t.stride(0))


def _values(t: Optional[torch.Tensor], name: str, shape, dtype, device) -> Optional[int]:
    """Address of a contiguous tensor of that shape and type."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError("%s is %s %s on %s: a contiguous %s %s on %s is wanted" % (
            name, t.dtype, tuple(t.shape), t.device, dtype, tuple(shape), device))
    return t.data_ptr()


def _scratch(nbytes: int, device) -> Tuple[Optional[torch.Tensor], Optional[int]]:
    """Scratch memory (torch's allocations start at multiples of 256 and more) that lives until the work on the current
    stream that was enqueued with it is done."""
    if nbytes == 0:
        return None, None
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if t.data_ptr() % 256:
        t = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    return t, (t.data_ptr() + 255) // 256 * 256


# ---- layer norm ------------------------------------------------------------------------------------------------------

def layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, out=None, stats: bool = True):
    """y = (x - mean) * rstd * gamma + beta over the last axis of x [k][rows][n]; gamma, beta: float32 [k][n] or None.

    Returns (y, mean, rstd), the latter float32 [k][rows] for layer_norm_grad, or None both with stats=False (a served
    model).  out: a tensor like x for y."""
    code = _type(x, "x")
    xp, x_ld, x_st = _matrix(x, "x")
    k, rows, n = x.shape
    dev = x.device
    stream, guard = _on(dev)
    if gamma is not None and beta is not None and k > 1 and gamma.stride(0) != beta.stride(0):
        raise ValueError("gamma and beta have different worker strides")
    gp, p_st = _param(gamma, "gamma", k, n, dev)
    bp, b_st = _param(beta, "beta", k, n, dev)
    if out is None:
        out = torch.empty((k, rows, n), dtype=x.dtype, device=dev)
    yp, y_ld, y_st = _matrix(out, "out", x.shape, x.dtype, dev)
    mean = torch.empty((k, rows), dtype=torch.float32, device=dev) if stats else None
    rstd = torch.empty((k, rows), dtype=torch.float32, device=dev) if stats else None
    with guard:
        _check(B.lib().dw_layer_norm(xp, x_ld, x_st, gp, bp, p_st if gp is not None else b_st, k, rows, n, code, eps, yp, y_ld,
                                     y_st, mean.data_ptr() if stats else None, rstd.data_ptr() if stats else None, stream),
               "dw_layer_norm")
    return out, mean, rstd


def layer_norm_grad(dy, x, gamma, mean, rstd, dx=None, dgamma=None, dbeta=None, want_dx: bool = True, want_params: bool = True):
    """(dx, dgamma, dbeta) of layer_norm from dy, its input and the statistics it returned.  dx, dgamma, dbeta: tensors to
    write into (float32 [k][n] for the latter two, such as views of the flat gradient of Handle.update_only); what is not
    wanted is returned as None."""
    code = _type(x, "x")
    xp, x_ld, x_st = _matrix(x, "x")
    k, rows, n = x.shape
    dev = x.device
    stream, guard = _on(dev)
    dyp, dy_ld, dy_st = _matrix(dy, "dy", x.shape, x.dtype, dev)
    gp, p_st = _param(gamma, "gamma", k, n, dev)
    mp = _values(mean, "mean", (k, rows), torch.float32, dev)
    rp = _values(rstd, "rstd", (k, rows), torch.float32, dev)
    dxp, dx_ld, dx_st = None, n, rows * n
    if want_dx:
        if dx is None:
            dx = torch.empty((k, rows, n), dtype=x.dtype, device=dev)
        dxp, dx_ld, dx_st = _matrix(dx, "dx", x.shape, x.dtype, dev)
    dgp = dbp = scratch = sp = None
    g_st, nbytes = n, 0
    if want_params:
        if dgamma is None:
            dgamma = torch.empty((k, n), dtype=torch.float32, device=dev)
        if dbeta is None:
            dbeta = torch.empty((k, n), dtype=torch.float32, device=dev)
        dgp, g_st = _param(dgamma, "dgamma", k, n, dev)
        dbp, b_st = _param(dbeta, "dbeta", k, n, dev)
        if b_st != g_st:
            raise ValueError("dgamma and dbeta have different worker strides")
        nbytes = B.lib().dw_layer_norm_grad_scratch_bytes(k, rows, n, code)
        scratch, sp = _scratch(nbytes, dev)
    with guard:
        _check(B.lib().dw_layer_norm_grad(dyp, dy_ld, dy_st, xp, x_ld, x_st, gp, p_st, mp, rp, k, rows, n, code, dxp, dx_ld,
                                          dx_st, dgp, dbp, g_st, sp, nbytes, stream), "dw_layer_norm_grad")
    return (dx if want_dx else None), (dgamma if want_params else None), (dbeta if want_params else None)


# ---- policy loss -----------------------------------------------------------------------------------------------------

def token_logp(logits, target, out=None):
    """Log probabilities, float32 [k][rows], of the tokens target (int32 [k][rows]) under logits [k][rows][vocab]; 0 where
    the target lies outside the vocabulary."""
    code = _type(logits, "logits")
    zp, ld, st = _matrix(logits, "logits")
    k, rows, vocab = logits.shape
    dev = logits.device
    stream, guard = _on(dev)
    tp = _values(target, "target", (k, rows), torch.int32, dev)
    if out is None:
        out = torch.empty((k, rows), dtype=torch.float32, device=dev)
    op = _values(out, "out", (k, rows), torch.float32, dev)
    with guard:
        _check(B.lib().dw_token_logp(zp, ld, st, tp, k, rows, vocab, code, op, stream), "dw_token_logp")
    return out


def policy_loss(logits, target, old_logp, advantage, weight=None, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, grad=None, want_grad: bool = True):
    """(loss [k], logp [k][rows], gradient of the logits) of the clipped policy loss with a KL term; see dw_policy_loss.

    weight (float32 [k][rows], None: 1/rows): mask and average in one, the loss is the weighted sum; rows of weight 0 are
    not read.  grad: a tensor like logits to write into, the logits themselves among them; want_grad=False: None."""
    code = _type(logits, "logits")
    zp, ld, st = _matrix(logits, "logits")
    k, rows, vocab = logits.shape
    dev = logits.device
    stream, guard = _on(dev)
    tp = _values(target, "target", (k, rows), torch.int32, dev)
    if old_logp is None or advantage is None:
        raise ValueError("old_logp and advantage are wanted")
    op, ap, wp, rp = (_values(t, name, (k, rows), torch.float32, dev) for t, name in (
        (old_logp, "old_logp"), (advantage, "advantage"), (weight, "weight"), (ref_logp, "ref_logp")))
    gp, g_ld, g_st = None, vocab, rows * vocab
    if want_grad:
        if grad is None:
            grad = torch.empty((k, rows, vocab), dtype=logits.dtype, device=dev)
        gp, g_ld, g_st = _matrix(grad, "grad", logits.shape, logits.dtype, dev)
    loss = torch.empty(k, dtype=torch.float32, device=dev)
    logp = torch.empty((k, rows), dtype=torch.float32, device=dev)
    nbytes = B.lib().dw_policy_loss_scratch_bytes(k, rows)
    scratch, sp = _scratch(nbytes, dev)
    with guard:
        _check(B.lib().dw_policy_loss(zp, ld, st, tp, op, rp, ap, wp, k, rows, vocab, code, clip_low, clip_high, kl_coef,
                                      loss.data_ptr(), logp.data_ptr(), gp, g_ld, g_st, sp, nbytes, stream), "dw_policy_loss")
    return loss, logp, (grad if want_grad else None)


# ---- gradient norm and clipping --------------------------------------------------------------------------------------

def _clip(grads, max_norm: float, workers: int, out, where: str):
    if workers < 1 or len(grads) % workers:
        raise ValueError("%d tensors for %d workers" % (len(grads), workers))
    per = len(grads) // workers
    if per == 0:
        raise ValueError("no tensors")
    dev = grads[0].device
    stream, guard = _on(dev)
    counts, types = [g.numel() for g in grads], [_TYPES.get(g.dtype, -1) for g in grads]
    if any(g.device != dev for g in grads) or -1 in types:
        raise ValueError("float32 or bfloat16 tensors on one device are wanted")
    if not all(g.is_contiguous() for g in grads):
        raise ValueError("a gradient is not contiguous")
    for w in range(1, workers):
        if counts[w * per:(w + 1) * per] != counts[:per] or types[w * per:(w + 1) * per] != types[:per]:
            raise ValueError("worker %d has tensors of other sizes or types than worker 0" % w)
    total = sum(counts[:per])
    op, o_st = None, total
    if out is not None:
        op, o_st = _param(out, "out", workers, total, dev)
    addresses = (C.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
    sizes = (C.c_int64 * per)(*counts[:per])
    kinds = None if types[:per] == [types[0]] * per else (C.c_int32 * per)(*types[:per])
    norm = torch.empty(workers, dtype=torch.float32, device=dev)
    nbytes = B.lib().dw_clip_grads_scratch_bytes(workers, per, sizes)
    scratch, sp = _scratch(nbytes, dev)
    with guard:
        _check(B.lib().dw_clip_grads(addresses, sizes, kinds, workers, per, types[0], max_norm, op, o_st, norm.data_ptr(), sp, nbytes,
                                     stream), where)
    return norm


def clip_grads(grads, max_norm: float, workers: int = 1, out=None):
    """Clip every worker's gradients to a global 2-norm of at most max_norm; returns the norms before, float32 [workers].

    grads: the tensors of worker 0, then those of worker 1 in the same order and so on (contiguous, float32 or bfloat16).
    They are scaled in place, or left alone with out, float32 [workers][total]: the clipped gradients one behind the other,
    as Handle.update_only takes them."""
    return _clip(grads, max_norm, workers, out, "dw_clip_grads")


def grad_norm(grads, workers: int = 1):
    """The global 2-norm of every worker's gradients, float32 [workers]; grads as for clip_grads."""
    return _clip(grads, float("inf"), workers, None, "dw_clip_grads")


# ---- products in 8 bits ----------------------------------------------------------------------------------------------

class Fp8Matrix:
    """[k][rows] rows of n numbers in e4m3, each row padded with zeros to whole blocks of 128, and their scales.

    q: float8_e4m3fn [k][rows][padded n]; scale: uint8 [k][rows][blocks, to a multiple of 4], 2^(scale - 127)."""

    __slots__ = ("q", "scale", "n")

    def __init__(self, k: int, rows: int, n: int, device):
        self.n = n
        self.q = torch.empty((k, rows, (n + 127) // 128 * 128), dtype=torch.float8_e4m3fn, device=device)
        self.scale = torch.empty((k, rows, (n + 511) // 512 * 4), dtype=torch.uint8, device=device)

    @property
    def shape(self):
        return (self.q.shape[0], self.q.shape[1], self.n)


def fp8_quantize(x, square: bool = False, transposed: bool = False):
    """x [k][rows][n] in 8 bits with a scale per block of 128 along its rows (square: per 128 x 128), an Fp8Matrix.
    transposed=True: (that, the same of x^T): [k][n] rows of `rows`, its blocks along those."""
    code = _type(x, "x")
    xp, x_ld, x_st = _matrix(x, "x")
    k, rows, n = x.shape
    dev = x.device
    stream, guard = _on(dev)
    m = Fp8Matrix(k, rows, n, dev)
    t = Fp8Matrix(k, n, rows, dev) if transposed else None
    with guard:
        _check(B.lib().dw_fp8_quantize(xp, x_ld, x_st, k, rows, n, code, int(square), m.q.data_ptr(), m.scale.data_ptr(),
                                       t.q.data_ptr() if t else None, t.scale.data_ptr() if t else None, stream), "dw_fp8_quantize")
    return (m, t) if transposed else m


def fp8_matmul(a: Fp8Matrix, b: Fp8Matrix, bias=None, dtype=torch.bfloat16, out=None):
    """a b^T (+ bias) per worker: a [k][m] and b [k][n] rows of the same length; [k][m][n] in dtype, or into out."""
    k, m, length = a.shape
    if b.shape[0] != k or b.n != length or b.q.device != a.q.device:
        raise ValueError("operands of %s and %s" % (a.shape, b.shape))
    n, dev = b.shape[1], a.q.device
    stream, guard = _on(dev)
    bp, b_st = _param(bias, "bias", k, n, dev)
    if out is None:
        out = torch.empty((k, m, n), dtype=dtype, device=dev)
    code = _type(out, "out")
    cp, c_ld, c_st = _matrix(out, "out", (k, m, n), None, dev)
    L = B.lib()
    nbytes = L.dw_fp8_matmul_scratch_bytes(k, m, n, length)
    scratch, sp = _scratch(nbytes, dev)
    with guard:
        _check(L.dw_fp8_matmul(a.q.data_ptr(), a.scale.data_ptr(), b.q.data_ptr(), b.scale.data_ptr(), bp, b_st, k, m, n, length,
                               code, cp, c_ld, c_st, sp, nbytes, stream), "dw_fp8_matmul")
    return out


def fp8_linear(x, weight: Fp8Matrix, bias=None, out=None):
    """x W^T (+ bias) with x [k][rows][n] quantised on the way and W kept in 8 bits; [k][rows][W's rows] in x's type."""
    return fp8_matmul(fp8_quantize(x), weight, bias, dtype=x.dtype, out=out)
