"""CPU-only checks of the handle-free operators: what the C entry points refuse, before anything touches a device, their
declarations, and the tensor-level wrappers' refusals."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000              # addresses that are never followed: every call below is refused
NULL, CONFIG, HYPER, WORKSPACE, ARG, LARGE = -1, -2, -3, -4, -5, -8


def test_binding_declares_as_many_arguments_as_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dw.h")).read(), flags=re.S)
    lib = B.lib()
    seen = 0
    for name, args in re.findall(r"\b(dw_[a-z_0-9]+)\s*\(([^)]*)\)\s*;", text):
        want = 0 if args.strip() in ("", "void") else args.count(",") + 1
        if name.startswith(("dw_layer", "dw_token", "dw_policy", "dw_clip", "dw_fp8")):
            assert len(getattr(lib, name).argtypes) == want, name
            seen += 1
    assert seen == 13


def _norm(**kw):
    a = dict(x=P, x_ld=8, x_st=24, gamma=P, beta=P, p_st=8, k=2, rows=3, n=8, dtype=0, eps=1e-5, y=2 * P, y_ld=8, y_st=24,
             mean=P, rstd=P, stream=None)
    a.update(kw)
    return B.lib().dw_layer_norm(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(k=65), CONFIG), (dict(dtype=2), CONFIG), (dict(rows=-1), ARG), (dict(n=0), ARG),
    (dict(n=(1 << 24) + 1), ARG), (dict(eps=-1.0), HYPER), (dict(eps=float("nan")), HYPER), (dict(eps=float("inf")), HYPER),
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(x=P + 2), ARG), (dict(x=P + 1, dtype=1), ARG), (dict(x_ld=7), ARG),
    (dict(x_ld=-8), ARG), (dict(x_st=-1), ARG), (dict(y_ld=7), ARG), (dict(y_st=23), ARG), (dict(y=P), ARG), (dict(gamma=P + 1), ARG),
    (dict(beta=P + 2), ARG), (dict(p_st=-1), ARG), (dict(mean=P + 1), ARG), (dict(rstd=P + 2), ARG), (dict(rows=0), 0),
])
def test_layer_norm(kw, status):
    assert _norm(**kw) == status


def _norm_grad(**kw):
    a = dict(dy=P, dy_ld=8, dy_st=24, x=P, x_ld=8, x_st=24, gamma=P, p_st=8, mean=P, rstd=P, k=2, rows=3, n=8, dtype=0, dx=2 * P,
             dx_ld=8, dx_st=24, dg=P, db=2 * P, g_st=8, scratch=P, bytes=1 << 20, stream=None)
    a.update(kw)
    return B.lib().dw_layer_norm_grad(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(k=65), CONFIG), (dict(dtype=-1), CONFIG), (dict(n=0), ARG), (dict(dy=None), NULL), (dict(x=None), NULL), (dict(mean=None), NULL),
    (dict(rstd=None), NULL), (dict(dx=P), ARG), (dict(dx_st=10), ARG), (dict(dx_ld=4), ARG), (dict(g_st=7), ARG), (dict(dg=2 * P), ARG),
    (dict(db=P + 2), ARG), (dict(scratch=None), WORKSPACE), (dict(scratch=P + 64), WORKSPACE), (dict(bytes=16), WORKSPACE),
    (dict(dx=None, dg=None, db=None), 0), (dict(rows=0, dg=None, db=None), 0),
])
def test_layer_norm_grad(kw, status):
    assert _norm_grad(**kw) == status


def test_scratch_sizes():
    lib = B.lib()
    assert lib.dw_layer_norm_grad_scratch_bytes(0, 4, 4, 0) == 0 and lib.dw_layer_norm_grad_scratch_bytes(1, 4, 4, 7) == 0
    for n in (1, 100, 5003, 40000):
        for dtype in (0, 1):
            b = lib.dw_layer_norm_grad_scratch_bytes(3, 1000, n, dtype)
            assert b % (3 * 2 * n * 4) == 0 and 0 < b <= 3 * 2 * n * 4 * 1000
    assert lib.dw_policy_loss_scratch_bytes(3, 100) == 1200 and lib.dw_policy_loss_scratch_bytes(65, 100) == 0
    sizes = (C.c_int64 * 3)(5, 0, 10000)
    assert lib.dw_clip_grads_scratch_bytes(2, 3, sizes) == 2 * (1 + 3 + 1) * 8
    assert lib.dw_clip_grads_scratch_bytes(2, 3, (C.c_int64 * 3)(5, -1, 3)) == 0
    assert lib.dw_fp8_matmul_scratch_bytes(1, 1, 4096, 4096) == 0                   # one token: read once, no slices
    s = lib.dw_fp8_matmul_scratch_bytes(1, 100, 100, 8192)                           # few tiles, long contraction: slices
    assert s > 0 and s % (100 * 100 * 4) == 0
    assert lib.dw_fp8_matmul_scratch_bytes(1, 0, 100, 8192) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=3), CONFIG), (dict(rows=-1), ARG), (dict(vocab=0), ARG), (dict(z=None), NULL), (dict(y=None), NULL),
    (dict(out=None), NULL), (dict(z=P + 2), ARG), (dict(ld=9), ARG), (dict(y=P + 2), ARG), (dict(out=P + 1), ARG), (dict(rows=0), 0),
])
def test_token_logp(kw, status):
    a = dict(z=P, ld=10, st=30, y=P, k=2, rows=3, vocab=10, dtype=0, out=P, stream=None)
    a.update(kw)
    assert B.lib().dw_token_logp(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=65), CONFIG), (dict(dtype=3), CONFIG), (dict(vocab=(1 << 24) + 1), ARG), (dict(low=-0.1), HYPER), (dict(low=1.1), HYPER),
    (dict(high=-0.1), HYPER), (dict(high=float("inf")), HYPER), (dict(kl=float("nan")), HYPER), (dict(z=None), NULL), (dict(old=None), NULL),
    (dict(adv=None), NULL), (dict(ref=None), NULL), (dict(adv=P + 1), ARG), (dict(grad=3 * P, g_ld=9), ARG), (dict(grad=3 * P, g_st=29), ARG),
    (dict(grad=P, g_ld=11, g_st=33), ARG), (dict(scratch=None), WORKSPACE), (dict(bytes=8), WORKSPACE), (dict(loss=P + 2), ARG),
])
def test_policy_loss(kw, status):
    a = dict(z=P, ld=10, st=30, y=P, old=P, ref=P, adv=P, w=None, k=2, rows=3, vocab=10, dtype=0, low=0.2, high=0.2, kl=0.1, loss=P, logp=P,
             grad=2 * P, g_ld=10, g_st=30, scratch=P, bytes=1 << 10, stream=None)
    a.update(kw)
    assert B.lib().dw_policy_loss(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(n=-1), ARG), (dict(n=(1 << 20) + 1), ARG), (dict(count=None), NULL), (dict(dtype=4), CONFIG),
    (dict(kinds=(C.c_int32 * 2)(0, 9)), CONFIG), (dict(max_norm=0.0), HYPER), (dict(max_norm=float("nan")), HYPER), (dict(norm=None), NULL),
    (dict(grad=None), NULL), (dict(grad=(C.c_void_p * 4)(P, P, None, P)), NULL), (dict(grad=(C.c_void_p * 4)(P, P + 2, P, P)), ARG),
    (dict(out=P, o_st=29), ARG), (dict(out=P + 2), ARG), (dict(scratch=None), WORKSPACE), (dict(bytes=8), WORKSPACE),
    (dict(count=(C.c_int64 * 2)(-1, 4)), ARG),
])
def test_clip_grads(kw, status):
    a = dict(grad=(C.c_void_p * 4)(P, P, P, P), count=(C.c_int64 * 2)(10, 20), kinds=None, k=2, n=2, dtype=0, max_norm=1.0, out=None, o_st=30,
             norm=P, scratch=P, bytes=1 << 10, stream=None)
    a.update(kw)
    assert B.lib().dw_clip_grads(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=2), CONFIG), (dict(rows=-1), ARG), (dict(n=0), ARG), (dict(square=2), ARG), (dict(x=None), NULL),
    (dict(q=None), NULL), (dict(s=None), NULL), (dict(qt=P, st=None), NULL), (dict(x=P + 2), ARG), (dict(q=P + 8), ARG), (dict(s=P + 2), ARG),
    (dict(qt=P + 8, st=P), ARG), (dict(x_ld=7), ARG), (dict(rows=0), 0),
])
def test_fp8_quantize(kw, status):
    a = dict(x=P, x_ld=8, x_st=24, k=2, rows=3, n=8, dtype=0, square=0, q=P, s=P, qt=None, st=None, stream=None)
    a.update(kw)
    assert B.lib().dw_fp8_quantize(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=65), CONFIG), (dict(dtype=2), CONFIG), (dict(m=-1), ARG), (dict(n=0), ARG), (dict(length=-1), ARG), (dict(a=None), NULL),
    (dict(sb=None), NULL), (dict(c=None), NULL), (dict(b=P + 8), ARG), (dict(sa=P + 1), ARG), (dict(c_ld=99), ARG), (dict(c_st=9999), ARG),
    (dict(bias=P + 2), ARG), (dict(m=1 << 20, n=1 << 20, c_ld=1 << 20, c_st=1 << 40), LARGE), (dict(length=8192), WORKSPACE),
    (dict(length=8192, scratch=P + 4, bytes=1 << 30), WORKSPACE), (dict(m=0), 0),
])
def test_fp8_matmul(kw, status):
    a = dict(a=P, sa=P, b=P, sb=P, bias=None, b_st=100, k=2, m=100, n=100, length=256, dtype=0, c=P, c_ld=100, c_st=10000, scratch=None, bytes=0,
             stream=None)
    a.update(kw)
    assert B.lib().dw_fp8_matmul(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=5), CONFIG), (dict(m=-1), ARG), (dict(length=0), ARG), (dict(x=None), NULL), (dict(w=None), NULL),
    (dict(sw=None), NULL), (dict(y=None), NULL), (dict(x=P + 2), ARG), (dict(w=P + 8), ARG), (dict(x_ld=255), ARG), (dict(y_ld=99), ARG),
    (dict(scratch=None), WORKSPACE), (dict(bytes=100), WORKSPACE), (dict(m=0), 0),
])
def test_fp8_linear(kw, status):
    a = dict(x=P, x_ld=256, x_st=25600, w=P, sw=P, bias=None, b_st=100, k=2, m=100, n=100, length=256, dtype=0, y=P, y_ld=100, y_st=10000,
             scratch=P, bytes=1 << 20, stream=None)
    a.update(kw)
    assert B.lib().dw_fp8_linear(*a.values()) == status
    assert B.lib().dw_fp8_linear_scratch_bytes(1, 1, 4096, 4096) == 0 and B.lib().dw_fp8_linear_scratch_bytes(2, 100, 100, 256) >= 2 * 100 * 260


def test_wrappers_want_tensors_on_a_gpu():
    x, f = torch.zeros(2, 3, 8), torch.zeros(2, 3)
    for call in (lambda: OPS.layer_norm(x), lambda: OPS.layer_norm_grad(x, x, None, f, f), lambda: OPS.token_logp(x, f.int()),
                 lambda: OPS.policy_loss(x, f.int(), f, f), lambda: OPS.clip_grads([x, x], 1.0, 2), lambda: OPS.grad_norm([x]),
                 lambda: OPS.fp8_quantize(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: OPS.layer_norm(x.half()), lambda: OPS.layer_norm(x[0]), lambda: OPS.layer_norm(x.transpose(1, 2)),
                 lambda: OPS.layer_norm([1.0]), lambda: OPS.clip_grads([], 1.0), lambda: OPS.clip_grads([x, x, x], 1.0, 2)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        OPS.clip_grads(5, 1.0)
