"""CPU-only checks of the operators around the residual stream and sampling: what the C entry points refuse, before anything touches a
device, and the tensor-level wrappers' refusals."""
import os
import re

import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000              # addresses that are never followed: every call below is refused, or has nothing to do
NULL, CONFIG, HYPER, WORKSPACE, ARG, TOO_LARGE = -1, -2, -3, -4, -5, -8
NAN, INF = float("nan"), float("inf")


def test_binding_declares_as_many_arguments_as_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dw.h")).read(), flags=re.S)
    seen = 0
    for name, args in re.findall(r"\b(dw_[a-z_0-9]+)\s*\(([^)]*)\)\s*;", text):
        if name.startswith(("dw_embedding", "dw_dropout", "dw_rms", "dw_adjust")):
            assert len(getattr(B.lib(), name).argtypes) == args.count(",") + 1, name
            seen += 1
    assert seen == 8


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(k=65), CONFIG), (dict(dtype=2), CONFIG), (dict(t_type=-1), CONFIG), (dict(rows=-1), ARG), (dict(n=0), ARG),
    (dict(n=(1 << 24) + 1), ARG), (dict(vocab=0), ARG), (dict(vocab=(1 << 24) + 1), ARG), (dict(scale=NAN), HYPER), (dict(scale=INF), HYPER),
    (dict(token=None), NULL), (dict(table=None), NULL), (dict(y=None), NULL), (dict(token=P + 2), ARG), (dict(table=P + 2), ARG),
    (dict(table=P + 1, t_type=1), ARG), (dict(t_ld=7), ARG), (dict(t_st=-1), ARG), (dict(y=P), ARG), (dict(y=2 * P + 2), ARG), (dict(y_ld=7), ARG),
    (dict(y_st=23), ARG), (dict(rows=0), 0),
])
def test_embedding(kw, status):
    a = dict(token=P, table=P, t_ld=8, t_st=80, t_type=0, k=2, rows=3, vocab=10, n=8, dtype=0, scale=1.0, y=2 * P, y_ld=8, y_st=24, stream=None)
    a.update(kw)
    assert B.lib().dw_embedding(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=3), CONFIG), (dict(rows=-1), ARG), (dict(vocab=0), ARG), (dict(n=0), ARG), (dict(acc=2), ARG),
    (dict(scale=NAN), HYPER), (dict(grad=None), NULL), (dict(dy=None), NULL), (dict(token=None), NULL), (dict(token=P + 1), ARG), (dict(dy=P + 2), ARG),
    (dict(dy=2 * P), ARG), (dict(ld=7), ARG), (dict(g_ld=7), ARG), (dict(g_st=79), ARG), (dict(g_st=0), ARG), (dict(grad=2 * P + 2), ARG),
    (dict(scratch=None), WORKSPACE), (dict(scratch=P + 64), WORKSPACE), (dict(bytes=16), WORKSPACE), (dict(rows=0, acc=1), 0),
    (dict(rows=(1 << 27) + 1), TOO_LARGE), (dict(rows=1 << 20, n=65537, ld=65537, st=65537 << 20, g_ld=65537, g_st=655370), TOO_LARGE),
])
def test_embedding_grad(kw, status):
    a = dict(dy=P, ld=8, st=24, token=P, k=2, rows=3, vocab=10, n=8, dtype=0, scale=1.0, acc=0, grad=2 * P, g_ld=8, g_st=80, scratch=P, bytes=1 << 20,
             stream=None)
    a.update(kw)
    assert B.lib().dw_embedding_grad(*a.values()) == status


def test_scratch_sizes():
    lib = B.lib()
    f = lib.dw_embedding_grad_scratch_bytes
    assert f(0, 10, 10, 8) == f(1, 0, 10, 8) == f(1, 10, 0, 8) == f(1, 10, 10, 0) == 0
    assert f(1, 10, 10, 8) >= 2 * 10 * 4
    assert f(1, 1 << 27, 10, 512) > 0 and f(1, (1 << 27) + 1, 10, 512) == f(1, 1 << 27, 10, 513) == 0
    for rows in (1, 31, 33, 1000, 8192, 8193, 100000):       # two lists of places, partial sums, and what sorting takes
        assert 2 * 3 * rows * 4 <= f(3, rows, 50, 64) <= 3 * (rows * (16 + 64) + 64 * 4 * 4) + (1 << 20)
    g = lib.dw_rms_norm_grad_scratch_bytes
    assert g(0, 4, 4, 0) == 0 and g(1, 4, 4, 7) == 0
    for n in (1, 100, 5003, 40000):
        for dtype in (0, 1):
            b = g(3, 1000, n, dtype)
            assert b % (3 * n * 4) == 0 and 0 < b <= 3 * n * 4 * 1000


@pytest.mark.parametrize("kw,status", [
    (dict(k=65), CONFIG), (dict(dtype=2), CONFIG), (dict(rows=-1), ARG), (dict(n=0), ARG), (dict(p=-0.1), HYPER), (dict(p=1.1), HYPER),
    (dict(p=NAN), HYPER), (dict(x=None), NULL), (dict(y=None), NULL), (dict(x=P + 2), ARG), (dict(x_ld=7), ARG), (dict(x_st=-1), ARG),
    (dict(y_ld=7), ARG), (dict(y_st=23), ARG), (dict(res=P + 1), ARG), (dict(r_ld=7), ARG), (dict(d_step=P + 4), ARG),
    (dict(y=P, y_ld=9, y_st=27), ARG), (dict(y=3 * P, y_st=25), ARG), (dict(x_st=0, y=P), ARG), (dict(rows=0), 0),
])
def test_dropout(kw, status):
    a = dict(x=P, x_ld=8, x_st=24, res=3 * P, r_ld=8, r_st=24, k=2, rows=3, n=8, dtype=0, p=0.1, seed=1, step=2, d_step=None, y=2 * P, y_ld=8, y_st=24,
             stream=None)
    a.update(kw)
    assert B.lib().dw_dropout(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=2), CONFIG), (dict(rows=-1), ARG), (dict(n=0), ARG), (dict(n=(1 << 24) + 1), ARG),
    (dict(q=P, s=P, rows=(1 << 24) + 1, x_st=1 << 40, r_st=1 << 40, h_st=1 << 40, y_st=1 << 40), ARG), (dict(eps=-1.0), HYPER), (dict(eps=NAN), HYPER),
    (dict(eps=INF), HYPER), (dict(p=2.0), HYPER), (dict(x=None), NULL), (dict(y=None, h=None, rstd=None), NULL), (dict(q=P), NULL), (dict(qt=P), NULL),
    (dict(qt=P, st=P, rstd=None), NULL), (dict(qt=P, st=P, h=None), NULL), (dict(qt=P, st=P, h=None, res=None, p=0.1), NULL), (dict(x=P + 2), ARG),
    (dict(x_ld=7), ARG), (dict(res=P + 2), ARG), (dict(r_ld=7), ARG), (dict(gamma=P + 1), ARG), (dict(p_st=-1), ARG), (dict(rstd=P + 2), ARG),
    (dict(d_step=P + 4), ARG), (dict(h=P, h_ld=9, h_st=27), ARG), (dict(h=3 * P, h_st=25), ARG), (dict(h_ld=7), ARG), (dict(h_st=23), ARG),
    (dict(y=P), ARG), (dict(y=3 * P), ARG), (dict(y=4 * P), ARG), (dict(y_ld=7), ARG), (dict(q=P + 8, s=P), ARG), (dict(q=P, s=P + 2), ARG),
    (dict(qt=P + 8, st=P), ARG), (dict(qt=P, st=P + 1), ARG), (dict(rows=0), 0),
])
def test_rms_norm(kw, status):
    a = dict(x=P, x_ld=8, x_st=24, res=3 * P, r_ld=8, r_st=24, gamma=P, p_st=8, k=2, rows=3, n=8, dtype=0, eps=1e-6, p=0.0, seed=1, step=2, d_step=None,
             h=4 * P, h_ld=8, h_st=24, y=2 * P, y_ld=8, y_st=24, q=None, s=None, qt=None, st=None, rstd=P, stream=None)
    a.update(kw)
    assert B.lib().dw_rms_norm(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=65), CONFIG), (dict(dtype=-1), CONFIG), (dict(n=0), ARG), (dict(p=-1.0), HYPER), (dict(dy=None), NULL), (dict(h=None), NULL),
    (dict(rstd=None), NULL), (dict(dy=P + 2), ARG), (dict(h_ld=7), ARG), (dict(dh=P + 2), ARG), (dict(dh_ld=7), ARG), (dict(gamma=P + 2), ARG),
    (dict(d_step=P + 4), ARG), (dict(dres=2 * P), ARG), (dict(dres=5 * P), ARG), (dict(dres=P, dres_st=25), ARG), (dict(dres=3 * P, dres_ld=9, dres_st=27), ARG),
    (dict(dres_ld=7), ARG), (dict(dx=2 * P), ARG), (dict(dx=3 * P), ARG), (dict(dx=P, dx_st=30), ARG), (dict(dx_st=10), ARG), (dict(dg=P + 2), ARG),
    (dict(g_st=7), ARG), (dict(scratch=None), WORKSPACE), (dict(scratch=P + 64), WORKSPACE), (dict(bytes=16), WORKSPACE),
    (dict(dres=None, dx=None, dg=None), 0), (dict(rows=0, dg=None), 0),
])
def test_rms_norm_grad(kw, status):
    a = dict(dy=P, dy_ld=8, dy_st=24, h=2 * P, h_ld=8, h_st=24, gamma=P, p_st=8, rstd=P, dh=3 * P, dh_ld=8, dh_st=24, k=2, rows=3, n=8, dtype=0, p=0.1,
             seed=1, step=2, d_step=None, dres=4 * P, dres_ld=8, dres_st=24, dx=5 * P, dx_ld=8, dx_st=24, dg=P, g_st=8, scratch=P, bytes=1 << 20,
             stream=None)
    a.update(kw)
    assert B.lib().dw_rms_norm_grad(*a.values()) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), CONFIG), (dict(dtype=3), CONFIG), (dict(rows=-1), ARG), (dict(vocab=0), ARG), (dict(vocab=(1 << 24) + 1), ARG), (dict(m=-1), ARG),
    (dict(m=(1 << 24) + 1), ARG), (dict(z=None), NULL), (dict(out=None), NULL), (dict(hist=None), NULL), (dict(z=P + 2), ARG), (dict(ld=39), ARG),
    (dict(out_ld=39), ARG), (dict(out_st=119), ARG), (dict(out=P, out_ld=41, out_st=123), ARG), (dict(st=0, out=P), ARG), (dict(hist=P + 1), ARG),
    (dict(h_ld=5), ARG), (dict(h_st=-1), ARG), (dict(filled=P + 1), ARG), (dict(answer=P + 2), ARG), (dict(rep=P + 2), ARG), (dict(pre=P + 1), ARG),
    (dict(freq=P + 3), ARG), (dict(bias=P + 2), ARG), (dict(b_ld=39), ARG), (dict(mask=P + 2), ARG), (dict(m_ld=1), ARG), (dict(m_st=-2), ARG),
    (dict(rows=0), 0),
])
def test_adjust_logits(kw, status):
    a = dict(z=P, ld=40, st=120, hist=P, h_ld=6, h_st=18, m=6, filled=P, answer=P, rep=P, pre=P, freq=P, bias=P, b_ld=40, b_st=120, mask=P, m_ld=2, m_st=6,
             k=2, rows=3, vocab=40, dtype=0, out=2 * P, out_ld=40, out_st=120, stream=None)
    a.update(kw)
    assert B.lib().dw_adjust_logits(*a.values()) == status


def test_wrappers_want_tensors_on_a_gpu():
    x, f, t = torch.zeros(2, 3, 8), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: OPS.embedding(t, x), lambda: OPS.embedding_grad(x, t, 5), lambda: OPS.dropout(x, 0.1, 1), lambda: OPS.rms_norm(x),
                 lambda: OPS.rms_norm_fp8(x), lambda: OPS.rms_norm_grad(x, x, None, f), lambda: OPS.adjust_logits(x)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: OPS.embedding(t, x.half()), lambda: OPS.embedding(t, x, dtype=torch.float16), lambda: OPS.embedding(t, [1.0]),
                 lambda: OPS.embedding_grad(x[0], t, 5), lambda: OPS.dropout(x.transpose(1, 2), 0.1, 1), lambda: OPS.rms_norm(x.int()),
                 lambda: OPS.rms_norm_grad(x, [x], None, f), lambda: OPS.adjust_logits(f)):
        with pytest.raises(ValueError):
            call()
