"""The operators of the residual stream where every group of threads takes several rows, one after another: the next row on its way while this
one is worked on and written (over its inputs too), what a row leaves in registers and LDS for the next.  Whole results against the
formulas in 64 bits; the bounds are those of the operators' own files, as a row's sums are the same however many rows follow.

With 64 workers a grid has at most 2048 threads a compute unit for all of them, 8192 threads a worker (lookup 16 blocks of 256 a unit, dropout
64): the rows below are two and a half times what such a grid takes at once, or more."""
import functools

import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, within
from stream_ref import kept
from test_gpu_dropout import _check as check_dropout
from test_gpu_rms_norm import _c, _check_h, _check_norm, _same8, _y32

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
K = 64

# 4, 16, 32, 64, 256, 512 and 1024 threads a row, with one to four pieces each and elements behind them; rows past the registers
ROWS = [(17, 5300), (100, 1300), (257, 670), (511, 330), (1003, 330), (2050, 84), (4097, 84), (5003, 42), (8200, 42), (16390, 22), (20001, 42),
        (33000, 36)]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@functools.lru_cache(maxsize=1)
def _kept(k, rows, n, p, seed, step):
    keep, factor = kept(k, rows, n, p, seed, step)
    return keep.to(DEV), factor


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows", ROWS)
def test_norm_forward(n, rows, dtype, monkeypatch):
    monkeypatch.setattr("test_gpu_rms_norm.kept", _kept)
    g = _gen(n)
    x, res = (torch.randn(K, rows, n, generator=g, device=DEV).to(dtype) for _ in range(2))
    gamma = torch.randn(K, n, generator=g, device=DEV)
    drop = dict(p=0.3, seed=5, step=2)
    y, h, rstd = OPS.rms_norm(x, gamma, 1e-6, residual=res, **drop)
    _check_h(h, x, res, 0.3, 5, 2)
    _check_norm(y, h, gamma, 1e-6, rstd)
    plain, same, r = OPS.rms_norm(x, gamma, 1e-6)            # nothing in front of the norm
    assert same is x
    _check_norm(plain, x, gamma, 1e-6, r)
    over = res.clone()                                       # the sum over the residual
    y2, h2, r2 = OPS.rms_norm(x, gamma, 1e-6, residual=over, sum_out=over, **drop)
    assert h2 is over and torch.equal(over, h) and torch.equal(y2, y) and torch.equal(r2, rstd)
    del y, y2, plain, over
    want, want_t = OPS.fp8_quantize(_y32(h, gamma, rstd), transposed=True)
    over = x.clone()                                         # and over x, with both 8-bit forms
    (q, qt), h3, r3 = OPS.rms_norm_fp8(over, gamma, 1e-6, residual=res, sum_out=over, transposed=True, **drop)
    assert torch.equal(h3, h)
    if not torch.equal(r3, rstd):                            # (where the 8-bit form divides a row among other threads: its sum's order)
        _check_norm(_y32(h, gamma, r3).to(F32), h.to(F32), gamma, 1e-6, r3)
        want, want_t = OPS.fp8_quantize(_y32(h, gamma, r3), transposed=True)
    assert _same8(q, want) and _same8(qt, want_t)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows", ROWS)
def test_norm_backward(n, rows, dtype):
    g = _gen(100 + n)
    h, dy, dh = (torch.randn(K, rows, n, generator=g, device=DEV).to(dtype) for _ in range(3))
    gamma = torch.randn(K, n, generator=g, device=DEV)
    rstd = (h.float().square().mean(-1) + 1e-6).rsqrt().contiguous()
    keep, factor = _kept(K, rows, n, 0.3, 5, 2)
    drop = dict(p=0.3, seed=5, step=2)
    dres, dx, dgamma = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=dh, **drop)
    for w0 in range(0, K, 8):                                # (a few workers at a time in 64 bits)
        w = slice(w0, w0 + 8)
        r = rstd[w].double()[..., None]
        t, d = h[w].double() * r, dy[w].double()
        a = d * gamma[w].double()[:, None]
        at = a * t
        m, dm = at.mean(-1, keepdim=True), (_c(n) + 4) * U * at.abs().mean(-1, keepdim=True)
        want = r * (a - t * m)
        bound = r * (5 * U * (a.abs() + (t * m).abs()) + 1.01 * t.abs() * dm)
        want = want + dh[w].double()
        bound = bound + U * (want.abs() + dh[w].double().abs())
        within(dres[w], want, bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "dres")
        wx, bx = torch.where(keep[w], want * factor, 0.0), (bound + 2 * U * want.abs()) * 1.01 * factor
        within(dx[w], wx, bx + out_rounding(dtype) * (wx.abs() + bx) + 1e-38, "dx")
        assert not bool(dx[w][~keep[w]].any())
        within(dgamma[w], (d * t).sum(1), (rows + 34) * U * (d * t).abs().sum(1) + 1e-38, "dgamma")
    for over in ("dh", "dy", "dx"):
        b, e = dy.clone(), dh.clone()
        more = {"dh": dict(dres=e), "dy": dict(dres=b), "dx": dict(dx=b)}[over]
        got = OPS.rms_norm_grad(b, h, gamma, rstd, dh=e, **drop, **more)
        assert torch.equal(got[0], dres) and torch.equal(got[1], dx) and torch.equal(got[2], dgamma), over


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows", [(3, 165000), (40, 21000), (1000, 1300), (2051, 660)])
def test_dropout(n, rows, dtype, monkeypatch):
    monkeypatch.setattr("test_gpu_dropout.kept", _kept)
    g = _gen(n)
    x, res = (torch.randn(K, rows, n, generator=g, device=DEV).to(dtype) for _ in range(2))
    y = OPS.dropout(x, 0.4, 7, 3, residual=res)
    check_dropout(y, x, res, 0.4, 7, 3)
    check_dropout(OPS.dropout(x, 0.4, 7, 3), x, None, 0.4, 7, 3)
    over = x.clone()
    assert torch.equal(OPS.dropout(over, 0.4, 7, 3, residual=res, out=over), y)
    over = res.clone()
    assert torch.equal(OPS.dropout(x, 0.4, 7, 3, residual=over, out=over), y)


@pytest.mark.parametrize("n,rows", [(3, 41000), (40, 6000), (1000, 330), (2051, 165)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("table_dtype", [F32, BF16])
def test_lookup(n, rows, table_dtype, dtype):
    g = _gen(n)
    vocab = 501
    table = torch.randn(K, vocab, n, generator=g, device=DEV).to(table_dtype)
    token = torch.randint(-1, vocab + 1, (K, rows), generator=g, device=DEV, dtype=torch.int32)
    y = OPS.embedding(token, table, 0.5, dtype=dtype)
    there = (token >= 0) & (token < vocab)
    at = torch.where(there, token, 0).long() + vocab * torch.arange(K, device=DEV)[:, None]
    want = (table.view(-1, n)[at].float() * 0.5 * there[..., None]).to(dtype)              # (half of a number is exact: one rounding, to the type)
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_histories_in_place(dtype):
    """More rows of a worker than a grid has blocks, in place by tokens and out of place by logits: whole numbers, exact."""
    g = _gen(8)
    rows, vocab = (1 << 20) + 77, 64
    z = torch.randint(-8, 9, (1, rows, vocab), generator=g, device=DEV).to(dtype)
    history = torch.randint(0, vocab, (1, rows, 2), generator=g, device=DEV, dtype=torch.int32)
    freq = torch.randint(1, 4, (1, rows), generator=g, device=DEV).float()
    count = torch.zeros(1, rows, vocab, device=DEV).scatter_add_(2, history.long(), torch.ones(1, rows, 2, device=DEV))
    want = (z.float() - freq[..., None] * count).to(dtype)
    assert torch.equal(OPS.adjust_logits(z, history, frequency=freq), want)
    OPS.adjust_logits(z, history, frequency=freq, out=z)
    assert torch.equal(z, want)
