"""Penalties, biases and masks on logits against the definition in 64 bits.

Bounds (U = 2^-24): the division or product, c times the frequency, the presence's addition, the subtraction and the bias's addition are
rounded once each: 5 roundings of at most the sum of the magnitudes, then the output's type."""
import math

import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _definition(z, history, filled, answer, rep, pre, freq, bias, mask):
    """(what it is, a bound of it before its rounding to a type, where nothing applies)"""
    k, rows, vocab = z.shape
    want, size = z.double().clone(), z.double().abs()
    seen, count = (torch.zeros(k, rows, vocab, dtype=torch.float64, device=DEV) for _ in range(2))
    if history is not None:
        m = history.shape[2]
        place = torch.arange(m, device=DEV)
        f = filled[..., None].clamp(0, m) if filled is not None else m
        a = answer[..., None] if answer is not None else 0
        real = (history >= 0) & (history < vocab) & (place < f)
        at = history.long().clamp(0, vocab - 1)
        seen.scatter_add_(2, at, real.double())
        count.scatter_add_(2, at, (real & (place >= a)).double())

    def of(t, other):
        return t.double()[..., None] if t is not None else torch.full((k, rows, 1), other, dtype=torch.float64, device=DEV)
    r, p, q = of(rep, 1.0), of(pre, 0.0), of(freq, 0.0)
    changed = torch.where(want > 0, want / r, want * r)
    want = torch.where(seen > 0, changed, want)
    want = torch.where(count > 0, want - (q * count + p), want)
    size = torch.maximum(size, changed.abs()) + torch.where(count > 0, q.abs() * count + p.abs(), 0.0)
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    same = (seen == 0) & (bias is None)
    if mask is not None:
        j = torch.arange(vocab, device=DEV)
        allowed = (mask.long()[..., j // 32] >> (j % 32)) & 1
        want = torch.where(allowed > 0, want, -math.inf)
        same &= allowed > 0
    return want, 5 * U * size, same


def _check(got, z, *rest):
    want, bound, same = _definition(z, *rest)
    low = want == -math.inf
    assert torch.equal(got == -math.inf, low)
    assert torch.equal(got[same], z[same])
    zero = torch.zeros_like(want)
    within(torch.where(low, zero, got.double()), torch.where(low, zero, want),
           torch.where(low, zero, bound + out_rounding(z.dtype) * (want.abs() + bound) + 1e-38), "logits")


def _request(k, rows, m, vocab, g):
    history = torch.randint(0, vocab, (k, rows, m), generator=g, device=DEV, dtype=torch.int32)
    history[..., ::3] = history[..., :1].clone()                    # one token again and again
    if m > 4:
        history[..., 4::9] = -1
        history[..., 3::10] = vocab
    filled = torch.randint(-1, m + 3, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    answer = torch.randint(-1, m + 2, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    rep, pre, freq = (torch.rand(k, rows, generator=g, device=DEV) + b for b in (0.5, -0.5, 0.0))
    return history, filled, answer, rep, pre, freq


def _bits(k, rows, vocab, g):
    mask = torch.randint(-(1 << 31), 1 << 31, (k, rows, (vocab + 31) // 32), generator=g, device=DEV).to(torch.int32)
    mask[:, ::3] = -1
    mask[:, 1::5] = 0                                        # nothing is allowed
    return mask


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 31, 32, 33, 100, 1000, 4097, 8191, 8192, 8193, 16385, 40003])
def test_everything_on_and_off(vocab, dtype):
    g = _gen(vocab)
    k, rows = 2, 7
    for m, with_bias, with_mask, pad, lead in ((1, False, False, 0, 0), (50, True, False, 3, 1), (300, False, True, 1, 5), (700, True, True, 0, 0)):
        z = padded((k, rows, vocab), pad, lead, dtype, g, 3.0)
        args = _request(k, rows, m, vocab, g) + (torch.randn(k, rows, vocab, generator=g, device=DEV) if with_bias else None,
                                                 _bits(k, rows, vocab, g) if with_mask else None)
        out = torch.full((k, rows, vocab + 2), 7.0, dtype=dtype, device=DEV)
        got = OPS.adjust_logits(z, *args, out=out[..., 1:vocab + 1])
        _check(got, z, *args)
        assert bool((out[..., 0] == 7).all()) and bool((out[..., -1] == 7).all())
        again = z.clone()
        OPS.adjust_logits(again, *args, out=again)           # in place
        assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parts_alone(dtype):
    g = _gen(1)
    k, rows, vocab, m = 3, 5, 9000, 600
    z = torch.randn(k, rows, vocab, generator=g, device=DEV).mul_(3).to(dtype)
    history, filled, answer, rep, pre, freq = _request(k, rows, m, vocab, g)
    bias, mask = torch.randn(k, rows, vocab, generator=g, device=DEV), _bits(k, rows, vocab, g)
    none = [None] * 8
    assert torch.equal(OPS.adjust_logits(z), z)
    for given in ({0: history}, {0: history, 3: rep}, {0: history, 4: pre}, {0: history, 5: freq}, {0: history, 1: filled, 5: freq},
                  {0: history, 2: answer, 3: rep, 4: pre}, {6: bias}, {7: mask}, {3: rep, 4: pre, 5: freq}, {0: history, 3: rep, 7: mask}):
        args = [given.get(i) for i in range(8)]
        _check(OPS.adjust_logits(z, *args), z, *args)
        again = z.clone()
        OPS.adjust_logits(again, *args, out=again)
        assert torch.equal(again, OPS.adjust_logits(z, *args)), sorted(given)
    empty = torch.empty(k, rows, 0, dtype=torch.int32, device=DEV)
    assert torch.equal(OPS.adjust_logits(z, empty, filled, answer, rep, pre, freq), z)
    assert none == [None] * 8


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_history_bias_and_mask(dtype):
    g = _gen(2)
    k, rows, vocab, m = 2, 6, 10001, 100
    z = torch.randn(k, rows, vocab, generator=g, device=DEV).to(dtype)
    history, _, _, rep, pre, freq = _request(k, rows, m, vocab, g)
    bias, mask = torch.randn(k, rows, vocab, generator=g, device=DEV), _bits(k, rows, vocab, g)
    for shape in ((1, 1), (k, 1), (1, rows)):
        h, b, w = (t[:shape[0], :shape[1]].expand(k, rows, t.shape[2]) for t in (history, bias, mask[:, ::3].repeat(1, 3, 1)))
        got = OPS.adjust_logits(z, h, None, None, rep, pre, freq, b, w)
        assert torch.equal(got, OPS.adjust_logits(z, h.contiguous(), None, None, rep, pre, freq, b.contiguous(), w.contiguous()))
        _check(got, z, h, None, None, rep, pre, freq, b, w)
    shared = z[:1].expand(k, rows, vocab)                    # one row of logits for the workers
    assert torch.equal(OPS.adjust_logits(shared, history, None, None, rep), OPS.adjust_logits(shared.contiguous(), history, None, None, rep))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_masked_nan(dtype):
    z = torch.randn(1, 1, 200, generator=_gen(3), device=DEV).to(dtype)
    z[0, 0, 3], z[0, 0, 5], z[0, 0, 7], z[0, 0, 9] = -math.inf, math.inf, math.nan, torch.finfo(dtype).min
    history = torch.tensor([[[3, 5, 9]]], dtype=torch.int32, device=DEV)
    two, half = torch.full((1, 1), 2.0, device=DEV), torch.full((1, 1), 0.5, device=DEV)
    got = OPS.adjust_logits(z, history, repetition=two, presence=half)
    assert float(got[0, 0, 3]) == -math.inf and float(got[0, 0, 5]) == math.inf and math.isnan(float(got[0, 0, 7]))
    assert float(got[0, 0, 9]) == -math.inf                  # twice the lowest number
    mask = torch.zeros(1, 1, 7, dtype=torch.int32, device=DEV)
    mask[0, 0, 0] = 1 << 2
    got = OPS.adjust_logits(z, history, repetition=two, presence=half, mask=mask)
    assert torch.equal(got[0, 0, 2], z[0, 0, 2]) and int((got == -math.inf).sum()) == 199


def test_then_a_row_without_a_choice_has_no_probability():
    z = torch.randn(1, 2, 100, generator=_gen(4), device=DEV)
    mask = torch.full((1, 2, 4), -1, dtype=torch.int32, device=DEV)
    mask[0, 1] = 0
    got = OPS.token_logp(OPS.adjust_logits(z, mask=mask), torch.zeros(1, 2, dtype=torch.int32, device=DEV))
    assert math.isfinite(float(got[0, 0])) and float(got[0, 1]) == -math.inf


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [1, 2, 63, 64, 65, 1023, 1024, 1025, 4096, 5000, 9000, 20000])
def test_long_histories(m, dtype):
    """Also alone and in place, where nothing but the history's tokens changes."""
    g = _gen(m)
    for vocab in (50, 40003, 300000):
        z = torch.randn(1, 3, vocab, generator=g, device=DEV).mul_(3).to(dtype)
        args = _request(1, 3, m, vocab, g)
        got = OPS.adjust_logits(z, *args)
        _check(got, z, *args, None, None)
        again = z.clone()
        OPS.adjust_logits(again, *args, out=again)
        assert torch.equal(again, got)
