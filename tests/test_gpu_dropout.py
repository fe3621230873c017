"""Dropout against its stream computed apart, element by element.

Bounds (U = 2^-24): the factor is rounded once, the product and the sum with the residual once each, then the output's type."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within
from stream_ref import kept

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _check(y, x, res, p, seed, step, what=""):
    keep, factor = kept(*x.shape, p, seed, step)
    keep = keep.to(DEV)
    want = torch.where(keep, x.double() * factor, 0.0)
    size = want.abs()
    if res is not None:
        want = want + res.double()
        size = size + res.double().abs()
    bound = 3 * U * size
    within(y, want, bound + out_rounding(x.dtype) * (want.abs() + bound) + 1e-38, what)
    if res is None:
        assert bool((y[~keep] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 3, 2), (3, 5, 3), (2, 37, 4), (1, 4, 5), (3, 9, 8), (2, 65, 17), (1, 3, 64), (2, 7, 100),
                                   (2, 300, 257), (1, 2, 1000), (3, 5, 2049), (1, 3, 4096), (2, 2, 5003), (64, 3, 12), (1, 20000, 8)])
def test_against_its_stream(shape, dtype):
    g = _gen(sum(shape))
    for pad, lead, p, seed, step, with_res in ((0, 0, 0.1, 7, 0, True), (3, 1, 0.5, (1 << 64) - 3, 12345678901, False), (1, 5, 0.9, 0, 1, True)):
        x = padded(shape, pad, lead, dtype, g)
        res = padded(shape, pad + 2, lead, dtype, g, 2.0) if with_res else None
        k, rows, n = shape
        out = torch.full((k, rows, n + 2), 7.0, dtype=dtype, device=DEV)
        y = OPS.dropout(x, p, seed, step, residual=res, out=out[..., 1:n + 1])
        _check(y, x, res, p, seed, step)
        assert bool((out[..., 0] == 7).all()) and bool((out[..., -1] == 7).all())
        assert torch.equal(OPS.dropout(x, p, seed, step, residual=res), y)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shares_at_the_ends(dtype):
    x = torch.randn(2, 9, 133, generator=_gen(1), device=DEV).to(dtype)
    assert torch.equal(OPS.dropout(x, 0.0, 3), x)
    assert torch.equal(OPS.dropout(x, 1.0, 3), torch.zeros_like(x))
    assert torch.equal(OPS.dropout(x, 1.0, 3, residual=x), x)
    tiny = OPS.dropout(x, 2.0 ** -17, 3)                     # less than half a step: nothing is dropped
    assert torch.equal(tiny, x)
    ones = torch.ones(1, 1000, 1000, device=DEV)
    share = float((OPS.dropout(ones, 0.25, 11) == 0).double().mean())
    assert abs(share - 0.25) < 5 * (0.25 * 0.75 / 1e6) ** 0.5
    # workers, steps and seeds draw apart: two masks agree in a share 0.25^2 + 0.75^2 of their places
    a = OPS.dropout(torch.ones(2, 1000, 500, device=DEV), 0.25, 11) == 0
    b, c = (OPS.dropout(torch.ones(2, 1000, 500, device=DEV), 0.25, s, t) == 0 for s, t in ((11, 1), (12, 0)))
    for other in (a[1], b[0], c[0]):
        assert abs(float((a[0] == other).double().mean()) - 0.625) < 5 * (0.625 * 0.375 / 5e5) ** 0.5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_dropped_leaves_no_trace(dtype):
    x = torch.randn(2, 20, 77, generator=_gen(2), device=DEV).to(dtype)
    y = OPS.dropout(x, 0.5, 5)
    keep, _ = kept(2, 20, 77, 0.5, 5, 0)
    bad = x.clone()
    bad[~keep.to(DEV)] = torch.tensor([float("nan"), float("inf"), -float("inf")], device=DEV, dtype=dtype).repeat(2 * 20 * 77)[:int((~keep).sum())]
    assert torch.equal(OPS.dropout(bad, 0.5, 5), y)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_shared_inputs(dtype):
    g = _gen(3)
    x, res = (torch.randn(3, 11, 50, generator=g, device=DEV).to(dtype) for _ in range(2))
    want = OPS.dropout(x, 0.3, 9, 4, residual=res)
    a, b = x.clone(), res.clone()
    assert OPS.dropout(a, 0.3, 9, 4, residual=b, out=a) is a
    assert torch.equal(a, want) and torch.equal(b, res)
    a = x.clone()
    OPS.dropout(a, 0.3, 9, 4, residual=b, out=b)
    assert torch.equal(b, want) and torch.equal(a, x)
    one = x[:1].expand(3, 11, 50)                            # one x for the workers, a mask for each
    got = OPS.dropout(one, 0.3, 9, 4)
    assert torch.equal(got, OPS.dropout(one.contiguous(), 0.3, 9, 4)) and not torch.equal(got[0], got[1])
    wide = torch.zeros(11, 3, 50, dtype=dtype, device=DEV)   # workers interleaved row by row
    OPS.dropout(x, 0.3, 9, 4, residual=res, out=wide.transpose(0, 1))
    assert torch.equal(wide.transpose(0, 1), want)


def test_backward_is_the_same_call():
    """y is linear in x: <dropout(dy), v> = <dy, dropout(v)> for any two."""
    g = _gen(4)
    dy, v = (torch.randn(2, 30, 41, generator=g, device=DEV) for _ in range(2))
    left = (OPS.dropout(dy, 0.2, 8, 3).double() * v.double()).sum()
    right = (OPS.dropout(v, 0.2, 8, 3).double() * dy.double()).sum()
    assert abs(float(left - right)) <= 2 * 2 * U * float((dy * v).double().abs().sum() / 0.8)


def test_a_step_on_the_device():
    x = torch.randn(2, 33, 60, generator=_gen(5), device=DEV)
    step = torch.tensor(6, dtype=torch.int64, device=DEV)
    assert torch.equal(OPS.dropout(x, 0.4, 2, step), OPS.dropout(x, 0.4, 2, 6))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step += 1
        y = OPS.dropout(x, 0.4, 2, step)
    for t in range(7, 11):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, OPS.dropout(x, 0.4, 2, t))
    for bad in (torch.tensor(6, device=DEV, dtype=torch.int32), torch.tensor([6, 7], device=DEV), torch.tensor(6)):
        with pytest.raises(ValueError, match="step"):
            OPS.dropout(x, 0.4, 2, bad)
