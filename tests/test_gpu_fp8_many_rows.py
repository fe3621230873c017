"""Matrices in 8 bits of more rows than a grid has blocks along y (65535, of 16 rows or 128): the same as of their parts, which lie below."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _x(k, rows, n, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    return torch.randn(k, rows, n, generator=g, device=DEV).to(dtype)


def _bytes(m):
    return m.q.view(torch.uint8), m.scale


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows(dtype):
    rows = 65535 * 16 + 37
    x = _x(2, rows, 35, dtype)
    q, scale = _bytes(OPS.fp8_quantize(x))
    for a, b in ((0, 1 << 19), (1 << 19, rows)):
        q1, s1 = _bytes(OPS.fp8_quantize(x[:, a:b]))
        assert torch.equal(q[:, a:b], q1) and torch.equal(scale[:, a:b], s1)


def _check_transposed(whole, part_of, rows, edge):
    """Blocks of 128 rows of x stand alone: those of the two parts of x, next to each other, and what fills a row of scales."""
    q, s = _bytes(whole)
    blocks = (rows + 127) // 128
    for a, b in ((0, edge), (edge, rows)):
        q1, s1 = _bytes(part_of(a, b))
        assert torch.equal(q[..., a:a + q1.shape[2]], q1)
        assert torch.equal(s[..., a // 128:(b + 127) // 128], s1[..., :(b - a + 127) // 128])
    assert bool((s[..., blocks:] == 127).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("square", [False, True])
def test_transposed(square, dtype):
    rows, edge = 65535 * 128 + 300, 1 << 22
    x = _x(1, rows, 3, dtype)
    q, qt = OPS.fp8_quantize(x, square=square, transposed=True)
    _check_transposed(qt, lambda a, b: OPS.fp8_quantize(x[:, a:b], square=square, transposed=True)[1], rows, edge)
    for a, b in ((0, edge), (edge, rows)):
        part = OPS.fp8_quantize(x[:, a:b], square=square, transposed=True)[0]
        assert torch.equal(_bytes(q)[0][:, a:b], _bytes(part)[0]) and torch.equal(q.scale[:, a:b], part.scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_transposed(dtype):
    rows, edge = 65535 * 128 + 300, 1 << 22
    x = _x(1, rows, 5, dtype)
    gamma = torch.randn(1, 5, device=DEV)
    (q, qt), h, rstd = OPS.rms_norm_fp8(x, gamma, transposed=True)
    assert h is x
    y = x.float() * rstd[..., None] * gamma[:, None]
    want = OPS.fp8_quantize(y)
    assert torch.equal(_bytes(q)[0], _bytes(want)[0]) and torch.equal(q.scale, want.scale)
    _check_transposed(qt, lambda a, b: OPS.fp8_quantize(y[:, a:b], transposed=True)[1], rows, edge)
