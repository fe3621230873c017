"""Operators on tensors whose elements lie further apart than 32 bits count, and on more rows than 16 bits count: the same bits
as on small contiguous copies."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _far(k, rows, n, dtype):
    """[k][rows][n] in one buffer of more than 2^32 elements: far workers, or far rows of one."""
    stride, pitch = ((2 ** 32 // (k - 1)) + 72, n + 8) if k > 1 else (0, (2 ** 32 // (rows - 1)) + 24)
    buf = torch.empty((k - 1) * stride + (rows - 1) * pitch + n, dtype=dtype, device=DEV)
    return buf.as_strided((k, rows, n), (stride, pitch, 1))


def _far_copy(x):
    return _far(*x.shape, x.dtype).copy_(x)


PLACES = [(2, 3, 1000), (1, 5, 1000)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PLACES)
def test_layer_norm(shape, dtype):
    g = _gen(1)
    k, rows, n = shape
    x, dy = (torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(2))
    gamma, beta = (torch.randn(k, n, generator=g, device=DEV) for _ in range(2))
    y, mean, rstd = OPS.layer_norm(x, gamma, beta)
    xf, out = _far_copy(x), _far(*shape, dtype)
    got = OPS.layer_norm(xf, gamma, beta, out=out)
    assert torch.equal(got[0], y) and torch.equal(out, y) and torch.equal(got[1], mean) and torch.equal(got[2], rstd)
    for want, have in zip(OPS.layer_norm_grad(dy, x, gamma, mean, rstd), OPS.layer_norm_grad(_far_copy(dy), xf, gamma, mean, rstd, dx=out)):
        assert torch.equal(want, have)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PLACES + [(1, 3, 40000)])
def test_policy_loss(shape, dtype):
    g = _gen(2)
    k, rows, vocab = shape
    z = torch.randn(shape, generator=g, device=DEV).to(dtype)
    target = torch.randint(0, vocab, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    old, adv = (torch.randn(k, rows, generator=g, device=DEV) for _ in range(2))
    old -= 7
    zf = _far_copy(z)
    assert torch.equal(OPS.token_logp(z, target), OPS.token_logp(zf, target))
    for want, have in zip(OPS.policy_loss(z, target, old, adv), OPS.policy_loss(zf, target, old, adv, grad=_far(*shape, dtype))):
        assert torch.equal(want, have)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PLACES)
def test_quantiser_and_linear_layer(shape, dtype):
    g = _gen(3)
    k, rows, n = shape
    x = torch.randn(shape, generator=g, device=DEV).to(dtype)
    xf = _far_copy(x)
    for square in (False, True):
        for want, have in zip(OPS.fp8_quantize(x, square, True), OPS.fp8_quantize(xf, square, True)):
            assert torch.equal(want.q.view(torch.uint8), have.q.view(torch.uint8)) and torch.equal(want.scale, have.scale)
    w = OPS.fp8_quantize(torch.randn(k, n, n, generator=g, device=DEV), square=True)
    y, out = OPS.fp8_linear(x, w), _far(*shape, dtype)
    OPS.fp8_linear(xf, w, out=out)
    assert torch.equal(out, y)
    a = OPS.fp8_quantize(torch.randn(k, rows, 9000, generator=g, device=DEV))      # tiles, their contraction cut
    b = OPS.fp8_quantize(torch.randn(k, n, 9000, generator=g, device=DEV))
    OPS.fp8_matmul(a, b, out=out)
    assert torch.equal(out, OPS.fp8_matmul(a, b, dtype=dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_of_operands_past_32_bits(dtype):
    """a and b of 2^32 numbers and more in turn: the last rows' products against those of a matrix that holds them alone."""
    g = _gen(4)
    rows, length, few = 2 ** 20 + 300, 4096, 200
    x = torch.randn(1, 1000, length, generator=g, device=DEV, dtype=BF16)
    long = OPS.fp8_quantize(torch.zeros(1, rows, length, device=DEV, dtype=BF16))
    some, other = OPS.fp8_quantize(x), OPS.fp8_quantize(torch.randn(1, few, length, generator=g, device=DEV, dtype=BF16))
    long.q[:, -1000:] = some.q
    long.scale[:, -1000:] = some.scale
    want = OPS.fp8_matmul(some, other, dtype=dtype).double()
    bound = (2.0 ** -8 if dtype == BF16 else 2.0 ** -20) * (want.abs() + float(want.abs().mean()))    # (tiles of other sizes add in another order)
    c = OPS.fp8_matmul(long, other, dtype=dtype)
    within(c[:, -1000:], want, bound, "rows of a")
    assert bool((c[:, :-1000] == 0).all())
    c = OPS.fp8_matmul(other, long, dtype=dtype)
    within(c[..., -1000:], want.transpose(1, 2), bound.transpose(1, 2), "rows of b")
    assert bool((c[..., :-1000] == 0).all())
    one = OPS.fp8_matmul(OPS.Fp8Matrix(other.q[:, :1], other.scale[:, :1], length), long, dtype=dtype)
    within(one[..., -1000:], want.transpose(1, 2)[:, :1], bound.transpose(1, 2)[:, :1], "a single row")


def test_quantiser_of_more_rows_than_16_bits_count():
    """128 x 65540 rows of one worker hold the numbers of 20 workers that divide them in whole blocks."""
    rows, n, parts = 128 * 65540, 8, 20
    x = torch.randn(1, rows, n, generator=_gen(5), device=DEV, dtype=BF16)
    for square in (False, True):
        whole, turned = OPS.fp8_quantize(x, square, True)
        part, part_turned = OPS.fp8_quantize(x.view(parts, rows // parts, n), square, True)
        assert torch.equal(whole.q.view(torch.uint8).view(parts, rows // parts, -1), part.q.view(torch.uint8))
        assert torch.equal(whole.scale.view(parts, rows // parts, -1), part.scale)
        blocks = rows // parts // 128
        assert torch.equal(turned.q.view(torch.uint8).view(n, parts, -1), part_turned.q.view(torch.uint8).transpose(0, 1))
        assert torch.equal(turned.scale[0, :, :parts * blocks].reshape(n, parts, blocks), part_turned.scale[..., :blocks].transpose(0, 1))
    alone = OPS.fp8_quantize(x)
    assert torch.equal(alone.q.view(torch.uint8).view(parts, rows // parts, -1), OPS.fp8_quantize(x.view(parts, rows // parts, n)).q.view(torch.uint8))


def test_gradients_past_32_bits():
    """Norms of a tensor of more than 2^32 elements, zero but for a few at its ends; clipped in place."""
    big = torch.zeros(2 ** 32 + 1000, dtype=BF16, device=DEV)
    big[:3] = 3.0
    big[-7:] = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0])
    norm = float(27 + 140) ** 0.5
    assert abs(float(OPS.grad_norm([big])[0]) - norm) < 1e-6 * norm
    OPS.clip_grads([big], 1.0)
    factor = 1.0 / (norm + 1e-6)
    assert torch.allclose(big[-7:].double(), torch.arange(1, 8, device=DEV).double() * factor, rtol=2.0 ** -8)
    assert torch.allclose(big[:3].double(), torch.full((3,), 3 * factor, device=DEV, dtype=torch.float64), rtol=2.0 ** -8)
