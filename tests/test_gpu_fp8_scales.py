"""Products of 8-bit matrices at the ends of the scales' range (bytes 1 to 247, powers -126 to 120), against 64 bits.

fp32 results come from numbers widened to bf16 at half their size, whose smallest step is 2^-133: a number is exact in steps of
2^-132 (half a step of rounding, 2^-133) and exact altogether from byte 4 on, whose step is 2^-9 2^-123.  bf16 results come
from the instruction that applies the scales by itself."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
# a single row, few rows, slices, tiles of 64, 128 and 256, as (m, n, contraction)
FORMS = [(1, 300, 200), (20, 300, 600), (100, 130, 5000), (254, 270, 130), (1600, 1700, 130), (4096, 4096, 130)]


def _two_to(e):
    return torch.ldexp(torch.ones((), dtype=torch.float64), torch.tensor(e)).to(DEV)


def _codes():
    c = torch.arange(256, device=DEV).to(torch.uint8)
    return c[(c & 127) != 127]                              # all finite numbers


def _matrix(q, byte, n):
    """[rows][padded] codes with one scale byte for all blocks."""
    scales = (n + 511) // 512 * 4
    s = torch.full((1, q.shape[0], scales), byte, dtype=torch.uint8, device=DEV)
    return OPS.Fp8Matrix(q[None].contiguous().view(torch.float8_e4m3fn), s, n)


def _operands(m, n, length, byte, other):
    """a: one number a row, each finite one in turn, in places all over the row; b: ones.  Their product is a's numbers."""
    padded = (length + 127) // 128 * 128
    r = torch.arange(m, device=DEV)
    code = _codes()[(r * 7 + 3) % 254]
    qa = torch.zeros(m, padded, dtype=torch.uint8, device=DEV)
    qa[r, (r * 37) % length] = code
    qb = torch.zeros(n, padded, dtype=torch.uint8, device=DEV)
    qb[:, :length] = 0x38                                    # 1.0
    value = code.view(torch.float8_e4m3fn).double() * _two_to(byte - 127) * _two_to(other - 127)
    return _matrix(qa, byte, length), _matrix(qb, other, length), value


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(map(str, f)))
@pytest.mark.parametrize("byte,other", [(1, 227), (2, 227), (3, 227), (4, 227), (9, 200), (120, 130), (240, 20), (245, 27), (246, 27), (247, 27),
                                        (247, 8)])
def test_every_number(form, byte, other):
    m, n, length = form
    a, b, value = _operands(m, n, length, byte, other)
    for dtype in (F32, BF16):
        want = value.to(dtype).double()
        assert bool(want.isfinite().all())
        # (the steps below byte 4 are of b's scale; a bf16 result is not made from widened numbers)
        bound = _two_to(other - 127 - 133) if dtype is F32 and byte < 4 else torch.zeros((), dtype=torch.float64, device=DEV)
        within(OPS.fp8_matmul(a, b, dtype=dtype)[0], want[:, None].expand(m, n), bound.expand(m, n), "numbers in a, %s" % dtype)
        within(OPS.fp8_matmul(b, a, dtype=dtype)[0], want[None].expand(n, m), bound.expand(n, m), "numbers in b, %s" % dtype)


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(map(str, f)))
def test_a_mask_of_the_lowest_value(form):
    """Numbers of the type's lowest value, which round to -2^128 in 8 bits, times small numbers and zeros: terms that fp32 holds,
    so the sum is right to (contraction) U of their magnitudes, and a product with zero is zero."""
    m, n, length = form
    g = torch.Generator(device=DEV).manual_seed(m)
    x = torch.randn(1, m, length, generator=g, device=DEV)
    x[:, :, length // 3] = torch.finfo(F32).min
    x[:, ::2, 5] = torch.finfo(BF16).min
    w = torch.randn(1, n, length, generator=g, device=DEV) * 2.0 ** -20
    w[:, ::3, length // 3] = 0
    w[:, ::3, 5] = 0
    a, b = OPS.fp8_quantize(x), OPS.fp8_quantize(w)

    def values(q):
        blocks = q.q.shape[2] // 128
        s = ((q.scale[..., :blocks].long() - 127 + 1023) << 52).view(torch.float64)
        return (q.q.double().unflatten(2, (blocks, 128)) * s[..., None]).flatten(2)[..., :length]
    va, vb = values(a), values(b)
    assert float(va.min()) == -2.0 ** 128
    want = torch.matmul(va, vb.transpose(1, 2).contiguous())
    size = torch.matmul(va.abs(), vb.abs().transpose(1, 2).contiguous())
    within(OPS.fp8_matmul(a, b, dtype=F32), want, length * U * size, "a b^T")
    within(OPS.fp8_matmul(b, a, dtype=F32), want.transpose(1, 2), length * U * size.transpose(1, 2), "b a^T")
    within(OPS.fp8_linear(x, b), want, length * U * size, "the linear layer")
    bias = torch.randn(1, n, generator=g, device=DEV) * 1e30
    within(OPS.fp8_linear(x, b, bias), want + bias.double()[:, None], (length + 1) * U * (size + bias.double().abs()[:, None]), "with a bias")
