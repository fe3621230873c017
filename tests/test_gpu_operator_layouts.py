"""Outputs whose workers are interleaved, [rows][k][n] seen as [k][rows][n]: the same bits as in outputs of their own, in every
form of the kernels, and nothing beside them."""
import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Interleaved:
    """[k][rows][n] inside [rows][k][n + 3], NaN between the rows."""

    def __init__(self, k, rows, n, dtype):
        self.buf = torch.full((rows, k, n + 3), float("nan"), dtype=dtype, device=DEV)
        self.view = self.buf.transpose(0, 1)[..., 1:n + 1]

    def holds(self, want):
        assert torch.equal(self.view, want)
        assert bool(self.buf[..., 0].isnan().all()) and bool(self.buf[..., -2:].isnan().all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [7, 39, 130, 1000, 4100, 40000])
def test_layer_norm(n, dtype):
    k, rows, g = 3, 9, _gen(n)
    x, dy = (torch.randn(k, rows, n, generator=g, device=DEV).to(dtype) for _ in range(2))
    gamma = torch.randn(k, n, generator=g, device=DEV)
    y, mean, rstd = OPS.layer_norm(x, gamma, gamma)
    out = Interleaved(k, rows, n, dtype)
    OPS.layer_norm(x, gamma, gamma, out=out.view)
    out.holds(y)
    want = OPS.layer_norm_grad(dy, x, gamma, mean, rstd)
    out = Interleaved(k, rows, n, dtype)
    got = OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dx=out.view)
    out.holds(want[0])
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [10, 203, 5003, 40001, 140003])
def test_policy_loss(vocab, dtype):
    k, rows, g = 3, 5, _gen(vocab)
    z = torch.randn(k, rows, vocab, generator=g, device=DEV).to(dtype)
    target = torch.randint(0, vocab, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    old, adv = OPS.token_logp(z, target) - 0.1, torch.randn(k, rows, generator=g, device=DEV)
    want = OPS.policy_loss(z, target, old, adv)[2]
    out = Interleaved(k, rows, vocab, dtype)
    OPS.policy_loss(z, target, old, adv, grad=out.view)
    out.holds(want)
    out = Interleaved(k, rows, vocab, dtype)                 # and over the logits
    out.view.copy_(z)
    OPS.policy_loss(out.view, target, old, adv, grad=out.view)
    out.holds(want)


# a single row, few rows, slices, tiles of each size, an empty contraction
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 1, 300, 1000), (2, 20, 130, 600), (2, 100, 130, 5000), (2, 200, 300, 500), (2, 1600, 1700, 300),
                                   (4, 2048, 2048, 300)])
def test_products(shape, dtype):
    k, m, n, length = shape
    g = _gen(m + n)
    x, w = (torch.randn(k, r, length, generator=g, device=DEV).to(dtype) for r in (m, n))
    bias = torch.randn(k, n, generator=g, device=DEV)
    wq = OPS.fp8_quantize(w, square=True)
    want = OPS.fp8_linear(x, wq, bias)
    out = Interleaved(k, m, n, dtype)
    OPS.fp8_linear(x, wq, bias, out=out.view)
    out.holds(want)
    out = Interleaved(k, m, n, dtype)
    OPS.fp8_matmul(OPS.fp8_quantize(x), wq, bias, out=out.view)
    out.holds(want)
    out = Interleaved(k, m, n, dtype)
    _, none = OPS.fp8_quantize(x[:, :0].reshape(k, 0, m), transposed=True)
    _, empty = OPS.fp8_quantize(x[:, :0].reshape(k, 0, n), transposed=True)
    OPS.fp8_matmul(none, empty, bias, out=out.view)
    out.holds(bias.to(dtype)[:, None].expand(-1, m, -1))


def test_rows_that_share_elements_are_refused():
    x = torch.zeros(3, 4, 8, device=DEV)
    buf = torch.zeros(200, device=DEV)
    for stride, ld in ((0, 8), (7, 24), (8, 23), (8, 16), (31, 8), (16, 8)):
        with pytest.raises(B.DwError) as e:
            OPS.layer_norm(x, out=buf.as_strided((3, 4, 8), (stride, ld, 1)))
        assert e.value.status == -5
    OPS.layer_norm(x, out=buf.as_strided((3, 4, 8), (8, 24, 1)))
