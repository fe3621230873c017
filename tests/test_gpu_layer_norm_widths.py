"""Layer norm and its backward pass at every short width, and at both sides of every width where a row changes hands, against
the formula in 64 bits.

A row is shared by 4 (in bf16 by 8 where more than 4 elements are odd), 16, 32, 64, 256, 512 or 1024 threads with one to four pieces of 16 bytes each (4 elements in
fp32, 8 in bf16), and what its whole pieces leave, up to 3 or 7 odd elements, goes to the first threads.  Outputs hold NaN
before each call, so that an element that nobody writes shows.

Bounds (U = 2^-24): a row sum goes through fewer than 64 + n/1024 roundings; what follows from it is the formula's
derivative times it."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within
from test_gpu_layer_norm import _check_forward

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
V = {F32: 4, BF16: 8}                                       # elements of a piece
LIMITS = [4, 16, 32, 64, 128, 256, 512, 1024, 1536, 2048, 4096]       # most pieces of a form
SHORT = [(n, t) for t in (F32, BF16) for n in range(1, 41)]
EDGES = [(p * V[t] + odd, t) for t in (F32, BF16) for p in LIMITS[1:] for odd in (V[t] - 1, V[t])]


def _name(c):
    return "%d-%s" % (c[0], "f32" if c[1] is F32 else "bf16")


def _nan(shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


@pytest.mark.parametrize("case", SHORT + EDGES, ids=_name)
def test_both_passes(case):
    n, dtype = case
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    k, rows = (3, 37) if n <= 1100 else (2, 5)
    x = padded((k, rows, n), 3, 1, dtype, g, 1.5, 0.4)
    gamma, beta = torch.randn(k, n, generator=g, device=DEV), torch.randn(k, n, generator=g, device=DEV)
    out = _nan((k, rows, n + 2), dtype)
    y, mean, rstd = OPS.layer_norm(x, gamma, beta, 1e-5, out=out[..., 1:n + 1])
    _check_forward(x, gamma, beta, 1e-5, (y, mean, rstd))
    assert bool(out[..., 0].isnan().all()) and bool(out[..., -1].isnan().all())

    dy = padded((k, rows, n), 2, 1, dtype, g, 0.3)
    out, flat = _nan((k, rows, n + 2), dtype), _nan((k, 2 * n + 3), F32)
    dx, dgamma, dbeta = OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dx=out[..., 1:n + 1], dgamma=flat[:, 1:n + 1],
                                            dbeta=flat[:, n + 2:2 * n + 2])
    m, r = mean.double()[..., None], rstd.double()[..., None]
    h, d = (x.double() - m) * r, dy.double()
    a = d * gamma.double()[:, None]
    c1, c2 = a.mean(-1, keepdim=True), (a * h).mean(-1, keepdim=True)
    dh = 3 * U * r * (x.double().abs() + m.abs())
    c = 64 + n / 1024
    d1 = c * U * a.abs().mean(-1, keepdim=True)
    d2 = c * U * (a * h).abs().mean(-1, keepdim=True) + (a.abs() * dh).mean(-1, keepdim=True)
    want = r * (a - c1 - h * c2)
    bound = r * (4 * U * (a.abs() + c1.abs() + (h * c2).abs()) + d1 + h.abs() * d2 + dh * c2.abs())
    within(dx, want, 1.01 * bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "dx")
    within(dgamma, (d * h).sum(1), (rows + 32) * U * (d * h).abs().sum(1) + (d.abs() * dh).sum(1) + 1e-38, "dgamma")
    within(dbeta, d.sum(1), (rows + 32) * U * d.abs().sum(1) + 1e-38, "dbeta")
    assert bool(out[..., 0].isnan().all()) and bool(out[..., -1].isnan().all())
    assert bool(flat[:, 0].isnan().all()) and bool(flat[:, n + 1].isnan().all()) and bool(flat[:, 2 * n + 2].isnan().all())
