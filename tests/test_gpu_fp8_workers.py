"""A worker's products depend on its own operands alone, in every form of the kernels."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
# a single row, few rows, slices, tiles of 64 and 128, tiles of 256 whose workers begin at different blocks of the contraction
FORMS = [(3, 1, 300, 900), (3, 40, 130, 600), (3, 70, 130, 5000), (3, 300, 270, 900), (3, 1000, 1100, 300), (4, 2048, 2048, 2048)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(map(str, f)))
def test_other_workers_do_not_matter(form, dtype):
    k, m, n, length = form
    g = torch.Generator(device=DEV).manual_seed(m)
    x, w = (torch.randn(k, r, length, generator=g, device=DEV).to(dtype) for r in (m, n))
    bias = torch.randn(k, n, generator=g, device=DEV)

    def results():
        a, at = OPS.fp8_quantize(x, transposed=True)
        b, bt = OPS.fp8_quantize(w, square=True, transposed=True)
        q = [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for v in (a, at, b, bt) for t in (v.q, v.scale)]
        return q + [OPS.fp8_matmul(a, b, bias, dtype=dtype), OPS.fp8_linear(x, b, bias)]
    first = results()
    assert all(torch.equal(u, v) for u, v in zip(first, results()))
    x[1], w[1], bias[1] = torch.randn(m, length, generator=g, device=DEV).to(dtype) * 50, float("nan"), float("inf")
    x[1, m // 2] = float("inf")
    second = results()
    others = [i for i in range(k) if i != 1]
    for u, v in zip(first, second):
        assert torch.equal(u[others], v[others])
    assert bool(second[-1][1].isnan().all()) and bool(second[-2][1].isnan().all()) and not bool(second[-1][others].isnan().any())
