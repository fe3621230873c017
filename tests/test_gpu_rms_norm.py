"""Root-mean-square norm behind residual and dropout, in both output types, and its backward pass against the formulas in 64 bits.

Bounds (U = 2^-24).  h: as a dropout's output.  A row's sum of squares in fp32 goes through at most 32 values of a thread (a thread of a
long row: n / 1024), 6 steps over the lanes and 16 waves: less than C = 64 + n/1024 roundings of positive terms, so the mean square
is off by C U of itself, its root's reciprocal by half of that and 3 U, and y by 2 U more."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within
from stream_ref import kept

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"

# every way a row is shared among threads and both sides of each change, whole and ragged
WIDTHS = [1, 3, 7, 16, 17, 31, 33, 64, 100, 127, 128, 129, 255, 256, 257, 511, 513, 784, 1000, 1024, 1027, 2048, 2050, 4096, 4097, 5003, 8192,
          8200, 16384, 16385, 32768, 33000]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _same8(a, b):
    return a.n == b.n and torch.equal(a.q.view(torch.uint8), b.q.view(torch.uint8)) and torch.equal(a.scale, b.scale)


def _c(n):
    return 64 + n / 1024


def _check_h(h, x, res, p, seed, step):
    keep, factor = kept(*x.shape, p, seed, step) if p else (None, 1.0)
    want = torch.where(keep.to(DEV), x.double() * factor, 0.0) if p else x.double()
    size = want.abs()
    if res is not None:
        want, size = want + res.double(), size + res.double().abs()
    bound = 3 * U * size
    within(h, want, bound + out_rounding(x.dtype) * (want.abs() + bound) + 1e-38, "h")


def _check_norm(y, h, gamma, eps, rstd):
    n = h.shape[-1]
    r = 1.0 / torch.sqrt(h.double().square().mean(-1) + eps)
    dr = (0.5 * _c(n) + 3) * U
    within(rstd, r, dr * r, "rstd")
    want = h.double() * r[..., None] * (gamma.double()[:, None] if gamma is not None else 1.0)
    bound = (dr + 2 * U) * 1.01 * want.abs()
    within(y, want, bound + out_rounding(h.dtype) * (want.abs() + bound) + 1e-38, "y")


def _y32(h, gamma, rstd):
    """The fp32 values of y, multiplied in the kernel's order."""
    y = h.float() * rstd[..., None]
    return y * gamma[:, None] if gamma is not None else y


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", WIDTHS)
def test_forward(n, dtype):
    g = _gen(n)
    k, rows = (2, 3) if n > 2000 else (3, 37)
    for pad, lead, p, with_res, affine in ((0, 0, 0.1, True, True), (5, 3, 0.0, True, True), (1, 1, 0.5, False, False), (0, 0, 0.0, False, True)):
        x = padded((k, rows, n), pad, lead, dtype, g, 1.5)
        res = padded((k, rows, n), pad + 1, lead, dtype, g, 2.0) if with_res else None
        gamma = torch.randn(k, n, generator=g, device=DEV) if affine else None
        out = torch.full((k, rows, n + 2), 7.0, dtype=dtype, device=DEV)
        hs = torch.full((k, rows, n + 2), 7.0, dtype=dtype, device=DEV)
        y, h, rstd = OPS.rms_norm(x, gamma, 1e-6, residual=res, p=p, seed=5, step=2, out=out[..., 1:n + 1],
                                  sum_out=hs[..., 1:n + 1] if with_res or p else None)
        _check_h(h, x, res, p, 5, 2)
        _check_norm(y, h, gamma, 1e-6, rstd)
        assert bool((out[..., 0] == 7).all()) and bool((out[..., -1] == 7).all())
        if with_res or p:
            assert bool((hs[..., 0] == 7).all()) and bool((hs[..., -1] == 7).all())
        else:
            assert h is x
        # in 8 bits: the same h and statistics, and what the quantiser makes of the fp32 values, both ways
        q, h8, r8 = OPS.rms_norm_fp8(x, gamma, 1e-6, residual=res, p=p, seed=5, step=2)
        assert torch.equal(h8, h)
        want, want_t = OPS.fp8_quantize(_y32(h, gamma, r8), transposed=True)
        assert _same8(q, want)
        (q2, qt), h2, r2 = OPS.rms_norm_fp8(x, gamma, 1e-6, residual=res, p=p, seed=5, step=2, transposed=True)
        assert torch.equal(h2, h) and torch.equal(r2, r8) and _same8(q2, want) and _same8(qt, want_t)
        dr = (0.5 * _c(n) + 3) * U
        within(r8, 1.0 / torch.sqrt(h.double().square().mean(-1) + 1e-6), dr * r8.double().abs() * 1.01, "rstd of the 8-bit form")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_forms_and_absent_outputs(dtype):
    g = _gen(1)
    for n in (100, 4096, 33000):
        x, res = (torch.randn(2, 5, n, generator=g, device=DEV).to(dtype) for _ in range(2))
        gamma = torch.randn(2, n, generator=g, device=DEV)
        y, h, rstd = OPS.rms_norm(x, gamma, residual=res, p=0.2, seed=3)
        for into_x in (False, True):
            a, b = x.clone(), res.clone()
            y2, h2, none = OPS.rms_norm(a, gamma, residual=b, p=0.2, seed=3, sum_out=a if into_x else b, stats=False)
            assert none is None and torch.equal(y2, y) and torch.equal(h2, h) and torch.equal(a if into_x else b, h)
            assert torch.equal(b, res) if into_x else torch.equal(a, x)
            a, b = x.clone(), res.clone()
            (q, qt), h3, r3 = OPS.rms_norm_fp8(a, gamma, residual=b, p=0.2, seed=3, sum_out=a if into_x else b, transposed=True)
            want, want_t = OPS.fp8_quantize(_y32(h, gamma, r3), transposed=True)
            assert torch.equal(h3, h) and _same8(q, want) and _same8(qt, want_t)
        one = torch.randn(1, n, generator=g, device=DEV).expand(2, n)          # one gamma and one residual for the workers
        y4, h4, _ = OPS.rms_norm(x, one, residual=res[:1].expand(2, 5, n))
        y5, h5, _ = OPS.rms_norm(x, one.contiguous(), residual=res[:1].repeat(2, 1, 1))
        assert torch.equal(y4, y5) and torch.equal(h4, h5)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_zeros_infinities_and_large_numbers(dtype):
    n = 300
    x = torch.zeros(1, 5, n, dtype=dtype, device=DEV)
    x[0, 1] = 1e18                                           # squares of 1e36: the largest sum that fits is 3.4e38
    x[0, 2, 7] = float("inf")
    x[0, 3, 7] = float("nan")
    x[0, 4] = 1e-30                                          # squares vanish: eps is left
    y, h, rstd = OPS.rms_norm(x, None, 1e-6)
    assert bool((y[0, 0] == 0).all()) and abs(float(rstd[0, 0]) - 1000) < 1e-2
    assert bool(((y[0, 1].float() - 1).abs() < 0.01).all())
    assert bool(y[0, 2, 7].isnan()) and bool((y[0, 2, :7] == 0).all()) and float(rstd[0, 2]) == 0
    assert bool(y[0, 3].isnan().all())
    assert bool(torch.isfinite(y[0, 4]).all())
    q, _, _ = OPS.rms_norm_fp8(x, None, 1e-6)
    want = OPS.fp8_quantize(_y32(h, None, rstd))
    assert _same8(q, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", WIDTHS)
def test_backward(n, dtype):
    g = _gen(100 + n)
    k, rows = (2, 5) if n > 2000 else (2, 150)
    for pad, lead, p, with_dh, affine in ((0, 0, 0.1, True, True), (3, 1, 0.0, True, True), (1, 2, 0.5, False, False)):
        h = padded((k, rows, n), pad, lead, dtype, g, 1.5)
        dy = padded((k, rows, n), pad + 1, lead, dtype, g, 0.3)
        dh = padded((k, rows, n), pad + 2, lead, dtype, g, 0.3) if with_dh else None
        gamma = torch.randn(k, n, generator=g, device=DEV) if affine else None
        rstd = (h.float().square().mean(-1) + 1e-6).rsqrt().contiguous()
        flat = torch.full((k, n + 2), 7.0, device=DEV)
        dres, dx, dgamma = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=dh, p=p, seed=5, step=2, dgamma=flat[:, 1:n + 1])
        r = rstd.double()[..., None]
        t, d = h.double() * r, dy.double()
        a = d * (gamma.double()[:, None] if affine else 1.0)
        m = (a * t).mean(-1, keepdim=True)
        dm = (_c(n) + 4) * U * (a * t).abs().mean(-1, keepdim=True)
        want = r * (a - t * m)
        bound = r * (5 * U * (a.abs() + (t * m).abs()) + 1.01 * t.abs() * dm)
        if with_dh:
            want = want + dh.double()
            bound = bound + U * (want.abs() + dh.double().abs())
        within(dres, want, bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "dres")
        if p:
            keep, factor = kept(k, rows, n, p, 5, 2)
            keep = keep.to(DEV)
            wx, bx = torch.where(keep, want * factor, 0.0), (bound + 2 * U * want.abs()) * 1.01 * factor
            within(dx, wx, bx + out_rounding(dtype) * (wx.abs() + bx) + 1e-38, "dx")
            assert bool((dx[~keep] == 0).all())
        else:
            assert dx is dres or dx.data_ptr() == dres.data_ptr()
        within(dgamma, (d * t).sum(1), (rows + 34) * U * (d * t).abs().sum(1) + 1e-38, "dgamma")
        assert bool((flat[:, 0] == 7).all()) and bool((flat[:, -1] == 7).all())
        # the parts alone are the same numbers
        only, onlyx, none = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=dh, p=p, seed=5, step=2, want_params=False)
        assert none is None and torch.equal(only, dres) and torch.equal(onlyx, dx)
        none, nothing, dg = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=dh, p=p, seed=5, step=2, want_dx=False)
        assert none is None and nothing is None and torch.equal(dg, dgamma)
        # in place: the stream's gradient over dh, or over dy; x's over dy
        for over in ("dh", "dy", "dx"):
            b, e = dy.contiguous().clone(), dh.contiguous().clone() if with_dh else None
            if over == "dh" and not with_dh:
                continue
            more = {"dh": dict(dres=e), "dy": dict(dres=b), "dx": dict(dx=b)}[over]
            got = OPS.rms_norm_grad(b, h, gamma, rstd, dh=e, p=p, seed=5, step=2, **more)
            assert torch.equal(got[0], dres) and torch.equal(got[1], dx) and torch.equal(got[2], dgamma)


# rows of partial sums around the sixteen waves that add them up and the eight of each at a time; rows past one for every block
@pytest.mark.parametrize("n", [70, 520, 4096])
@pytest.mark.parametrize("rows", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400, 1100, 5000])
def test_column_sums(rows, n):
    """Whole numbers, whose sums are exact whatever their order."""
    g = _gen(rows + n)
    for dtype in (F32, BF16):
        dy, h = (torch.randint(-8, 9, (2, rows, n), generator=g, device=DEV).to(dtype) for _ in range(2))
        rstd = torch.exp2(torch.randint(-1, 2, (2, rows), generator=g, device=DEV).float())
        dgamma = OPS.rms_norm_grad(dy, h, None, rstd)[2]
        assert torch.equal(dgamma.double(), (dy.double() * h.double() * rstd.double()[..., None]).sum(1))


def test_gradients_against_differences():
    """Quotients of differences of L = <dy, y> + <dh, h> in 64 bits, in directions for x, the residual and gamma."""
    g = _gen(9)
    k, rows, n, p = 2, 12, 77, 0.3
    x, res, dy, dh, vx, vr = (torch.randn(k, rows, n, generator=g, device=DEV) for _ in range(6))
    gamma, vg = (torch.randn(k, n, generator=g, device=DEV) for _ in range(2))
    keep, factor = kept(k, rows, n, p, 21, 4)
    keep = keep.to(DEV).double() * factor

    def loss(x, res, gamma):
        h = res.double() + keep * x.double()
        y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * gamma.double()[:, None]
        return float((dy.double() * y + dh.double() * h).sum())
    y, h, rstd = OPS.rms_norm(x, gamma, residual=res, p=p, seed=21, step=4)
    dres, dx, dgamma = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=dh, p=p, seed=21, step=4)
    e = 1e-5
    for got, v, at in ((dx, vx, 0), (dres, vr, 1), (dgamma, vg, 2)):
        args = [x.double(), res.double(), gamma.double()]
        up, down = list(args), list(args)
        up[at] = args[at] + e * v.double()
        down[at] = args[at] - e * v.double()
        quotient = (loss(*up) - loss(*down)) / (2 * e)
        inner = float((got.double() * v.double()).sum())
        # fp32 of the gradient: 100 U of its terms; h was rounded, which moves the slope by as much; the quotient's own error is e^2
        assert abs(inner - quotient) <= 400 * U * float((got.double() * v.double()).abs().sum()) + 1e-6 * (1 + abs(quotient)), at


def test_many_rows_and_many_workers():
    g = _gen(5)
    for k, rows, n, dtype in ((1, 20011, 96, BF16), (64, 41, 260, F32), (1, 3001, 1030, F32)):
        x = torch.randn(k, rows, n, generator=g, device=DEV).to(dtype)
        gamma = torch.randn(k, n, generator=g, device=DEV)
        y, h, rstd = OPS.rms_norm(x, gamma, residual=x)
        _check_norm(y, h, gamma, 1e-6, rstd)
        dy = torch.randn(k, rows, n, generator=g, device=DEV).to(dtype)
        _, _, dg = OPS.rms_norm_grad(dy, h, gamma, rstd)
        dt = dy.double() * h.double() * rstd.double()[..., None]
        within(dg, dt.sum(1), (rows + 34) * U * dt.abs().sum(1), "dgamma")


def test_no_rows():
    x = torch.empty(2, 0, 40, device=DEV)
    y, h, rstd = OPS.rms_norm(x, None, residual=x)
    assert y.shape == h.shape == (2, 0, 40) and rstd.shape == (2, 0)
    _, _, dg = OPS.rms_norm_grad(x, x, None, rstd)
    assert torch.equal(dg, torch.zeros(2, 40, device=DEV))
    assert OPS.dropout(x, 0.5, 1).shape == (2, 0, 40)
