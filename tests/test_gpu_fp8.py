"""Numbers in e4m3 with power-of-two scales, and their products, against the definition in 64 bits.

The quantised numbers are equal bit for bit.  A product's terms are exact in fp32 (two numbers of 4 significant bits and
powers of two), so in fp32 its error is that of adding K of them, at most K U sum|terms|.  In bf16 the 8-bit instruction
adds eight neighbouring terms with bits down to 2^-13 of the largest one's power: up to 8 2^-13 of the largest for each
eight on top of that, which is at most the product of the operands' largest in those places; then the output's rounding."""
import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _up(n, a=128):
    return (n + a - 1) // a * a


def _two_to(e):
    """2^e in 64 bits from its bits (the GPU's power function is an ulp off for some e)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantized(x, square=False):
    """(codes uint8 [k][r][up(n)], scale bytes [k][r][up(n)/128]) by search over the e4m3 numbers' neighbours in 64 bits."""
    k, r, n = x.shape
    rb = 128 if square else 1
    v = torch.zeros(k, _up(r, rb), _up(n), dtype=torch.float64, device=x.device)
    v[:, :r, :n] = x.double()
    v = v.view(k, v.shape[1] // rb, rb, _up(n) // 128, 128)
    top = v.abs().amax((2, 4), keepdim=True)
    e = torch.zeros_like(top)
    for i in range(-126, 121):                              # the least e with top <= 448 2^e
        e = torch.where((top > 448 * 2.0 ** (i - 1)) & (top <= 448 * 2.0 ** i), float(i), e)
    e = torch.where((top > 0) & (top <= 448 * 2.0 ** -126), -126.0, e)
    table = torch.arange(127, device=x.device).to(torch.uint8).view(torch.float8_e4m3fn).double()    # 0 .. 448, rising
    s = (v * _two_to(-e)).abs()
    hi = torch.searchsorted(table, s.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = s - table[lo], table[hi] - s
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = torch.where((v < 0) | ((v == 0) & torch.signbit(v)), code + 128, code).to(torch.uint8)
    scales = (e + 127).to(torch.uint8).expand(-1, -1, rb, -1, -1)
    return code.reshape(k, -1, _up(n))[:, :r], scales.reshape(k, -1, _up(n) // 128)[:, :r]


def _values(m):
    """What an Fp8Matrix stands for, [k][rows][n] in 64 bits."""
    blocks = m.q.shape[2] // 128
    s = _two_to(m.scale[..., :blocks].long() - 127)
    return (m.q.double().unflatten(2, (blocks, 128)) * s[..., None]).flatten(2)[..., :m.n]


def _eights(va, vb):
    """Sum over groups of eight places of the largest |a| there times the largest |b|, [k][m][n]."""
    def top(v):
        v = torch.nn.functional.pad(v.abs(), (0, -v.shape[2] % 8))
        return v.unflatten(2, (-1, 8)).amax(3)
    return torch.matmul(top(va), top(vb).transpose(1, 2).contiguous())


def _check_quantized(m, x, square):
    code, scale = _quantized(x, square)
    got = m.q.view(torch.uint8)
    same = (got == code) | ((got & 127 == 0) & (code & 127 == 0))       # the sign of a zero does not count
    assert bool(same.all())
    blocks = scale.shape[2]
    assert torch.equal(m.scale[..., :blocks], scale) and bool((m.scale[..., blocks:] == 127).all())


SHAPES = [(1, 1, 1), (2, 3, 127), (1, 16, 128), (2, 130, 129), (3, 33, 784), (1, 257, 1000), (2, 128, 512), (1, 500, 1030)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantized_numbers(shape, dtype):
    g = _gen(sum(shape))
    k, rows, n = shape
    for pad, lead in ((0, 0), (3, 1)):
        x = padded(shape, pad, lead, dtype, g)
        x.mul_(torch.exp(4 * torch.randn(k, rows, n, generator=g, device=DEV)).to(dtype))     # e4m3's whole range, subnormals too
        x[:, :: 2, n // 2:] = 0
        for square in (False, True):
            m = OPS.fp8_quantize(x, square=square)
            _check_quantized(m, x, square)
            m2, t = OPS.fp8_quantize(x, square=square, transposed=True)
            assert torch.equal(m2.q.view(torch.uint8), m.q.view(torch.uint8)) and torch.equal(m2.scale, m.scale)
            _check_quantized(t, x.transpose(1, 2), square)
            assert t.shape == (k, n, rows)
            if square:
                assert torch.equal(_values(t), _values(m).transpose(1, 2))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 2100, 2050), (1, 2048, 2048), (5, 900, 1000)])
def test_quantized_numbers_of_many_tiles(shape, dtype):
    """Both forms of more tiles than compute units, and of as many: by one block, and by one for each."""
    x = padded(shape, 3, 1, dtype, _gen(sum(shape)))
    for square in (False, True):
        m, t = OPS.fp8_quantize(x, square=square, transposed=True)
        _check_quantized(m, x, square)
        _check_quantized(t, x.transpose(1, 2), square)


def test_rounding_scales_and_extremes():
    x = torch.zeros(1, 8, 128, device=DEV)
    x[0, 0, :4] = torch.tensor([448.0, 447.0, 1.0625, 1.1875])             # ties to even at the fourth bit
    x[0, 1, :2] = torch.tensor([448.01, -448.01])                          # past the largest number: one binade up
    x[0, 2, 0] = 3e38
    x[0, 3, 0] = 1e-38
    x[0, 4, :3] = torch.tensor([1e-44, -1e-45, 0.0])                       # subnormal fp32
    x[0, 5, :3] = torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10])             # the smallest number, and a tie with zero
    x[0, 6, :2] = torch.tensor([-1.0, 1.0])
    m = OPS.fp8_quantize(x)
    _check_quantized(m, x, False)
    v = _values(m)[0]
    assert v[0, :4].tolist() == [448, 448, 1.0, 1.25] and v[5, :3].tolist() == [448, 2.0 ** -9, 0]
    assert m.scale[0, :, 0].tolist()[:2] == [127, 128] and int(m.scale[0, 7, 0]) == 127
    for bad in (float("inf"), float("nan"), -float("inf")):
        y = torch.ones(1, 130, 300, device=DEV)
        y[0, 5, 140] = bad
        q, t = OPS.fp8_quantize(y, transposed=True)
        nan = q.q.float().isnan()
        assert bool(nan[0, 5, 128:256].all()) and int(nan.sum()) == 128
        nan = t.q.float().isnan()
        assert bool(nan[0, 140, :128].all()) and int(nan.sum()) == 128
        c = OPS.fp8_matmul(q, OPS.fp8_quantize(torch.ones(1, 70, 300, device=DEV)), dtype=F32)
        assert bool(c[0, 5].isnan().all()) and int(c.isnan().sum()) == 70


PRODUCTS = [(1, 1, 1, 1), (1, 1, 128, 128), (2, 3, 5, 7), (1, 16, 64, 300), (2, 33, 65, 129), (3, 64, 64, 640), (1, 100, 200, 784),
            (2, 129, 257, 1000), (1, 17, 4100, 512), (1, 300, 20, 3000), (5, 1, 1000, 520), (2, 8, 96, 9000), (1, 1, 5000, 4100),
            (4, 600, 1100, 384), (2, 2100, 4200, 200), (3, 1025, 520, 2060), (1, 4096, 4096, 256), (2, 2048, 2304, 640)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_products(shape, dtype):
    k, m, n, length = shape
    g = _gen(m + n)
    a = OPS.fp8_quantize(padded((k, m, length), 0, 0, F32, g) * torch.exp(torch.randn(k, m, 1, generator=g, device=DEV)))
    b = OPS.fp8_quantize(padded((k, n, length), 0, 0, F32, g) * 0.1)
    va, vb = _values(a), _values(b)
    for bias in (None, torch.randn(k, n, generator=g, device=DEV)):
        out = torch.full((k, m, n + 3), 7.0, dtype=dtype, device=DEV)
        got = OPS.fp8_matmul(a, b, bias, out=out[..., 1:n + 1])
        want = torch.matmul(va, vb.transpose(1, 2).contiguous())
        size = torch.matmul(va.abs(), vb.abs().transpose(1, 2).contiguous())
        if bias is not None:
            want, size = want + bias.double()[:, None], size + bias.double().abs()[:, None]
        bound = (length + 2) * U * size + (8 * 2.0 ** -13 * _eights(va, vb) if dtype == BF16 else 0)
        within(got, want, bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "product")
        assert bool((out[..., 0] == 7).all()) and bool((out[..., n + 1:] == 7).all())
        assert torch.equal(got, OPS.fp8_matmul(a, b, bias, dtype=dtype))
    assert float((got.double() - want).norm() / want.norm()) < (2e-6 if dtype == F32 else 4e-3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(3, 2400, 2500, 100), (3, 2400, 2500, 200), (3, 2433, 2311, 330), (3, 2400, 2500, 1300), (1, 8192, 4096, 520)])
def test_products_of_more_tiles_than_run_at_once(shape, dtype):
    """Ragged ends and whole tiles of the largest size, contractions of one block and of many."""
    k, m, n, length = shape
    g = _gen(m + n + length)
    a = OPS.fp8_quantize(padded((k, m, length), 0, 0, F32, g) * torch.exp(torch.randn(k, m, 1, generator=g, device=DEV)))
    b = OPS.fp8_quantize(padded((k, n, length), 0, 0, F32, g) * 0.1)
    bias = torch.randn(k, n, generator=g, device=DEV)
    va, vb = _values(a), _values(b)
    product = torch.matmul(va, vb.transpose(1, 2).contiguous())
    terms = torch.matmul(va.abs(), vb.abs().transpose(1, 2).contiguous())
    for bias in (None, bias):
        want = product if bias is None else product + bias.double()[:, None]
        size = terms if bias is None else terms + bias.double().abs()[:, None]
        bound = ((length + 2) * U + (8 * 2.0 ** -13 if dtype == BF16 else 0)) * size    # (of eight products the largest is at most their sum)
        out = torch.full((k, m, n + 3), 7.0, dtype=dtype, device=DEV)
        got = OPS.fp8_matmul(a, b, bias, out=out[..., 1:n + 1])
        within(got, want, bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "product")
        assert bool((out[..., 0] == 7).all()) and bool((out[..., n + 1:] == 7).all())
        for _ in range(3):
            assert torch.equal(got, OPS.fp8_matmul(a, b, bias, dtype=dtype))


def test_scales_apply_to_their_blocks():
    """Integers that fp32 holds exactly: rows and blocks of very different scales, compared for equality."""
    g = _gen(3)
    k, m, n, length = 2, 70, 150, 1152
    ints = lambda rows: torch.randint(-7, 8, (k, rows, length), generator=g, device=DEV).float()
    a, b = ints(m), ints(n)
    for blk in range(length // 128):                        # every block on its own: the others are zero
        one_a, one_b = torch.zeros_like(a), torch.zeros_like(b)
        s = slice(blk * 128, blk * 128 + 128)
        up = _two_to(torch.randint(-20, 20, (k, m, 1), generator=g, device=DEV)).float()
        down = _two_to(torch.randint(-20, 20, (k, n, 1), generator=g, device=DEV)).float()
        one_a[..., s], one_b[..., s] = a[..., s] * up, b[..., s] * down
        got = OPS.fp8_matmul(OPS.fp8_quantize(one_a), OPS.fp8_quantize(one_b), dtype=F32)
        assert torch.equal(got.double(), torch.matmul(one_a.double(), one_b.double().transpose(1, 2).contiguous()))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_linear_layer_and_its_gradients(dtype):
    """y, dx and dW from quantised operands are the products of the numbers those stand for."""
    g = _gen(7)
    k, m, i, o = 2, 150, 200, 330
    x, w, dy = (padded(s, 0, 0, dtype, g) for s in ((k, m, i), (k, o, i), (k, m, o)))
    bias = torch.randn(k, o, generator=g, device=DEV)
    wq, wt = OPS.fp8_quantize(w, square=True, transposed=True)
    xq, xt = OPS.fp8_quantize(x, transposed=True)
    dq, dt = OPS.fp8_quantize(dy, transposed=True)
    y = OPS.fp8_linear(x, wq, bias)
    assert y.dtype == dtype and torch.equal(y, OPS.fp8_matmul(xq, wq, bias, dtype=dtype))
    for got, a, b, extra in ((y, xq, wq, bias), (OPS.fp8_matmul(dq, wt, dtype=dtype), dq, wt, None), (OPS.fp8_matmul(dt, xt, dtype=F32), dt, xt, None)):
        want = torch.matmul(_values(a), _values(b).transpose(1, 2).contiguous())
        size = torch.matmul(_values(a).abs(), _values(b).abs().transpose(1, 2).contiguous())
        if extra is not None:
            want, size = want + extra.double()[:, None], size + extra.double().abs()[:, None]
        bound = 400 * U * size + (8 * 2.0 ** -13 * _eights(_values(a), _values(b)) if got.dtype == BF16 else 0)
        within(got, want, bound + out_rounding(got.dtype) * (want.abs() + bound), "linear")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 1, 64, 128), (1, 1, 4096, 4096), (2, 3, 100, 131), (3, 16, 50, 1000), (1, 5, 17, 7), (2, 9, 300, 2050),
                                   (1, 17, 64, 300), (2, 100, 130, 500), (1, 4, 96, 9000)])
def test_a_linear_layer_quantises_on_the_way(shape, dtype):
    """With few rows in one launch: the same bits as quantiser and product, from any view of x."""
    k, m, n, length = shape
    g = _gen(m + length)
    wq = OPS.fp8_quantize(padded((k, n, length), 0, 0, F32, g), square=True)
    bias = torch.randn(k, n, generator=g, device=DEV)
    for pad, lead in ((0, 0), (3, 1)):
        x = padded((k, m, length), pad, lead, dtype, g, 2.0)
        x[:, m // 2, :200] = 0
        out = torch.full((k, m, n + 2), 7.0, dtype=dtype, device=DEV)
        y = OPS.fp8_linear(x, wq, bias, out=out[..., 1:n + 1])
        assert torch.equal(y, OPS.fp8_matmul(OPS.fp8_quantize(x), wq, bias, dtype=dtype))
        assert bool((out[..., 0] == 7).all()) and bool((out[..., -1] == 7).all())
    x[0, 0, length - 1] = float("nan")
    y = OPS.fp8_linear(x, wq)
    assert bool(y[0, 0].isnan().all()) and not bool(y[0, 1:].isnan().any())


def test_results_do_not_change_and_other_workers_do_not_matter():
    g = _gen(11)
    a, b = padded((3, 70, 900), 0, 0, BF16, g), padded((3, 300, 900), 0, 0, BF16, g)
    first = OPS.fp8_matmul(OPS.fp8_quantize(a), OPS.fp8_quantize(b))
    for _ in range(3):
        assert torch.equal(first, OPS.fp8_matmul(OPS.fp8_quantize(a), OPS.fp8_quantize(b)))


def test_empty_matrices():
    """No rows: nothing comes out.  No tokens: the weight gradient of a layer that saw none is zero."""
    g = _gen(13)
    x, w = padded((3, 5, 200), 0, 0, BF16, g), padded((3, 300, 200), 0, 0, BF16, g)
    assert OPS.fp8_linear(x[:, :0], OPS.fp8_quantize(w)).shape == (3, 0, 300)
    _, xt = OPS.fp8_quantize(x[:, :0], transposed=True)
    _, dt = OPS.fp8_quantize(padded((3, 5, 300), 0, 0, F32, g)[:, :0], transposed=True)
    bias = torch.randn(3, 200, generator=g, device=DEV)
    for dtype in (F32, BF16):
        assert bool((OPS.fp8_matmul(dt, xt, dtype=dtype) == 0).all())
        assert torch.equal(OPS.fp8_matmul(dt, xt, bias, dtype=dtype), bias.to(dtype)[:, None].expand(-1, 300, -1))


def test_refusals():
    x = torch.zeros(2, 4, 8, device=DEV)
    q = OPS.fp8_quantize(x)
    for bad in (lambda: OPS.fp8_quantize(x.half()), lambda: OPS.fp8_quantize(x[0]), lambda: OPS.fp8_matmul(q, OPS.fp8_quantize(x[:1])),
                lambda: OPS.fp8_matmul(q, OPS.fp8_quantize(x[..., :7])), lambda: OPS.fp8_matmul(q, q, torch.zeros(2, 5, device=DEV)),
                lambda: OPS.fp8_matmul(q, q, out=torch.zeros(2, 4, 5, device=DEV)), lambda: OPS.fp8_matmul(q, q, dtype=torch.float16)):
        with pytest.raises(ValueError):
            bad()


def test_flags_are_taken_by_their_truth():
    x = torch.ones(1, 4, 200, device=DEV)
    m, t = OPS.fp8_quantize(x, square=1, transposed=1)
    want, turned = OPS.fp8_quantize(x, square=True, transposed=True)
    assert torch.equal(m.scale, want.scale) and torch.equal(t.scale, turned.scale) and t.shape == (1, 200, 4)
    assert OPS.layer_norm(x, stats=0)[1] is None and OPS.layer_norm(x, stats=1)[1].shape == (1, 4)
