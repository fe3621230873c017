"""Operators around the residual stream and sampling on a caller's stream, in graphs that are replayed with other inputs, on tensors
past 32 bits of elements and rows past 16 bits, and what they do to the versions of tensors that they write into."""
import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _flat(r):
    """The tensors of a result, 8-bit numbers as bytes."""
    if isinstance(r, OPS.Fp8Matrix):
        return [r.q.view(torch.uint8), r.scale]
    if isinstance(r, (tuple, list)):
        return [t for e in r for t in _flat(e)]
    return [] if r is None else [r]


def _norm(n):
    def make(dtype):
        k, rows = 3, 70
        inputs = [torch.empty(k, rows, n, dtype=dtype, device=DEV) for _ in range(3)] + [torch.empty(k, n, device=DEV)]

        def run(x, res, dy, gamma):
            y, h, rstd = OPS.rms_norm(x, gamma, residual=res, p=0.2, seed=3)
            return (y, h, rstd, OPS.rms_norm_fp8(x, gamma, residual=res, p=0.2, seed=3, transposed=True),
                    OPS.rms_norm_grad(dy, h, gamma, rstd, dh=res, p=0.2, seed=3), OPS.dropout(x, 0.4, 7, 1, residual=dy))
        return inputs, run
    make.__name__ = "norm %d" % n
    return make


def _embed(rows, vocab, n):
    def make(dtype):
        k = 2
        token = torch.randint(-1, vocab, (k, rows), generator=_gen(9), device=DEV, dtype=torch.int32)
        inputs = [torch.empty(k, vocab, n, dtype=dtype, device=DEV), torch.empty(k, rows, n, dtype=dtype, device=DEV), torch.empty(k, vocab, n, device=DEV)]

        def run(table, dy, base):
            tied = base.clone()
            OPS.embedding_grad(dy, token, out=tied, accumulate=True)
            return OPS.embedding(token, table, 2.0, dtype=F32), OPS.embedding_grad(dy, token, vocab), tied
        return inputs, run
    make.__name__ = "embedding %d of %d" % (rows, vocab)
    return make


def _adjust(dtype):
    k, rows, vocab, m = 2, 9, 20001, 300
    history = torch.randint(0, vocab, (k, rows, m), generator=_gen(8), device=DEV, dtype=torch.int32)
    mask = torch.randint(-(1 << 31), 1 << 31, (k, rows, (vocab + 31) // 32), generator=_gen(7), device=DEV).to(torch.int32)
    inputs = [torch.empty(k, rows, vocab, dtype=dtype, device=DEV), torch.empty(k, rows, vocab, device=DEV), torch.empty(k, rows, device=DEV)]

    def run(z, bias, freq):
        rep = freq.abs() + 0.5
        here = z.clone()
        OPS.adjust_logits(here, history, None, None, rep, freq, freq, out=here)
        return OPS.adjust_logits(z, history, None, None, rep, freq, freq, bias, mask), here
    return inputs, run


# rows of a wave, of a block, too long for registers; places sorted by counting and by digits
CASES = [_norm(64), _norm(1003), _norm(33000), _embed(300, 50, 33), _embed(9000, 700, 8), _embed(20000, 700, 8), _adjust]


def _fill(inputs, g):
    for t in inputs:
        t.copy_(torch.randn(t.shape, generator=g, device=DEV))


def _same(got, want):
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("make", CASES, ids=lambda m: m.__name__.strip("_"))
def test_on_a_stream_of_the_callers(make, dtype):
    g = _gen(1)
    inputs, run = make(dtype)
    _fill(inputs, g)
    want = [t.clone() for t in _flat(run(*inputs))]
    _fill(inputs, g)
    other = [t.clone() for t in _flat(run(*inputs))]
    assert not all(torch.equal(a, b) for a, b in zip(want, other))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):                              # inputs, calls and copies one behind the other on that stream
        _fill(inputs, _gen(1))
        got = [t.clone() for t in _flat(run(*inputs))]
    s.synchronize()
    _same(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("make", CASES, ids=lambda m: m.__name__.strip("_"))
def test_in_graphs(make, dtype):
    """Two graphs of one memory pool in turn, every replay with other inputs and eager work in between."""
    g = _gen(2)
    inputs, run = make(dtype)
    _fill(inputs, g)
    run(*inputs)
    torch.cuda.synchronize()
    graphs, results, pool = [], [], None
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            results.append(_flat(run(*inputs)))
        pool = graph.pool()
        graphs.append(graph)
    for turn in range(4):
        _fill(inputs, g)
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results[turn % 2]]
        _same(got, _flat(run(*inputs)))
        torch.cuda.synchronize()


def _far(k, rows, n, dtype):
    """[k][rows][n] in one buffer of more than 2^32 elements: far workers, or far rows of one."""
    stride, pitch = ((2 ** 32 // (k - 1)) + 72, n + 8) if k > 1 else (0, (2 ** 32 // (rows - 1)) + 24)
    return torch.empty((k - 1) * stride + (rows - 1) * pitch + n, dtype=dtype, device=DEV).as_strided((k, rows, n), (stride, pitch, 1))


def _far_copy(x):
    return _far(*x.shape, x.dtype).copy_(x)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(2, 3, 1000), (1, 5, 1000)])
def test_past_32_bits(shape, dtype):
    g = _gen(3)
    k, rows, n = shape
    x, res, dy = (torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(3))
    gamma = torch.randn(k, n, generator=g, device=DEV)
    far, out = _far_copy(x), _far(*shape, dtype)
    want = OPS.rms_norm(x, gamma, residual=res, p=0.3, seed=1)
    got = OPS.rms_norm(far, gamma, residual=res, p=0.3, seed=1, out=out)
    _same(_flat(got), _flat(want))
    got = OPS.rms_norm(x, gamma, residual=res, p=0.3, seed=1, sum_out=out)
    _same(_flat(got), _flat(want))
    _same(_flat(OPS.rms_norm_fp8(far, gamma, transposed=True)), _flat(OPS.rms_norm_fp8(x, gamma, transposed=True)))
    back = OPS.rms_norm_grad(dy, x, gamma, want[2], dh=res, p=0.3, seed=1)
    _same(_flat(OPS.rms_norm_grad(dy, far, gamma, want[2], dh=res, p=0.3, seed=1, dx=out)), _flat(back))
    _same(_flat(OPS.rms_norm_grad(far, dy, gamma, want[2], p=0.3, seed=1, dres=out)), _flat(OPS.rms_norm_grad(x, dy, gamma, want[2], p=0.3, seed=1)))
    drop = OPS.dropout(x, 0.3, 5, residual=res)
    assert torch.equal(OPS.dropout(far, 0.3, 5, residual=res, out=out), drop)
    token = torch.tensor([[2, 0, 1, 0, 2, -1, 2]] * k, dtype=torch.int32, device=DEV)
    assert torch.equal(OPS.embedding(token, far, 1.5), OPS.embedding(token, x, 1.5))
    rows7 = torch.randn(k, 7, n, generator=g, device=DEV).to(dtype)
    want = OPS.embedding_grad(rows7, token, rows)
    assert torch.equal(OPS.embedding_grad(_far_copy(rows7), token, rows), want)
    del far, out
    grad = _far(k, rows, n, F32)
    assert torch.equal(OPS.embedding_grad(rows7, token, out=grad), want)
    OPS.embedding_grad(rows7, token, out=grad, accumulate=True)
    assert torch.equal(grad, want + want)
    del grad
    history = torch.randint(0, n, (k, rows, 40), generator=g, device=DEV, dtype=torch.int32)
    freq = torch.rand(k, rows, generator=g, device=DEV)
    want = OPS.adjust_logits(x, history, frequency=freq, bias=dy.float())
    far = _far_copy(x)
    assert torch.equal(OPS.adjust_logits(far, history, frequency=freq, bias=dy.float()), want)
    OPS.adjust_logits(far, history, frequency=freq, out=far)
    assert torch.equal(far, OPS.adjust_logits(x, history, frequency=freq))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_table_past_32_bits(dtype):
    """Rows at the end of a table of more than 2^32 elements."""
    vocab, n = 2 ** 22 + 50, 1026
    table = torch.empty(1, vocab, n, dtype=dtype, device=DEV)
    last = torch.randn(50, n, generator=_gen(4), device=DEV).to(dtype)
    table[0, -50:] = last
    token = torch.randint(0, 50, (1, 200), generator=_gen(5), device=DEV, dtype=torch.int32)
    assert torch.equal(OPS.embedding(token + (vocab - 50), table)[0], last[token[0].long()])


def test_more_rows_than_16_bits_count():
    g = _gen(6)
    rows, n = 70001, 12
    x, dy = (torch.randn(1, rows, n, generator=g, device=DEV) for _ in range(2))
    part = OPS.rms_norm(x[:, 65000:], None, residual=dy[:, 65000:])
    whole = OPS.rms_norm(x, None, residual=dy)
    assert all(torch.equal(a[:, 65000:], b) for a, b in zip(whole, part))
    z, history = x, torch.randint(0, n, (1, rows, 3), generator=g, device=DEV, dtype=torch.int32)
    rep = torch.rand(1, rows, generator=g, device=DEV) + 0.5
    want = OPS.adjust_logits(z[:, 65000:], history[:, 65000:], repetition=rep[:, 65000:].contiguous())
    assert torch.equal(OPS.adjust_logits(z, history, repetition=rep)[:, 65000:], want)
    token = torch.arange(rows, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    assert torch.equal(OPS.embedding(token, x), x.flip(1)) and torch.equal(OPS.embedding_grad(dy, token, rows), dy.flip(1))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_workers_interleaved_row_by_row(dtype):
    """Tensors [rows][k][n] seen as [k][rows][n], as inputs and outputs."""
    g = _gen(12)
    k, rows, n = 3, 41, 203

    def woven(like=None):
        t = torch.randn(rows, k, n, generator=g, device=DEV).to(dtype).transpose(0, 1)
        return t if like is None else t.copy_(like)
    x, res, dy = woven(), woven(), woven()
    gamma = torch.randn(k, n, generator=g, device=DEV)
    plain = [t.contiguous() for t in (x, res, dy)]
    want = OPS.rms_norm(plain[0], gamma, residual=plain[1], p=0.3, seed=1)
    got = OPS.rms_norm(x, gamma, residual=res, p=0.3, seed=1, out=woven(), sum_out=woven())
    _same(_flat(got), _flat(want))
    _same(_flat(OPS.rms_norm_fp8(x, gamma, residual=res, transposed=True, sum_out=woven())), _flat(OPS.rms_norm_fp8(plain[0], gamma, residual=plain[1], transposed=True)))
    want = OPS.rms_norm_grad(plain[2], plain[0], gamma, want[2], dh=plain[1], p=0.3, seed=1)
    _same(_flat(OPS.rms_norm_grad(dy, x, gamma, got[2], dh=res, p=0.3, seed=1, dres=woven(), dx=woven())), _flat(want))
    assert torch.equal(OPS.dropout(x, 0.3, 2, residual=res, out=woven()), OPS.dropout(plain[0], 0.3, 2, residual=plain[1]))
    token = torch.randint(-1, rows, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    assert torch.equal(OPS.embedding(token, x, 2.0, out=woven()), OPS.embedding(token, plain[0], 2.0))
    for vocab in (rows, 40 * rows):                          # zeros at the end, and in front
        grad = torch.full((vocab, k, n), 7.0, device=DEV).transpose(0, 1)
        assert torch.equal(OPS.embedding_grad(dy, token, out=grad), OPS.embedding_grad(plain[2], token, vocab))
    history = torch.randint(0, n, (rows, k, 9), generator=g, device=DEV, dtype=torch.int32).transpose(0, 1)
    bias, mask = torch.randn(rows, k, n, generator=g, device=DEV).transpose(0, 1), torch.randint(-9, 9, (rows, k, 7), generator=g, device=DEV, dtype=torch.int32).transpose(0, 1)
    rep = torch.rand(k, rows, generator=g, device=DEV) + 0.5
    want = OPS.adjust_logits(plain[0], history.contiguous(), repetition=rep, bias=bias.contiguous(), mask=mask.contiguous())
    assert torch.equal(OPS.adjust_logits(x, history, repetition=rep, bias=bias, mask=mask, out=woven()), want)
    OPS.adjust_logits(x, history, repetition=rep, bias=bias, mask=mask, out=x)
    assert torch.equal(x, want)


def test_written_tensors_count_as_changed():
    """A graph that saved a tensor which a call has written into since refuses its backward pass."""
    x, g = torch.randn(1, 4, 40, device=DEV), torch.randn(1, 40, device=DEV)
    token, rstd = torch.zeros(1, 4, dtype=torch.int32, device=DEV), torch.ones(1, 4, device=DEV)
    calls = [lambda t: OPS.dropout(x, 0.5, 1, out=t), lambda t: OPS.rms_norm(x, g, out=t), lambda t: OPS.rms_norm(x, g, residual=x, sum_out=t),
             lambda t: OPS.rms_norm_fp8(x, g, residual=x, sum_out=t), lambda t: OPS.rms_norm_grad(x, x, g, rstd, dres=t),
             lambda t: OPS.rms_norm_grad(x, x, g, rstd, p=0.5, dx=t), lambda t: OPS.embedding(token, x, out=t),
             lambda t: OPS.embedding_grad(x, token, out=t), lambda t: OPS.embedding_grad(x, token, out=t, accumulate=True),
             lambda t: OPS.adjust_logits(x, out=t)]
    for i, call in enumerate(calls):
        t = torch.randn(1, 4, 40, device=DEV)
        leaf = torch.randn(1, 4, 40, device=DEV, requires_grad=True)
        loss = (leaf * t).sum()
        before = t._version
        call(t)
        assert t._version > before, i
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    dg = torch.zeros(1, 40, device=DEV)
    OPS.rms_norm_grad(x, x, g, rstd, dgamma=dg)
    assert dg._version == 1 and x._version == 0 and g._version == 0


def test_wrappers_refuse_what_does_not_fit():
    x, g, f = torch.zeros(2, 3, 40, device=DEV), torch.zeros(2, 40, device=DEV), torch.zeros(2, 3, device=DEV)
    i, wide = f.int(), torch.zeros(2, 3, 80, device=DEV)
    words, history = torch.zeros(2, 3, 2, dtype=torch.int32, device=DEV), torch.zeros(2, 3, 5, dtype=torch.int32, device=DEV)
    bad = [lambda: OPS.embedding(i.long(), x), lambda: OPS.embedding(i[0], x), lambda: OPS.embedding(i[:1], x), lambda: OPS.embedding(i.cpu(), x),
           lambda: OPS.embedding(i, x, out=x[:, :2]), lambda: OPS.embedding(i, x.transpose(1, 2)), lambda: OPS.embedding(i.t().contiguous().t(), x),
           lambda: OPS.embedding_grad(x, i), lambda: OPS.embedding_grad(x, i, 9, accumulate=True), lambda: OPS.embedding_grad(x, i, 0),
           lambda: OPS.embedding_grad(x, i, out=g), lambda: OPS.embedding_grad(x, i, 9, out=x), lambda: OPS.embedding_grad(x, i, out=x.bfloat16()),
           lambda: OPS.dropout(x, 0.1, 1, residual=x.bfloat16()), lambda: OPS.dropout(x, 0.1, 1, residual=wide), lambda: OPS.dropout(x, 0.1, 1, out=wide),
           lambda: OPS.rms_norm(x, g[:1]), lambda: OPS.rms_norm(x, g.bfloat16()), lambda: OPS.rms_norm(x, g, residual=wide),
           lambda: OPS.rms_norm(x, g, sum_out=wide), lambda: OPS.rms_norm(x, g, out=x.bfloat16()), lambda: OPS.rms_norm_fp8(x, g, sum_out=x.double()),
           lambda: OPS.rms_norm_grad(x, x, g, f[:, :2]), lambda: OPS.rms_norm_grad(wide, x, g, f), lambda: OPS.rms_norm_grad(x, x, g, f, dh=wide),
           lambda: OPS.rms_norm_grad(x, x, g, f, dgamma=f), lambda: OPS.rms_norm_grad(x, x, g, f, dres=wide),
           lambda: OPS.adjust_logits(x, history[..., 0]), lambda: OPS.adjust_logits(x, history.long()), lambda: OPS.adjust_logits(x, history, filled=f),
           lambda: OPS.adjust_logits(x, repetition=i), lambda: OPS.adjust_logits(x, bias=x[..., :39]), lambda: OPS.adjust_logits(x, bias=x.bfloat16()),
           lambda: OPS.adjust_logits(x, mask=words[..., :1]), lambda: OPS.adjust_logits(x, mask=words.long()), lambda: OPS.adjust_logits(x, out=wide)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was taken" % n)
    refused = [lambda: OPS.dropout(x, 1.5, 1), lambda: OPS.rms_norm(x, eps=-1.0), lambda: OPS.rms_norm(x, out=x), lambda: OPS.embedding(i, x, float("nan")),
               lambda: OPS.dropout(x, 0.1, 1, out=x[:1].expand(2, 3, 40)), lambda: OPS.rms_norm_grad(x, x, g, f, dres=x), lambda: OPS.embedding(i, x, out=x),
               lambda: OPS.adjust_logits(x, out=x[:1].expand(2, 3, 40)), lambda: OPS.embedding_grad(x, i, out=x[:1].expand(2, 3, 40))]
    for n, call in enumerate(refused):
        with pytest.raises(B.DwError):
            call()
            pytest.fail("call %d was taken" % n)
