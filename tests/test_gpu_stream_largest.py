"""The longest rows, vocabularies and histories that the operators around the residual stream and sampling take, and calls on two streams at
once.  Bounds as in the operators' own files."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, within
from stream_ref import kept
from test_gpu_adjust_logits import _check as check_logits
from test_gpu_rms_norm import _c, _check_h, _check_norm, _same8, _y32

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
N = 1 << 24


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("n", [N, N - 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_and_dropout(n, dtype):
    g = _gen(1)
    k, rows, p = 1, 3, 0.25
    x, res, dy = (torch.randn(k, rows, n, generator=g, device=DEV).to(dtype) for _ in range(3))
    gamma = torch.randn(k, n, generator=g, device=DEV)
    y, h, rstd = OPS.rms_norm(x, gamma, residual=res, p=p, seed=5, step=2)
    _check_h(h, x, res, p, 5, 2)
    _check_norm(y, h, gamma, 1e-6, rstd)
    assert torch.equal(OPS.dropout(x, p, 5, 2, residual=res), h)
    (q, qt), h8, r8 = OPS.rms_norm_fp8(x, gamma, residual=res, p=p, seed=5, step=2, transposed=True)
    want, want_t = OPS.fp8_quantize(_y32(h, gamma, r8), transposed=True)
    assert torch.equal(h8, h) and _same8(q, want) and _same8(qt, want_t)
    del q, qt, want, want_t, y
    dres, dx, dgamma = OPS.rms_norm_grad(dy, h, gamma, rstd, dh=res, p=p, seed=5, step=2)
    r = rstd.double()[..., None]
    t, d = h.double() * r, dy.double()
    a = d * gamma.double()[:, None]
    m = (a * t).mean(-1, keepdim=True)
    dm = (_c(n) + 4) * U * (a * t).abs().mean(-1, keepdim=True)
    want = r * (a - t * m)
    bound = r * (5 * U * (a.abs() + (t * m).abs()) + 1.01 * t.abs() * dm)
    want = want + res.double()
    bound = bound + U * (want.abs() + res.double().abs())
    within(dres, want, bound + out_rounding(dtype) * (want.abs() + bound) + 1e-38, "dres")
    keep, factor = kept(k, rows, n, p, 5, 2)
    wx, bx = torch.where(keep.to(DEV), want * factor, 0.0), (bound + 2 * U * want.abs()) * 1.01 * factor
    within(dx, wx, bx + out_rounding(dtype) * (wx.abs() + bx) + 1e-38, "dx")
    within(dgamma, (d * t).sum(1), (rows + 34) * U * (d * t).abs().sum(1) + 1e-38, "dgamma")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [N, N - 1])
def test_embedding(n, dtype):
    """Whole numbers: exact sums, over three chunks of places, whole and added; no rows, where pages of zeros are all there is."""
    g = _gen(2)
    vocab, rows = 2, 35
    table = torch.randint(-8, 9, (1, vocab, n), generator=g, device=DEV).to(dtype)
    token = torch.randint(-1, vocab + 1, (1, rows), generator=g, device=DEV, dtype=torch.int32)
    y = OPS.embedding(token, table)
    ok = ((token >= 0) & (token < vocab))[0]
    assert torch.equal(y[0, ok], table[0][token[0, ok].long()]) and not bool(y[0, ~ok].any())
    want = torch.stack([y[0, token[0] == v].double().sum(0) for v in range(vocab)])
    grad = OPS.embedding_grad(y, token, vocab)
    assert torch.equal(grad[0].double(), want)
    OPS.embedding_grad(y, token, out=grad, accumulate=True)
    assert torch.equal(grad[0].double(), 2 * want)
    OPS.embedding_grad(y[:, :0], token[:, :0].contiguous(), out=grad)
    assert not bool(grad.any())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits(dtype):
    g = _gen(3)
    vocab, m = N, 5000
    z = torch.randn(1, 2, vocab, generator=g, device=DEV).mul_(3).to(dtype)
    history = torch.randint(0, vocab, (1, 2, m), generator=g, device=DEV, dtype=torch.int32)
    history[..., ::3] = vocab - 1
    answer = torch.tensor([[100, 4000]], dtype=torch.int32, device=DEV)
    rep, pre, freq = (torch.rand(1, 2, generator=g, device=DEV) + b for b in (0.5, 0.0, 0.0))
    bias, mask = torch.randn(1, 2, vocab, generator=g, device=DEV), torch.randint(-(1 << 31), 1 << 31, (1, 2, vocab // 32), generator=g, device=DEV).to(torch.int32)
    few = (history, None, answer, rep, pre, freq)
    check_logits(OPS.adjust_logits(z, *few, bias, mask), z, *few, bias, mask)
    got = OPS.adjust_logits(z, *few)
    check_logits(got, z, *few, None, None)
    OPS.adjust_logits(z, *few, out=z)
    assert torch.equal(z, got)


def test_the_longest_history():
    """2^24 tokens, of which all but a prompt count: whole numbers, exact."""
    g = _gen(4)
    vocab, m, prompt = 1000, 1 << 24, 12345
    history = torch.randint(-1, vocab + 1, (1, 1, m), generator=g, device=DEV, dtype=torch.int32)
    z = torch.zeros(1, 1, vocab, device=DEV)
    got = OPS.adjust_logits(z, history, answer=torch.tensor([[prompt]], dtype=torch.int32, device=DEV), frequency=torch.ones(1, 1, device=DEV))
    said = history[0, 0, prompt:]
    said = said[(said >= 0) & (said < vocab)]
    assert torch.equal(-got[0, 0].long(), torch.bincount(said.long(), minlength=vocab))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_streams_at_once(dtype):
    """The same operators on two streams with nothing between them: every call has scratch of its own."""
    g = _gen(5)
    k, rows, n, vocab = 2, 3000, 520, 700

    def step(x, res, gamma, token, z, history):
        (q, qt), h, rstd = OPS.rms_norm_fp8(x, gamma, residual=res, p=0.2, seed=3, transposed=True)
        dres, dx, dgamma = OPS.rms_norm_grad(x, h, gamma, rstd, dh=res, p=0.2, seed=3)
        table = OPS.embedding_grad(dx, token, vocab)
        OPS.embedding_grad(dres, token, out=table, accumulate=True)
        return [q.q.view(torch.uint8), qt.q.view(torch.uint8), q.scale, qt.scale, dres, dx, dgamma, table, OPS.embedding(token, table), OPS.dropout(x, 0.3, 4),
                OPS.adjust_logits(z, history, frequency=rstd[:, :40].contiguous())]
    given = []
    for _ in range(2):
        given.append((torch.randn(k, rows, n, generator=g, device=DEV).to(dtype), torch.randn(k, rows, n, generator=g, device=DEV).to(dtype),
                      torch.randn(k, n, generator=g, device=DEV), torch.randint(0, vocab, (k, rows), generator=g, device=DEV, dtype=torch.int32),
                      torch.randn(k, 40, 9000, generator=g, device=DEV).to(dtype),
                      torch.randint(0, 9000, (k, 40, 300), generator=g, device=DEV, dtype=torch.int32)))
    want = [[t.clone() for t in step(*a)] for a in given]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(*given[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for turn in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(turn, want[i]))
