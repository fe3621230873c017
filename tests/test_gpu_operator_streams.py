"""Operators on a stream of the caller's and in a graph: the same bits as on the default stream, replay after replay."""
import pytest
import torch

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


def _norm(dtype):
    k, rows, n = 3, 70, 1003
    inputs = [torch.empty(k, rows, n, dtype=dtype, device=DEV), torch.empty(k, rows, n, dtype=dtype, device=DEV), torch.empty(k, n, device=DEV)]

    def run(x, dy, gamma):
        y, mean, rstd = OPS.layer_norm(x, gamma, gamma)
        return y, mean, rstd, OPS.layer_norm_grad(dy, x, gamma, mean, rstd)
    return inputs, run


def _policy(dtype):
    k, rows, vocab = 2, 60, 5003
    inputs = [torch.empty(k, rows, vocab, dtype=dtype, device=DEV)] + [torch.empty(k, rows, device=DEV) for _ in range(2)]
    target = torch.randint(0, vocab, (k, rows), generator=_gen(9), device=DEV, dtype=torch.int32)

    def run(z, old, adv):
        return OPS.token_logp(z, target), OPS.policy_loss(z, target, old, adv, None, adv, 0.2, 0.28, 0.04)
    return inputs, run


def _clip(dtype):
    sizes, k = [1, 5003, 70000, 64], 3
    inputs = [torch.empty(s, dtype=dtype, device=DEV) for _ in range(k) for s in sizes]
    out = torch.empty(k, sum(sizes), device=DEV)

    def run(*grads):
        return OPS.clip_grads(grads, 1.0, k, out), out, OPS.grad_norm(grads, k)
    return inputs, run


def _fp8(k, m, n, length):
    def make(dtype):
        inputs = [torch.empty(k, m, length, dtype=dtype, device=DEV), torch.empty(k, n, length, dtype=dtype, device=DEV), torch.empty(k, n, device=DEV)]

        def run(x, w, bias):
            wq, wt = OPS.fp8_quantize(w, square=True, transposed=True)
            xq = OPS.fp8_quantize(x)
            return wq, wt, xq, OPS.fp8_linear(x, wq, bias), OPS.fp8_matmul(xq, wq, bias, dtype=F32), OPS.fp8_matmul(xq, wq)
        return inputs, run
    make.__name__ = "fp8 %d x %d x %d x %d" % (k, m, n, length)
    return make


# a single row, few tiles in slices, tiles of each size
CASES = [_norm, _policy, _clip, _fp8(2, 1, 300, 1000), _fp8(1, 100, 130, 5000), _fp8(2, 200, 300, 500), _fp8(1, 1600, 1700, 300), _fp8(4, 2048, 2048, 300)]


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
def test_in_a_graph(make, dtype):
    """Every replay, with other inputs and eager work in between, gives what the calls give outside."""
    g = _gen(2)
    inputs, run = make(dtype)
    _fill(inputs, g)
    run(*inputs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = _flat(run(*inputs))
    for _ in range(4):
        _fill(inputs, g)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in results]
        want = _flat(run(*inputs))
        _same(got, want)
        torch.cuda.synchronize()
