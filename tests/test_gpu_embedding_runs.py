"""The table's gradient where a token's rows go on over more chunks of 16 places than one look ahead (64) takes, in rows so wide that one thread
adds all partial sums of its columns, and in narrow ones that several share."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from operators_ref import U, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


# (vocabulary, the lengths of the runs in sorted order): one token alone, runs that end with a chunk or one place beside, at 64 chunks and beside
RUNS = [(1, [3000]), (7, [3000]), (3, [1, 2999]), (3, [1023, 1024, 1025]), (5, [16, 1040, 15, 1056, 17]), (4, [2048, 0, 2049, 31])]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [5, 130, 1019, 1021, 1028, 2050, 4096])
@pytest.mark.parametrize("vocab,runs", RUNS)
def test_long_runs(vocab, runs, n, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    token = torch.cat([torch.full((m,), v, dtype=torch.int32) for v, m in enumerate(runs)])
    rows = len(token)
    token = torch.stack([token[torch.randperm(rows, generator=torch.Generator().manual_seed(s))] for s in range(2)]).to(DEV)
    whole = torch.randint(-8, 9, (2, rows, n), generator=g, device=DEV).to(dtype)          # sums exact whatever their order
    want = torch.stack([torch.zeros(vocab, n, dtype=torch.float64, device=DEV).index_add_(0, token[w].long(), whole[w].double()) for w in range(2)])
    got = OPS.embedding_grad(whole, token, vocab)
    assert torch.equal(got.double(), want)
    OPS.embedding_grad(whole, token, scale=2.0, out=got, accumulate=True)
    assert torch.equal(got.double(), 3 * want)
    dy = torch.randn(2, rows, n, generator=g, device=DEV).to(dtype)
    got = OPS.embedding_grad(dy, token, vocab)
    m = torch.tensor(runs + [0] * (vocab - len(runs)), device=DEV, dtype=torch.float64)[:vocab, None]
    for w in range(2):                                       # a term goes through at most as many additions as its token has rows
        want, size = (torch.zeros(vocab, n, dtype=torch.float64, device=DEV).index_add_(0, token[w].long(), t) for t in (dy[w].double(), dy[w].double().abs()))
        within(got[w], want, (m + 1) * U * size, "worker %d" % w)
    assert torch.equal(got, OPS.embedding_grad(dy, token, vocab))
