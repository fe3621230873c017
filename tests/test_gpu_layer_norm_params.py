"""Where the gradients of layer norm's weight and bias go: one of them given, both, or neither, in any layout."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [5, 130, 1003])
@pytest.mark.parametrize("k", [1, 3])
def test_one_of_them_given(k, n):
    """One goes into a flat gradient, the other comes back in a tensor of its own."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x, dy = (torch.randn(k, 11, n, generator=g, device=DEV) for _ in range(2))
    gamma = torch.randn(k, n, generator=g, device=DEV)
    _, mean, rstd = OPS.layer_norm(x, gamma)
    dx, dgamma, dbeta = OPS.layer_norm_grad(dy, x, gamma, mean, rstd)
    flat = torch.full((k, 2 * n + 5), float("nan"), device=DEV)
    mine = flat[:, 2:n + 2]
    got = OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dgamma=mine)
    assert got[1] is mine and torch.equal(mine, dgamma) and torch.equal(got[2], dbeta) and torch.equal(got[0], dx)
    assert got[2].shape == (k, n) and bool(flat[:, :2].isnan().all()) and bool(flat[:, n + 2:].isnan().all())
    got = OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dbeta=mine)
    assert got[2] is mine and torch.equal(mine, dbeta) and torch.equal(got[1], dgamma) and got[1].shape == (k, n)
    assert bool(flat[:, :2].isnan().all()) and bool(flat[:, n + 2:].isnan().all())


def test_different_worker_strides_are_refused():
    x = torch.zeros(2, 3, 8, device=DEV)
    own, view = torch.ones(2, 8, device=DEV), torch.ones(2, 20, device=DEV)[:, :8]
    y, mean, rstd = OPS.layer_norm(x, own)
    for bad in (lambda: OPS.layer_norm(x, own, view), lambda: OPS.layer_norm_grad(x, x, own, mean, rstd, dgamma=own, dbeta=view)):
        with pytest.raises(ValueError, match="different worker strides"):
            bad()


def test_rows_that_overlap_are_refused():
    x = torch.zeros(2, 3, 8, device=DEV)
    _, mean, rstd = OPS.layer_norm(x)
    for bad in (torch.ones(1, 8, device=DEV).expand(2, 8), torch.ones(20, device=DEV).as_strided((2, 8), (7, 1))):
        for kw in (dict(dgamma=bad), dict(dbeta=bad)):
            with pytest.raises(ValueError, match="overlap"):
                OPS.layer_norm_grad(x, x, None, mean, rstd, **kw)
