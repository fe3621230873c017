"""Tensors that the operators write into count as changed in place: their version goes up, and a graph of autograd's that
saved one refuses its backward pass.  Tensors that are only read keep theirs."""
import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _x(*shape):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)


def _calls():
    """name -> (tensors that are written, tensors that are read, the call)"""
    x, dy, gamma = _x(2, 5, 130), _x(2, 5, 130), _x(2, 130)
    y, mean, rstd = OPS.layer_norm(x, gamma)
    out, dgamma, dbeta = _x(2, 5, 130), _x(2, 130), _x(2, 130)
    target, row, logp = torch.zeros(2, 5, dtype=torch.int32, device=DEV), _x(2, 5), _x(2, 5)
    grads, flat = [_x(40), _x(7), _x(40), _x(7)], _x(2, 50)
    m, c = OPS.fp8_quantize(x), _x(2, 5, 5)
    return {
        "layer_norm": ([out], [x, gamma], lambda: OPS.layer_norm(x, gamma, out=out)),
        "layer_norm_grad": ([out, dgamma, dbeta], [dy, x, gamma, mean, rstd],
                            lambda: OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dx=out, dgamma=dgamma, dbeta=dbeta)),
        "layer_norm_grad dx": ([out], [dgamma, dbeta], lambda: OPS.layer_norm_grad(dy, x, gamma, mean, rstd, dx=out, dgamma=dgamma,
                                                                                  dbeta=dbeta, want_params=False)),
        "token_logp": ([logp], [x, target], lambda: OPS.token_logp(x, target, out=logp)),
        "policy_loss": ([out], [x, target, row], lambda: OPS.policy_loss(x, target, row, row, grad=out)),
        "policy_loss in place": ([dy], [row], lambda: OPS.policy_loss(dy, target, row, row, grad=dy)),
        "policy_loss alone": ([], [x, out], lambda: OPS.policy_loss(x, target, row, row, grad=out, want_grad=False)),
        "clip in place": (grads, [], lambda: OPS.clip_grads(grads, 1.0, 2)),
        "clip packed": ([flat], grads, lambda: OPS.clip_grads(grads, 1.0, 2, out=flat[:, 1:48])),
        "grad_norm": ([], grads, lambda: OPS.grad_norm(grads, 2)),
        "fp8_matmul": ([c], [m.q, m.scale], lambda: OPS.fp8_matmul(m, m, out=c)),
        "fp8_linear": ([c], [x, m.q, m.scale], lambda: OPS.fp8_linear(x, m, out=c)),
    }


NAMES = ["layer_norm", "layer_norm_grad", "layer_norm_grad dx", "token_logp", "policy_loss", "policy_loss in place", "policy_loss alone",
         "clip in place", "clip packed", "grad_norm", "fp8_matmul", "fp8_linear"]


@pytest.mark.parametrize("name", NAMES)
def test_versions(name):
    calls = _calls()
    assert set(calls) == set(NAMES)
    written, read, call = calls[name]
    before = [t._version for t in written + read]
    call()
    after = [t._version for t in written + read]
    n = len(written)
    assert all(a > b for a, b in zip(after[:n], before[:n])) and after[n:] == before[n:]


def test_a_graph_that_saved_a_clipped_tensor_refuses():
    g = [torch.ones(100, device=DEV)]
    w = torch.ones(100, device=DEV, requires_grad=True)
    product = (w * g[0]).sum()                                # keeps g[0] for the gradient of w
    OPS.clip_grads(g, 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()


def test_a_graph_that_saved_logits_refuses():
    z = torch.randn(1, 4, 9, device=DEV, requires_grad=True)
    probs = torch.softmax(z, -1)                              # keeps its output
    row = torch.zeros(1, 4, device=DEV)
    OPS.policy_loss(probs.detach(), row.int(), row, row, grad=probs.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        probs.sum().backward()


def test_a_refused_call_changes_nothing():
    g = [torch.ones(10, device=DEV)]
    with pytest.raises(B.DwError):
        OPS.clip_grads(g, -1.0)
    assert g[0]._version == 0


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        g = [torch.full((100,), 2.0, device=DEV)]
        OPS.clip_grads(g, 1.0)
    OPS.clip_grads(g, 0.5)
    assert abs(float(g[0].norm()) - 0.5) < 1e-5
