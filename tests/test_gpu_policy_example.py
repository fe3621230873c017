"""The operators together, as a training loop uses them."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from paper_2409_09242_amd import policy_example as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_of_the_whole_model():
    """The flat gradient against automatic differentiation in 64 bits of the model without quantisation.  A number in e4m3 is
    off by at most 2^-4 of itself (1/27 rms over a binade's fractions at 3 bits), a product of two by sqrt(2) of that, 5 %; the
    logits that two such products feed move the gradient of the softmax by the like, bf16 by 0.4 %: 20 % covers them."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    k, rows, n, v = 3, 200, 130, 410
    w = E.PolicyWorkers(k, n, v, max_norm=1e9, seed=5)
    x = torch.randn(k, rows, n, generator=g, device=DEV, dtype=torch.bfloat16)
    token = torch.randint(0, v, (k, rows), generator=g, device=DEV).to(torch.int32)
    adv = torch.randn(k, rows, generator=g, device=DEV)
    z, kept = w.logits(x)
    old = OPS.token_logp(z, token)
    loss, logp, dz = OPS.policy_loss(z, token, old, adv, kl_coef=0.0)
    norm = w.gradient(dz, kept)
    for i in range(k):
        theta = w.theta[i].double().cpu().requires_grad_()
        ga, be, W, b = theta[:n], theta[n:2 * n], theta[2 * n:2 * n + v * n].view(v, n), theta[2 * n + v * n:w.used]
        X = x[i].double().cpu()
        y = torch.nn.functional.layer_norm(X, (n,), ga, be, 1e-5)
        lp = torch.log_softmax(y @ W.t() + b, -1).gather(1, token[i].long().cpu()[:, None])[:, 0]
        (-(lp * adv[i].double().cpu()).mean()).backward()        # ratio 1: the clipped loss has the gradient of -A lp
        want = theta.grad
        assert float((w.flat[i].double().cpu() - want).norm() / want.norm()) < 0.2
        assert abs(float(norm[i]) / float(want.norm()) - 1) < 0.2
        cos = float((w.flat[i].double().cpu() * want).sum() / (want.norm() * w.flat[i].double().cpu().norm()))
        assert cos > 0.98


def test_the_policy_learns():
    rewards = E.train(k=3, rounds=12, updates=3, seed=1)
    assert rewards.shape == (12, 3) and bool(torch.isfinite(rewards).all())
    # rewards of random tokens are N(0, 1) over states: a mean over 512 is 0 +- 0.05
    assert bool((rewards[0].abs() < 0.3).all()) and bool((rewards[-3:].mean(0) > 0.3).all())
