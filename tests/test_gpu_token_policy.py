"""The example whose states are tokens: its flat gradient, and that it runs."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from paper_2409_09242_amd import policy_example as E
from stream_ref import kept

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_of_the_whole_model():
    """The flat gradient against automatic differentiation in 64 bits of the model without quantisation, its dropout's mask computed
    apart.  A number in e4m3 is off by at most 2^-4 of itself (1/27 rms over a binade's fractions at 3 bits), a product of two by
    sqrt(2) of that, 5 %; the logits that two such products feed move the gradient of the softmax by the like, bf16 by 0.4 %: 20 % covers
    them."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    k, rows, n, v = 3, 200, 130, 210
    w = E.TokenPolicyWorkers(k, n, v, max_norm=1e9, p=0.2, seed=5)
    state = torch.randint(0, v, (k, rows), generator=g, device=DEV, dtype=torch.int32)
    history = torch.randint(0, v, (k, rows, 5), generator=g, device=DEV, dtype=torch.int32)
    presence = torch.rand(k, rows, generator=g, device=DEV)
    adv = torch.randn(k, rows, generator=g, device=DEV)
    token = torch.randint(0, v, (k, rows), generator=g, device=DEV).to(torch.int32)
    for step in range(2):
        z, had = w.logits(state)
        OPS.adjust_logits(z, history, presence=presence, out=z)
        loss, logp, dz = OPS.policy_loss(z, token, OPS.token_logp(z, token), adv, kl_coef=0.0)
        norm = w.gradient(dz, had)
        keep, factor = kept(k, rows, n, 0.2, 6, step)
        for i in range(k):
            theta = w.theta[i].double().cpu().requires_grad_()
            table, W = theta[:v * n].view(v, n), theta[v * n:2 * v * n].view(v, n)
            gamma, b = theta[2 * v * n:2 * v * n + n], theta[2 * v * n + n:w.used]
            h = table[state[i].long().cpu()] * keep[i] * factor
            y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * gamma
            seen = torch.zeros(rows, v, dtype=torch.float64).scatter_(1, history[i].long().cpu(), 1.0)
            lp = torch.log_softmax(y @ W.t() + b - seen * presence[i].double().cpu()[:, None], -1).gather(1, token[i].long().cpu()[:, None])[:, 0]
            (-(lp * adv[i].double().cpu()).mean()).backward()
            got, want = w.flat[i].double().cpu(), theta.grad
            assert float((got - want).norm() / want.norm()) < 0.2
            assert abs(float(norm[i]) / float(want.norm()) - 1) < 0.2
            unused = torch.bincount(state[i].long().cpu(), minlength=v) == 0
            assert bool((got[:v * n].view(v, n)[unused] == 0).all())


def test_it_runs():
    rewards = E.train_tokens(k=3, rounds=3, updates=2, seed=1)
    assert rewards.shape == (3, 3) and bool(torch.isfinite(rewards).all())
