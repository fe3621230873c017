"""Every part of the token example's flat gradient against its own norm, for workers whose parameters differ.

Bound: a number in e4m3 is off by at most 2^-4 of its binade's lower end, 2^-4/sqrt(3) = 3.7 % rms of it, a product of two such
operands by sqrt(2) of that, 5.2 % of its norm.  W's gradient is one such product, the gradient of the norm's output another, which
gamma's and the table's are linear in; b's is a sum of what the loss returns.  The forward product moves the logits (of
about one) by 0.052, and a row of the loss' gradient by that times sqrt(sum p^2) <= 0.2 of its norm: 1 %.  Four roundings to bf16 on the
way, 2^-8 each: 1.6 %.  Together below 8 %; 12 % leaves half as much again."""
import pytest
import torch

from paper_2409_09242_amd import operators as OPS
from paper_2409_09242_amd import policy_example as E
from stream_ref import kept

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOUND = 0.12


def _parts(flat, v, n):
    return {"table": flat[:v * n], "W": flat[v * n:2 * v * n], "gamma": flat[2 * v * n:2 * v * n + n], "b": flat[2 * v * n + n:2 * v * n + n + v]}


def _oracle(theta, v, n, state, factor, penalty, token, adv):
    """The flat gradient in 64 bits on the CPU; factor: what the dropout multiplies by, element by element."""
    theta = theta.double().cpu().requires_grad_()
    p = _parts(theta, v, n)
    h = p["table"].view(v, n)[state] * factor
    y = h / torch.sqrt(h.square().mean(-1, keepdim=True) + 1e-6) * p["gamma"]
    lp = torch.log_softmax(y @ p["W"].view(v, n).t() + p["b"] - penalty, -1).gather(1, token[:, None])[:, 0]
    (-(lp * adv).mean()).backward()
    return theta.grad


def _off(got, want):
    return float((got - want).norm() / want.norm())


def test_parts_of_the_gradient():
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    k, rows, n, v = 3, 200, 130, 210
    w = E.TokenPolicyWorkers(k, n, v, max_norm=1e9, p=0.2, seed=5)
    w.theta[:, 2 * v * n:w.used] += 0.2 * torch.randn(k, w.used - 2 * v * n, generator=g, device=DEV)      # gamma and b are not all alike
    w.theta[:, :2 * v * n] *= 1.0 + 0.1 * torch.arange(k, device=DEV)[:, None]
    w._split()
    state, token = (torch.randint(0, v, (k, rows), generator=g, device=DEV, dtype=torch.int32) for _ in range(2))
    history = torch.randint(0, v, (k, rows, 5), generator=g, device=DEV, dtype=torch.int32)
    presence, adv = torch.rand(k, rows, generator=g, device=DEV), torch.randn(k, rows, generator=g, device=DEV)
    for step in range(3):
        z, had = w.logits(state)
        OPS.adjust_logits(z, history, presence=presence, out=z)
        _, _, dz = OPS.policy_loss(z, token, OPS.token_logp(z, token), adv, kl_coef=0.0)
        w.gradient(dz, had)
        keep, factor = kept(k, rows, n, 0.2, 6, step)
        for i in range(k):
            penalty = torch.zeros(rows, v, dtype=torch.float64).scatter_(1, history[i].long().cpu(), 1.0) * presence[i].double().cpu()[:, None]
            rest = (penalty, token[i].long().cpu(), adv[i].double().cpu())
            got = _parts(w.flat[i].double().cpu(), v, n)
            want = _parts(_oracle(w.theta[i], v, n, state[i].long().cpu(), keep[i].double() * factor, *rest), v, n)
            for name in want:
                assert _off(got[name], want[name]) < BOUND, (step, i, name)
            # an oracle with another step's mask is told apart by every part behind the dropout
            other, _ = kept(k, rows, n, 0.2, 6, step + 1)
            wrong = _parts(_oracle(w.theta[i], v, n, state[i].long().cpu(), other[i].double() * factor, *rest), v, n)
            for name in ("table", "W", "gamma"):
                assert _off(wrong[name], want[name]) > 2 * BOUND, (step, i, name)
