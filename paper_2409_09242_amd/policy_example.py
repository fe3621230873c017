"""k workers train a small policy over a vocabulary by the clipped policy loss, under elastic averaging.

    python -m paper_2409_09242_amd.policy_example [--workers K] [--rounds N]

The model of a worker is a layer norm and a linear layer on states x: logits = LN(x) W^T + b.  A round samples one token for
every state, takes a few clipped updates on them and lets the workers exchange with the centre:

    layer_norm -> fp8_linear -> token_logp (the policy that sampled), then, per update,
    layer_norm -> fp8_linear -> policy_loss -> fp8 products for W and its input -> layer_norm_grad -> clip_grads into the
    flat gradient -> Handle.update_only (momentum) -> Handle.elastic_sync

The task is synthetic: a fixed random teacher gives every state its best tokens; the reward of a token is the teacher's
score of it, standardised.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from . import operators as OPS


class PolicyWorkers:
    """k replicas of the model over one handle; parameters are a worker's [gamma, beta, W, b] in one flat vector."""

    def __init__(self, k: int, width: int, vocab: int, lr: float = 2.0, momentum: float = 0.5, max_norm: float = 1.0, seed: int = 0,
                 device="cuda:0"):
        self.k, self.width, self.vocab, self.max_norm = k, width, vocab, max_norm
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        theta0 = torch.cat([torch.ones(width, device=device), torch.zeros(width, device=device),
                            torch.randn(vocab * width, generator=g, device=device) * width ** -0.5, torch.zeros(vocab, device=device)])
        self.used = theta0.numel()
        theta0 = torch.nn.functional.pad(theta0, (0, -self.used % 4))       # the handle's vectors are multiples of four
        cfg = B.make_config(dims=None, k=k, n_params=theta0.numel(), lr=lr, optimizer=B.DW_OPT_MOMENTUM, momentum=momentum)
        self.handle = B.Handle(cfg, theta0, device)
        self.flat = torch.zeros(k, theta0.numel(), device=device)
        self.theta = theta0.expand(k, -1).contiguous()
        self._split()

    def _split(self):
        """Views of the workers' parameters, and the weights in 8 bits, both ways, as they have just moved."""
        n, v = self.width, self.vocab
        self.gamma, self.beta = self.theta[:, :n], self.theta[:, n:2 * n]
        self.w = self.theta[:, 2 * n:2 * n + v * n].view(self.k, v, n)
        self.b = self.theta[:, 2 * n + v * n:self.used]
        self.w8, self.w8t = OPS.fp8_quantize(self.w, square=True, transposed=True)

    def logits(self, x):
        """(logits, what the backward pass needs) for states x [k][rows][width] in bf16."""
        y, mean, rstd = OPS.layer_norm(x, self.gamma, self.beta)
        y8, y8t = OPS.fp8_quantize(y, transposed=True)
        return OPS.fp8_matmul(y8, self.w8, self.b), (x, mean, rstd, y8t)

    def gradient(self, dlogits, kept):
        """The workers' flat clipped gradients from that of the logits; returns their norms before clipping."""
        x, mean, rstd, y8t = kept
        d8, d8t = OPS.fp8_quantize(dlogits, transposed=True)
        dy = OPS.fp8_matmul(d8, self.w8t)
        dw = OPS.fp8_matmul(d8t, y8t, dtype=torch.float32)
        db = dlogits.sum(1, dtype=torch.float32)
        _, dgamma, dbeta = OPS.layer_norm_grad(dy, x, self.gamma, mean, rstd, want_dx=False)
        parts = [t[w] for w in range(self.k) for t in (dgamma, dbeta, dw, db)]
        return OPS.clip_grads(parts, self.max_norm, workers=self.k, out=self.flat[:, :self.used])

    def update(self, exchange: bool):
        """One momentum step from the flat gradients, and a round of communication."""
        self.handle.update_only(self.flat, None)
        if exchange:
            self.handle.elastic_sync(B.DW_DYNAMIC, tau=1)
        self.theta = torch.from_numpy(self.handle.all_state(B.DW_S_THETA)).to(self.flat.device)
        self._split()


def draw_tokens(z, g):
    """A draw from softmax(z) for every row of logits, int32: the largest of z plus Gumbel noise (an index in range whatever
    z holds)."""
    waits = -torch.rand(z.shape, generator=g, device=z.device).clamp_min(1e-20).log()       # exponentially distributed
    return (z.float() - waits.clamp_min(1e-20).log()).argmax(-1).to(torch.int32)


def train(k: int = 4, rows: int = 512, width: int = 72, vocab: int = 75, rounds: int = 20, updates: int = 3, seed: int = 0,
          lr: float = 2.0, device="cuda:0"):
    """Mean reward of the sampled tokens in every round, [rounds][k]."""
    g = torch.Generator(device=device)
    g.manual_seed(seed + 1)
    workers = PolicyWorkers(k, width, vocab, lr=lr, seed=seed, device=device)
    teacher = torch.randn(vocab, width, generator=g, device=device) * width ** -0.5
    rewards = []
    for _ in range(rounds):
        x = torch.randn(k, rows, width, generator=g, device=device, dtype=torch.bfloat16)
        z, _ = workers.logits(x)
        token = draw_tokens(z, g)
        old = OPS.token_logp(z, token)
        score = x.float() @ teacher.t()
        reward = score.gather(-1, token.long()[..., None])[..., 0]
        advantage = (reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-6)
        for u in range(updates):
            z, kept = workers.logits(x)
            _, _, dlogits = OPS.policy_loss(z, token, old, advantage, ref_logp=old, kl_coef=0.01, grad=z)
            workers.gradient(dlogits, kept)
            workers.update(exchange=u == updates - 1)
        rewards.append(reward.mean(1))
    return torch.stack(rewards)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--workers", type=int, default=4)
    p.add_argument("--rounds", type=int, default=20)
    a = p.parse_args()
    for i, r in enumerate(train(k=a.workers, rounds=a.rounds).tolist()):
        print("round %3d  mean reward %s" % (i, "  ".join("%+.3f" % v for v in r)))


if __name__ == "__main__":
    main()
