"""Token log probabilities, the clipped policy loss and its gradient against the formula in 64 bits.

Bounds (U = 2^-24).  With x_j = z_j - max the kernel's exp(x_j) is right to (|x_j| + 3) U, the sum of them goes through at
most 128 + 1 terms of a thread, 6 steps and 16 waves (a vocabulary past the registers: as many terms more as are read
again; a thread that adds its pieces' sums relative to a running maximum has 4 + 3 for each of 16 pieces and 1), so log sum is
off by (152 + more + mean|x|) U, the mean over the softmax; the rest follows by differentiating."""
import pytest
import torch

from paper_2409_09242_amd import binding as B
from paper_2409_09242_amd import operators as OPS
from operators_ref import U, out_rounding, padded, within

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
# every way a row is shared among threads, whole and ragged, the form that reads a part again (both types)
VOCABS = [1, 2, 7, 9, 64, 100, 511, 513, 1000, 2048, 5003, 8192, 20001, 32000, 40009, 70001, 131072, 140003]
RATIOS = torch.tensor([0.3, 0.75, 0.9, 1.0, 1.1, 1.25, 2.5], dtype=torch.float64)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _reference(z, target, old, adv, weight, ref, lo, hi, kl):
    """(lp, loss, grad) and their bounds, in 64 bits; rows of weight 0 or without a valid target are zero."""
    z = z.double()
    k, rows, vocab = z.shape
    ok = (target >= 0) & (target < vocab) & (weight != 0)
    y = target.long().clamp(0, vocab - 1)[..., None]
    z = torch.where(ok[..., None], z, torch.zeros_like(z))
    top = z.amax(-1, keepdim=True)
    none = torch.isneginf(top)
    x = torch.where(none, torch.full_like(z, -float("inf")), z - top)
    p = torch.exp(x)
    total = p.sum(-1, keepdim=True)
    p = torch.where(none, torch.zeros_like(p), p / total)
    lp = torch.where(none[..., 0], torch.full_like(old, -float("inf")).double(), (x.gather(-1, y) - total.log())[..., 0])
    size = torch.where(p > 0, x.abs(), torch.zeros_like(x))
    dsum = (160 + vocab / 1024 + (p * size).sum(-1)) * U
    dlp = dsum + U * (x.gather(-1, y)[..., 0].abs() + 3 * total.log()[..., 0].abs() + lp.abs())
    live = ok & ~none[..., 0]
    lp_out = torch.where(ok, lp, torch.zeros_like(lp))
    old, adv, weight = old.double(), adv.double(), weight.double()
    q = torch.exp(lp - old)
    dq = torch.where(q > 0, q * (dlp + U * (lp - old).abs() + 3 * U), torch.zeros_like(q))     # (a chosen -inf: the ratio is 0)
    free, held = torch.where(adv == 0, torch.zeros_like(q), q * adv), q.clamp(1 - lo, 1 + hi) * adv
    clipped = held < free
    ell = -torch.where(clipped, held, free)
    slope = -torch.where(clipped, torch.zeros_like(free), free)
    dl = adv.abs() * dq + 3 * U * ell.abs()
    ds = torch.where(clipped, torch.zeros_like(q), dl)
    if kl != 0:
        gap = ref.double() - lp
        em1 = torch.expm1(gap)
        dgap = dlp + U * gap.abs()
        ell = ell + kl * (em1 - gap)
        slope = slope - kl * em1
        dl = dl + abs(kl) * (em1.abs() * dgap + 4 * U * (em1.abs() + gap.abs())) + 2 * U * ell.abs()
        ds = ds + abs(kl) * ((1 + em1) * dgap + 4 * U * em1.abs()) + 2 * U * slope.abs()
    zero = torch.zeros_like(lp)
    ell, slope, dl, ds = (torch.where(live, weight * v, zero) for v in (ell, slope, dl, ds))
    dl, ds = dl.abs() + U * ell.abs(), ds.abs() + U * slope.abs()
    hot = torch.zeros_like(z).scatter_(-1, y, 1.0)
    grad = slope[..., None] * (hot - p)
    dgrad = ds[..., None] * (hot + p) + slope.abs()[..., None] * p * ((size + 6) * U + dsum[..., None]) + U * slope.abs()[..., None] * hot
    return lp_out, ell.sum(-1), grad, torch.where(live, dlp, zero), dl.sum(-1) + U * ell.sum(-1).abs(), dgrad


def _inputs(g, k, rows, vocab, dtype, pad=0, lead=0, scale=3.0):
    z = padded((k, rows, vocab), pad, lead, dtype, g, scale)
    target = torch.randint(0, vocab, (k, rows), generator=g, device=DEV).to(torch.int32)
    lp = torch.log_softmax(z.double(), -1).gather(-1, target.long()[..., None])[..., 0]
    pick = torch.randint(0, len(RATIOS), (k, rows), generator=g, device=DEV)
    old = (lp - RATIOS.to(DEV)[pick].log()).float()          # ratios away from the clip's bounds
    ref = (lp + 0.5 * torch.randn(k, rows, generator=g, device=DEV)).float()
    adv = torch.randn(k, rows, generator=g, device=DEV)
    weight = torch.rand(k, rows, generator=g, device=DEV) + 0.1
    weight[torch.rand(k, rows, generator=g, device=DEV) < 0.2] = 0.0
    return z, target, old, adv, weight, ref


def _check(z, target, old, adv, weight, ref, lo, hi, kl, got):
    loss, logp, grad = got
    lp, want, dz, dlp, dloss, dgrad = _reference(z, target, old, adv, weight, ref, lo, hi, kl)
    finite = torch.isfinite(lp)
    assert bool((logp[~finite] == lp[~finite].float()).all())
    within(logp[finite], lp[finite], 1.01 * dlp[finite] + 1e-38, "logp")
    within(loss, want, 1.01 * dloss + 1e-38, "loss")
    if grad is not None:
        within(grad, dz, 1.01 * dgrad + out_rounding(grad.dtype) * (dz.abs() + dgrad) + 1e-38, "grad")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_loss_and_gradient(vocab, dtype):
    g = _gen(vocab)
    k, rows = (2, 9) if vocab > 10000 else (3, 41)
    for pad, lead, kl in ((0, 0, 0.1), (3, 1, 0.0)):
        z, target, old, adv, weight, ref = _inputs(g, k, rows, vocab, dtype, pad, lead)
        grad = torch.full((k, rows, vocab + 2), 7.0, dtype=dtype, device=DEV)
        got = OPS.policy_loss(z, target, old, adv, weight, ref if kl else None, 0.2, 0.28, kl, grad=grad[..., 1:vocab + 1])
        _check(z, target, old, adv, weight, ref, 0.2, 0.28, kl, got)
        assert bool((grad[..., 0] == 7).all()) and bool((grad[..., -1] == 7).all())
        again = OPS.policy_loss(z, target, old, adv, weight, ref if kl else None, 0.2, 0.28, kl, want_grad=False)
        assert again[2] is None and torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
        alone = OPS.token_logp(z, target)
        assert torch.equal(torch.where(weight != 0, alone, 0.0), got[1])


@pytest.mark.parametrize("vocab", [5, 300, 4096, 33000, 132000])
def test_in_place(vocab):
    g = _gen(3)
    for dtype in (F32, BF16):
        z, target, old, adv, weight, ref = _inputs(g, 2, 6, vocab, dtype)
        want = OPS.policy_loss(z, target, old, adv, weight, ref, kl_coef=0.05)
        copy = z.clone()
        got = OPS.policy_loss(copy, target, old, adv, weight, ref, kl_coef=0.05, grad=copy)
        assert all(torch.equal(a, b) for a, b in zip(want, got)) and got[2] is copy


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [6, 203, 3000, 9001, 50001, 135001])
def test_masked_logits(vocab, dtype):
    """Banned tokens at -inf or at the type's lowest value, rows with one choice, rows with none, rows that do not count
    and hold NaN."""
    g = _gen(17 + vocab)
    z, target, old, adv, weight, ref = _inputs(g, 2, 8, vocab, dtype)
    z = z.clone()
    weight = weight.abs() + 0.1
    low = torch.finfo(dtype).min
    z[0, 0, 1:] = -float("inf"); target[0, 0] = 0
    z[0, 1] = -float("inf")
    z[0, 2, vocab // 2:] = low; target[0, 2] = 1
    z[0, 3] = low                                            # all equal: a uniform choice
    z[0, 4] = float("nan"); weight[0, 4] = 0
    z[0, 5] = float("nan"); target[0, 5] = -1
    z[0, 6] = float("nan"); target[0, 6] = vocab
    z[1, 0, ::2] = -float("inf"); target[1, 0] = 1
    z[1, 1, 0] = -float("inf"); target[1, 1] = 0             # a banned token that was chosen all the same: ratio 0
    lp = torch.log_softmax(z.double(), -1).gather(-1, target.long().clamp(0, vocab - 1)[..., None])[..., 0]
    old = torch.where(torch.isfinite(lp), lp - 0.05, -torch.ones_like(lp)).float()
    got = OPS.policy_loss(z, target, old, adv, weight, None, 0.2, 0.2, 0.0)
    assert float(got[1][0, 1]) == -float("inf") and float(got[1][1, 1]) == -float("inf")
    assert bool((got[2][0, 1] == 0).all()) and bool((got[2][0, 4:7] == 0).all()) and bool((got[2][1, 1] == 0).all())
    assert not bool(got[2].isnan().any()) and bool(torch.isfinite(got[0]).all())
    assert bool((got[1][0, 4:7] == 0).all())
    _check(z, target, old, adv, weight, ref, 0.2, 0.2, 0.0, got)


def test_not_a_number_shows():
    """A NaN logit in a row that counts reaches the loss, the log probability and the gradient, wherever it sits."""
    g = _gen(23)
    for vocab in (9, 700, 9001, 140003):
        z, target, old, adv, weight, ref = _inputs(g, 1, 3, vocab, F32)
        z = z.clone()
        weight = weight + 1.0
        z[0, 1, vocab - 1] = float("nan")
        loss, logp, grad = OPS.policy_loss(z, target, old, adv, weight, ref, kl_coef=0.1)
        assert bool(loss.isnan().all()) and logp.isnan().tolist() == [[False, True, False]]
        assert bool(grad[0, 1].isnan().all()) and not bool(grad[0, 0].isnan().any()) and not bool(grad[0, 2].isnan().any())
        z[0, 1] = float("nan")
        loss, logp, grad = OPS.policy_loss(z, target, old, adv, weight)
        assert bool(loss.isnan().all()) and bool(grad[0, 1].isnan().all())


def test_default_weight_is_the_mean_and_extreme_ratios():
    g = _gen(29)
    z, target, old, adv, weight, ref = _inputs(g, 2, 50, 333, F32)
    mean = torch.full_like(weight, 1.0) / 50
    a, b = OPS.policy_loss(z, target, old, adv), OPS.policy_loss(z, target, old, adv, mean)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    far = old - 200.0                                        # the ratio overflows: clipped where the advantage is positive
    up = OPS.policy_loss(z, target, far, adv.abs() + 0.1)
    assert bool(torch.isfinite(up[0]).all()) and bool((up[2] == 0).all())
    zero = OPS.policy_loss(z, target, far, adv * 0)
    assert bool((zero[0] == 0).all()) and bool((zero[2] == 0).all())


@pytest.mark.parametrize("vocab", [40, 1500])
def test_gradient_against_differences(vocab):
    """Along a random direction, step h in the logits: the loss is right to a few hundred U, over 2h, and the third
    derivative of a row's loss along it is at most of the order of 10."""
    g = _gen(31)
    z, target, old, adv, weight, ref = _inputs(g, 1, 12, vocab, F32)
    weight = weight + 0.1
    v = torch.randn(z.shape, generator=g, device=DEV)
    h = 1e-2
    grad = OPS.policy_loss(z, target, old, adv, weight, ref, kl_coef=0.2)[2]
    along = float((grad.double() * v).sum())
    up, down = (float(OPS.policy_loss(z + s * v, target, old, adv, weight, ref, kl_coef=0.2)[0]) for s in (h, -h))
    total = float(weight.sum())
    assert abs((up - down) / (2 * h) - along) <= total * (400 * U * 4 / (2 * h) + 40 * h * h)


def test_rows_of_many_workers_and_none():
    g = _gen(37)
    z, target, old, adv, weight, ref = _inputs(g, 64, 33, 70, BF16)
    _check(z, target, old, adv, weight, ref, 0.2, 0.2, 0.3, OPS.policy_loss(z, target, old, adv, weight, ref, kl_coef=0.3))
    z = torch.zeros(3, 0, 10, device=DEV)
    e = torch.zeros(3, 0, device=DEV)
    loss, logp, grad = OPS.policy_loss(z, e.int(), e, e, e)
    assert loss.tolist() == [0, 0, 0] and logp.shape == (3, 0) and grad.shape == (3, 0, 10)
    assert OPS.token_logp(z, e.int()).shape == (3, 0)


def test_refusals():
    z = torch.zeros(2, 3, 8, device=DEV)
    y = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    f = torch.zeros(2, 3, device=DEV)
    for bad in (lambda: OPS.token_logp(z, y.long()), lambda: OPS.token_logp(z, y[:1]), lambda: OPS.token_logp(z.half(), y),
                lambda: OPS.policy_loss(z, y, f, None), lambda: OPS.policy_loss(z, y, f.double(), f),
                lambda: OPS.policy_loss(z, y, f, f, f.t().contiguous().t()), lambda: OPS.policy_loss(z, y, f, f, grad=z.bfloat16())):
        with pytest.raises(ValueError):
            bad()
    for kw, status in ((dict(kl_coef=0.1), -1), (dict(clip_low=1.5), -3), (dict(clip_high=-0.1), -3), (dict(kl_coef=float("nan")), -3)):
        with pytest.raises(B.DwError) as e:
            OPS.policy_loss(z, y, f, f, **kw)
        assert e.value.status == status
    wide = torch.zeros(2, 4, 8, device=DEV)
    with pytest.raises(B.DwError) as e:                       # in place, but not the same rows
        OPS.policy_loss(wide[:, :3], y, f, f, grad=wide.view(-1)[:48].view(2, 3, 8))
    assert e.value.status == -5
