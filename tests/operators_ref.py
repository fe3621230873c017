"""Helpers of the operators' tests: element-wise comparison against 64-bit references with derived bounds."""
import torch

U = 2.0 ** -24                   # unit roundoff of float32
U16 = 2.0 ** -8                  # of bfloat16: half a unit in the last place, relative to the value, is 2^-9 .. 2^-8


def out_rounding(dtype):
    return U16 if dtype == torch.bfloat16 else U


def within(got, want, bound, what=""):
    """|got - want| <= bound element by element, in 64 bits."""
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    if bool(bad.any()):
        at = int(torch.argmax(torch.where(bad, err / bound.clamp_min(1e-300), torch.zeros_like(err)).reshape(-1)))
        raise AssertionError("%s: %d of %d outside, worst at %d: got %.9g, wanted %.9g, bound %.3g" % (
            what, int(bad.sum()), bad.numel(), at, float(got.reshape(-1)[at]), float(want.reshape(-1)[at]),
            float(bound.expand_as(want).reshape(-1)[at])))


def padded(shape, pad, lead, dtype, g, scale=1.0, shift=0.0, device="cuda:0"):
    """A [k][rows][n] view inside a wider buffer filled with NaN: rows `pad` apart beyond n, the first element `lead`
    elements into the buffer."""
    k, rows, n = shape
    buf = torch.full((k * rows * (n + pad) + lead,), float("nan"), dtype=dtype, device=device)
    view = buf[lead:].view(k, rows, n + pad)[..., :n]
    view.copy_((torch.randn(shape, generator=g, device=device) * scale + shift).to(dtype))
    return view
