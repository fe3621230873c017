"""The tokens that the policy example samples follow softmax of the logits."""
import pytest
import torch

from paper_2409_09242_amd import policy_example as E

N = 200_000


@pytest.mark.parametrize("p", [[0.5, 0.3, 0.15, 0.05], [0.9, 0.1], [0.25] * 4, [0.6, 0.0, 0.4]])
def test_frequencies(p):
    """A token's count over N draws is binomial: 5 of its standard deviations, and one for its being whole."""
    g = torch.Generator()
    g.manual_seed(7)
    p = torch.tensor(p, dtype=torch.float64)
    z = (p.log() + 3.0).float().expand(2, N, -1)
    token = E.draw_tokens(z, g)
    assert token.dtype == torch.int32 and token.shape == (2, N)
    for w in range(2):
        count = torch.bincount(token[w].long(), minlength=len(p)).double()
        assert bool(((count - N * p).abs() <= 5 * (N * p * (1 - p)).sqrt() + (p > 0)).all()), (count / N, p)
    assert not torch.equal(token[0], token[1])


def test_any_logits_give_a_token():
    g = torch.Generator()
    g.manual_seed(8)
    for fill in (-float("inf"), float("inf"), float("nan"), torch.finfo(torch.bfloat16).min):
        token = E.draw_tokens(torch.full((3, 5, 7), fill, dtype=torch.bfloat16), g)
        assert bool((token >= 0).all()) and bool((token < 7).all())
