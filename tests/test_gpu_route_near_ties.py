"""GPU: routing by FP64 keys of which many differ by hardly more than what the keys keep (44 bits)."""
import pytest
import torch

from blocks_ref import gen
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu


def _keys(logits, bias, sigmoid):
    x = logits.double()
    if sigmoid:
        s = torch.exp(-x.abs())
        s = torch.where(x < 0, s, 1.0) / (1.0 + s)
    else:
        s = torch.softmax(x, -1)
    return s + bias.double()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("span", [2.0 ** -7, 8.0])
@pytest.mark.parametrize("E", [32, 512])
def test_keys_that_nearly_agree(sigmoid, span, E):
    # Scores that differ by up to a factor exp(span), and a bias that brings all keys to the same value but for its own rounding to
    # 32 bits: neighbouring keys are 2^-30 to 2^-44 of their value apart.  The choice may change places only where two keys agree
    # in what is kept of them: 2^-43 of the value, and a few 2^-50 for FP64's own roundings (exp, sum, quotient, sum: each at most
    # some 2^-52 of a score, and scores at most exp(8) times the key).
    g = gen(17 + E)
    k, close = 32, 0
    for step in range(40):
        x0 = -30.0 + 1.5 * step if sigmoid else 0.0
        logits = (x0 + span * torch.rand((1, E), generator=g, device="cuda")).float()
        zero = torch.zeros((E,), device="cuda")
        s = _keys(logits, zero, sigmoid)[0]
        bias = (s.min() - s).float()          # (exact but for one rounding)
        key = _keys(logits, bias, sigmoid)[0]
        ids = binding.route_experts(logits, k, score=binding.SCORE_SIGMOID if sigmoid else binding.SCORE_SOFTMAX, bias=bias)[0][0].long()
        assert ids.unique().numel() == k
        tol = 2.0 ** -43 * key.abs().max() + 2.0 ** -50 * s.max()
        chosen = key[ids]
        assert bool((chosen[1:] <= chosen[:-1] + tol).all()), step
        rest = torch.ones((E,), dtype=torch.bool, device="cuda")
        rest[ids] = False
        assert bool((key[rest] <= chosen[-1] + tol).all()), step
        if E == k:
            close += int(((chosen[:-1] - chosen[1:]) < 2.0 ** -28 * key.abs().max()).sum())
        else:
            close += int(((chosen[:-1] - chosen[1:]) < 2.0 ** -32 * key.abs().max()).sum())
    assert binding.query_device_status() == 0
    assert close > 40 or span > 1             # neighbours that an error of 2^-32 would mix up
