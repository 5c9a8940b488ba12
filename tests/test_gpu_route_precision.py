"""GPU: how exact the routing's scores, weights and keys are."""
import math

import pytest
import torch

from blocks_ref import gen, route64
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def _route(logits, k, sigmoid=False, **kw):
    got = binding.route_experts(logits, k, score=binding.SCORE_SIGMOID if sigmoid else binding.SCORE_SOFTMAX, **kw)
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
    return got


@pytest.mark.parametrize("M,E,k", [(1, 8, 2), (16, 64, 6), (130, 96, 4), (33, 512, 32), (300, 200, 16), (700, 128, 8)])
@pytest.mark.parametrize("scale", [0.5, 6.0])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_softmax_weights_that_are_not_renormalised(M, E, k, scale, dtype):
    # With a bias (of zeros) scores and their sum are in FP64, rounded once (2^-24); without one the sum over all experts is in FP32:
    # every exp within 2 ulp (2^-22); the differences to the largest logit 2^-24 of themselves, averaged over the terms (whose shares
    # are exp(-difference) / sum) at most ln E <= 6.3 times 2^-24; at most E / 32 + 5 sums of 2^-24; and the one rounding.
    logits = (torch.randn((M, E), generator=gen(M + E), device="cuda") * scale).to(dtype)
    if M > 2:
        logits[1, : E - 2] = -math.inf
        logits[2, 0] = math.nan
    ids, weights, _, _ = route64(logits, k, renormalize=False)
    for bias, tol in ((torch.zeros((E,), device="cuda"), 2.0 ** -24 * 1.01), (None, (E / 32 + 17) * 2.0 ** -24)):
        got = _route(logits, k, renormalize=False, bias=bias)
        assert torch.equal(got[0].cpu().long(), ids)
        assert bool(((got[1].cpu().double() - weights).abs() <= tol * weights + 2.0 ** -149).all())
    # and with groups by their best two
    groups = dict(groups=4, top_groups=3, group_best=2) if E % 4 == 0 and k <= E // 4 * 3 else dict()
    if groups:
        ids, weights, _, _ = route64(logits, k, renormalize=False, **groups)
        got = _route(logits, k, renormalize=False, **groups)
        assert torch.equal(got[0].cpu().long(), ids)
        assert bool(((got[1].cpu().double() - weights).abs() <= 2.0 ** -24 * 1.01 * weights + 2.0 ** -149).all())
