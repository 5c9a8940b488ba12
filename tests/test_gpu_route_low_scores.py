"""GPU: sigmoid scores near the end of FP64's range."""
import pytest
import torch

from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_bias", [False, True])
def test_scores_near_the_end_of_64_bits_keep_their_order(with_bias):
    # sigmoids of 1e-313 to 1e-296, which have the order of the logits (keys: a bias of zeros, or groups by their best two)
    low = torch.tensor([[-720.0, -700.0, -695.0, -705.0, -710.0, -691.0, -682.0, -715.0]], device="cuda")
    order = low[0].argsort(descending=True).tolist()
    kw = dict(bias=torch.zeros((8,), device="cuda")) if with_bias else dict(groups=2, top_groups=2, group_best=2)
    for roll in range(8):
        logits = low.roll(roll, 1)
        ids, weights, _, _ = binding.route_experts(logits, 8, score=binding.SCORE_SIGMOID, **kw)
        assert ids[0].tolist() == [(e + roll) % 8 for e in order]
        # shares of the sum: FP64 scores (the least has 36 bits) rounded once
        s = torch.exp(low[0, order].double() + 700.0)
        assert bool(((weights[0].double() - s / s.sum()).abs() <= 2.0 ** -23 * s / s.sum() + 2.0 ** -149).all())
    if not with_bias:       # the group with the two highest
        logits = torch.tensor([[-700.0, -701.0, -699.0, -708.0, -600.0, -709.0, -698.0, -699.5]], device="cuda")
        ids = binding.route_experts(logits, 2, score=binding.SCORE_SIGMOID, groups=4, top_groups=1, group_best=2)[0]
        assert ids[0].tolist() == [4, 5]
        logits[0, 4] = -900.0
        ids = binding.route_experts(logits, 2, score=binding.SCORE_SIGMOID, groups=4, top_groups=1, group_best=2)[0]
        assert ids[0].tolist() == [6, 7]
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
