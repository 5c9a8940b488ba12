"""GPU: tensors of one row (or one expert), whose stride from row to row PyTorch leaves open."""
import pytest
import torch

from blocks_ref import activation, gen, random_rows, random_weights
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu


def _row(t, stride):
    """The same single row (or layer) with another stride in front."""
    return t.as_strided(t.shape, (stride,) + t.stride()[1:])


@pytest.mark.parametrize("stride", [1, 7, 1 << 42])
def test_single_rows_of_any_stride(stride):
    N, K, k = 272, 400, 3
    g = gen(5)
    x, gu = activation(g, 1, K), activation(g, 1, 2 * K)
    want = binding.quantize_act_blocks(x)
    for a, b in zip(binding.quantize_act_blocks(_row(x, stride), out=tuple(_row(torch.zeros_like(t), stride) for t in want)), want):
        assert torch.equal(a, b)
    for a, b in zip(binding.quantize_act_blocks(_row(gu, stride), input_kind=binding.CHAIN_INPUT_SILU_MUL),
                    binding.quantize_act_blocks(gu, input_kind=binding.CHAIN_INPUT_SILU_MUL)):
        assert torch.equal(a, b)
    x8, s_x = random_rows(g, 1, K)
    w8, s_w = random_weights(g, (1, N, K))
    y = binding.linear_fp8_blocks(x8, s_x, w8[0], s_w[0])
    out = _row(torch.zeros_like(y), stride)
    assert torch.equal(binding.linear_fp8_blocks(_row(x8, stride), _row(s_x, stride), w8[0], s_w[0], out=out), y)
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    assert torch.equal(binding.linear_fp8_experts(_row(x8, stride), _row(s_x, stride), off, _row(w8, stride), s_w), y)
    logits = torch.randn((1, 64), generator=g, device="cuda")
    for a, b in zip(binding.route_experts(_row(logits, stride), k), binding.route_experts(logits, k)):
        assert torch.equal(a, b)
    rows, add = torch.randn((1, N), generator=g, device="cuda"), torch.randn((1, N), generator=g, device="cuda")
    slots, weights = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1, 1), 0.5, device="cuda")
    want = binding.combine_experts(rows, slots, weights, add=add, out_dtype=binding.OUT_FP32)
    out = _row(torch.zeros_like(want), stride)
    assert torch.equal(binding.combine_experts(_row(rows, stride), slots, weights, add=_row(add, stride), out=out), want)
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
