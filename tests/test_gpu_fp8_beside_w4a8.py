"""FP8 layers with block scales between W4A8 layers on one stream: each of these kernels starts its set-up (tensor memory among it)
while the one before it still runs."""
import pytest
import torch

from blocks_ref import activation, gen, random_weights
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [(1, 1), (16, 1), (1, 77), (77, 200), (300, 5), (520, 600)])
def test_layers_in_turn_give_what_each_gives_alone(tokens):
    few, many = tokens
    K, N = 1024, 1536
    g = gen(41 + few + many)
    codes, gscale, gzero, s_w4 = binding.quantize_weight_rtn(torch.randn((N, K), generator=g, device="cuda"))
    tw = binding.prepack_weight(codes, gscale, gzero, s_w4)
    w8, s_w = random_weights(g, (N, K))
    e8, s_e = random_weights(g, (4, N, K))

    steps, keep = [], []
    for M in (few, many):
        x = activation(g, M, K)
        a, b = binding.quantize_act(x), binding.quantize_act_blocks(x)
        off = torch.tensor([0, M // 2, M // 2, M - 1, M], dtype=torch.int32, device="cuda")
        ws = binding.new_workspace(M, N, K, tw.fmt)
        keep.append((x, ws))
        steps += [lambda out, a=a, ws=ws: binding.linear_tiled(*a[:2], tw, out=out, workspace=ws),
                  lambda out, b=b: binding.linear_fp8_blocks(*b, w8, s_w, out=out),
                  lambda out, b=b, off=off: binding.linear_fp8_experts(*b, off, e8, s_e, out=out)]
    outs = [torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for M in (few, many) for _ in range(3)]
    want = []
    for step, out in zip(steps, outs):
        step(out)
        torch.cuda.synchronize()
        want.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    order = [0, 1, 3, 2, 4, 0, 5, 1, 1, 4, 4, 2, 2, 5, 3, 0, 2, 3, 4, 1, 5, 5, 0, 4, 3, 1, 2, 0]
    for _ in range(3):
        for i in order:
            steps[i](outs[i])
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
    for out, w in zip(outs, want):
        assert torch.equal(out, w)
