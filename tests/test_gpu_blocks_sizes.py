"""Many tokens in the routing (several rounds of rows per CTA, more choices than shared memory keeps), and rows behind four
gigabytes in the quantization and the weighted sum."""
import math

import pytest
import torch

from blocks_ref import activation, gen, quantize_fp32
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("M,E,k,sigmoid", [(128, 512, 32, True), (5000, 512, 32, False), (20001, 48, 16, True), (66000, 64, 8, False), (80007, 100, 8, True)])
def test_routing_of_many_tokens(M, E, k, sigmoid):
    g = gen(M)
    logits = torch.randn((M, E), generator=g, device="cuda")
    logits[M // 3:M // 3 + 40] = -math.inf                      # tokens of no expert
    logits[M // 2] = -math.inf
    logits[M // 2, E // 2] = 1.0                                # and of one
    ids, weights, offsets, slots = binding.route_experts(logits, k, score=binding.SCORE_SIGMOID if sigmoid else binding.SCORE_SOFTMAX)
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
    x = logits.double()
    order = x.sort(dim=-1, descending=True, stable=True)
    there = order.values[:, :k] > -math.inf
    want = torch.where(there, order.indices[:, :k], -1)
    assert torch.equal(ids.long(), want)
    s = torch.where(there, 1.0 / (1.0 + torch.exp(-order.values[:, :k])) if sigmoid else torch.exp(order.values[:, :k] - order.values[:, :1]), 0.0)
    total = s.sum(-1, keepdim=True)
    w = torch.where(total > 0, s / total, 0.0)
    # scores and sums in FP64, rounded once
    assert bool(((weights.double() - w).abs() <= 2.0 ** -24 * 1.01 * w + 2.0 ** -149).all())
    flat = want.view(-1)
    counts = torch.bincount(flat[flat >= 0], minlength=E)
    assert torch.equal(offsets.long(), torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]))
    by_expert = torch.where(flat >= 0, flat, E).sort(dim=0, stable=True).indices
    rows = torch.full_like(flat, -1)
    n = int(counts.sum())
    rows[by_expert[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(slots.long().view(-1), rows)


def test_rows_behind_four_gigabytes():
    M, K, far = 520, 272, 1 << 23                               # values from a row to the next
    g = gen(7)
    x, gate_up = activation(g, M, K), activation(g, M, 2 * K)
    wide = torch.zeros((M, far), dtype=BF16, device="cuda")     # 8.7 GB
    wide[:, :K] = x
    x8 = torch.zeros((M, far), dtype=torch.uint8, device="cuda")
    s = torch.zeros((M, 3), device="cuda")
    binding.quantize_act_blocks(wide[:, :K], out=(x8[:, :K], s))
    want8, want_s = quantize_fp32(x)
    assert torch.equal(x8[:, :K], want8) and torch.equal(s, want_s) and not bool(x8[:, K].any())
    wide[:, :2 * K] = gate_up
    slots = torch.randperm(M, generator=g, device="cuda").to(torch.int32).view(M, 1)
    binding.quantize_act_blocks(wide[:, :2 * K], input_kind=binding.CHAIN_INPUT_SILU_MUL, slots=slots, out=(x8[:, :K], s))
    want8, want_s = binding.quantize_act_blocks(gate_up, input_kind=binding.CHAIN_INPUT_SILU_MUL)
    assert torch.equal(x8[:, :K][slots[:, 0].long()], want8) and torch.equal(s[slots[:, 0].long()], want_s)
    # the products' activations so far apart too: a tile of few tokens, and of many
    w8 = torch.randint(-3, 4, (256, K), generator=g, device="cuda").float().to(torch.float8_e4m3fn).view(torch.uint8)
    s_w = torch.rand((2, 3), generator=g, device="cuda")
    for rows in (5, M):
        near = binding.linear_fp8_blocks(x8[:, :K][M - rows:].contiguous(), s[M - rows:].contiguous(), w8, s_w)
        assert torch.equal(binding.linear_fp8_blocks(x8[M - rows:, :K], s[M - rows:], w8, s_w), near)
    weights = torch.rand((M, 1), generator=g, device="cuda")
    out = torch.zeros((M, far), dtype=BF16, device="cuda")
    binding.combine_experts(wide[:, :K], slots, weights, add=wide[:, K:2 * K], out=out[:, :K])
    near = binding.combine_experts(wide[:, :K].contiguous(), slots, weights, add=wide[:, K:2 * K].contiguous())
    assert torch.equal(out[:, :K], near)
    # one fused multiply-add of 2^-24, and half a step of BF16
    y, add = wide[:, :K].double()[slots[:, 0].long()], wide[:, K:2 * K].double()
    want, mag = weights.double() * y + add, (weights.double() * y).abs() + add.abs()
    tol = 2.0 ** -24 * mag
    assert bool(((near.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all())
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
