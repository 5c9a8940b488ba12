"""GPU parity: routing to experts and the weighted sum of their outputs against the definitions in 64 bits."""
import math

import pytest
import torch

from blocks_ref import gen, route64
from gpu_utils import Guarded
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def _check(logits, top_k, **kw):
    M, E = logits.shape
    got = binding.route_experts(logits, top_k, score=binding.SCORE_SIGMOID if kw.get("sigmoid") else binding.SCORE_SOFTMAX,
                                **{k: v for k, v in kw.items() if k != "sigmoid"})
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0
    ids, weights, offsets, slots = route64(logits, top_k, **kw)
    assert torch.equal(got[0].cpu().long(), ids)
    assert torch.equal(got[2].cpu().long(), offsets) and torch.equal(got[3].cpu().long(), slots)
    # scores in FP64, rounded once (2^-24) -- except the softmax's sum over all experts where it is not renormalised: FP32, each
    # exp within 2 ulp (2^-22), at most experts / 32 + 5 sums of 2^-24
    tol = 2.0 ** -24 * 1.01
    if not kw.get("renormalize", True) and not kw.get("sigmoid"):
        tol += 2.0 ** -22 + (E / 32 + 6) * 2.0 ** -24
    assert bool(((got[1].cpu().double() - weights).abs() <= tol * weights.abs() + 2.0 ** -149).all())
    return got


@pytest.mark.parametrize("M,E,k", [(1, 8, 2), (1, 256, 8), (16, 64, 6), (17, 2, 1), (64, 256, 8), (130, 96, 4), (33, 512, 32), (700, 128, 8), (3, 1, 1), (2500, 40, 3)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_plain_choice(M, E, k, sigmoid, dtype):
    logits = torch.randn((M, E), generator=gen(M + E), device="cuda").to(dtype)
    _check(logits, k, sigmoid=sigmoid)
    _check(logits, k, sigmoid=sigmoid, renormalize=False, scale=2.5)


@pytest.mark.parametrize("M,E,k,groups,top_groups", [(1, 256, 8, 8, 4), (64, 256, 8, 8, 4), (40, 64, 3, 4, 1), (19, 160, 6, 8, 3), (600, 32, 4, 16, 8), (5, 512, 16, 32, 5)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("with_bias", [False, True])
def test_groups_and_bias(M, E, k, groups, top_groups, sigmoid, best, with_bias):
    g = gen(M + E + groups)
    logits = torch.randn((M, E), generator=g, device="cuda")
    bias = 0.3 * torch.randn((E,), generator=g, device="cuda") if with_bias else None
    _check(logits, k, sigmoid=sigmoid, bias=bias, groups=groups, top_groups=top_groups, group_best=best, scale=1.5)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_equal_scores_go_to_the_lower_index(sigmoid):
    g = gen(5)
    logits = torch.randint(-2, 3, (50, 64), generator=g, device="cuda").float()
    logits[logits == 0] *= -1.0                                   # zeros of both signs are equal
    logits[0] = 1.0
    _check(logits, 8, sigmoid=sigmoid)
    _check(logits, 8, sigmoid=sigmoid, groups=8, top_groups=3, group_best=2)
    bias = torch.randint(-1, 2, (64,), generator=g, device="cuda").float()
    _check(logits, 8, sigmoid=sigmoid, bias=bias, groups=8, top_groups=3, group_best=1)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
def test_experts_that_cannot_be_chosen_and_tokens_of_none(sigmoid, with_bias):
    g = gen(9)
    logits = torch.randn((70, 32), generator=g, device="cuda")
    logits[0] = -math.inf                       # a padded token
    logits[1, 3:] = -math.inf                   # three experts left for four choices
    logits[2] = math.nan
    logits[3, 7] = math.nan
    logits[4, :] = torch.finfo(FP32).min        # masks of the lowest value are values
    logits[5, 4] = math.inf
    logits[6, 4] = logits[6, 9] = math.inf
    logits[7, :16] = -math.inf
    logits[69] = -math.inf
    bias = None
    if with_bias:
        bias = 0.1 * torch.randn((32,), generator=g, device="cuda")
        bias[12] = -math.inf
        bias[13] = math.nan
        bias[14] = math.inf
    got = _check(logits, 4, sigmoid=sigmoid, bias=bias)
    assert got[0][0].tolist() == [-1] * 4 and got[1][0].tolist() == [0.0] * 4 and got[3][0].tolist() == [-1] * 4
    for best in (1, 2):
        _check(logits, 4, sigmoid=sigmoid, bias=bias, groups=8, top_groups=2, group_best=best)
    _check(logits, 4, sigmoid=sigmoid, bias=bias, renormalize=False)


def test_scores_beyond_the_range_of_32_bits():
    logits = torch.tensor([[-200.0, -300.0, -250.0, -220.0], [90.0, -90.0, 0.0, 80.0], [-1000.0, -2000.0, -1500.0, -900.0]], device="cuda")
    _check(logits, 2, sigmoid=True)
    _check(logits, 2, sigmoid=False)
    _check(logits, 3, sigmoid=True, renormalize=False)


def test_logits_in_wider_rows_and_buffers_of_exact_size():
    g = gen(77)
    M, E, k = 90, 72, 5
    wide = torch.full((M, E + 7), math.inf, device="cuda")
    wide[:, :E] = torch.randn((M, E), generator=g, device="cuda")
    out = [Guarded((M, k), torch.int32), Guarded((M, k), FP32), Guarded((E + 1,), torch.int32), Guarded((M, k), torch.int32)]
    ws = Guarded((binding.route_experts_workspace_bytes(M, E),), torch.uint8)
    binding.route_experts(wide[:, :E], k, out=tuple(o.t for o in out), workspace=ws.t)
    want = route64(wide[:, :E], k)
    for o, w in zip(out, want):
        assert torch.allclose(o.t.cpu().double(), w.double(), rtol=1e-6)
        o.check()
    ws.check()


def test_two_streams_and_a_captured_call():
    logits = [torch.randn((400, 64), generator=gen(i), device="cuda") for i in range(2)]
    want = [binding.route_experts(x, 6) for x in logits]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            for _ in range(4):
                got[i] = binding.route_experts(logits[i], 6)
    torch.cuda.synchronize()
    graph, x = torch.cuda.CUDAGraph(), torch.zeros_like(logits[0])
    out = tuple(torch.zeros_like(t) for t in want[0])
    with torch.cuda.graph(graph):
        binding.route_experts(x, 6, out=out)
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
        x.copy_(logits[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))


def test_refusals():
    x = torch.randn((4, 64), device="cuda")
    for kw in (dict(top_k=0), dict(top_k=33), dict(top_k=9, groups=8), dict(top_k=4, groups=7), dict(top_k=4, groups=8, top_groups=9),
               dict(top_k=4, group_best=3), dict(top_k=4, score=7), dict(top_k=4, groups=64, top_groups=64)):
        with pytest.raises(binding.W4A8Error):
            binding.route_experts(x, **kw)
    with pytest.raises(binding.W4A8Error):
        binding.route_experts(torch.randn((4, 513), device="cuda"), 2)
    with pytest.raises(binding.W4A8Error):
        binding.route_experts(torch.randn((400, 64), device="cuda"), 2, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(AssertionError):
        binding.route_experts(x.double(), 2)
    with pytest.raises(AssertionError):
        binding.route_experts(x, 2, bias=torch.zeros(63, device="cuda"))


# ------------------------------------------------------------------------------ weighted sum
@pytest.mark.parametrize("M,N,k", [(1, 16, 1), (16, 4096, 8), (33, 272, 3), (700, 2064, 6), (5, 7168, 10)])
@pytest.mark.parametrize("y_dtype", [BF16, FP32])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("with_add", [False, True])
def test_combine(M, N, k, y_dtype, dtype, with_add):
    g = gen(M + N + k)
    y = torch.randn((M * k + 3, N), generator=g, device="cuda").to(y_dtype)
    slots = torch.randperm(M * k + 3, generator=g, device="cuda")[:M * k].to(torch.int32).view(M, k)
    weights = torch.rand((M, k), generator=g, device="cuda")
    add = torch.randn((M, N), generator=g, device="cuda").to(dtype) if with_add else None
    out = Guarded((M, N), dtype)
    binding.combine_experts(y, slots, weights, add=add, out=out.t)
    terms = weights.double().unsqueeze(-1) * y.double()[slots.long()]
    want, mag = terms.sum(1), terms.abs().sum(1)
    if with_add:
        want, mag = want + add.double(), mag + add.double().abs()
    # k fused multiply-adds of 2^-24 each, relative to at most the sum of magnitudes; BF16: half a step more
    tol = (k + 1) * 2.0 ** -24 * mag
    if dtype == BF16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert bool(((out.t.double() - want).abs() <= tol).all())
    out.check()


def test_tokens_without_experts_and_rows_that_are_not_finite():
    g = gen(3)
    M, N, k = 12, 144, 4
    y = torch.randn((M * k, N), generator=g, device="cuda").to(BF16)
    y[0] = math.nan
    slots = torch.arange(M * k, device="cuda", dtype=torch.int32).view(M, k).clone()
    weights = torch.rand((M, k), generator=g, device="cuda")
    slots[0, 0] = -1                               # row 0 is named by nothing
    weights[0, 0] = math.nan                       # and its weight is not looked at
    slots[1] = -1
    slots[2, 1] = M * k                            # outside
    slots[3, 3] = 2 ** 31 - 1
    add = torch.randn((M, N), generator=g, device="cuda").to(BF16)
    got = binding.combine_experts(y, slots, weights, add=add)
    assert bool(got.isfinite().all()) and torch.equal(got[1], add[1])
    assert torch.equal(binding.combine_experts(y, slots, weights)[1], torch.zeros(N, dtype=BF16, device="cuda"))
    have = (slots >= 0) & (slots < M * k)
    safe = torch.where(have, slots, 1).long()
    want = add.double() + (torch.where(have, weights.nan_to_num(), 0.0).double().unsqueeze(-1) * y.double()[safe]).sum(1)
    assert bool(((got.double() - want).abs() <= 2.0 ** -7 * (want.abs() + 1)).all())
    same = add.clone()
    assert torch.equal(binding.combine_experts(y, slots, weights, add=same, out=same), got)      # in place


def test_strides_of_the_sum():
    g = gen(6)
    M, N, k = 20, 272, 2
    y = torch.randn((M * k, N + 16), generator=g, device="cuda").to(BF16)
    slots = torch.randperm(M * k, generator=g, device="cuda").to(torch.int32).view(M, k)
    weights = torch.rand((M, k), generator=g, device="cuda")
    out = torch.full((M, N + 8), 7.0, dtype=BF16, device="cuda")
    binding.combine_experts(y[:, :N], slots, weights, out=out[:, :N])
    assert torch.equal(out[:, :N], binding.combine_experts(y[:, :N].contiguous(), slots, weights))
    assert bool((out[:, N:] == 7.0).all())
    with pytest.raises(binding.W4A8Error):
        binding.combine_experts(y[:, 1:N + 1], slots, weights)     # rows not 16-byte aligned
    with pytest.raises(AssertionError):
        binding.combine_experts(y[:, :N], slots, weights.double())
