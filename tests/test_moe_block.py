"""The mixture-of-experts block: its sequence of steps and its checks with a plain stand-in for the library (no GPU), and the
block on the library against 64 bits."""
import types

import pytest
import torch

from paper_2505_14638_b200.moe import BlockWeights, MoeMlpBlock


def _weights(*shape):
    s = shape[:-2] + (-(-shape[-2] // 128), -(-shape[-1] // 128))
    return BlockWeights(torch.zeros(shape, dtype=torch.uint8), torch.ones(s))


class _Recorder:
    CHAIN_INPUT_SILU_MUL = 1

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args, **kw):
            self.calls.append((name, args, kw))
            return {"route_experts": ("ids", "weights", "offsets", "slots"), "quantize_act_blocks": ("x8", "s")}.get(name, name)
        return call


def test_steps_in_order():
    ops = _Recorder()
    gu, down = _weights(4, 64, 32), _weights(4, 32, 32)
    shared = (_weights(96, 32), _weights(32, 48))
    block = MoeMlpBlock(gu, down, 2, shared=shared, ops=ops, scale=2.5)
    x, logits = torch.zeros((3, 32), dtype=torch.bfloat16), torch.zeros((3, 4))
    assert block.forward(x, logits) == "combine_experts"
    names = [c[0] for c in ops.calls]
    assert names == ["route_experts", "quantize_act_blocks", "linear_fp8_experts", "quantize_act_blocks", "linear_fp8_experts",
                     "quantize_act_blocks", "linear_fp8_blocks", "quantize_act_blocks", "linear_fp8_blocks", "combine_experts"]
    assert ops.calls[0][1] == (logits, 2) and ops.calls[0][2] == {"scale": 2.5}
    assert ops.calls[1][2] == {"slots": "slots"} and ops.calls[3][2] == {"input_kind": 1}
    assert ops.calls[2][1][2:] == ("offsets", gu.w8, gu.s_w) and ops.calls[4][1][2:] == ("offsets", down.w8, down.s_w)
    assert ops.calls[-1][1] == ("linear_fp8_experts", "slots", "weights") and ops.calls[-1][2] == {"add": "linear_fp8_blocks", "out": None}


def test_shapes_that_do_not_fit_are_refused():
    ops = types.SimpleNamespace()
    gu, down = _weights(4, 64, 32), _weights(4, 32, 32)
    for a, b, kw in ((_weights(64, 32), down, {}), (gu, _weights(3, 32, 32), {}), (gu, _weights(4, 48, 32), {}), (gu, _weights(4, 32, 48), {}),
                     (gu, down, dict(shared=(_weights(64, 48), _weights(48, 32)))), (gu, down, dict(shared=(_weights(64, 32), _weights(32, 48))))):
        with pytest.raises(ValueError):
            MoeMlpBlock(a, b, 2, ops=ops, **kw)
    block = MoeMlpBlock(gu, down, 2, ops=ops)
    for logits in (torch.zeros((3, 5)), torch.zeros((2, 4))):
        with pytest.raises(ValueError):
            block.forward(torch.zeros((3, 32), dtype=torch.bfloat16), logits)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 64, 777])
@pytest.mark.parametrize("with_shared", [False, True])
def test_block_on_the_library(M, with_shared):
    from blocks_ref import activation, gen, quantize_fp32, random_weights, route64, rows64, weights64
    from paper_2505_14638_b200 import binding
    E, k, H, F = 16, 4, 272, 400
    g = gen(M)
    gu, down = BlockWeights(*random_weights(g, (E, 2 * F, H))), BlockWeights(*random_weights(g, (E, H, F)))
    shared = (BlockWeights(*random_weights(g, (2 * 144, H))), BlockWeights(*random_weights(g, (H, 144)))) if with_shared else None
    routing = dict(score=binding.SCORE_SIGMOID, bias=0.1 * torch.randn((E,), generator=g, device="cuda"), groups=4, top_groups=2,
                   group_best=2, scale=2.5)
    block = MoeMlpBlock(gu, down, k, shared=shared, **routing)
    x, logits = activation(g, M, H), torch.randn((M, E), generator=g, device="cuda")
    if M > 1:
        logits[1] = -torch.inf                  # a padded token: nothing but the shared MLP
    got = block.forward(x, logits)
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0

    def mlp(rows, gate_up, w_down):
        """In 64 bits, but for the first quantization and the BF16 output of gate/up.  Returns (y, largest error)."""
        y = (rows64(*quantize_fp32(rows)) @ weights64(*gate_up).T).to(torch.bfloat16).double()
        half = y.shape[1] // 2
        g, u = y[:, :half], y[:, half:]
        h = g / (1.0 + torch.exp(-g)) * u
        # gate and up may each be the neighbouring BF16 value (2^-7 of it; silu has a slope of at most 1.1); h is rounded to E4M3
        # (2^-4 of it, 2^-10 of the block's scale where that is more)
        low = torch.nn.functional.pad(h, (0, -half % 128)).view(h.shape[0], -1, 128).abs().amax(-1).repeat_interleave(128, 1)[:, :half] / 448.0
        off = (2.0 ** -4 + 2.0 ** -7) * h.abs() + 1.1 * 2.0 ** -7 * (g * u).abs() * 1.1 + 2.0 ** -10 * low
        w = weights64(*w_down)
        return h @ w.T, off @ w.abs().T + 2.0 ** -8 * (h.abs() @ w.abs().T)      # (and y to BF16)

    ids, weights, _, _ = route64(logits, k, sigmoid=True, **{n: v for n, v in routing.items() if n != "score"})
    want, tol = torch.zeros((M, H), dtype=torch.float64, device="cuda"), torch.zeros((M, H), dtype=torch.float64, device="cuda")
    for e in range(E):
        m, j = (ids == e).nonzero(as_tuple=True)
        if m.numel():
            y, a = mlp(x[m.cuda()], (gu.w8[e], gu.s_w[e]), (down.w8[e], down.s_w[e]))
            w = weights[m, j].cuda().unsqueeze(1)
            want.index_add_(0, m.cuda(), w * y)
            tol.index_add_(0, m.cuda(), w * a)
    if shared is not None:
        y, a = mlp(x, (shared[0].w8, shared[0].s_w), (shared[1].w8, shared[1].s_w))
        want, tol = want + y, tol + a
    assert bool(((got.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all())
    if M > 1 and shared is None:
        assert bool((got[1] == 0).all())
    # the steps one by one give the same bits
    _, w, off, slots = binding.route_experts(logits, k, **routing)
    x8, s = binding.quantize_act_blocks(x, slots=slots)
    h = binding.quantize_act_blocks(binding.linear_fp8_experts(x8, s, off, gu.w8, gu.s_w), input_kind=binding.CHAIN_INPUT_SILU_MUL)
    y = binding.linear_fp8_experts(*h, off, down.w8, down.s_w)
    assert torch.equal(binding.combine_experts(y, slots, w, add=None if shared is None else block._shared_mlp(x)), got)
    # and so does a captured pass, with other tokens in between
    graph, xs, ls, out = torch.cuda.CUDAGraph(), x.clone(), logits.clone(), torch.empty_like(got)
    with torch.cuda.graph(graph):
        block.forward(xs, ls, out=out)
    for order in (torch.arange(M - 1, -1, -1, device="cuda"), torch.arange(M, device="cuda")):
        xs.copy_(x[order])
        ls.copy_(logits[order])
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, got)
