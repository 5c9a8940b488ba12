"""FP8 layers of many tokens, whose kernel takes all tensor memory of an SM, between W4A8 layers and FP8 layers of few tokens: on one
stream, on two, captured; and on rows that lie megabytes apart."""
import pytest
import torch

from blocks_neighbours import EXPERTS, FAR_FEW, FAR_MANY, FEW_TOKENS, LAYER, MANY_TOKENS
from blocks_ref import E4M3, activation, blocks, gen, linear64, linear_tolerance, random_rows, random_weights
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


class _Steps:
    """W4A8, FP8 and experts' products of few and of many tokens, each into an output of its own."""

    def __init__(self, few, many):
        N, K = LAYER
        g = gen(few + many)
        tw = binding.prepack_weight(*binding.quantize_weight_rtn(torch.randn((N, K), generator=g, device="cuda")))
        w8, s_w = random_weights(g, (N, K))
        e8, s_e = random_weights(g, (EXPERTS, N, K))
        self.calls = []
        for M in (few, many):
            x = activation(g, M, K)
            a, b = binding.quantize_act(x)[:2], binding.quantize_act_blocks(x)
            off = torch.tensor([0, M // 3, M // 3, M - 1, M], dtype=torch.int32, device="cuda")
            self.calls += [lambda out, ws, a=a: binding.linear_tiled(*a, tw, out=out, workspace=ws),
                           lambda out, ws, b=b: binding.linear_fp8_blocks(*b, w8, s_w, out=out),
                           lambda out, ws, b=b, off=off: binding.linear_fp8_experts(*b, off, e8, s_e, out=out)]
        self.shapes = [(few, N)] * 3 + [(many, N)] * 3
        self.fmt = tw.fmt
        alone = self.buffers()
        for i in range(6):
            self.run(i, alone)
            torch.cuda.synchronize()
        self.want = alone[0]

    def buffers(self):
        N, K = LAYER
        return ([torch.zeros(s, dtype=BF16, device="cuda") for s in self.shapes],
                [binding.new_workspace(s[0], N, K, self.fmt) for s in self.shapes])

    def run(self, i, buffers):
        self.calls[i](buffers[0][i], buffers[1][i])

    def check(self, buffers):
        torch.cuda.synchronize()
        assert binding.query_device_status() == 0
        for out, w in zip(buffers[0], self.want):
            assert torch.equal(out, w)


ORDER = [4, 0, 4, 1, 4, 3, 4, 4, 5, 5, 2, 5, 3, 5, 1, 3, 4, 2, 0, 5, 4, 3, 3, 1, 4, 5, 0, 2]


@pytest.mark.parametrize("few,many", list(zip(FEW_TOKENS, MANY_TOKENS)))
def test_in_turn_on_one_stream(few, many):
    s = _Steps(few, many)
    got = s.buffers()
    for _ in range(3):
        for i in ORDER:
            s.run(i, got)
    s.check(got)


@pytest.mark.parametrize("few,many", list(zip(FEW_TOKENS, MANY_TOKENS)))
def test_on_two_streams_and_captured(few, many):
    s = _Steps(few, many)
    got = [s.buffers(), s.buffers(), s.buffers()]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, j in zip(ORDER, reversed(ORDER)):       # the two streams' calls alternate
            for stream, step, buffers in ((side[0], i, got[0]), (side[1], j, got[1])):
                with torch.cuda.stream(stream):
                    s.run(step, buffers)
    s.check(got[0])
    s.check(got[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in ORDER:
            s.run(i, got[2])
    for out in got[2][0]:
        out.zero_()
    for _ in range(2):
        graph.replay()
    s.check(got[2])


def test_rows_far_apart():
    # 8 MB from one row of activations to the next, 16 MB between those of the result: the last of 520 lie 4.3 and 8.7 GB off
    far = 1 << 23
    rows, N, K = FAR_MANY
    g = gen(3)
    x8, s_x = random_rows(g, rows, K)
    w8, s_w = random_weights(g, (2, N, K))
    wide = torch.zeros((rows, far), dtype=torch.uint8, device="cuda")
    wide[:, :K] = x8
    wide[:, K:K + 128] = 0x7F                          # NaN behind the rows
    out = torch.zeros((rows, far), dtype=BF16, device="cuda")
    for few in (FAR_MANY[0], FAR_FEW[0]):
        at = rows - few                                # the last rows
        y, mag = linear64(x8[at:], s_x[at:], w8[0], s_w[0])
        out[:, :N + 16] = 7.0
        binding.linear_fp8_blocks(wide[at:, :K], s_x[at:], w8[0], s_w[0], out=out[at:, :N])
        torch.cuda.synchronize()
        assert binding.query_device_status() == 0
        assert bool(((out[at:, :N].double() - y).abs() <= linear_tolerance(mag, K, BF16, y)).all())
        assert bool((out[:at, :N] == 7.0).all()) and bool((out[:, N:N + 16] == 7.0).all())
        # experts: bulk stores where 32 rows are there, a warp's own where an expert ends
        off = torch.tensor([0, few // 2 + 1, few - 1], dtype=torch.int32, device="cuda")
        out[:, :N + 16] = 7.0
        binding.linear_fp8_experts(wide[at:, :K], s_x[at:], off, w8, s_w, out=out[at:, :N])
        torch.cuda.synchronize()
        assert binding.query_device_status() == 0
        cut = at + few // 2 + 1
        for e, (a, b) in enumerate(((at, cut), (cut, rows - 1))):
            y, mag = linear64(x8[a:b], s_x[a:b], w8[e], s_w[e])
            assert bool(((out[a:b, :N].double() - y).abs() <= linear_tolerance(mag, K, BF16, y)).all())
        assert bool((out[rows - 1, :N] == 7.0).all()) and bool((out[:at, :N] == 7.0).all()) and bool((out[:, N:N + 16] == 7.0).all())
    assert blocks(K) == s_x.shape[1] and x8.view(E4M3).float().isfinite().all()
