"""GPU parity: block quantization and FP8 linear layers with block scales, of one layer and of several experts, against the
definitions in 64 bits."""
import pytest
import torch

from blocks_ref import (E4M3, activation, blocks, gen, linear64, linear_tolerance, quantize_fp32, random_rows, random_weights)
from blocks_shapes import EXPERTS_FEW, EXPERTS_MANY, EXPERTS_MANY_LAYERS, FEW, MANY
from gpu_utils import Guarded
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def _same_bits(a, b):
    return torch.equal(a.view(torch.uint8) if a.dtype != torch.uint8 else a, b.view(torch.uint8) if b.dtype != torch.uint8 else b)


def _out(M, N, dtype):
    return Guarded((M, N), dtype, fill=7.0)


def _clean():
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0


# ------------------------------------------------------------------------------ quantization
@pytest.mark.parametrize("M,K", [(1, 16), (1, 128), (3, 144), (7, 1040), (16, 4096), (130, 656), (513, 2816), (2, 14336)])
def test_plain_quantization_is_the_definition_bit_for_bit(M, K):
    x = activation(gen(M + K), M, K)
    x[0] = 0                                   # a token of zeros
    if M > 2:
        x[1, :128] = 0
        x[1, 0] = 1e-38                        # below the least maximum
        x[2, :16] = 3e38
    x8, s = Guarded((M, K), torch.uint8), Guarded((M, blocks(K)), FP32)
    binding.quantize_act_blocks(x, out=(x8.t, s.t))
    _clean()
    want8, want_s = quantize_fp32(x)
    assert torch.equal(x8.t, want8) and _same_bits(s.t, want_s)
    x8.check(), s.check()


def test_values_that_are_not_finite_stay_visible():
    x = activation(gen(1), 4, 256)
    x[0, 3] = float("nan")
    x[1, 130] = float("inf")
    x[2, 0] = -float("inf")
    x8, s = binding.quantize_act_blocks(x)
    v = x8.view(E4M3).float() * s.repeat_interleave(128, 1)
    assert bool(v[0, 3].isnan()) and int(v[0].isnan().sum()) == 1
    assert bool(v[1, 130].isnan()) and not bool(v[1, :128].isnan().any())
    assert bool(v[2, 0].isnan()) and not bool(v[2, 128:].isnan().any()) and not bool(v[3].isnan().any())
    want8, want_s = quantize_fp32(x)
    assert torch.equal(s, want_s) and torch.equal(x8[3], want8[3]) and torch.equal(x8[0, 128:], want8[0, 128:])


@pytest.mark.parametrize("M,F", [(1, 16), (5, 256), (16, 1408), (300, 2064), (3, 14336)])
def test_gated_quantization(M, F):
    # silu in FP32: exp within 2 ulp (2^-22), then a sum, a division and a product of 2^-24 each: together within 2^-21
    gu = activation(gen(M * 3 + F), M, 2 * F, 2.0)
    x8, s = binding.quantize_act_blocks(gu, input_kind=binding.CHAIN_INPUT_SILU_MUL)
    _clean()
    g, u = gu[:, :F].double(), gu[:, F:].double()
    h = g / (1.0 + torch.exp(-g)) * u
    amax = torch.nn.functional.pad(h, (0, blocks(F) * 128 - F)).view(M, -1, 128).abs().amax(-1)
    assert bool(((s.double() - amax / 448.0).abs() <= (2.0 ** -21 + 2.0 ** -23) * amax / 448.0).all())
    sd = s.double().repeat_interleave(128, 1)[:, :F]
    off = (x8.view(E4M3).double() * sd - h).abs()
    # half a step of E4M3 (2^-4 of the value, 2^-10 of the scale where it is subnormal) and what h itself is off
    assert bool((off <= h.abs() * (2.0 ** -4 + 2.0 ** -20) + sd * 2.0 ** -10 * (1 + 2.0 ** -20)).all())


def test_extreme_gates():
    gu = torch.zeros((1, 256), dtype=BF16, device="cuda")
    gu[0, :4] = torch.tensor([-100.0, 100.0, -3e38, 0.0])
    gu[0, 128:132] = torch.tensor([3.0, 2.0, 1.0, 5.0])
    x8, s = binding.quantize_act_blocks(gu, input_kind=binding.CHAIN_INPUT_SILU_MUL)
    assert x8.view(E4M3).float()[0, :4].tolist() == [0.0, 448.0, 0.0, 0.0]
    assert abs(float(s[0, 0]) * 448.0 - 200.0) < 1e-3


@pytest.mark.parametrize("M,K,k", [(1, 128, 1), (5, 144, 3), (64, 2048, 8), (300, 656, 6)])
@pytest.mark.parametrize("gated", [False, True])
def test_rows_of_the_experts_and_rows_that_nothing_names(M, K, k, gated):
    g = gen(M + K + k)
    x = activation(g, M, K * (2 if gated else 1))
    kind = binding.CHAIN_INPUT_SILU_MUL if gated else binding.CHAIN_INPUT_PLAIN
    rows = M * k + 5
    slots = torch.randperm(rows, generator=g, device="cuda")[:M * k].to(torch.int32).view(M, k)
    slots[0, 0] = -1
    if M > 1:
        slots[1, k - 1] = rows                 # outside: skipped
    if M > 2:
        slots[2] = torch.iinfo(torch.int32).min
    x8, s = Guarded((rows, K), torch.uint8, fill=0x5A), Guarded((rows, blocks(K)), FP32, fill=3.5)
    binding.quantize_act_blocks(x, input_kind=kind, slots=slots, out=(x8.t, s.t))
    _clean()
    one8, one_s = binding.quantize_act_blocks(x, input_kind=kind)
    want8, want_s = torch.full_like(x8.t, 0x5A), torch.full_like(s.t, 3.5)
    for m in range(M):
        for r in slots[m].tolist():
            if 0 <= r < rows:
                want8[r], want_s[r] = one8[m], one_s[m]
    assert torch.equal(x8.t, want8) and torch.equal(s.t, want_s)
    x8.check(), s.check()


def test_strides_of_the_quantization():
    M, K = 9, 272
    g = gen(4)
    wide = activation(g, M, K + 24)
    x8 = torch.full((M + 2, K + 16), 0xAA, dtype=torch.uint8, device="cuda")
    s = torch.full((M + 2, 5), -1.0, device="cuda")
    binding.quantize_act_blocks(wide[:, 8:8 + K], out=(x8[:, :K], s[:, :3]))
    want8, want_s = quantize_fp32(wide[:, 8:8 + K])
    assert torch.equal(x8[:M, :K], want8) and torch.equal(s[:M, :3], want_s)
    assert bool((x8[:, K:] == 0xAA).all()) and bool((x8[M:] == 0xAA).all())
    assert bool((s[:, 3:] == -1.0).all()) and bool((s[M:] == -1.0).all())


# ------------------------------------------------------------------------------ one layer
SHAPES = FEW + MANY


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_linear(M, N, K, dtype):
    g = gen(M + 7 * N + 3 * K)
    (x8, s_x), (w8, s_w) = random_rows(g, M, K), random_weights(g, (N, K))
    out = _out(M, N, dtype)
    od = binding.OUT_FP32 if dtype == FP32 else binding.OUT_BF16
    binding.linear_fp8_blocks(x8, s_x, w8, s_w, out_dtype=od, out=out.t)
    _clean()
    y, mag = linear64(x8, s_x, w8, s_w)
    off = (out.t.double() - y).abs() - linear_tolerance(mag, K, dtype, y)
    assert bool((off <= 0).all()), float(off.max())
    out.check()
    again = binding.linear_fp8_blocks(x8, s_x, w8, s_w, out_dtype=od)
    assert _same_bits(again, out.t)


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_whole_numbers_are_exact(M, N, K):
    # codes and scales whose products and sums are whole numbers below 2^24 (scales powers of two): exact in any order
    g = gen(M + N + K)
    x8 = torch.randint(-2, 3, (M, K), generator=g, device="cuda").float().to(E4M3).view(torch.uint8)
    w8 = torch.randint(-3, 4, (N, K), generator=g, device="cuda").float().to(E4M3).view(torch.uint8)
    s_x = 2.0 ** torch.randint(0, 3, (M, blocks(K)), generator=g, device="cuda").float()
    s_w = 2.0 ** torch.randint(0, 3, (blocks(N), blocks(K)), generator=g, device="cuda").float()
    y, mag = linear64(x8, s_x, w8, s_w)
    assert float(mag.max()) < 2 ** 24
    got = binding.linear_fp8_blocks(x8.view(E4M3), s_x, w8.view(E4M3), s_w, out_dtype=binding.OUT_FP32)
    _clean()
    assert torch.equal(got.double(), y)


@pytest.mark.parametrize("M,N", [(37, 400), (300, 400), (2000, 4112)])
def test_strides_of_the_linear_layer(M, N):
    K = 656
    g = gen(8)
    x8, s_x = random_rows(g, M, K)
    w8, s_w = random_weights(g, (N, K))
    xw = torch.full((M, K + 48), 0x7F, dtype=torch.uint8, device="cuda")     # NaN behind the rows
    ww = torch.full((N, K + 16), 0x7F, dtype=torch.uint8, device="cuda")
    sw = torch.full((M, 9), float("nan"), device="cuda")
    xw[:, :K], ww[:, :K], sw[:, :blocks(K)] = x8, w8, s_x
    for dtype, od in ((BF16, binding.OUT_BF16), (FP32, binding.OUT_FP32)):
        out = torch.full((M, N + 3), 7.0, dtype=dtype, device="cuda")
        binding.linear_fp8_blocks(xw[:, :K], sw[:, :blocks(K)], ww[:, :K], s_w, out_dtype=od, out=out[:, :N])
        assert torch.equal(out[:, :N], binding.linear_fp8_blocks(x8, s_x, w8, s_w, out_dtype=od))
        assert bool((out[:, N:] == 7.0).all())


@pytest.mark.parametrize("M,N", [(5, 272), (300, 272), (2000, 4112)])
def test_what_is_not_finite_stays_in_its_row_or_channel(M, N):
    K = 528
    g = gen(M)
    x8, s_x = random_rows(g, M, K)
    w8, s_w = random_weights(g, (N, K))
    clean = binding.linear_fp8_blocks(x8, s_x, w8, s_w)
    x8[1, 5] = 0x7F
    s_x[3, 1] = float("inf")
    w8[130, 500] = 0xFF
    y = binding.linear_fp8_blocks(x8, s_x, w8, s_w)
    assert bool(y[1].isnan().all()) and bool(y[:, 130].isnan().all()) and not bool(y[3].isfinite().any())
    rows = [m for m in range(M) if m not in (1, 3)]
    cols = [n for n in range(N) if n != 130]
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])


# ------------------------------------------------------------------------------ experts
def _experts_ref(x8, s_x, counts, w8, s_w):
    y = torch.zeros((x8.shape[0], w8.shape[1]), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(y)
    at = 0
    for e, n in enumerate(counts):
        if n:
            y[at:at + n], mag[at:at + n] = linear64(x8[at:at + n], s_x[at:at + n], w8[e], s_w[e])
        at += n
    return y, mag


def _offsets(counts, first=0):
    return torch.tensor([first] + counts, device="cuda").cumsum(0).to(torch.int32)


EXPERTS = [(c, N, K) for c in EXPERTS_FEW for N, K in ((16, 16), (272, 400), (1408, 2048), (128, 4096))] + \
          [(c, N, K) for c in EXPERTS_MANY for N, K in EXPERTS_MANY_LAYERS]


@pytest.mark.parametrize("counts,N,K", EXPERTS)
def test_experts(counts, N, K):
    rows, E = sum(counts) + 6, len(counts)
    g = gen(sum(counts) + N + K)
    x8, s_x = random_rows(g, rows, K)
    w8, s_w = random_weights(g, (E, N, K))
    for dtype, od in ((BF16, binding.OUT_BF16), (FP32, binding.OUT_FP32)):
        out = _out(rows, N, dtype)
        binding.linear_fp8_experts(x8, s_x, _offsets(counts), w8, s_w, out_dtype=od, out=out.t)
        _clean()
        used = rows - 6
        y, mag = _experts_ref(x8, s_x, counts, w8, s_w)
        off = (out.t.double() - y).abs()[:used] - linear_tolerance(mag, K, dtype, y)[:used]
        assert bool((off <= 0).all()), float(off.max())
        assert bool((out.t[used:] == 7.0).all())       # rows behind the last expert's
        out.check()


@pytest.mark.parametrize("N,K", [(512, 1664), (384, 2048), (400, 2064), (256, 1040)])
@pytest.mark.parametrize("counts", [[129, 129, 129, 121, 1, 1, 1, 1], [1] * 7 + [505], [64] * 8, [0, 300, 0, 0, 212, 0, 0, 0]])
def test_more_tiles_than_expected_where_k_is_cut(counts, N, K):
    # few channels, so that clusters share K, and experts with more rows than the plan expects: clusters with several tiles
    rows = sum(counts)
    g = gen(N + K + counts[0])
    x8, s_x = random_rows(g, rows, K)
    w8, s_w = random_weights(g, (8, N, K))
    out = _out(rows, N, FP32)
    for _ in range(3):
        binding.linear_fp8_experts(x8, s_x, _offsets(counts), w8, s_w, out_dtype=binding.OUT_FP32, out=out.t)
    _clean()
    y, mag = _experts_ref(x8, s_x, counts, w8, s_w)
    off = (out.t.double() - y).abs() - linear_tolerance(mag, K, FP32, y)
    assert bool((off <= 0).all()), float(off.max())
    out.check()


def test_experts_agree_with_single_layers_and_take_strides():
    counts, N, K = [40, 0, 9, 200], 400, 656
    g = gen(12)
    x8, s_x = random_rows(g, 260, K)
    w8, s_w = random_weights(g, (4, N, K))
    wide = torch.full((4, N + 2, K + 32), 0x7F, dtype=torch.uint8, device="cuda")
    wide[:, :N, :K] = w8
    got = torch.full((260, N), 7.0, device="cuda")
    binding.linear_fp8_experts(x8, s_x, _offsets(counts, first=4), wide[:, :N, :K], s_w, out_dtype=binding.OUT_FP32, out=got)
    assert bool((got[:4] == 7.0).all()) and bool((got[253:] == 7.0).all())
    at = 4
    for e, n in enumerate(counts):
        if n:
            y, mag = linear64(x8[at:at + n], s_x[at:at + n], w8[e], s_w[e])
            assert bool(((got[at:at + n].double() - y).abs() <= linear_tolerance(mag, K, FP32, y)).all())
        at += n


def test_offsets_that_are_not_in_order_reach_nothing_outside():
    # descending, negative and too large offsets: as the documented ones they stand for
    N, K, rows = 144, 256, 50
    g = gen(3)
    x8, s_x = random_rows(g, rows, K)
    w8, s_w = random_weights(g, (6, N, K))
    bad = torch.tensor([-9, 10, 4, 30, -(2 ** 31), 2 ** 31 - 1, 2], dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 10, 10, 30, 30, 50, 50], dtype=torch.int32, device="cuda")
    a, b = _out(rows, N, FP32), _out(rows, N, FP32)
    binding.linear_fp8_experts(x8, s_x, bad, w8, s_w, out_dtype=binding.OUT_FP32, out=a.t)
    binding.linear_fp8_experts(x8, s_x, good, w8, s_w, out_dtype=binding.OUT_FP32, out=b.t)
    _clean()
    assert torch.equal(a.t, b.t)
    a.check(), b.check()
    none = torch.zeros(7, dtype=torch.int32, device="cuda")
    a.t.fill_(7.0)
    binding.linear_fp8_experts(x8, s_x, none, w8, s_w, out_dtype=binding.OUT_FP32, out=a.t)
    _clean()
    assert bool((a.t == 7.0).all())


def test_weights_behind_four_gigabytes():
    # 70 experts of 8192 x 8192, the last of which has rows; then 36 000 outputs of 65 552 channels
    E, N, K = 70, 8192, 8192
    w8 = torch.zeros((E, N, K), dtype=torch.uint8, device="cuda")
    g = gen(2)
    w8[69, 8000:8010] = torch.randint(-3, 4, (10, K), generator=g, device="cuda").float().to(E4M3).view(torch.uint8)
    s_w = torch.ones((E, 64, 64), device="cuda")
    x8 = torch.randint(-2, 3, (3, K), generator=g, device="cuda").float().to(E4M3).view(torch.uint8)
    s_x = torch.ones((3, 64), device="cuda")
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[E] = 3
    y = binding.linear_fp8_experts(x8, s_x, offsets, w8, s_w, out_dtype=binding.OUT_FP32)
    want, _ = linear64(x8, s_x, w8[69], s_w[69])
    assert torch.equal(y.double(), want)
    del w8
    N, M = 65552, 36000
    w8 = torch.zeros((N, 128), dtype=torch.uint8, device="cuda")
    w8[:, 0] = torch.tensor([1.0]).to(E4M3).view(torch.uint8).item()
    x8 = torch.zeros((M, 128), dtype=torch.uint8, device="cuda")
    x8[:, 0] = torch.tensor([2.0]).to(E4M3).view(torch.uint8).item()
    s_x = (torch.arange(M, device="cuda") % 251 + 1).float().view(M, 1)
    y = binding.linear_fp8_blocks(x8, s_x, w8, torch.ones((513, 1), device="cuda"))
    want = (2.0 * s_x).to(BF16)
    for m in (0, 32767, 32768, 35999):
        assert bool((y[m] == want[m]).all())
    assert torch.equal(y[:, 65551:], want)


# ------------------------------------------------------------------------------ streams, graphs, refusals
def test_other_streams_and_captured_calls():
    counts, N, K = [3, 0, 40, 9], 528, 1040
    g = gen(31)
    x = activation(g, 52, K)
    w8, s_w = random_weights(g, (4, N, K))
    off = _offsets(counts)

    def step(x, out):
        x8, s_x = binding.quantize_act_blocks(x, out=out[0])
        binding.linear_fp8_experts(x8, s_x, off, w8, s_w, out=out[1])
        binding.linear_fp8_blocks(x8, s_x, w8[2], s_w[2], out=out[2])
        return out

    def buffers():
        return ((torch.zeros((52, K), dtype=torch.uint8, device="cuda"), torch.zeros((52, blocks(K)), device="cuda")),
                torch.zeros((52, N), dtype=BF16, device="cuda"), torch.zeros((52, N), dtype=BF16, device="cuda"))

    want = step(x, buffers())
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [buffers(), buffers()]
    torch.cuda.synchronize()
    for s, out in zip(side, got):
        with torch.cuda.stream(s):
            for _ in range(5):
                step(x, out)
    torch.cuda.synchronize()
    for out in got:
        assert torch.equal(out[1], want[1]) and torch.equal(out[2], want[2])
    graph, out, xs = torch.cuda.CUDAGraph(), buffers(), torch.zeros_like(x)
    with torch.cuda.graph(graph):
        step(xs, out)
    for _ in range(2):
        xs.copy_(x)
        graph.replay()
        xs.zero_()
    torch.cuda.synchronize()
    assert torch.equal(out[1], want[1]) and torch.equal(out[2], want[2])
    _clean()


def test_tensors_of_the_wrong_kind_are_refused():
    g = gen(1)
    x8, s_x = random_rows(g, 4, 256)
    w8, s_w = random_weights(g, (32, 256))
    bad = [(x8[:, :128], s_x, w8, s_w), (x8, s_x[:, :1], w8, s_w), (x8, s_x, w8, s_w[:, :1]), (x8.cpu(), s_x, w8, s_w),
           (x8, s_x.double(), w8, s_w), (x8.float(), s_x, w8, s_w), (x8, s_x, w8.t().contiguous().t(), s_w)]
    for a in bad:
        with pytest.raises(AssertionError):
            binding.linear_fp8_blocks(*a)
    with pytest.raises(binding.W4A8Error):
        binding.linear_fp8_blocks(x8, s_x, w8[:24], s_w)          # N % 16
    with pytest.raises(AssertionError):
        binding.linear_fp8_blocks(x8, s_x, w8, s_w, out_dtype=binding.OUT_FP32, out=torch.empty((4, 32), dtype=BF16, device="cuda"))
    with pytest.raises(AssertionError):
        binding.linear_fp8_experts(x8, s_x, torch.zeros(3, dtype=torch.int32, device="cuda"), w8[None], s_w[None])
    with pytest.raises(AssertionError):
        binding.linear_fp8_experts(x8, s_x, torch.zeros(2, dtype=torch.int64, device="cuda"), w8[None], s_w[None])
    with pytest.raises(AssertionError):
        binding.quantize_act_blocks(torch.zeros((2, 256), device="cuda"))
    with pytest.raises(binding.W4A8Error):
        binding.quantize_act_blocks(torch.zeros((2, 24), dtype=BF16, device="cuda"))
    with pytest.raises(TypeError):
        binding.linear_fp8_blocks(x8, 3, w8, s_w)
