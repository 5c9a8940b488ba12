"""GPU: the gated block quantization over every BF16 gate, each alone in a block, so that the block's scale shows silu(gate) * up."""
import pytest
import torch

from blocks_ref import E4M3, blocks
from paper_2505_14638_b200 import binding

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _alone(gates, up):
    """(code, scale) of silu(gate) * up for each of `gates` in a block of its own, at varying places of it."""
    n, per = gates.numel(), 64
    rows = -(-n // per)
    gu = torch.zeros((rows * per, 2, 128), dtype=BF16, device="cuda")
    at, place = torch.arange(n, device="cuda"), (torch.arange(n, device="cuda") * 37) % 128
    gu[at, 0, place], gu[at, 1, place] = gates, up
    gu = gu.view(rows, per, 2, 128).transpose(1, 2).reshape(rows, 2 * per * 128)
    x8, s = binding.quantize_act_blocks(gu.contiguous(), input_kind=binding.CHAIN_INPUT_SILU_MUL)
    torch.cuda.synchronize()
    assert binding.query_device_status() == 0 and blocks(per * 128) == per
    return x8.view(E4M3).float().view(rows * per, 128)[at, place], s.view(-1)[:n]


@pytest.mark.parametrize("up", [1.0, -0.75, 2.0 ** -30])
def test_every_finite_gate(up):
    bits = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16)
    gates = bits.view(BF16)
    gates = gates[gates.isfinite()]
    code, s = _alone(gates, torch.full_like(gates, up))
    g = gates.double()
    h = torch.where(g < -87, 0.0, g / (1.0 + torch.exp(-g))) * up
    a = h.abs()
    # silu(gate) * up within 2^-20, then the scale's division (2^-24); at least 2^-100 is divided, and a block of zeros has scale 1
    least = 2.0 ** -100
    zero = a < 2.0 ** -151                # (2^-150 and more may round up to FP32's least number, 2^-149)
    big = a >= least * (1 + 2.0 ** -19)
    assert int(big.sum()) > 30000
    assert bool(code.isfinite().all()) and bool(s.isfinite().all())
    assert bool(((s.double() * 448.0 - a).abs() <= (2.0 ** -20 + 2.0 ** -23) * a)[big].all())
    assert bool((code == 448.0 * torch.sign(h).float())[big].all())
    assert bool((s == 1.0)[zero].all()) and bool((code == 0.0)[zero].all())


def test_gates_next_to_the_largest():
    # finite, however large: silu(gate) = gate; the neighbours in the block are rounded with that scale
    gates = torch.tensor([2.3e38, 2.37e38, 2.5e38, 3e38, 3.3895313892515355e38], device="cuda").to(BF16)
    for up in (1.0, 2.0 ** -100, -2.0 ** -40):
        code, s = _alone(gates, torch.full_like(gates, up))
        want = gates.double() * abs(up)
        assert bool(((s.double() * 448.0 - want).abs() <= 2.0 ** -20 * want).all())
        assert bool((code == (448.0 if up > 0 else -448.0)).all())


def test_gates_that_are_not_finite():
    gates = torch.tensor([float("inf"), float("nan"), -float("inf")], device="cuda").to(BF16)
    code, _ = _alone(gates, torch.ones_like(gates))
    assert bool(code.isnan().all())
