"""Host-side checks of the entry points for FP8 layers with block scales and mixture-of-experts blocks: bad arguments are refused
before a device is touched, and the plan of a layer holds for any size (no GPU needed)."""
import ctypes
import math

import pytest

from paper_2505_14638_b200 import binding, build

INVALID, SHAPE, ALIGN, WORKSPACE = (binding.ERR_INVALID_ARG, binding.ERR_BAD_SHAPE, binding.ERR_BAD_ALIGNMENT,
                                    binding.ERR_WORKSPACE_TOO_SMALL)


@pytest.fixture(scope="module")
def L():
    build.build()
    return binding.lib()


def _p(addr=0x1000):
    return ctypes.c_void_p(addr)


def test_quantize_act_blocks_refuses(L):
    def call(x=_p(), M=4, K=256, ldx=256, kind=0, slots=None, k=0, x8=_p(), rows=4, ldx8=256, s=_p(), lds=2):
        return L.w4a8_quantize_act_blocks(x, M, K, ldx, kind, slots, k, x8, rows, ldx8, s, lds, None)
    for kw in (dict(x=None), dict(x8=None), dict(s=None), dict(M=0), dict(K=0), dict(rows=0), dict(kind=2), dict(k=1), dict(slots=_p()), dict(slots=_p(), k=-1)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(K=100, ldx=128), dict(ldx=128), dict(ldx8=128), dict(lds=1), dict(rows=3), dict(kind=1), dict(M=2 ** 31, rows=2 ** 31), dict(K=2 ** 31, ldx=2 ** 32)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(x=_p(0x1008)), dict(x8=_p(0x1004)), dict(ldx=260), dict(ldx8=264), dict(s=_p(0x1002)), dict(slots=_p(0x1001), k=2)):
        assert call(**kw) == ALIGN, kw


def test_linear_fp8_refuses(L):
    def layer(x8=_p(), ldx8=256, s_x=_p(), lds=2, M=4, w8=_p(), ldw=256, s_w=_p(), N=32, K=256, y=_p(), ldy=32, od=0):
        return L.w4a8_linear_fp8_blocks(x8, ldx8, s_x, lds, M, w8, ldw, s_w, N, K, y, ldy, od, None)

    def experts(x8=_p(), ldx8=256, s_x=_p(), lds=2, M=4, off=_p(), E=2, w8=_p(), ldw=256, ws=32 * 256, s_w=_p(), N=32, K=256, y=_p(), ldy=32, od=0):
        return L.w4a8_linear_fp8_experts(x8, ldx8, s_x, lds, M, off, E, w8, ldw, ws, s_w, N, K, y, ldy, od, None)
    for call in (layer, experts):
        for kw in (dict(x8=None), dict(s_x=None), dict(w8=None), dict(s_w=None), dict(y=None), dict(M=0), dict(N=0), dict(K=-16), dict(od=2)):
            assert call(**kw) == INVALID, kw
        for kw in (dict(K=248), dict(N=24), dict(ldx8=240), dict(ldw=128), dict(ldy=16), dict(lds=1), dict(M=2 ** 31), dict(N=2 ** 31, ldy=2 ** 31)):
            assert call(**kw) == SHAPE, kw
        for kw in (dict(x8=_p(0x1008)), dict(w8=_p(0x1008)), dict(y=_p(0x1002)), dict(ldx8=264), dict(s_x=_p(0x1002)), dict(s_w=_p(0x1002))):
            assert call(**kw) == ALIGN, kw
    assert experts(off=None) == INVALID and experts(E=0) == INVALID
    assert experts(E=513) == SHAPE and experts(ws=31 * 256) == SHAPE
    assert layer(ldw=264) == ALIGN and experts(ldw=264, ws=32 * 264) == ALIGN
    assert experts(off=_p(0x1002)) == ALIGN and experts(ws=32 * 256 + 8) == ALIGN


def test_route_and_combine_refuse(L):
    def route(x=_p(), xd=1, M=4, ldl=64, E=64, k=4, score=0, bias=None, groups=1, tg=1, best=1, renorm=1, ids=_p(), w=_p(), off=_p(), slots=_p(), ws=None, wsn=0):
        return L.w4a8_route_experts(x, xd, M, ldl, E, k, score, bias, groups, tg, best, renorm, 1.0, ids, w, off, slots, ws, wsn, None)
    for kw in (dict(x=None), dict(ids=None), dict(w=None), dict(off=None), dict(slots=None), dict(M=0), dict(E=0), dict(k=0), dict(groups=0), dict(tg=0),
               dict(xd=2), dict(score=2), dict(best=0), dict(best=3), dict(renorm=2)):
        assert route(**kw) == INVALID, kw
    for kw in (dict(E=513, ldl=513), dict(k=33), dict(groups=33, tg=33), dict(groups=7), dict(groups=8, tg=9), dict(groups=8, k=9), dict(ldl=63), dict(M=2 ** 30)):
        assert route(**kw) == SHAPE, kw
    for kw in (dict(x=_p(0x1002)), dict(bias=_p(0x1001)), dict(ids=_p(0x1002)), dict(w=_p(0x1002)), dict(off=_p(0x1002)), dict(slots=_p(0x1002)), dict(ws=_p(0x1001))):
        assert route(**kw) == ALIGN, kw
    need = L.w4a8_route_experts_workspace_bytes(4096, 64)
    assert need > 0 and route(M=4096) == WORKSPACE and route(M=4096, ws=_p(), wsn=need - 1) == WORKSPACE

    def combine(y=_p(), yd=0, rows=8, ldy=32, slots=_p(), w=_p(), M=4, k=2, N=32, add=None, ldadd=0, out=_p(), ldo=32, od=0):
        return L.w4a8_combine_experts(y, yd, rows, ldy, slots, w, M, k, N, add, ldadd, out, ldo, od, None)
    for kw in (dict(y=None), dict(slots=None), dict(w=None), dict(out=None), dict(M=0), dict(k=0), dict(N=0), dict(rows=0), dict(yd=2), dict(od=-1)):
        assert combine(**kw) == INVALID, kw
    for kw in (dict(N=24), dict(ldy=16), dict(ldo=16), dict(add=_p(), ldadd=16), dict(M=2 ** 31), dict(rows=2 ** 31)):
        assert combine(**kw) == SHAPE, kw
    for kw in (dict(y=_p(0x1008)), dict(out=_p(0x1008)), dict(add=_p(0x1008), ldadd=32), dict(ldy=36), dict(ldo=36), dict(add=_p(), ldadd=36), dict(slots=_p(0x1002))):
        assert combine(**kw) == ALIGN, kw


def test_workspace_of_the_routing_is_at_most_a_count_per_expert_and_sixteen_tokens(L):
    for M in (1, 16, 17, 64, 148 * 16, 148 * 16 + 1, 8192, 10 ** 6, 2 ** 31 - 1):
        for E in (1, 2, 64, 256, 512):
            need = L.w4a8_route_experts_workspace_bytes(M, E)
            assert 0 <= need <= 4 * E * math.ceil(M / 16) and need <= 148 * 4 * E
            assert need == 0 or M > 16
    assert L.w4a8_route_experts_workspace_bytes(0, 64) == 0 and L.w4a8_route_experts_workspace_bytes(4096, 513) == 0


def test_tensors_that_are_not_on_a_device_are_refused(L):
    import torch
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    x8, s = torch.zeros((4, 256), dtype=torch.uint8), torch.zeros((4, 2))
    i, w = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2))
    with pytest.raises(AssertionError):
        binding.quantize_act_blocks(x)
    with pytest.raises(AssertionError):
        binding.linear_fp8_blocks(x8, s, x8[:2], s[:1])
    with pytest.raises(AssertionError):
        binding.route_experts(torch.zeros((4, 8)), 2)
    with pytest.raises(AssertionError):
        binding.combine_experts(x, i, w)
    with pytest.raises(TypeError):
        binding.combine_experts(3, i, w, out=x)
