"""Mixture-of-experts MLP block on FP8 weights with block scales (one per 128 x 128): the form in which such layers are kept in
8 bits beside a model's W4A8 ones.

    route -> quantize x, written to the rows of its experts -> gate/up of every expert -> silu(gate) * up fused with the
    quantization of the down projections' inputs -> down of every expert -> weighted sum of each token's experts

The router's logits are the caller's (a small product in the model's own precision).  `shared` adds an MLP that every token
passes, as one more layer without routing.  The arithmetic runs in the CUDA library through `ops` (the binding, or any object with
the same functions); nothing here computes, and no step looks at a tensor on the host, so a forward pass can be captured into a
CUDA graph.
"""
from dataclasses import dataclass


@dataclass
class BlockWeights:
    """w8: E4M3 [E, N, K] (or [N, K] of a single layer; uint8 or torch.float8_e4m3fn), s_w: float32 with one scale per 128 x 128
    weights, [E, ceil(N / 128), ceil(K / 128)]."""
    w8: object
    s_w: object

    @property
    def N(self):
        return self.w8.shape[-2]

    @property
    def K(self):
        return self.w8.shape[-1]


def _check_mlp(gate_up, down, what):
    if gate_up.N % 2 != 0 or gate_up.N // 2 != down.K or gate_up.K != down.N:
        raise ValueError("%s: gate/up [%d, %d] and down [%d, %d] do not form an MLP" % (what, gate_up.N, gate_up.K, down.N, down.K))


class MoeMlpBlock:
    """Gated MLP experts with routing.  gate_up [E, 2F, H] (gate first) and down [E, H, F]: BlockWeights; the keyword arguments
    behind top_k are those of route_experts.  shared: (gate_up, down) of an MLP for all tokens, or None."""

    def __init__(self, gate_up, down, top_k, shared=None, ops=None, **routing):
        if len(gate_up.w8.shape) != 3 or len(down.w8.shape) != 3 or gate_up.w8.shape[0] != down.w8.shape[0]:
            raise ValueError("experts: [E, N, K] weights of as many experts each")
        _check_mlp(gate_up, down, "experts")
        if shared is not None:
            _check_mlp(*shared, "shared")
            if shared[0].K != gate_up.K:
                raise ValueError("shared MLP of %d columns beside experts of %d" % (shared[0].K, gate_up.K))
        if ops is None:
            from . import binding as ops
            ops.lib()
        self.gate_up, self.down, self.shared = gate_up, down, shared
        self.top_k, self.routing, self.ops = top_k, routing, ops

    @property
    def experts(self):
        return self.gate_up.w8.shape[0]

    def forward(self, x, logits, out=None):
        """x BF16 [M, H] of at least one token, logits BF16 or FP32 [M, E]; returns BF16 [M, H]."""
        if logits.shape[1] != self.experts or x.shape[0] != logits.shape[0]:
            raise ValueError("logits %s for %d tokens and %d experts" % (tuple(logits.shape), x.shape[0], self.experts))
        o = self.ops
        _, weights, offsets, slots = o.route_experts(logits, self.top_k, **self.routing)
        x8, s_x = o.quantize_act_blocks(x, slots=slots)
        gu = o.linear_fp8_experts(x8, s_x, offsets, self.gate_up.w8, self.gate_up.s_w)
        h8, s_h = o.quantize_act_blocks(gu, input_kind=o.CHAIN_INPUT_SILU_MUL)
        y = o.linear_fp8_experts(h8, s_h, offsets, self.down.w8, self.down.s_w)
        return o.combine_experts(y, slots, weights, add=None if self.shared is None else self._shared_mlp(x), out=out)

    def _shared_mlp(self, x):
        o, (gate_up, down) = self.ops, self.shared
        x8, s_x = o.quantize_act_blocks(x)
        gu = o.linear_fp8_blocks(x8, s_x, gate_up.w8, gate_up.s_w)
        h8, s_h = o.quantize_act_blocks(gu, input_kind=o.CHAIN_INPUT_SILU_MUL)
        return o.linear_fp8_blocks(h8, s_h, down.w8, down.s_w)
