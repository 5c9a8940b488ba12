"""FP8 layers with a scale per block of 128, and mixture-of-experts blocks made of them, as measurable cases.

The kinds, each one operator of `paper_2505_14638_b200.binding`:

  quantize  BF16 activations to E4M3 with one scale per token and 128 columns; plain or gated (silu(gate) * up), and
            optionally written to the rows that the experts of each token read
  linear    FP8 product with block scales of one layer
  experts   the same for the rows of several experts, sorted by expert
  route     choice of experts from router logits, their weights, and the rows' order by expert
  combine   the weighted sum of the experts' outputs of each token

Activations are N(0, 1) with one channel in a hundred scaled by 20; weights have the codes that N(0, 0.02^2) takes in
blocks of 128 x 128 (maximum of a block: four standard deviations and a little more).
"""
import math
import random

import torch

own = False

MAX_QUANTIZED = 2 * 4096 * 14336           # values read by the largest quantization
MAX_FLOPS = 2.0 * 8192 * 8192 * 28672      # the largest prefill layer
MAX_EXPERT_WEIGHTS = 128 * 4096 * 4096     # weights of the largest set of experts
MAX_EXPERT_FLOPS = 2.0 * 32768 * 4096 * 2048
MAX_ROUTED = 8192 * 128                    # logits
MAX_COMBINED = 4096 * 8 * 4096             # values read by the largest sum


def listed():
    return [
        # decoding sixteen sequences: every token's activations written to the rows of its eight experts
        dict(name="quantize_experts_m16", kind="quantize", M=16, K=4096, gated=False, top_k=8),
        # prefill: the gated activation of an MLP on its way to the down projection
        dict(name="quantize_gated_m4096", kind="quantize", M=4096, K=14336, gated=True, top_k=0),
        # decoding one token: the qkv projection
        dict(name="linear_qkv_m1", kind="linear", M=1, N=6144, K=4096, out="bf16"),
        # a ragged batch of sequences: the up projection, FP32 result
        dict(name="linear_up_m77", kind="linear", M=77, N=14336, K=4096, out="fp32"),
        # the largest prefill layer
        dict(name="linear_large_m8192", kind="linear", M=8192, N=28672, K=8192, out="bf16"),
        # decoding one token: eight experts of 128, each with one row (gate and up of 1408 channels)
        dict(name="experts_8_rows", kind="experts", rows=8, experts=128, active=8, N=2816, K=2048),
        # a decode batch of 64 tokens: most experts have a few rows, some have none
        dict(name="experts_512_rows", kind="experts", rows=512, experts=128, active=120, N=4096, K=4096),
        # prefill of 4096 tokens over 64 experts, unevenly loaded
        dict(name="experts_32768_rows", kind="experts", rows=32768, experts=64, active=64, N=4096, K=2048),
        # decoding 64 sequences: sigmoid scores, a bias for balance, the best groups
        dict(name="route_groups_m64", kind="route", M=64, experts=256, top_k=8, score="sigmoid", bias=True, groups=8,
             top_groups=4, group_best=2, renormalize=True, logits="fp32"),
        # prefill: softmax scores
        dict(name="route_softmax_m8192", kind="route", M=8192, experts=128, top_k=8, score="softmax", bias=False, groups=1,
             top_groups=1, group_best=1, renormalize=True, logits="bf16"),
        # decoding sixteen sequences, with the output of an expert that all tokens share
        dict(name="combine_m16", kind="combine", M=16, N=4096, top_k=8, add=True),
        # prefill
        dict(name="combine_m4096", kind="combine", M=4096, N=4096, top_k=8, add=False),
    ]


def _log_int(rng, lo, hi, mult=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // mult * mult, max(-(-lo // mult) * mult, int(round(v / mult)) * mult))


def draw(rng):
    while True:
        kind = rng.choice(["quantize", "linear", "linear", "experts", "experts", "route", "combine"])
        if kind == "quantize":
            case = dict(kind=kind, M=_log_int(rng, 1, 4096), K=_log_int(rng, 128, 14336, 16), gated=rng.random() < 0.5,
                        top_k=rng.choice([0, 0, 1, 2, 6, 8]))
            if case["M"] * case["K"] * max(1 + case["gated"], case["top_k"]) > MAX_QUANTIZED:
                continue
        elif kind == "linear":
            case = dict(kind=kind, M=_log_int(rng, 1, 8192), N=_log_int(rng, 256, 28672, 16), K=_log_int(rng, 512, 14336, 16),
                        out=rng.choice(["bf16", "bf16", "fp32"]))
            if work(case)["flops"] > MAX_FLOPS:
                continue
        elif kind == "experts":
            experts, rows = _log_int(rng, 2, 256), _log_int(rng, 1, 32768)
            active = max(1, min(experts, rows, int(experts * rng.uniform(0.3, 1.2))))
            case = dict(kind=kind, rows=rows, experts=experts, active=active, N=_log_int(rng, 512, 7168, 16),
                        K=_log_int(rng, 512, 7168, 16))
            if experts * case["N"] * case["K"] > MAX_EXPERT_WEIGHTS or work(case)["flops"] > MAX_EXPERT_FLOPS:
                continue
        elif kind == "route":
            groups = rng.choice([1, 1, 4, 8])
            experts = groups * _log_int(rng, 2, 256 // groups)
            top_groups = rng.randint(1, groups) if groups > 1 else 1
            case = dict(kind=kind, M=_log_int(rng, 1, 16384), experts=experts,
                        top_k=rng.randint(1, min(16, experts // groups * top_groups)), score=rng.choice(["softmax", "sigmoid"]),
                        bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_best=rng.choice([1, 2]),
                        renormalize=rng.random() < 0.7, logits=rng.choice(["fp32", "bf16"]))
            if case["M"] * experts > MAX_ROUTED:
                continue
        else:
            case = dict(kind=kind, M=_log_int(rng, 1, 16384), N=_log_int(rng, 256, 8192, 16), top_k=rng.randint(1, 10),
                        add=rng.random() < 0.5)
            if case["M"] * case["N"] * case["top_k"] > MAX_COMBINED:
                continue
        return case


def _blocks(k):
    return -(-k // 128)


def work(case):
    c = case
    if c["kind"] == "quantize":
        rows = c["M"] * max(1, c["top_k"])
        read = 2 * c["M"] * c["K"] * (2 if c["gated"] else 1) + 4 * c["M"] * c["top_k"]
        return {"bytes": read + rows * (c["K"] + 4 * _blocks(c["K"])), "flops": 2.0 * c["M"] * c["K"]}
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        scales = 4 * _blocks(K) * (M + _blocks(N))
        return {"bytes": M * K + N * K + scales + M * N * (2 if c["out"] == "bf16" else 4), "flops": 2.0 * M * N * K}
    if c["kind"] == "experts":
        R, A, N, K = c["rows"], c["active"], c["N"], c["K"]
        scales = 4 * _blocks(K) * (R + A * _blocks(N))
        return {"bytes": R * K + A * N * K + scales + 4 * (c["experts"] + 1) + 2 * R * N, "flops": 2.0 * R * N * K}
    if c["kind"] == "route":
        M, E, k = c["M"], c["experts"], c["top_k"]
        return {"bytes": M * E * (4 if c["logits"] == "fp32" else 2) + (4 * E if c["bias"] else 0) + 12 * M * k + 4 * (E + 1),
                "flops": 10.0 * M * E}
    M, N, k = c["M"], c["N"], c["top_k"]
    return {"bytes": 2 * M * N * (k + 1 + c["add"]) + 8 * M * k, "flops": 2.0 * M * N * k}


# ---- preparation ---------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activation(g, M, K):
    x = torch.randn((M, K), generator=g, device="cuda")
    cols = torch.randperm(K, generator=g, device="cuda")[:max(1, K // 100)]
    x[:, cols] *= 20.0
    return x.to(torch.bfloat16)


def _quantized_rows(g, M, K):
    """E4M3 activations with their block scales, as the layer before leaves them."""
    nb = _blocks(K)
    x = torch.zeros((M, nb * 128), dtype=torch.float32, device="cuda")
    x[:, :K] = _activation(g, M, K).float()
    x = x.view(M, nb, 128)
    s = x.abs().amax(-1, keepdim=True).clamp_min(1e-20) / 448.0
    x8 = (x / s).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(M, nb * 128)
    return x8.view(torch.uint8)[:, :K].contiguous(), s.view(M, nb).contiguous()


def _weights(g, E, N, K):
    w8 = torch.empty((E, N, K), dtype=torch.uint8, device="cuda")
    for e in range(E):
        w = torch.randn((N, K), generator=g, device="cuda", dtype=torch.bfloat16).mul_(105.0).clamp_(-448.0, 448.0)
        w8[e] = w.to(torch.float8_e4m3fn).view(torch.uint8)
    s_w = (0.02 / 105.0) * (0.9 + 0.2 * torch.rand((E, _blocks(N), _blocks(K)), generator=g, device="cuda"))
    return w8, s_w


def _row_counts(case, seed):
    """Rows of each expert: every active one has at least one, the others fall unevenly."""
    r = random.Random(seed)
    active = r.sample(range(case["experts"]), case["active"])
    counts = [0] * case["experts"]
    for e in active:
        counts[e] = 1
    weights = [math.exp(r.gauss(0.0, 0.5)) for _ in active]
    for e in r.choices(active, weights, k=case["rows"] - case["active"]):
        counts[e] += 1
    return counts


def _row_slots(g, M, k):
    """Where the k copies of each token's row lie among M * k rows."""
    return torch.randperm(M * k, generator=g, device="cuda").to(torch.int32).view(M, k)


def prepare(case, seed):
    g = _gen(seed)
    c, kind = case, case["kind"]
    if kind == "quantize":
        rows = c["M"] * max(1, c["top_k"])
        x = _activation(g, c["M"], c["K"] * (2 if c["gated"] else 1))
        slots = _row_slots(g, c["M"], c["top_k"]) if c["top_k"] else None
        out = (torch.empty((rows, c["K"]), dtype=torch.uint8, device="cuda"),
               torch.empty((rows, _blocks(c["K"])), dtype=torch.float32, device="cuda"))
        return dict(case=c, x=x, slots=slots, out=out)
    if kind == "linear":
        x8, s_x = _quantized_rows(g, c["M"], c["K"])
        w8, s_w = _weights(g, 1, c["N"], c["K"])
        out = torch.empty((c["M"], c["N"]), dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32, device="cuda")
        return dict(case=c, x8=x8, s_x=s_x, w8=w8[0], s_w=s_w[0], out=out)
    if kind == "experts":
        counts = _row_counts(c, seed)
        x8, s_x = _quantized_rows(g, c["rows"], c["K"])
        w8, s_w = _weights(g, c["experts"], c["N"], c["K"])
        offsets = torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)
        out = torch.empty((c["rows"], c["N"]), dtype=torch.bfloat16, device="cuda")
        return dict(case=c, x8=x8, s_x=s_x, w8=w8, s_w=s_w, offsets=offsets, most=max(counts), counts=counts, out=out)
    if kind == "route":
        M, E, k = c["M"], c["experts"], c["top_k"]
        logits = torch.randn((M, E), generator=g, device="cuda") + 0.5 * torch.randn((1, E), generator=g, device="cuda")
        logits = logits.to(torch.float32 if c["logits"] == "fp32" else torch.bfloat16)
        bias = 0.1 * torch.randn((E,), generator=g, device="cuda") if c["bias"] else None
        out = (torch.empty((M, k), dtype=torch.int32, device="cuda"), torch.empty((M, k), dtype=torch.float32, device="cuda"),
               torch.empty((E + 1,), dtype=torch.int32, device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"))
        # room for a count per expert and sixteen tokens
        workspace = torch.empty((4 * E * (M // 16 + 2) + 4096,), dtype=torch.uint8, device="cuda")
        return dict(case=c, logits=logits, bias=bias, out=out, workspace=workspace)
    M, N, k = c["M"], c["N"], c["top_k"]
    y = torch.randn((M * k, N), generator=g, device="cuda").to(torch.bfloat16)
    slots = _row_slots(g, M, k)
    weights = torch.softmax(torch.randn((M, k), generator=g, device="cuda"), -1)
    add = torch.randn((M, N), generator=g, device="cuda").to(torch.bfloat16) if c["add"] else None
    out = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    return dict(case=c, y=y, slots=slots, weights=weights, add=add, out=out)


# ---- one pass ------------------------------------------------------------------------------------
def _plain_quantize(s):
    c = s["case"]
    M, K, nb = c["M"], c["K"], _blocks(c["K"])
    x = s["x"].float()
    if c["gated"]:
        gate, up = x[:, :K], x[:, K:]
        x = gate / (1.0 + torch.exp(-gate)) * up
    x = torch.nn.functional.pad(x, (0, nb * 128 - K)).view(M, nb, 128)
    a = x.abs().amax(-1, keepdim=True)
    a_safe = a.clamp_min(2.0 ** -100)
    scale = torch.where(a == 0, 1.0, a_safe / 448.0).view(M, nb)
    inv = torch.where(a == 0, 1.0, 448.0 / a_safe)
    x8 = (x * inv).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).view(M, nb * 128)[:, :K]
    if not c["top_k"]:
        return x8.contiguous().view(torch.float8_e4m3fn), scale
    k = c["top_k"]
    at = s["slots"].long().view(-1)
    rows8 = torch.empty((M * k, K), dtype=torch.uint8, device="cuda")
    rows_scale = torch.empty((M * k, nb), dtype=torch.float32, device="cuda")
    rows8[at] = x8.unsqueeze(1).expand(M, k, K).reshape(M * k, K)
    rows_scale[at] = scale.unsqueeze(1).expand(M, k, nb).reshape(M * k, nb)
    return rows8.view(torch.float8_e4m3fn), rows_scale


def _plain_rows(x8, s_x):
    K = x8.shape[-1]
    return x8.view(torch.float8_e4m3fn).float() * s_x.repeat_interleave(128, dim=-1)[..., :K]


def _plain_weights(w8, s_w):
    N, K = w8.shape[-2:]
    scale = s_w.repeat_interleave(128, dim=-2)[..., :N, :].repeat_interleave(128, dim=-1)[..., :K]
    return scale.mul_(w8.view(torch.float8_e4m3fn).float())


def _plain_linear(s):
    y = _plain_rows(s["x8"], s["s_x"]) @ _plain_weights(s["w8"], s["s_w"]).t()
    return y.to(s["out"].dtype)


def _plain_experts(s):
    c, off = s["case"], s["offsets"].long()
    row = torch.arange(c["rows"], device="cuda")
    e = torch.searchsorted(off[1:], row, right=True)
    x = torch.zeros((c["experts"], s["most"], c["K"]), device="cuda")
    x[e, row - off[e]] = _plain_rows(s["x8"], s["s_x"])
    y = torch.bmm(x, _plain_weights(s["w8"], s["s_w"]).transpose(1, 2))
    return y[e, row - off[e]].to(torch.bfloat16)


def _plain_route(s):
    c = s["case"]
    M, E, k, G = c["M"], c["experts"], c["top_k"], c["groups"]
    logits = s["logits"].double()        # a choice between two nearly equal experts is lost in 32 bits
    if c["score"] == "softmax":
        p = torch.exp(logits - logits.amax(-1, keepdim=True))
        score = p / p.sum(-1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    key = score if s["bias"] is None else score + s["bias"].double()
    if G > 1:
        best = key.view(M, G, E // G).sort(dim=-1, descending=True).values[..., :c["group_best"]].sum(-1)
        chosen = best.sort(dim=-1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros((M, G), dtype=torch.bool, device="cuda").scatter_(1, chosen, True)
        key = torch.where(keep.repeat_interleave(E // G, dim=1), key, -math.inf)
    ids = key.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, ids)
    if c["renormalize"]:
        w = w / w.sum(-1, keepdim=True)
    order = ids.reshape(-1).sort(dim=-1, stable=True)
    slots = torch.empty((M * k,), dtype=torch.int64, device="cuda")
    slots[order.indices] = torch.arange(M * k, device="cuda")
    offsets = torch.searchsorted(order.values, torch.arange(E + 1, device="cuda"))
    return ids.int(), (w * ROUTE_SCALE).float(), offsets.int(), slots.view(M, k).int()


ROUTE_SCALE = 2.5     # the factor on the weights of the chosen experts


def _plain_combine(s):
    out = (s["weights"].unsqueeze(-1) * s["y"].float()[s["slots"].long()]).sum(1)
    if s["add"] is not None:
        out = out + s["add"].float()
    return out.to(torch.bfloat16)


def _own(s):
    from paper_2505_14638_b200 import binding as b
    c, kind = s["case"], s["case"]["kind"]
    if kind == "quantize":
        x8, s_x = b.quantize_act_blocks(s["x"], input_kind=b.CHAIN_INPUT_SILU_MUL if c["gated"] else b.CHAIN_INPUT_PLAIN,
                                        slots=s["slots"], out=s["out"])
        return x8.view(torch.float8_e4m3fn), s_x
    if kind == "linear":
        return b.linear_fp8_blocks(s["x8"], s["s_x"], s["w8"], s["s_w"],
                                   out_dtype=b.OUT_BF16 if c["out"] == "bf16" else b.OUT_FP32, out=s["out"])
    if kind == "experts":
        return b.linear_fp8_experts(s["x8"], s["s_x"], s["offsets"], s["w8"], s["s_w"], out=s["out"])
    if kind == "route":
        return b.route_experts(s["logits"], c["top_k"],
                               score=b.SCORE_SOFTMAX if c["score"] == "softmax" else b.SCORE_SIGMOID, bias=s["bias"],
                               groups=c["groups"], top_groups=c["top_groups"], group_best=c["group_best"],
                               renormalize=c["renormalize"], scale=ROUTE_SCALE, out=s["out"], workspace=s["workspace"])
    return b.combine_experts(s["y"], s["slots"], s["weights"], add=s["add"], out=s["out"])


_PLAIN = dict(quantize=_plain_quantize, linear=_plain_linear, experts=_plain_experts, route=_plain_route, combine=_plain_combine)


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["kind"]](state)


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _to_e4m3_grid(v):
    """The nearest value of E4M3 (ties to even), saturated at 448."""
    mag = v.abs()
    e = torch.floor(torch.log2(mag.clamp_min(2.0 ** -20))).clamp_min(-6.0)
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=v.device), e - 3.0)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = case, case["kind"]
    if kind == "quantize":
        M, K, nb = c["M"], c["K"], _blocks(c["K"])
        x = s["x"].double()
        if c["gated"]:
            x = x[:, :K] * torch.sigmoid(x[:, :K]) * x[:, K:]
        x8, scale = torch.zeros_like(x), torch.empty((M, nb), dtype=torch.float64, device="cuda")
        for b in range(nb):
            part = x[:, 128 * b:128 * b + 128]
            a = part.abs().max(dim=1).values
            scale[:, b] = a / 448.0
            x8[:, 128 * b:128 * b + 128] = _to_e4m3_grid(part / scale[:, b:b + 1])
        if c["top_k"]:
            token = torch.empty((M * c["top_k"],), dtype=torch.int64, device="cuda")
            token[s["slots"].long().view(-1)] = torch.arange(M * c["top_k"], device="cuda") // c["top_k"]
            x8, scale = x8[token], scale[token]
        return x8, scale
    if kind in ("linear", "experts"):
        K = c["K"]
        x = s["x8"].view(torch.float8_e4m3fn).double()
        s_x, s_w = s["s_x"].double(), s["s_w"].double()
        counts = s.get("counts", [x.shape[0]])
        w8, s_w = (s["w8"], s_w) if kind == "experts" else (s["w8"][None], s_w[None])
        y = torch.zeros((x.shape[0], c["N"]), dtype=torch.float64, device="cuda")
        at = 0
        for e, n in enumerate(counts):
            if n:
                w = w8[e].view(torch.float8_e4m3fn).double()
                xe = x[at:at + n].clone()
                for b in range(_blocks(K)):
                    cols = slice(128 * b, min(K, 128 * b + 128))
                    xe[:, cols] *= s_x[at:at + n, b:b + 1]
                    for nb in range(_blocks(c["N"])):
                        w[128 * nb:128 * nb + 128, cols] *= s_w[e, nb, b]
                y[at:at + n] = torch.matmul(xe, w.t())
            at += n
        return y
    if kind == "route":
        logits = s["logits"].double()
        score = torch.softmax(logits, -1) if c["score"] == "softmax" else torch.sigmoid(logits)
        key = score if s["bias"] is None else score + s["bias"].double()
        M, E, size = c["M"], c["experts"], c["experts"] // c["groups"]
        if c["groups"] > 1:
            groups = key.reshape(M, c["groups"], size)
            value = groups.topk(min(size, c["group_best"]), dim=-1).values.sum(-1)
            least = value.topk(c["top_groups"], dim=-1).values[:, -1:]
            key = key.masked_fill((value < least).repeat_interleave(size, dim=1), -math.inf)
        w = score.gather(1, key.sort(dim=-1, descending=True, stable=True).indices[:, :c["top_k"]])
        w = 2.5 * (w / w.sum(-1, keepdim=True) if c["renormalize"] else w)
        return None, w, None, None
    y, slots, out = s["y"].double(), s["slots"].long(), 0.0
    for j in range(c["top_k"]):
        out = out + s["weights"][:, j:j + 1].double() * y[slots[:, j]]
    return out if s["add"] is None else out + s["add"].double()
