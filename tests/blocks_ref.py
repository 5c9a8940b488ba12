"""Plain forms in 64 bits of the FP8 layers with block scales and of the mixture-of-experts steps, for the GPU tests."""
import math

import torch

E4M3 = torch.float8_e4m3fn


def blocks(n):
    return -(-n // 128)


def gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def activation(g, M, K, scale=1.0):
    """N(0, 1) with outlier channels, BF16."""
    x = torch.randn((M, K), generator=g, device="cuda") * scale
    x[:, torch.randperm(K, generator=g, device="cuda")[:max(1, K // 100)]] *= 20.0
    return x.to(torch.bfloat16)


def quantize_fp32(x):
    """The definition of the plain kind, operation by operation in FP32: (codes uint8 [M, K], scales)."""
    M, K = x.shape
    nb = blocks(K)
    v = torch.nn.functional.pad(x.float(), (0, nb * 128 - K)).view(M, nb, 128)
    amax = torch.nan_to_num(v.abs(), nan=0.0, posinf=math.inf).amax(-1, keepdim=True)
    a = amax.clamp_min(2.0 ** -100)
    most = torch.full_like(a, 448.0)      # (torch multiplies with the inverse of a number, and of what a number is divided by)
    s, inv = torch.where(amax == 0, 1.0, a / most), torch.where(amax == 0, 1.0, most / a)
    q = (v * inv).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)
    return q.view(M, nb * 128)[:, :K].contiguous(), s.view(M, nb)


def random_rows(g, M, K):
    """Codes and scales of M activations as the quantizer gives them."""
    return quantize_fp32(activation(g, M, K))


def random_weights(g, shape):
    """E4M3 weights [..., N, K] (uint8) and block scales."""
    w = (torch.randn(shape, generator=g, device="cuda") * 105.0).clamp(-448.0, 448.0).to(E4M3).view(torch.uint8)
    s = 2e-4 * (0.5 + torch.rand(shape[:-2] + (blocks(shape[-2]), blocks(shape[-1])), generator=g, device="cuda"))
    return w, s


def rows64(x8, s_x):
    K = x8.shape[-1]
    return x8.view(E4M3).double() * s_x.double().repeat_interleave(128, -1)[..., :K]


def weights64(w8, s_w):
    N, K = w8.shape[-2:]
    return w8.view(E4M3).double() * s_w.double().repeat_interleave(128, -2)[..., :N, :].repeat_interleave(128, -1)[..., :K]


def linear64(x8, s_x, w8, s_w):
    """(y, sum of the magnitudes of its products)."""
    x, w = rows64(x8, s_x), weights64(w8, s_w)
    return x @ w.T, x.abs() @ w.abs().T


def linear_tolerance(mag, K, out_dtype, y):
    """Largest error of an output.  A block's up to 128 products are exact; their sum in the tensor core takes at most 128 roundings
    or truncations of 2^-23, the scales' product one of 2^-24, the sum over blocks one of 2^-24 each and one per CTA that shares
    K (8 at most) -- each relative to at most the sum of magnitudes.  BF16: half a step more (2^-8 of the value)."""
    t = (128 + 0.5 * (1 + blocks(K) + 8)) * 2.0 ** -23 * mag
    if out_dtype == torch.bfloat16:
        t = t + 2.0 ** -8 * (y.abs() + t)
    return t


def route64(logits, top_k, sigmoid=False, bias=None, groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0):
    """ids, weights (float64), offsets, slots by the definition, one token after the other."""
    M, E = logits.shape
    x = logits.double().cpu()
    x = torch.where(torch.isnan(x), -math.inf, x)
    b = None if bias is None else bias.double().cpu()
    by_logit = b is None and (groups == 1 or group_best == 1)
    ids = torch.full((M, top_k), -1, dtype=torch.int64)
    weights = torch.zeros((M, top_k), dtype=torch.float64)
    size = E // groups
    for m in range(M):
        if sigmoid:
            s = 1.0 / (1.0 + torch.exp(-x[m]))
        else:
            most = x[m].max()
            e = torch.where(x[m] == most, 1.0, torch.exp(x[m] - most))
            e = torch.where(x[m] == -math.inf, 0.0, e)
            s = e / e.sum()
        key = x[m].clone() if by_logit else (s if b is None else s + b)
        key = torch.where((x[m] == -math.inf) | torch.isnan(key), -math.inf, key)
        if groups > 1:
            best = key.view(groups, size).sort(-1, descending=True).values[:, :group_best]
            score = torch.where((best == -math.inf).any(-1), -math.inf, best.sum(-1))
            kept = score.sort(descending=True, stable=True).indices[:top_groups]
            keep = torch.zeros(groups, dtype=torch.bool)
            keep[kept] = True
            key = torch.where(keep.repeat_interleave(size), key, -math.inf)
        order = key.sort(descending=True, stable=True)
        n = int((order.values[:top_k] > -math.inf).sum())
        ids[m, :n] = order.indices[:n]
        w = s[ids[m, :n]]
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else torch.zeros_like(w)
        weights[m, :n] = w * scale
    flat = ids.view(-1)
    counts = torch.tensor([int((flat == e).sum()) for e in range(E)])
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    slots = torch.full((M * top_k,), -1, dtype=torch.int64)
    for e in range(E):
        at = (flat == e).nonzero().view(-1)
        slots[at] = offsets[e] + torch.arange(at.numel())
    return ids, weights, offsets, slots.view(M, top_k)
