"""The operators around the decoders' attention in 64 bits on the CPU, and how far a kernel's result may lie from them.

  rotate     the sum of d squares has d + 2 roundings of 2^-24, half of that in its root, which has 2^-22 of its own (mean, root, division); two products: en = (d + 2) 2^-25 +
             2^-21 of the element, nothing without a weight.  Cosine and sine are within 2^-21, the angle within 2^-51 of itself, products and sum have 2^-23:
             |y - exact| <= (|a| + |b|) (en + 2^-21 + 2^-51 |angle| + 2^-23) + h |y|, h half a step of the type.
  fp4        whole numbers: no bound.  What is read is the value itself, rounded where bfloat16's denormals end it.
  logprobs   x = f(scale * logit) is off by e = 2^-23 |x|, 2^-20 |x| under a cap; a term exp(x - top) by e + e(top) + 2^-23 |x - top| + 2^-21 of itself, sums of V terms in chunks of
             4096 by (96 + V / 4096) 2^-24.  log S by the mean of these over the terms and 2^-23 of itself; log p by that, e, e(top) and 2^-23 of itself; the entropy's second
             sum by the mean of |x - top| (term) + e + e(top), its quotient by 2^-22 of itself."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------------------------------------------------------------------ rotate
def rotate(x, B, S, heads, freq, gamma, pos, start, sections, interleaved, eps):
    """One of the two: rows [M, B S, heads d] -> result and bound, in 64 bits."""
    M, d = x.shape[0], x.shape[2] // heads
    h = half_step(x.dtype)
    y = x.detach().cpu().double().reshape(M, B, S, heads, d)
    en = 0.0
    if gamma is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * gamma.cpu().double().view(M, 1, 1, 1, d)
        en = (d + 2) * 2.0 ** -25 + 2.0 ** -21
    out, tol = y.clone(), y.abs() * (en + h)
    P = 0 if freq is None else freq.numel()
    if P:
        sections = [P] if sections is None else sections
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
        if pos is None:
            where = ((torch.zeros(M, B, dtype=torch.int64) if start is None else start.cpu().long())[..., None] + torch.arange(S))[..., None].expand(M, B, S, len(sections))
        else:
            where = pos.cpu().long().reshape(M, B, S, -1)
        angle = (where[..., axis].double() * freq.cpu().double())[:, :, :, None]
        i = torch.arange(P)
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
        room = (a.abs() + b.abs()) * (en + 2.0 ** -21 + 2.0 ** -23 + 2.0 ** -51 * angle.abs())
        tol[..., ia], tol[..., ib] = room + h * out[..., ia].abs(), room + h * out[..., ib].abs()
    return out.reshape(M, B * S, -1), tol.reshape(M, B * S, -1) + 1e-37


# --------------------------------------------------------------------------------------------------------------------------------------- fp4
def quantise(x):
    """[..., d] -> codes [..., 16 G], scales [..., G or G + 1], from the definition: the exponent is looked for, and each code is the nearest of the eight."""
    d = x.shape[-1]
    G = (d + 31) // 32
    y = torch.zeros(x.shape[:-1] + (32 * G,), dtype=torch.float64)
    y[..., :d] = x.detach().cpu().double()
    y = y.unflatten(-1, (G, 32))
    top = y.abs().amax(-1)
    odd = ~torch.isfinite(y).all(-1)
    top = torch.where(odd, 0.0, top)
    e = torch.full(top.shape, 125, dtype=torch.int64)
    for k in range(125, -126, -1):
        e = torch.where(top <= 7 * 2.0 ** k, k, e)
    y = torch.where(odd[..., None], 0.0, y) * torch.exp2(-e.double())[..., None]
    off = (y.abs()[..., None] - GRID).abs()
    off[..., 1::2] += 1e-18 * (off[..., 1::2] > 0)                 # halfway: the even code
    low = torch.stack([off[..., c] for c in (0, 2, 4, 6, 1, 3, 5, 7)], -1)
    code = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])[low.argmin(-1)]  # the even codes first: they win what is equally near
    code = (code + 8 * torch.signbit(y)).masked_fill(odd[..., None], 0)
    code = code.flatten(-2).to(torch.uint8)
    scale = torch.where(odd, 255, e + 127).to(torch.uint8)
    if G % 2:
        scale = torch.cat((scale, torch.zeros_like(scale[..., :1])), -1)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def dequantise(codes, scales, d):
    c = torch.stack((codes.cpu() % 16, codes.cpu() // 16), -1).flatten(-2).long()
    s = scales.cpu().long().repeat_interleave(32, -1)[..., :d]
    v = GRID[c[..., :d] % 8] * torch.where(c[..., :d] >= 8, -1.0, 1.0) * torch.exp2((s - 127).double())
    return torch.where(s == 255, math.nan, v)


# ---------------------------------------------------------------------------------------------------------------------------------- logprobs
def logprobs(logits, token, k, vocab, nodes, scale, cap):
    """(logp, bound, entropy, bound, top, top_logp, bound); rows with NaN or +infinity are as the 64-bit sums have them."""
    M, N, V = logits.shape
    B = 1 if nodes is None else nodes.shape[1]
    n = 0 if token is None else token.shape[2]
    f64 = torch.float64
    logp, entropy, top_logp = torch.full((M, N, n), -math.inf, dtype=f64), torch.zeros(M, N, dtype=f64), torch.full((M, N, k), -math.inf, dtype=f64)
    tl, te, tt = torch.zeros(M, N, n, dtype=f64), torch.zeros(M, N, dtype=f64), torch.zeros(M, N, k, dtype=f64)
    top = torch.full((M, N, k), -1, dtype=torch.int32)
    for m in range(M):
        size = V if vocab is None else min(max(int(vocab[m]), 0), V)
        for r in range(N):
            T = N // B
            if size == 0 or (nodes is not None and r % T >= int(nodes[m, r // T])):
                continue
            raw = logits[m, r, :size].cpu().double()
            x = raw * scale
            x = cap * torch.tanh(x / cap) if cap else x
            x = torch.where(raw == -math.inf, -math.inf, x)
            if (raw == -math.inf).all():
                continue
            order = torch.where(torch.isnan(raw), -math.inf, raw)
            order = [int(j) for j in torch.sort(order, descending=True, stable=True).indices[:k] if order[int(j)] > -math.inf]
            top[m, r, :len(order)] = torch.tensor(order, dtype=torch.int32)
            best = x[~torch.isnan(x)].max() if (~torch.isnan(x)).any() else torch.tensor(math.nan)
            diff = x - best
            w = torch.exp(diff)
            S = w.sum()
            p = w / S
            lse = best + torch.log(S)
            unit = 2.0 ** -20 if cap else 2.0 ** -23
            e, e_top = unit * x.abs(), unit * best.abs()
            live = p > 0
            term = e[live] + e_top + 2.0 ** -23 * diff[live].abs() + 2.0 ** -21
            many = (96 + size / 4096) * 2.0 ** -24
            off = (p[live] * term).sum() + many + 2.0 ** -23 * torch.log(S).abs() + 2.0 ** -24
            lp = torch.where(raw == -math.inf, -math.inf, x - lse)
            room = torch.where(lp == -math.inf, 0.0, off + e + e_top + 2.0 ** -22 * lp.abs())
            entropy[m, r] = -(p[live] * lp[live]).sum() if torch.isfinite(S) else math.nan
            te[m, r] = off + (p[live] * (diff[live].abs() * (term + many) + e[live] + e_top)).sum() + 2.0 ** -22 * (torch.log(S).abs() + (p[live] * diff[live].abs()).sum())
            for i in range(n):
                j = int(token[m, r, i])
                if 0 <= j < size:
                    logp[m, r, i], tl[m, r, i] = lp[j], room[j]
            top_logp[m, r, :len(order)], tt[m, r, :len(order)] = lp[order], room[order]
    return logp, tl, entropy, te, top, top_logp, tt


def near(got, want, tol):
    """Equal where `want` is not finite, within the bound elsewhere; the worst ratio is the message."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN elsewhere"
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)]), "another infinity"
    off = (got - want).abs()[~odd]
    assert torch.isfinite(got[~odd]).all(), "not finite"
    if off.numel():
        ratio = (off / tol[~odd].clamp(min=1e-300)).max()
        assert (off <= tol[~odd]).all(), "%.3g of the bound" % float(ratio)
