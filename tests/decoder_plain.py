"""The decoders' operators in 64 bits on the CPU, one sequence and head at a time, and how far a kernel's result may lie from them.

Bounds, for a row of n keys and d features in a type of half step h (2^-8 for bfloat16, 2^-24 for float32):
  - a dot product has d products and sums of 2^-24 each; scaling, tanh, bias and the change to log2 units add at most 2^-20 of the
    magnitudes that enter the score: e = (d + 2) 2^-24 scale sum |q k| + 2^-20 (|f(x)| + slope * distance), the largest over the keys;
  - a weight exp(s - max) is off by e for s, e for the maximum (which cancels between sum and products) and 2^-20 for exp itself;
    weights enter the second product in the storage type: h for bfloat16, nothing for float32;
  - sums of n terms: n 2^-24 each for the sum and the product;
  - the result is rounded once: h.
So |O - exact| <= (2 e + 2^-19 + h' + n 2^-23) sum p |v| + h |O|, and |lse - exact| <= e + 2^-20 + n 2^-24 + 2^-23 |lse|."""
import math

import torch


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def heads_of(x, B, N, heads):
    """[M, B N, heads d] -> [M, B, heads, N, d] in 64 bits."""
    M, _, w = x.shape
    return x.detach().cpu().double().reshape(M, B, N, heads, w // heads).permute(0, 1, 3, 2, 4)


def row_scores(q, k, scale, cap, slope, dist):
    """Scores and the bound e of each, from q[n, d], k[j, d], dist[n, j]."""
    d = q.shape[1]
    x = q @ k.T * scale
    f = cap * torch.tanh(x / cap) if cap else x
    bias = slope * dist
    e = (d + 2) * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().T) + 2.0 ** -20 * (f.abs() + bias.abs())
    return f - bias, e


def attend(q, k, v, seen, scale, cap, slope, dist, dtype):
    """One head: output, its bound, lse, its bound."""
    s, e = row_scores(q, torch.where(seen.any(0)[:, None], k, 0.0), scale, cap, slope, dist)
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    n, h = k.shape[0], half_step(dtype)
    e = torch.where(seen, e, 0.0).amax(1) if n else torch.zeros(q.shape[0], dtype=torch.float64)
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
    # a value counts only where it is seen, whatever the others hold
    clean = torch.isfinite(v).all()
    o = p @ v if clean else torch.stack([p[r][seen[r]] @ v[seen[r]] for r in range(q.shape[0])])
    a = p @ v.abs() if clean else torch.stack([p[r][seen[r]] @ v[seen[r]].abs() for r in range(q.shape[0])])
    rel = 2 * e + 2.0 ** -19 + (h if dtype == torch.bfloat16 else 0.0) + n * 2.0 ** -23
    return o, rel[:, None] * a + h * o.abs() + 1e-37, lse, e + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -23 * lse.abs()


def prompt(Q, K, V, B, S, heads, kv, causal=True, scale=None, cap=0.0, slope=None, length=None, prefix=None, doc=None):
    q, k, v = heads_of(Q, B, S, heads), heads_of(K, B, S, kv), heads_of(V, B, S, kv)
    M, d = q.shape[0], q.shape[-1]
    scale = d ** -0.5 if scale is None else scale
    out, tol = torch.zeros(M, B, S, heads, d, dtype=torch.float64), torch.zeros(M, B, S, heads, d, dtype=torch.float64)
    at = torch.arange(S)
    for m in range(M):
        for b in range(B):
            L = S if length is None else min(max(int(length[m, b]), 0), S)
            first = 0 if prefix is None else int(prefix[m, b])
            seen = (at[:, None] < L) & (at[None] < L)
            if causal:
                seen &= (at[None] <= at[:, None]) | (at[None] < first)
            if doc is not None:
                x = doc[m, b].cpu()
                seen &= (x[:, None] == x[None]) & (x[:, None] >= 0)
            for h in range(heads):
                g = h // (heads // kv)
                w = 0.0 if slope is None else float(slope[m, h])
                dist = (at[:, None] - at[None]).abs().double()
                out[m, b, :, h], tol[m, b, :, h], _, _ = attend(q[m, b, h], k[m, b, g], v[m, b, g], seen, scale, cap, w, dist, Q.dtype)
    return out.reshape(M, B * S, -1), tol.reshape(M, B * S, -1)


def paths(parent, T):
    """Which nodes each node sees, and how many ancestors it has."""
    see, depth = torch.zeros(T, T, dtype=torch.bool), [0] * T
    for t in range(T):
        p = t - 1 if parent is None else int(parent[t])
        if 0 <= p < t:
            see[t], depth[t] = see[p], depth[p] + 1
        see[t, t] = True
    return see, torch.tensor(depth)


def tree(Q, K, V, Kc, Vc, length, start=None, parent=None, nodes=None, pos=None, slope=None, scale=None, cap=0.0):
    M, B, kv, C, d = Kc.shape
    T, heads = Q.shape[1] // B, Q.shape[2] // d
    q, k, v = heads_of(Q, B, T, heads), heads_of(K, B, T, kv), heads_of(V, B, T, kv)
    kc, vc = Kc.detach().cpu().double(), Vc.detach().cpu().double()
    scale = d ** -0.5 if scale is None else scale
    out, tol = torch.zeros(M, B, T, heads, d, dtype=torch.float64), torch.zeros(M, B, T, heads, d, dtype=torch.float64)
    lse, ltol = torch.full((M, B, T, heads), -math.inf, dtype=torch.float64), torch.zeros(M, B, T, heads, dtype=torch.float64)
    for m in range(M):
        for b in range(B):
            L = min(max(int(length[m, b]), 0), C)
            there = T if nodes is None else min(max(int(nodes[m, b]), 0), T)
            see, depth = paths(None if parent is None else parent[m, b], T)
            mine = (L if start is None else int(start[m, b])) + depth
            seen = torch.cat((torch.ones(T, L, dtype=torch.bool), see), 1)
            seen &= (torch.arange(T) < there)[:, None]
            for h in range(heads):
                g = h // (heads // kv)
                w = 0.0 if slope is None else float(slope[m, h])
                at = torch.arange(L) if pos is None else pos[m, b, g, :L].cpu()
                dist = (mine[:, None] - torch.cat((at, mine))[None]).abs().double()
                r = attend(q[m, b, h], torch.cat((kc[m, b, g, :L], k[m, b, g])), torch.cat((vc[m, b, g, :L], v[m, b, g])), seen, scale, cap, w, dist, Q.dtype)
                out[m, b, :, h], tol[m, b, :, h], lse[m, b, :, h], ltol[m, b, :, h] = r
    return out.reshape(M, B * T, -1), tol.reshape(M, B * T, -1), lse.reshape(M, B * T, heads), ltol.reshape(M, B * T, heads)


def weigh(Q, lse, Kc, weight, length, start=None, index=None, count=None, pos=None, slope=None, scale=None, cap=0.0):
    M, B, kv, C, d = Kc.shape
    T, heads = Q.shape[1] // B, Q.shape[2] // d
    q, kc, ls = heads_of(Q, B, T, heads), Kc.detach().cpu().double(), lse.detach().cpu().double().reshape(M, B, T, heads)
    n = T if index is None else index.shape[2]
    scale = d ** -0.5 if scale is None else scale
    out = weight.detach().cpu().double().clone()
    tol = torch.zeros_like(out)
    for m in range(M):
        for b in range(B):
            L = min(max(int(length[m, b]), 0), C)
            cnt = n if count is None else min(max(int(count[m, b]), 0), n)
            for i in range(cnt):
                row = i if index is None else int(index[m, b, i])
                if not 0 <= row < T:
                    continue
                end = min(L + i + 1, C)
                for h in range(heads):
                    g, z = h // (heads // kv), ls[m, b, row, h]
                    if z == -math.inf:
                        continue
                    at = torch.arange(end) if pos is None else pos[m, b, g, :end].cpu()
                    dist = ((L if start is None else int(start[m, b])) + i - at).abs().double()[None]
                    s, e = row_scores(q[m, b, h, row][None], kc[m, b, g, :end], scale, cap, 0.0 if slope is None else float(slope[m, h]), dist)
                    p = torch.exp(s[0] - z)
                    out[m, b, g, :end] += p
                    tol[m, b, g, :end] += p * (e[0] + 2.0 ** -20 + 2.0 ** -22 * abs(z))
    return out, tol + (n * heads // kv + 1) * 2.0 ** -24 * out.abs()


def append(K, V, Kc, Vc, pos, weight, length, start=None, index=None, count=None):
    """New copies of the caches."""
    M, B, kv, C, d = Kc.shape
    T = K.shape[1] // B
    Kc, Vc, pos, weight = (None if x is None else x.clone().cpu() for x in (Kc, Vc, pos, weight))
    n = T if index is None else index.shape[2]
    for m in range(M):
        for b in range(B):
            L = min(max(int(length[m, b]), 0), C)
            for i in range(n if count is None else min(max(int(count[m, b]), 0), n)):
                row = i if index is None else int(index[m, b, i])
                if L + i >= C or not 0 <= row < T:
                    continue
                Kc[m, b, :, L + i] = K[m, b * T + row].cpu().view(kv, d)
                Vc[m, b, :, L + i] = V[m, b * T + row].cpu().view(kv, d)
                if pos is not None:
                    pos[m, b, :, L + i] = (L if start is None else int(start[m, b])) + i
                if weight is not None:
                    weight[m, b, :, L + i] = 0.0
    return Kc, Vc, pos, weight


def evict(Kc, Vc, pos, weight, length, budget, start=None, recent=0):
    """New copies of the caches; slots that no entry moved into are as they were."""
    M, B, kv, C, d = Kc.shape
    Kc, Vc, weight = Kc.clone().cpu(), Vc.clone().cpu(), weight.clone().cpu()
    pos = None if pos is None else pos.clone().cpu()
    for m in range(M):
        for b in range(B):
            L = min(max(int(length[m, b]), 0), C)
            bound = (L if start is None else int(start[m, b])) - recent
            for g in range(kv):
                w = [math.inf if x != x else x for x in weight[m, b, g, :L].tolist()]
                odd = [x != x for x in weight[m, b, g, :L].tolist()]
                guard = [recent > 0 and int(pos[m, b, g, j]) >= bound for j in range(L)]
                order = sorted(range(L), key=lambda j: (guard[j], odd[j], w[j], j))
                gone = set(order[:max(0, L - budget)])
                to, come = [j for j in range(min(L, budget)) if j in gone], [j for j in range(budget, L) if j not in gone]
                assert len(to) == len(come)
                for x in (Kc, Vc) + (() if pos is None else (pos,)) + (weight,):
                    x[m, b, g, to] = x[m, b, g, come]
    return Kc, Vc, pos, weight
