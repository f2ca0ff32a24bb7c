"""The merged decoder operators, as they are measured: attention of prompts with capped, biased and masked scores, attention of a tree
of drafted tokens over a cache, and the cache that this attention reads -- rows appended, keys weighed, entries evicted.

All of them act on M models of B sequences each; a model's queries meet its own keys only.  With rows of `heads` query heads over
`kv_heads` key heads (query head h reads key head h / (heads / kv_heads)) the score of query i and key j is

    s_ij = f(scale q_i . k_j) - slope_h |pos_i - pos_j|,    f(x) = cap tanh(x / cap), or x where cap is 0,

a row's weights are the softmax over the keys that it sees, and a row that sees none gives 0."""
import math

import numpy as np
import torch

own = False

BF, F32 = "bfloat16", "float32"


# ---------------------------------------------------------------------------------------------------------------------------- cases
def listed():
    """Two cases or more of each operator; sizes of 64 features and 12 heads are those of the encoder workloads."""
    return [
        # a short prompt for each of 8 merged models, in float32: what latency allows
        dict(name="prompt_short_f32", op="prompt", M=8, B=1, S=128, heads=12, kv=12, d=64, dtype=F32, causal=True, cap=0.0, slopes=True, docs=0, prefix=True, ragged=False),
        # 32 models, several documents packed into each sequence of 512, capped scores, sequences of different lengths
        dict(name="prompt_documents", op="prompt", M=32, B=1, S=512, heads=12, kv=12, d=64, dtype=BF, causal=True, cap=30.0, slopes=False, docs=3, prefix=False, ragged=True),
        # a long prompt of odd length, four query heads to a key head, a bias by distance
        dict(name="prompt_long", op="prompt", M=2, B=1, S=8191, heads=32, kv=8, d=128, dtype=BF, causal=True, cap=0.0, slopes=True, docs=0, prefix=False, ragged=False),
        # one token for each of 8 models over a short cache, in float32: what latency allows
        dict(name="tree_token_f32", op="tree", M=8, B=1, T=1, C=1024, heads=12, kv=12, d=64, dtype=F32, cap=0.0, slopes=True, ragged=True, start=0, lse=True),
        # trees of 26 drafted tokens, capped scores, caches that have been evicted from
        dict(name="tree_draft", op="tree", M=4, B=8, T=26, C=4096, heads=32, kv=8, d=128, dtype=BF, cap=50.0, slopes=False, ragged=True, start=9000, lse=True),
        # one token over long caches of two sequences: the keys have to be shared out
        dict(name="tree_long", op="tree", M=1, B=2, T=1, C=100003, heads=32, kv=8, d=128, dtype=BF, cap=0.0, slopes=True, ragged=True, start=0, lse=False),
        # the accepted path of a draft goes into the cache
        dict(name="append_path", op="append", M=8, B=4, T=26, n=6, C=2048, kv=8, d=64, dtype=F32, ragged=True, start=5000),
        # whole prompts go into the cache
        dict(name="append_prompt", op="append", M=8, B=4, T=2039, n=0, C=4096, kv=8, d=128, dtype=BF, ragged=True, start=0),
        # the accepted tokens' attention is added to the weights of the keys: a path in float32, and single tokens of a batch
        dict(name="weigh_path_f32", op="weigh", M=8, B=1, T=26, n=6, C=1000, heads=12, kv=12, d=64, dtype=F32, cap=0.0, slopes=True, ragged=True, start=0),
        dict(name="weigh_token", op="weigh", M=4, B=8, T=1, n=1, C=8192, heads=32, kv=8, d=128, dtype=BF, cap=50.0, slopes=False, ragged=True, start=20000),
        # caches cut back by an eighth, and long prompts cut to a small budget
        dict(name="evict_some", op="evict", M=8, B=2, C=1024, budget=896, recent=64, kv=12, d=64, dtype=F32, ragged=False, start=3000),
        dict(name="evict_prompt", op="evict", M=4, B=4, C=32768, budget=4096, recent=256, kv=8, d=128, dtype=BF, ragged=True, start=0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """A case between the listed ones: its operator, then sizes over the logarithm of their range, made smaller until it costs no more than the largest listed one."""
    op = rng.choice(("prompt", "tree", "append", "weigh", "evict"))
    kv, group = rng.choice((1, 2, 3, 4, 8, 12)), rng.choice((1, 1, 2, 4, 8))
    c = dict(op=op, M=rng.choice((1, 2, 3, 4, 8, 16, 32)), B=rng.choice((1, 1, 2, 3, 4, 8)), kv=kv, d=rng.choice((32, 64, 64, 80, 128, 128)), dtype=rng.choice((F32, BF, BF)), ragged=rng.random() < 0.6)
    if op in ("prompt", "tree", "weigh"):
        c.update(heads=kv * group, cap=rng.choice((0.0, 0.0, 15.0, 30.0, 50.0)), slopes=rng.random() < 0.5)
    if op == "prompt":
        c.update(S=_log(rng, 16, 8191), causal=rng.random() < 0.8, docs=rng.choice((0, 0, 2, 5)), prefix=False)
        c["prefix"] = c["causal"] and not c["docs"] and rng.random() < 0.3
    else:
        c.update(C=_log(rng, 64, 100003), start=rng.choice((0, 0, 7000)))
    if op in ("tree", "weigh"):
        c["T"] = _log(rng, 1, 64)
    if op == "tree":
        c["lse"] = rng.random() < 0.5
    if op == "weigh":
        c["n"] = rng.randint(1, min(c["T"], 12))
    if op == "append":
        c["T"] = _log(rng, 1, c["C"])
        c["n"] = rng.choice((0, rng.randint(1, c["T"])))
    if op == "evict":
        c["budget"] = max(1, int(c["C"] * rng.uniform(0.1, 0.95)))
        c["recent"] = rng.choice((0, 1, 64, 256))
    top = max((work(x) for x in listed() if x["op"] == op), key=lambda w: w["bytes"] + w["flops"] / 50)
    while work(c)["bytes"] > top["bytes"] or work(c)["flops"] > top["flops"] or _elements(c) > 1 << 29:
        big = max((k for k in ("M", "B", "kv") if c[k] > 1), key=lambda k: c[k], default=None)
        if big is None or (big == "kv" and c["kv"] < 2):
            for k in ("S", "C", "T", "budget", "n"):
                if c.get(k, 0) > 1:
                    c[k] = max(1, c[k] // 2)
        elif big == "kv":
            c["kv"] //= 2
            c.update({"heads": c["kv"] * group} if "heads" in c else {})
        else:
            c[big] = c[big] // 2
    return c


def _elements(c):
    """Of the largest tensor of the case: cache, rows or, for the plain form of a prompt and of a tree, a quarter of the scores."""
    rows = c["M"] * c["B"]
    if c["op"] == "prompt":
        return rows * max(c["heads"] * c["S"] * c["S"] // 8, c["S"] * (c["heads"] + 2 * c["kv"]) * c["d"])
    return rows * max(c["kv"] * c["C"] * c["d"] * (4 if c["op"] == "evict" else 1), c.get("T", 1) * c.get("heads", 0) * c["C"] // 4)


# -------------------------------------------------------------------------------------------------- lengths, from the case alone
def _lengths(c, full, least=1):
    """Valid tokens of each of the M B sequences: all of them, or between a half and all."""
    k = torch.arange(c["M"] * c["B"])
    off = (k * 37 + 11) % 64 * (full // 2) // 64 if c["ragged"] else k * 0
    return (full - off).clamp(min=least).view(c["M"], c["B"]).to(torch.int32)


def _documents(c):
    """Document of every token: `docs` of them per sequence, of unequal lengths that differ from sequence to sequence."""
    S, k = c["S"], torch.arange(c["M"] * c["B"])[:, None]
    at = torch.arange(S)[None] + (k * 29) % (S // (2 * c["docs"]) + 1)
    return (at * c["docs"] // S).view(c["M"], c["B"], S).to(torch.int32)


def _prefixes(c):
    return (_lengths(c, c["S"]) // 3).to(torch.int32)


def _cached(c):
    """Entries of each cache before the step: room is left for what is appended."""
    room = c["n"] or c["T"] if c["op"] in ("append", "weigh") else 0
    return _lengths(c, max(c["C"] - room, 0), 0)


def _counts(c):
    return (_lengths(c, c["n"] or c["T"])).to(torch.int32)


def _nodes(c):
    return _lengths(c, c["T"])


def work(case):
    """Bytes: inputs and outputs that belong to a valid token, once.  Operations: two products over the pairs that see each other (one for weigh)."""
    c, e = case, 4 if case["dtype"] == F32 else 2
    rows, d, kv = c["M"] * c["B"], c["d"], c["kv"]
    if c["op"] == "prompt":
        n = _lengths(c, c["S"]).double().view(-1)
        if c["docs"]:
            doc, i = _documents(c).view(rows, -1).long(), torch.arange(c["S"])[None]
            doc = torch.where(i < n[:, None], doc, c["docs"] + 1)
            size = torch.zeros(rows, c["docs"] + 2, dtype=torch.float64).scatter_add_(1, doc, torch.ones(doc.shape, dtype=torch.float64))[:, :c["docs"] + 1]
            pairs = (size * (size + 1) / 2 if c["causal"] else size * size).sum()
        elif c["causal"]:
            p = _prefixes(c).double().view(-1) if c["prefix"] else n * 0
            pairs = (n * (n + 1) / 2 + p * (p - 1) / 2 * (p > 0)).sum()
        else:
            pairs = (n * n).sum()
        small = (rows * c["S"] * 4 if c["docs"] else 0) + (c["M"] * c["heads"] * 4 if c["slopes"] else 0) + 8 * rows
        return {"bytes": float(n.sum()) * (c["heads"] + 2 * kv) * d * e + rows * c["S"] * c["heads"] * d * e + small, "flops": 4.0 * float(pairs) * c["heads"] * d}
    L = _cached(c).double().view(-1)
    if c["op"] == "tree":
        t = _nodes(c).double().view(-1)
        cache = float(L.sum()) * kv * (2 * d * e + (4 if c["slopes"] and c["start"] else 0))
        own_rows = float(t.sum()) * (c["heads"] + 2 * kv) * d * e + rows * c["T"] * c["heads"] * (d * e + (4 if c["lse"] else 0))
        return {"bytes": cache + own_rows + 4.0 * rows * (c["T"] + 3), "flops": 4.0 * float((t * (L + (t + 1) / 2)).sum()) * c["heads"] * d}
    if c["op"] == "append":
        return {"bytes": float(_counts(c).sum()) * kv * (4 * d * e + 8) + 12.0 * rows, "flops": 0.0}
    if c["op"] == "weigh":
        t = _counts(c).double().view(-1)
        return {"bytes": float((L + t).sum()) * kv * (d * e + 8 + (4 if c["slopes"] and c["start"] else 0)) + float(t.sum()) * c["heads"] * (d * e + 4),
                "flops": 2.0 * float((t * (L + (t + 1) / 2)).sum()) * c["heads"] * d}
    # evict: position and weight of every entry are read, those that stay are written; half of what leaves lies below the budget at most,
    # and each of these places is filled with one row of keys and one of values
    gone = (L - c["budget"]).clamp(min=0)
    filled = gone * torch.minimum(L, torch.tensor(float(c["budget"]))) / L.clamp(min=1)
    return {"bytes": float((L * 8 + torch.minimum(L, torch.tensor(float(c["budget"]))) * 8 + filled * 4 * d * e).sum()) * kv, "flops": 0.0}


# --------------------------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if c["dtype"] == F32 else torch.bfloat16
    M, B, kv, d = c["M"], c["B"], c["kv"], c["d"]
    s = dict(c, seed=seed, scale=d ** -0.5)
    randn = lambda *n: torch.randn(n, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    dev = lambda t: t.to("cuda").contiguous()  # noqa: E731
    s["slope"] = None
    if c.get("slopes"):  # the usual powers of two between 2^-1 and 2^-8 over the heads, another factor for each model
        s["slope"] = (2.0 ** -(1 + 7 * torch.arange(c["heads"], device="cuda") / max(1, c["heads"] - 1)) * (1 + 0.1 * torch.rand((M, 1), generator=g, device="cuda"))).float().contiguous()
    if c["op"] in ("prompt", "tree", "weigh"):  # one projection gives the three, side by side; queries of about half as much again as unit size
        N, H = B * c.get("S", c.get("T", 0)), c["heads"]
        qkv = randn(M, N, (H + 2 * kv) * d)
        qkv[:, :, :H * d] *= 1.5
        qkv = qkv.to(dt)
        s.update(qkv=qkv, Q=qkv[:, :, :H * d], K=qkv[:, :, H * d:(H + kv) * d], V=qkv[:, :, (H + kv) * d:], out=torch.empty((M, N, H * d), dtype=dt, device="cuda"))
    if c["op"] == "prompt":
        s["length"] = dev(_lengths(c, c["S"])) if c["ragged"] else None
        s["doc"] = dev(_documents(c)) if c["docs"] else None
        s["prefix_len"] = dev(_prefixes(c)) if c["prefix"] else None
        return s
    L = _cached(c)
    s["length"] = dev(L)
    s["begin"] = dev(L + c["start"]) if c["start"] else None
    s["Kc"] = randn(M, B, kv, c["C"], d).to(dt)
    s["pos"] = None
    if c["op"] == "weigh":
        s["weight"] = randn(M, B, kv, c["C"]).square()
    else:
        s["Vc"] = randn(M, B, kv, c["C"], d).to(dt)
    if c["start"] or c["op"] in ("append", "evict"):  # evicted caches are in no order: any positions below the next one's
        order = torch.rand((M, B, kv, c["C"]), generator=g, device="cuda").argsort(-1)
        s["pos"] = (order * (1 + c["start"] // c["C"])).to(torch.int32)
    if c["op"] in ("tree", "weigh"):
        T = c["T"]
        host = torch.Generator().manual_seed(seed)
        parent = (torch.rand((M, B, T), generator=host) * torch.arange(T)).floor().to(torch.int32)  # one root, children of earlier nodes
        parent[:, :, 0] = -1
        s["parent"] = dev(parent)
    if c["op"] == "tree":
        s["nodes"] = dev(_nodes(c)) if c["ragged"] and T > 1 else None
        s["lse_out"] = torch.empty((M, B * T, c["heads"]), dtype=torch.float32, device="cuda") if c["lse"] else None
    if c["op"] in ("append", "weigh"):
        n = c["n"] or c["T"]
        pick = torch.rand((M, B, c["T"]), generator=g, device="cuda").argsort(-1)[:, :, :n].sort(-1).values
        s["index"] = pick.to(torch.int32).contiguous() if c["n"] else None
        s["count"] = dev(_counts(c))
    if c["op"] == "append":
        kvs = randn(M, B * c["T"], 2 * kv * d).to(dt)
        s.update(K=kvs[:, :, :kv * d], V=kvs[:, :, kv * d:], weight=randn(M, B, kv, c["C"]).square())
    if c["op"] == "weigh":  # the sums that the attention of these tokens gave, from the scores themselves
        s["out"] = torch.empty_like(s["weight"])
        s["lse"] = torch.zeros((M, B * T, c["heads"]), device="cuda")
        sc, seen = _weigh_scores(s)
        lse = torch.logsumexp(sc.masked_fill(~seen, -math.inf), -1).nan_to_num(neginf=0.0)  # [M, B, kv, n, group]
        lse = lse.permute(0, 1, 3, 2, 4).reshape(M, B, n, -1)
        s["lse"].view(M, B, T, -1).scatter_(2, s["index"].long()[..., None].expand(lse.shape), lse)
    if c["op"] == "evict":
        w = randn(M, B, kv, c["C"]).square()
        s["weight"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.02, torch.zeros_like(w), w)  # some were never looked at
        s["pos_out"], s["weight_out"] = torch.zeros_like(s["pos"]), torch.zeros_like(s["weight"])
    return s


# ------------------------------------------------------------------------------------------------------------------------------ run
def run(state):
    s = state
    if own:
        import paper_2009_13062_amd as nf
        M, B = s["M"], s["B"]
        if s["op"] == "prompt":
            return nf.attention_prompt(s["Q"], s["K"], s["V"], B, s["S"], s["heads"], s["kv"], causal=s["causal"], scale=s["scale"], cap=s["cap"], slope=s["slope"], length=s["length"],
                                       prefix=s["prefix_len"], doc=s["doc"], out=s["out"])
        if s["op"] == "tree":
            O = nf.attention_tree(s["Q"], s["K"], s["V"], s["Kc"], s["Vc"], s["length"], start=s["begin"], parent=s["parent"], nodes=s["nodes"], pos=s["pos"], slope=s["slope"],
                                  scale=s["scale"], cap=s["cap"], out=s["out"], lse=s["lse_out"])
            return {"O": O, "lse": s["lse_out"]}
        if s["op"] == "append":
            nf.cache_append(s["K"], s["V"], s["Kc"], s["Vc"], s["pos"], s["weight"], s["length"], start=s["begin"], index=s["index"], count=s["count"])
            return {"Kc": s["Kc"], "Vc": s["Vc"], "pos": s["pos"], "weight": s["weight"]}
        if s["op"] == "weigh":
            return nf.cache_weigh(s["Q"], s["lse"], s["Kc"], s["weight"], s["length"], start=s["begin"], index=s["index"], count=s["count"], pos=s["pos"], slope=s["slope"],
                                  scale=s["scale"], cap=s["cap"], out=s["out"])
        nf.cache_evict(s["Kc"], s["Vc"], s["pos"], s["weight"], s["length"], s["budget"], start=s["begin"], recent=s["recent"], pos_out=s["pos_out"], weight_out=s["weight_out"])
        return {"Kc": s["Kc"], "Vc": s["Vc"], "pos": s["pos_out"], "weight": s["weight_out"]}
    return {"prompt": _plain_prompt, "tree": _plain_tree, "append": _plain_append, "weigh": _plain_weigh, "evict": _plain_evict}[s["op"]](s)


def _capped(x, cap):
    return x.div_(cap).tanh_().mul_(cap) if cap else x


def _softmax_product(s, seen, v):
    """Rows of weights over the keys that they see, times the values, and the logarithm of the sum."""
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.masked_fill(total == 0, 1.0)
    return out, (top + total.log()).squeeze(-1)


def _by_head(x, M, B, S, kv, d):
    """[M, B S, heads d] -> [M, B, kv, group, S, d] in 32 bits."""
    return x.float().view(M, B, S, kv, -1, d).permute(0, 1, 3, 4, 2, 5)


def _plain_prompt(s):
    M, B, S, kv, d = s["M"], s["B"], s["S"], s["kv"], s["d"]
    G = s["heads"] // kv
    q = _by_head(s["Q"], M, B, S, kv, d).reshape(M, B, kv, G * S, d)
    k = _by_head(s["K"], M, B, S, kv, d).reshape(M, B, kv, S, d)
    v = _by_head(s["V"], M, B, S, kv, d).reshape(M, B, kv, S, d)
    sc = _capped(torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]), s["cap"]).view(M, B, kv, G, S, S)
    at = torch.arange(S, device="cuda")
    if s["slope"] is not None:
        sc.addcmul_(s["slope"].view(M, 1, kv, G, 1, 1), (at[:, None] - at[None]).abs().float(), value=-1.0)
    seen = torch.ones((M, B, S, S), dtype=torch.bool, device="cuda")
    if s["causal"]:
        low = at[None] <= at[:, None]
        seen &= low if s["prefix_len"] is None else low | (at < s["prefix_len"][..., None])[:, :, None]
    if s["doc"] is not None:
        seen &= s["doc"][:, :, :, None] == s["doc"][:, :, None]
        seen &= (s["doc"] >= 0)[:, :, None]
    if s["length"] is not None:
        valid = at < s["length"][..., None]
        seen &= valid[:, :, None] & valid[..., None]
    o, _ = _softmax_product(sc, seen[:, :, None, None], v[:, :, :, None])
    return o.permute(0, 1, 4, 2, 3, 5).reshape(M, B * S, s["heads"] * d).to(s["Q"].dtype)


def _ancestors(parent):
    """[M, B, T] parents -> which node sees which [M, B, T, T] (itself and its ancestors), and depths, by squaring the relation."""
    T = parent.shape[-1]
    at = torch.arange(T, device=parent.device)
    see = (parent[..., None] == at).float() + torch.eye(T, device=parent.device)
    for _ in range(T.bit_length()):  # a path of 2^k steps after k of them
        see = (torch.matmul(see, see) > 0).float()
    return see > 0, see.sum(-1).to(torch.int32) - 1


def _plain_tree(s):
    M, B, T, C, kv, d = s["M"], s["B"], s["T"], s["C"], s["kv"], s["d"]
    G = s["heads"] // kv
    q = _by_head(s["Q"], M, B, T, kv, d).reshape(M, B, kv, G * T, d)
    k = torch.cat((s["Kc"].float(), _by_head(s["K"], M, B, T, kv, d).reshape(M, B, kv, T, d)), 3)
    v = torch.cat((s["Vc"].float(), _by_head(s["V"], M, B, T, kv, d).reshape(M, B, kv, T, d)), 3)
    sc = _capped(torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]), s["cap"]).view(M, B, kv, G, T, C + T)
    see, depth = _ancestors(s["parent"])
    slot, node = torch.arange(C, device="cuda"), torch.arange(T, device="cuda")
    valid = node < (s["nodes"] if s["nodes"] is not None else torch.full_like(s["length"], T))[..., None]
    seen = torch.cat(((slot < s["length"][..., None])[:, :, None].expand(M, B, T, C), see & valid[:, :, None]), 3) & valid[..., None]
    if s["slope"] is not None:
        mine = (s["begin"] if s["begin"] is not None else s["length"])[..., None] + depth  # [M, B, T]
        cached = s["pos"] if s["pos"] is not None else slot.to(torch.int32).expand(M, B, kv, C)
        theirs = torch.cat((cached, mine[:, :, None].expand(M, B, kv, T)), 3)
        sc.addcmul_(s["slope"].view(M, 1, kv, G, 1, 1), (mine[:, :, None, None, :, None] - theirs[:, :, :, None, None]).abs().float(), value=-1.0)
    o, lse = _softmax_product(sc, seen[:, :, None, None], v[:, :, :, None])
    o = o.permute(0, 1, 4, 2, 3, 5).reshape(M, B * T, s["heads"] * d).to(s["Q"].dtype)
    return {"O": o, "lse": lse.permute(0, 1, 4, 2, 3).reshape(M, B * T, s["heads"]) if s["lse"] else None}


def _plain_append(s):
    M, B, T, C, kv, d = s["M"], s["B"], s["T"], s["C"], s["kv"], s["d"]
    n = s["n"] or T
    i = torch.arange(n, device="cuda")
    pick = s["index"].long() if s["index"] is not None else i.expand(M, B, n)
    # every slot of the cache asks which of the new rows it holds: none for those before the length and behind the count
    which = torch.arange(C, device="cuda") - s["length"][..., None]                                      # [M, B, C]
    new = ((which >= 0) & (which < s["count"][..., None]))[:, :, None]                                   # [M, B, 1, C]
    row = torch.gather(pick, 2, which.clamp(0, n - 1))[:, :, None, :, None].expand(M, B, kv, C, d)
    rows = lambda x: torch.gather(x.reshape(M, B, T, kv, d).transpose(2, 3), 3, row)  # noqa: E731
    s["Kc"].copy_(torch.where(new[..., None], rows(s["K"]), s["Kc"]))
    s["Vc"].copy_(torch.where(new[..., None], rows(s["V"]), s["Vc"]))
    begin = s["begin"] if s["begin"] is not None else s["length"]
    s["pos"].copy_(torch.where(new, (begin[..., None] + which)[:, :, None].to(torch.int32), s["pos"]))
    s["weight"].masked_fill_(new, 0.0)
    return {"Kc": s["Kc"], "Vc": s["Vc"], "pos": s["pos"], "weight": s["weight"]}


def _weigh_scores(s):
    """Scores of the counted rows against the cache and which of them count: [M, B, kv, n, group, C] each."""
    M, B, T, C, kv, d, n = s["M"], s["B"], s["T"], s["C"], s["kv"], s["d"], s["n"] or s["T"]
    G = s["heads"] // kv
    pick = s["index"].long()[:, :, None, :, None, None].expand(M, B, kv, n, G, d)
    q = torch.gather(s["Q"].float().view(M, B, T, kv, G, d).permute(0, 1, 3, 2, 4, 5), 3, pick).reshape(M, B, kv, n * G, d)
    sc = _capped(torch.matmul(q, s["Kc"].float().transpose(-1, -2).contiguous()).mul_(s["scale"]), s["cap"]).view(M, B, kv, n, G, C)
    i, slot = torch.arange(n, device="cuda"), torch.arange(C, device="cuda")
    seen = (slot <= s["length"][..., None, None] + i[:, None]) & (i < s["count"][..., None])[..., None]   # [M, B, n, C]
    if s["slope"] is not None:
        mine = (s["begin"] if s["begin"] is not None else s["length"])[..., None] + i
        theirs = s["pos"] if s["pos"] is not None else slot.expand(M, B, kv, C)
        sc.addcmul_(s["slope"].view(M, 1, kv, 1, G, 1), (mine[:, :, None, :, None, None] - theirs[:, :, :, None, None]).abs().float(), value=-1.0)
    return sc, seen[:, :, None, :, None].expand(sc.shape)


def _plain_weigh(s):
    M, B, T, kv, n = s["M"], s["B"], s["T"], s["kv"], s["n"] or s["T"]
    sc, seen = _weigh_scores(s)
    pick = s["index"].long()[..., None].expand(M, B, n, s["heads"])
    lse = torch.gather(s["lse"].view(M, B, T, -1), 2, pick).view(M, B, n, kv, -1).permute(0, 1, 3, 2, 4)[..., None]
    return s["weight"] + sc.sub_(lse).exp_().masked_fill_(~seen, 0.0).sum((3, 4))


def _plain_evict(s):
    C, budget = s["C"], s["budget"]
    slot = torch.arange(C, device="cuda")
    L = s["length"][:, :, None, None].long()                                                            # [M, B, 1, 1]
    begin = (s["begin"] if s["begin"] is not None else s["length"])[:, :, None, None].long()
    held = slot < L
    guarded = held & (s["pos"] >= begin - s["recent"]) if s["recent"] else torch.zeros_like(s["pos"], dtype=torch.bool)
    # the order of leaving: entries not guarded by their weight, lowest slot first among equals, then the guarded ones, then what is no entry
    order = s["weight"].argsort(dim=-1, stable=True)
    rank = torch.gather((guarded.int() + 2 * (~held).int()), 3, order).argsort(dim=-1, stable=True)
    order = torch.gather(order, 3, rank)
    leaves = torch.zeros_like(guarded).scatter_(3, order, (slot < L - budget).expand(order.shape))
    stays = held & ~leaves
    # places below the budget that became free, in order, take the entries above it that stay, in order; the rest are moves of the last slot onto itself
    free, mover = leaves & (slot < budget), stays & (slot >= budget)
    pairs = slot < free.sum(-1, keepdim=True)
    to = torch.where(pairs, (~free).int().argsort(dim=-1, stable=True), C - 1)
    come = torch.where(pairs, (~mover).int().argsort(dim=-1, stable=True), C - 1)
    wide = lambda x: x[..., None].expand(s["Kc"].shape)  # noqa: E731
    s["Kc"].scatter_(3, wide(to), torch.gather(s["Kc"], 3, wide(come)))
    s["Vc"].scatter_(3, wide(to), torch.gather(s["Vc"], 3, wide(come)))
    kept = slot < torch.minimum(L, torch.tensor(budget, device="cuda"))
    for new, old in ((s["pos_out"], s["pos"]), (s["weight_out"], s["weight"])):
        new.copy_(torch.where(kept, old.scatter(3, to, torch.gather(old, 3, come)), new))
    return {"Kc": s["Kc"], "Vc": s["Vc"], "pos": s["pos_out"], "weight": s["weight_out"]}


# ---------------------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions one sequence and head at a time in 64 bits (copies of whole rows as they are)."""
    s = prepare(case, seed)
    c, M, B, kv, d = case, case["M"], case["B"], case["kv"], case["d"]
    if c["op"] in ("append", "evict"):
        return _exact_cache(s)
    G = c["heads"] // kv
    N = c["S"] if c["op"] == "prompt" else c["T"]
    slope = s["slope"].double().cpu() if s["slope"] is not None else torch.zeros((M, c["heads"]), dtype=torch.float64)
    if c["op"] == "weigh":
        out = s["weight"].double()
    else:
        out = torch.zeros((M, B, N, c["heads"], d), dtype=torch.float64, device="cuda")
    lse = torch.full((M, B, N, c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    rows = lambda x, m, b, h: x[m].view(B, N, -1)[b, :, h * d:(h + 1) * d].double()  # noqa: E731
    for m in range(M):
        for b in range(B):
            length = int(s["length"][m, b]) if s["length"] is not None else N
            begin = int(s["begin"][m, b]) if s.get("begin") is not None else length
            if c["op"] == "prompt":
                i = j = torch.arange(length, device="cuda")
                q_at, take = i, i
                ok = (j[None] <= i[:, None]) if c["causal"] else torch.ones((length, length), dtype=torch.bool, device="cuda")
                if s["prefix_len"] is not None:
                    ok = ok | (j < int(s["prefix_len"][m, b]))[None]
                if s["doc"] is not None:
                    doc = s["doc"][m, b, :length]
                    ok = ok & (doc[:, None] == doc[None]) & (doc >= 0)[None]
            elif c["op"] == "tree":
                t = int(s["nodes"][m, b]) if s["nodes"] is not None else N
                par, see, depth = s["parent"][m, b].tolist(), torch.zeros((t, t), dtype=torch.bool), [0] * t
                for a in range(t):
                    if par[a] >= 0:
                        see[a], depth[a] = see[par[a]], depth[par[a]] + 1
                    see[a, a] = True
                take = torch.arange(t, device="cuda")
                q_at = begin + torch.tensor(depth, device="cuda")
                ok = torch.cat((torch.ones((t, length), dtype=torch.bool), see), 1).cuda()
            else:
                t = int(s["count"][m, b])
                take = s["index"][m, b, :t].long() if s["index"] is not None else torch.arange(t, device="cuda")
                q_at = begin + torch.arange(t, device="cuda")
                ok = torch.arange(length + t, device="cuda")[None] <= length + torch.arange(t, device="cuda")[:, None]
            for h in range(kv):
                if c["op"] == "prompt":
                    k, v, k_at = rows(s["K"], m, b, h)[:length], rows(s["V"], m, b, h)[:length], j
                else:
                    held = ok.shape[1] if c["op"] == "weigh" else length
                    k = s["Kc"][m, b, h, :held].double()
                    k_at = s["pos"][m, b, h, :held].long() if s["pos"] is not None else torch.arange(held, device="cuda")
                    if c["op"] == "tree":
                        k, k_at = torch.cat((k, rows(s["K"], m, b, h)[:t])), torch.cat((k_at, q_at))
                        v = torch.cat((s["Vc"][m, b, h, :held].double(), rows(s["V"], m, b, h)[:t]))
                far = (q_at[:, None] - k_at[None]).abs().double()
                for x in range(h * G, h * G + G):
                    sc = torch.mm(rows(s["Q"], m, b, x)[take], k.t()) * s["scale"]
                    if c["cap"]:
                        sc = c["cap"] * torch.tanh(sc / c["cap"])
                    sc = (sc - float(slope[m, x]) * far).masked_fill(~ok, -math.inf)
                    if c["op"] == "weigh":
                        out[m, b, h, :held] += torch.exp(sc - s["lse"].view(M, B, N, -1)[m, b, take, x].double()[:, None]).sum(0)
                        continue
                    total = torch.logsumexp(sc, 1)
                    lse[m, b, take, x] = total
                    out[m, b, take, x] = torch.mm(torch.softmax(sc, 1).nan_to_num(0.0), v)
    if c["op"] == "weigh":
        return out
    out = out.view(M, B * N, c["heads"] * d)
    return out if c["op"] == "prompt" else {"O": out, "lse": lse.view(M, B * N, -1) if c["lse"] else None}


def _exact_cache(s):
    kv, d = s["kv"], s["d"]
    pos, weight = (s["pos"], s["weight"]) if s["op"] == "append" else (s["pos_out"], s["weight_out"])
    for m in range(s["M"]):
        for b in range(s["B"]):
            length = int(s["length"][m, b])
            begin = int(s["begin"][m, b]) if s["begin"] is not None else length
            if s["op"] == "append":
                t = int(s["count"][m, b])
                take = s["index"][m, b, :t].long() if s["index"] is not None else torch.arange(t, device="cuda")
                for to, rows in ((s["Kc"], s["K"]), (s["Vc"], s["V"])):
                    to[m, b, :, length:length + t] = rows[m].view(s["B"], s["T"], kv, d)[b, take].transpose(0, 1)
                pos[m, b, :, length:length + t] = begin + torch.arange(t, device="cuda", dtype=torch.int32)
                weight[m, b, :, length:length + t] = 0.0
                continue
            for h in range(kv):
                w, p = s["weight"][m, b, h, :length].cpu().numpy(), s["pos"][m, b, h, :length].cpu().numpy()
                guard = (p >= begin - s["recent"]) & (s["recent"] > 0)
                gone = np.zeros(length, dtype=bool)
                gone[np.lexsort((np.arange(length), w, guard))[:max(0, length - s["budget"])]] = True
                to, come = np.nonzero(gone[:s["budget"]])[0], s["budget"] + np.nonzero(~gone[s["budget"]:])[0]
                stay = min(length, s["budget"])
                pos[m, b, h, :stay], weight[m, b, h, :stay] = s["pos"][m, b, h, :stay], s["weight"][m, b, h, :stay]
                to, come = torch.from_numpy(to).cuda(), torch.from_numpy(come).cuda()
                for x, y in ((s["Kc"], s["Kc"]), (s["Vc"], s["Vc"]), (pos, s["pos"]), (weight, s["weight"])):
                    x[m, b, h, to] = y[m, b, h, come]
    return {"Kc": s["Kc"], "Vc": s["Vc"], "pos": pos, "weight": weight.double()}
