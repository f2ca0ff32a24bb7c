"""Weights of the entries of many long caches, where a wavefront takes one block of keys after the other: against calls of one model, which are
small enough for a block each, and a sequence of each model against 64 bits."""
import math

import pytest
import torch

import decoder_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


# With heads = M B kv and pieces of 256 keys (128 in float32; half as many above 64 features) a wavefront takes heads * pieces / 4096 turns, 8 at most:
# 2, 4, 8 and 8, 3, 2.  C is no multiple of the keys of a workgroup's turns; a model alone stays below 8192 pieces, one turn.
SIZES = [(BF, 8, 8, 16, 4, 4500), (F32, 8, 8, 16, 4, 4500), (F32, 8, 16, 16, 4, 4700), (BF, 8, 16, 32, 4, 4321), (BF, 72, 8, 10, 4, 5111), (F32, 80, 8, 8, 2, 5003)]


@pytest.mark.parametrize("T,n,group", [(1, None, 2), (6, 4, 4), (12, 9, 4)], ids=["token", "16 rows", "36 rows"])
@pytest.mark.parametrize("dtype,d,M,B,kv,C", SIZES, ids=str)
def test_weigh_in_turns(nf, dtype, d, M, B, kv, C, T, n, group):
    g = torch.Generator(device="cuda").manual_seed(C + T)
    heads, N, dev = kv * group, T if n is None else n, "cuda"
    Q = torch.randn(M, B * T, heads * d, generator=g, device=dev).to(dtype)
    Kc = torch.randn(M, B, kv, C, d, generator=g, device=dev).to(dtype)
    at = torch.arange(M * B, device=dev).view(M, B)
    length = ((at * 977 + 13) % (C + 1)).int()                # of every size, so that they end in every turn
    length[0, 0], length[0, 1], length[1, 0], length[1, 1] = C, 0, C - N, C - 1
    count = (at % (N + 2)).int()
    held = (length + count).clamp(max=C)
    behind = torch.arange(C, device=dev) >= held[:, :, None, None]
    Kc.masked_fill_(behind[..., None], math.nan)
    weight = torch.rand(M, B, kv, C, generator=g, device=dev).masked_fill_(behind, math.nan)
    index = None if n is None else torch.rand(M, B, T, generator=g, device=dev).argsort(-1)[:, :, :n].sort(-1).values.int().contiguous()
    pos = torch.randint(0, 9000, (M, B, kv, C), generator=g, device=dev, dtype=torch.int32)
    lse = torch.rand(M, B * T, heads, generator=g, device=dev) * 3 + 5
    lse[1, 0] = -math.inf
    slope = torch.rand(M, heads, generator=g, device=dev) * 0.001
    for kw in (dict(cap=3.0), dict(pos=pos, start=length + 5, slope=slope)):
        kw["count"] = count
        cut = lambda m, b: {k: (v[m:m + 1] if k == "slope" else v[m:m + 1, b].contiguous()) if torch.is_tensor(v) else v for k, v in kw.items()}  # noqa: E731
        if index is not None:
            kw["index"] = index
        got = nf.cache_weigh(Q, lse, Kc, weight, length, **kw)
        inplace = weight.clone()
        nf.cache_weigh(Q, lse, Kc, inplace, length, out=inplace, **kw)
        assert torch.equal(got.nan_to_num(-1.0), inplace.nan_to_num(-1.0))
        every = slice(None)
        for m in range(M):
            one = nf.cache_weigh(Q[m:m + 1], lse[m:m + 1], Kc[m:m + 1], weight[m:m + 1], length[m:m + 1], **cut(m, every))
            assert torch.equal(one.nan_to_num(-1.0), got[m:m + 1].nan_to_num(-1.0)), m
        assert (got.isnan() == behind).all()
        for m, b in ((0, 0), (0, 1), (1, 0), (1, 1), (M - 1, B - 1), (M // 2, B // 2)):
            r, s = slice(b * T, b * T + T), slice(b, b + 1)
            want, tol = plain.weigh(Q[m:m + 1, r], lse[m:m + 1, r], Kc[m:m + 1, s], weight[m:m + 1, s], length[m:m + 1, s], **cut(m, s))
            there = ~behind[m:m + 1, s].expand(want.shape).cpu()
            off = (got[m:m + 1, s].cpu().double() - want).abs()
            assert (off[there] <= tol[there]).all(), (m, b)
