"""Caps and scales at the ends of their ranges: what scale / cap is not a float32 number, or hardly one, the score is one all the same."""
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


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def near(got, want, tol):
    assert ((got.cpu().double() - want).abs() <= tol).all()


# scale / cap: infinite, largest, below the normal numbers.  `size` is that of the queries, so that scores lie about the cap or far below it.
ENDS = [(1e9, 1e-30, 1.0), (1e30, 1e-30, 1.0), (3e38, 0.5, 1.0), (1e-10, 1e30, 3e10), (1e-20, 1e25, 1e20), (1e-8, 1e30, 1e7)]


@pytest.mark.parametrize("scale,cap,size", ENDS, ids=str)
@pytest.mark.parametrize("biased", [False, True], ids=["", "biased"])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 20), (F32, 64)], ids=str)
def test_caps_and_scales_of_any_ratio(nf, dtype, d, biased, scale, cap, size):
    """Every third query is 0, and so are its scores: the mean of what it sees, but for the bias.  The others as the definition in 64 bits has them."""
    g = torch.Generator().manual_seed(d)
    B, S, heads, kv, C = 2, 70, 4, 2, 90
    zero = torch.arange(S) % 3 == 0

    def rows(N, where):
        Q = torch.randn(1, B * N, heads * d, generator=g) * size / d ** 0.5
        Q[:, where.repeat(B)] = 0
        return (x.to(dtype).cuda() for x in (Q, torch.randn(1, B * N, kv * d, generator=g), torch.randn(1, B * N, kv * d, generator=g)))
    kw = dict(scale=scale, cap=cap, slope=(torch.rand(1, heads, generator=g) * 0.1).cuda() if biased else None)
    # scores that the cap or an overflow of scale q k decides are right in sign alone: those rows hold to the bound of the definition where q k is far from 0
    Q, K, V = rows(S, zero)
    want, tol = plain.prompt(Q, K, V, B, S, heads, kv, **kw)
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw)
    assert got.isfinite().all()
    keep = slice(None) if scale < 1 else zero.repeat(B)
    near(got[0, keep], want[0, keep], tol[0, keep])
    Kc, Vc = (torch.randn(1, B, kv, C, d, generator=g).to(dtype).cuda() for _ in range(2))
    L = ints([[C - 20, 33]])
    for T in (1, 6, 20):
        Q, K, V = rows(T, zero[:T])
        lse = torch.empty(1, B * T, heads, device="cuda")
        o, tol, z, ztol = plain.tree(Q, K, V, Kc, Vc, L, **kw)
        got = nf.attention_tree(Q, K, V, Kc, Vc, L, lse=lse, **kw)
        assert got.isfinite().all() and lse.isfinite().all()
        keep = slice(None) if scale < 1 else zero[:T].repeat(B)
        near(got[0, keep], o[0, keep], tol[0, keep])
        near(lse[0, keep], z[0, keep], ztol[0, keep])
        after = [Kc.clone(), Vc.clone()]
        nf.cache_append(K, V, *after, None, None, L)
        w = torch.zeros(1, B, kv, C, device="cuda")
        only = zero[:T].nonzero().flatten().int() if scale >= 1 else torch.arange(T).int()
        index = only.expand(1, B, len(only)).contiguous().cuda()
        args = (Q, z.float().cuda(), after[0], w, L)
        got = nf.cache_weigh(*args, index=index, **kw)
        w, tol = plain.weigh(*args, index=index, **kw)
        assert got.isfinite().all()
        near(got, w, tol)
