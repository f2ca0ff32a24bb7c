"""Attention weights of bfloat16 caches that few rows read: the product with the values holds 15 bits of each, so a result is off by its own rounding."""
import pytest
import torch

import decoder_plain as plain

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


ROWS = [(1, 4, 1), (1, 16, 1), (1, 3, 3), (4, 8, 2), (5, 4, 1), (8, 4, 1)]      # the last two have more than 16 to a key head


@pytest.mark.parametrize("d,T,heads,kv", [(d, *r) for d in (64, 72, 128, 256) for r in (ROWS[:4] if d <= 64 else ROWS)])
@pytest.mark.parametrize("L", [40, 700, 3000])
def test_weights_of_few_rows_are_not_rounded_to_bfloat16(nf, d, L, T, heads, kv):
    """The bound of tests/decoder_plain.py with 2^-15 for the weights' parts in place of their rounding (the upper part is the weight less 2^-9 of it, cut
    off after 8 bits, so the rest is below 2^-6.5 of it and rounded to 9 bits).  16 rows to a key head at most up to 64 features, 32 above: more take their keys through LDS."""
    g = torch.Generator().manual_seed(d + L)
    x = torch.randn(1, T, (heads + 2 * kv) * d, generator=g).to(BF).cuda()
    Q, K, V = x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d], x[:, :, (heads + kv) * d:]
    Kc, Vc = (torch.randn(1, 1, kv, L, d, generator=g).to(BF).cuda() for _ in range(2))
    length = torch.tensor([[L]], dtype=torch.int32).cuda()
    want, tol, _, _ = plain.tree(Q, K, V, Kc, Vc, length)
    # tol = (2 e + 2^-19 + h + n 2^-23) sum p |v| + h |O|: the h of the weights, h sum p |v|, becomes 2^-15 sum p |v|
    h = plain.half_step(BF)
    a, _, _, _ = plain.tree(Q, K, V.abs(), Kc, Vc.abs(), length)              # sum p |v|
    got = nf.attention_tree(Q, K, V, Kc, Vc, length).cpu().double()
    assert ((got - want).abs() <= tol - (h - 2.0 ** -15) * a).all()
