"""Caches that are shared out in chunks, and infinite values in them: a value under a weight gives that infinity whichever chunk holds it,
and the other features keep their bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


# Chunks hold 512 or 1024 entries.  The lengths fill 1 to 18 of them: batches of eight that are full, that are not, and one chunk alone; with the
# first capacity a row's chunks are one group's work, with the second all groups of a workgroup share them.
CACHES = [(4000, [1500, 2600, 4000, 700]), (8800, [1500, 4500, 8192, 8800, 8200, 300])]


@pytest.mark.parametrize("C,lengths", CACHES, ids=["one group", "shared"])
@pytest.mark.parametrize("T", [1, 20])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 256), (F32, 64), (F32, 128), (F32, 256)], ids=str)
def test_infinite_values_of_a_shared_out_cache(nf, dtype, d, T, C, lengths):
    """Feature 0: an infinity in the last entry; 1: in the middle; 2: in the first drafted token, which every later one descends from; 3: one of
    either sign, NaN; 4: in the first entry."""
    g = torch.Generator().manual_seed(C + T)
    B, heads, kv = len(lengths), 4, 1
    x = torch.randn(1, B * T, (heads + 2 * kv) * d, generator=g).to(dtype).cuda()
    Q, K, V = x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d], x[:, :, (heads + kv) * d:]
    Kc, Vc = (torch.randn(1, B, kv, C, d, generator=g).to(dtype).cuda() for _ in range(2))
    length = torch.tensor([lengths], dtype=torch.int32).cuda()
    ok = nf.attention_tree(Q, K, V, Kc, Vc, length)
    for b, L in enumerate(lengths):
        Vc[0, b, 0, L - 1, 0], Vc[0, b, 0, L // 2, 1], V[0, b * T, 2] = INF, -INF, INF
        Vc[0, b, 0, 1, 3], Vc[0, b, 0, L - 2, 3], Vc[0, b, 0, 0, 4] = INF, -INF, -INF
    got = nf.attention_tree(Q, K, V, Kc, Vc, length)
    got, ok = (t.cpu().float().view(B, T, heads, d) for t in (got, ok))
    for f, want in ((0, INF), (1, -INF), (2, INF), (4, -INF)):
        assert (got[..., f] == want).all(), (f, got[:, 0, 0, f])
    assert got[..., 3].isnan().all()
    assert torch.equal(got[..., 5:], ok[..., 5:])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_values_that_are_nan_stay_in_their_feature(nf, dtype):
    """NaN in the last of 2, 3 and 9 chunks: that feature of every row that sees it, no other."""
    g = torch.Generator().manual_seed(3)
    for lengths in ([700], [1300], [4500]):
        L, d = lengths[0], 64
        x = torch.randn(1, 3, 3 * d, generator=g).to(dtype).cuda()
        Kc, Vc = (torch.randn(1, 1, 1, L, d, generator=g).to(dtype).cuda() for _ in range(2))
        Vc[0, 0, 0, L - 1, 7] = math.nan
        got = nf.attention_tree(x[:, :, :d], x[:, :, d:2 * d], x[:, :, 2 * d:], Kc, Vc, torch.tensor([lengths], dtype=torch.int32).cuda()).cpu()[0]
        assert got[:, 7].isnan().all() and got.isfinite().sum() == 3 * (d - 1)
