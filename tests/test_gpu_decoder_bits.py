"""What a row does not see changes none of its bits, under every form of the scores: later tokens, other documents, other nodes and rows past the
lengths hold large finite numbers, which choose other ways through a tile for themselves but not for their neighbours."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FORMS = {"plain": (0.0, False), "biased": (0.0, True), "cap 5": (5.0, False), "cap 50": (50.0, False), "cap 5 biased": (5.0, True), "cap 50 biased": (50.0, True)}
TYPES = [(BF, 64), (BF, 128), (BF, 256), (BF, 20), (F32, 64), (F32, 128)]


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def different(a, b):
    """Rows of a and b (compared as they are) with any bit that differs."""
    return (a != b).view(a.shape[0], -1).any(1).nonzero().flatten().tolist()


@pytest.mark.parametrize("factor", [1.6, 6.0, 40.0, 1e10])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,d", TYPES, ids=str)
def test_prompt_rows_keep_their_bits(nf, dtype, d, form, factor):
    cap, biased = FORMS[form]
    g = torch.Generator().manual_seed(d)
    B, S, heads, kv = 3, 400, 4, 2
    Q, K, V = ((torch.randn(1, B * S, n * d, generator=g) * s).to(dtype).cuda() for n, s in ((heads, 1.5), (kv, 1.0), (kv, 1.0)))
    doc = torch.zeros(1, B, S, dtype=torch.int32)
    doc[0, 1, 150:290] = 1                                    # three documents, two of them one
    kw = dict(cap=cap, slope=(torch.rand(1, heads, generator=g) * 0.2).cuda() if biased else None, length=ints([[S, S, 333]]), doc=ints(doc))
    ok = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw).cpu()[0]
    hurt = torch.zeros(B, S, dtype=torch.bool)
    hurt[0, 201:], hurt[1, 150:290:3], hurt[2, 333:] = True, True, True
    for x in (Q, K, V):
        x[:, hurt.view(-1).cuda()] *= factor
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw).cpu()[0]
    same = torch.ones(B, S, dtype=torch.bool)
    same[0, 201:], same[1, 150:290] = False, False
    assert not different(got[same.view(-1)], ok[same.view(-1)])


@pytest.mark.parametrize("factor", [1.6, 6.0, 40.0, 1e10])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T", [6, 20])
@pytest.mark.parametrize("dtype,d", TYPES, ids=str)
def test_tree_rows_keep_their_bits(nf, dtype, d, T, form, factor):
    """24 rows of a key head, and 80: the kernels for few rows and for many."""
    cap, biased = FORMS[form]
    g = torch.Generator().manual_seed(d + T)
    B, C, heads, kv = 2, 1300, 4, 1
    Q, K, V = ((torch.randn(1, B * T, n * d, generator=g) * s).to(dtype).cuda() for n, s in ((heads, 1.5), (kv, 1.0), (kv, 1.0)))
    Kc, Vc = (torch.randn(1, B, kv, C, d, generator=g).to(dtype).cuda() for _ in range(2))
    length = ints([[C, 37]])
    parent = torch.arange(T).expand(1, B, T) - 2              # two chains, of even nodes and of odd ones
    lse = torch.empty(1, B * T, heads, device="cuda")
    kw = dict(cap=cap, slope=(torch.rand(1, heads, generator=g) * 0.2).cuda() if biased else None, parent=ints(parent), nodes=ints([[T, T - 2]]), lse=lse)
    ok = nf.attention_tree(Q, K, V, Kc, Vc, length, **kw).cpu()[0]
    ok_lse = lse.cpu()[0]
    hurt = torch.zeros(B, T, dtype=torch.bool)
    hurt[0, 1::2], hurt[1, T - 2:] = True, True               # the odd chain of the first sequence, nodes past the second's
    for x in (Q, K, V):
        x[:, hurt.view(-1).cuda()] *= factor
    got = nf.attention_tree(Q, K, V, Kc, Vc, length, **kw).cpu()[0]
    keep = ~hurt.view(-1)
    assert not different(got[keep], ok[keep])
    assert not different(lse.cpu()[0][keep], ok_lse[keep])


@pytest.mark.parametrize("cap", [0.0, 5.0, 50.0])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_a_row_alone_has_the_bits_that_it_has_among_others(nf, dtype, cap):
    """Cached tokens and prompts, where neighbours of a tile hold scores of every size: each model alone against all of them."""
    g = torch.Generator().manual_seed(11)
    M, S, heads, d = 4, 300, 2, 128
    size = torch.tensor([0.1, 1.0, 8.0, 60.0]).view(M, 1, 1)
    Q, K, V = ((torch.randn(M, S, heads * d, generator=g) * s).to(dtype).cuda() for s in (size, 1.0, 1.0))
    want = nf.attention_prompt(Q, K, V, 1, S, heads, cap=cap)
    for m in range(M):
        assert torch.equal(nf.attention_prompt(Q[m:m + 1], K[m:m + 1], V[m:m + 1], 1, S, heads, cap=cap), want[m:m + 1])
