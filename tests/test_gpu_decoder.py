"""The decoders' operators against their definitions in 64 bits (tests/decoder_plain.py, which also derives how far they may be off):
sizes around the tiles, head layouts, masks that leave rows empty, what lies in masked places and behind the last entry, strides,
streams, captured graphs, and a run of all of them together."""
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


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows(g, M, N, heads, kv, d, dtype, std=1.0):
    """Q, K, V as column blocks of one packed projection."""
    x = (torch.randn(M, N, (heads + 2 * kv) * d, generator=g) * std).to(dtype).cuda()
    return x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d], x[:, :, (heads + kv) * d:]


def ints(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def slopes(g, M, heads):
    return (torch.rand(M, heads, generator=g) * 0.5).float().cuda()


def near(got, want, tol, what=""):
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    off = (got - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its tolerance" % (what, int(bad.sum()), bad.numel(), float((off / tol)[bad].max()))


# ---------------------------------------------------------------------------------------------------------------------------- prompts
SIZES = [(1, 1, 1), (2, 1, 2), (1, 2, 31), (1, 1, 63), (2, 1, 64), (1, 1, 65), (1, 2, 127), (1, 1, 128), (1, 1, 129), (2, 1, 200), (1, 1, 333)]


@pytest.mark.parametrize("M,B,S", SIZES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_lengths(nf, dtype, M, B, S):
    g = gen(S)
    heads, kv, d = 4, 2, 64
    Q, K, V = rows(g, M, B * S, heads, kv, d, dtype)
    kw = dict(slope=slopes(g, M, heads), cap=5.0)
    near(nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw), *plain.prompt(Q, K, V, B, S, heads, kv, **kw))


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 1), (16, 2)])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_heads(nf, dtype, heads, kv):
    g = gen(heads)
    Q, K, V = rows(g, 2, 100, heads, kv, 64, dtype)
    s = slopes(g, 2, heads)
    near(nf.attention_prompt(Q, K, V, 1, 100, heads, kv, slope=s), *plain.prompt(Q, K, V, 1, 100, heads, kv, slope=s))


@pytest.mark.parametrize("d", [1, 7, 8, 20, 32, 40, 64, 72, 80, 96, 100, 120, 128, 136, 192, 256])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_head_sizes(nf, dtype, d):
    g = gen(d)
    Q, K, V = rows(g, 1, 2 * 75, 2, 1, d, dtype)
    near(nf.attention_prompt(Q, K, V, 2, 75, 2, 1, cap=2.0), *plain.prompt(Q, K, V, 2, 75, 2, 1, cap=2.0))


MASKS = {
    "causal": dict(causal=True), "all": dict(causal=False), "lengths": dict(causal=True, length=True), "lengths of all": dict(causal=False, length=True),
    "prefix": dict(causal=True, prefix=True), "prefix and lengths": dict(causal=True, prefix=True, length=True), "documents": dict(causal=True, doc="runs"),
    "documents of all": dict(causal=False, doc="runs", length=True), "mixed documents": dict(causal=True, doc="mixed"), "mixed documents of all": dict(causal=False, doc="mixed"),
    "prefix and documents": dict(causal=True, prefix=True, doc="runs"), "padding": dict(causal=True, doc="padding"),
}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("S", [40, 150, 300])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_masks(nf, dtype, S, mask):
    g, spec = gen(S), dict(MASKS[mask])
    M, B, heads, kv, d = 2, 3, 2, 1, 64
    kw = dict(causal=spec["causal"], slope=slopes(g, M, heads))
    if spec.get("length"):
        kw["length"] = ints([[S, 0, S // 2 + 1], [1, S + 7, -3]])
    if spec.get("prefix"):
        kw["prefix"] = ints([[0, S // 3, S], [S + 5, 65 % S, -1]])
    if spec.get("doc") == "runs":
        kw["doc"] = ints((torch.arange(S)[None, None] * torch.tensor([[2, 3, 5], [1, 7, 4]])[..., None] // S) + 1000)
    elif spec.get("doc") == "mixed":
        kw["doc"] = ints(torch.randint(-1, 3, (M, B, S), generator=g))
    elif spec.get("doc") == "padding":
        doc = torch.zeros(M, B, S, dtype=torch.int32)
        doc[:, 1, S // 2:] = -1
        doc[0, 2] = -5
        kw["doc"] = ints(doc)
    Q, K, V = rows(g, M, B * S, heads, kv, d, dtype)
    want, tol = plain.prompt(Q, K, V, B, S, heads, kv, **kw)
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw)
    near(got, want, tol)
    empty = (want == 0).all(-1)
    assert (got.cpu()[empty] == 0).all()                      # rows that see nothing are 0, not nearly so


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 192), (F32, 64), (F32, 128), (F32, 256), (BF, 20)], ids=str)
def test_prompt_what_is_not_seen_has_no_part(nf, dtype, d, bad):
    """Later tokens, other documents, padding and rows past the length hold NaN or infinities: the other rows' bits stay."""
    g = gen(3)
    M, B, S, heads, kv = 1, 3, 150, 4, 2
    Q, K, V = (x.contiguous() for x in rows(g, M, B * S, heads, kv, d, dtype))
    doc = torch.zeros(M, B, S, dtype=torch.int32)
    doc[0, 1, 50:] = 1
    doc[0, 2, 70:90] = -1
    kw = dict(length=ints([[S, S, 120]]), doc=ints(doc))
    ok = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw)
    hurt = torch.zeros(B, S, dtype=torch.bool)
    hurt[0, 101], hurt[1, 20], hurt[2, 75], hurt[2, 120:] = True, True, True, True
    for x in (Q, K, V):
        x[:, hurt.view(-1).cuda()] = bad
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw)
    same = torch.ones(B, S, dtype=torch.bool)
    same[0, 101:] = False                                     # those that see row 101 of the first sequence
    same[1, 20:50] = False                                    # the rest of the first document of the second
    assert torch.equal(got.cpu()[0][same.view(-1)], ok.cpu()[0][same.view(-1)])
    if math.isnan(bad):
        assert got.cpu()[0].view(B, S, -1)[1, 20:50].isnan().all()


@pytest.mark.parametrize("scale", [0.0, 1e-38, -0.125, 30.0, 1e30])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_scales(nf, dtype, scale):
    """Scores of any finite size: none, tiny, negative, and so far apart that one key takes all the weight."""
    g = gen(4)
    Q, K, V = rows(g, 1, 90, 2, 2, 64, dtype)
    got = nf.attention_prompt(Q, K, V, 1, 90, 2, scale=scale).cpu().double()
    want, tol = plain.prompt(Q, K, V, 1, 90, 2, 2, scale=scale)
    if scale < 1e6:
        near(got, want, tol)
    else:
        assert torch.isfinite(got).all()
        near(got, want, 2 * plain.half_step(dtype) * want.abs())          # distinct scores: 1e30 apart and more


@pytest.mark.parametrize("cap", [1e-3, 1.0, 50.0, 3e4])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompt_caps(nf, dtype, cap):
    """Scores far below the cap, about it and far above."""
    g = gen(5)
    Q, K, V = rows(g, 1, 140, 2, 2, 64, dtype, std=3.0)
    near(nf.attention_prompt(Q, K, V, 1, 140, 2, cap=cap), *plain.prompt(Q, K, V, 1, 140, 2, 2, cap=cap))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 80), (F32, 64), (F32, 20)], ids=str)
def test_prompt_layouts_change_no_bit(nf, dtype, d):
    """Packed, dense and padded rows, rows at odd elements, and models merged or alone."""
    g = gen(6)
    M, B, S, heads, kv = 3, 2, 70, 4, 2
    Q, K, V = rows(g, M, B * S, heads, kv, d, dtype)
    want = nf.attention_prompt(Q, K, V, B, S, heads, kv)
    assert torch.equal(nf.attention_prompt(Q.contiguous(), K.contiguous(), V.contiguous(), B, S, heads, kv), want)
    for m in range(M):
        assert torch.equal(nf.attention_prompt(Q[m:m + 1], K[m:m + 1], V[m:m + 1], B, S, heads, kv), want[m:m + 1])

    def at_odd(x):                                            # the same rows, one element into a wider buffer of an odd row length
        wide = torch.zeros(M, B * S, x.shape[2] + 3, dtype=dtype, device="cuda")
        wide[:, :, 1:-2] = x
        return wide[:, :, 1:-2]
    ref, tol = plain.prompt(Q, K, V, B, S, heads, kv)
    near(nf.attention_prompt(at_odd(Q), at_odd(K), at_odd(V), B, S, heads, kv), ref, tol)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128), (F32, 200)], ids=str)
def test_prompt_infinite_values_add_up(nf, dtype, d):
    """One infinity under a weight gives that infinity, two of opposite signs NaN, and neither reaches the rows before it."""
    g = gen(15)
    S = 420
    Q, K, V = (x.contiguous() for x in rows(g, 1, S, 1, 1, d, dtype))
    ok = nf.attention_prompt(Q, K, V, 1, S, 1)
    V[0, 300, 3], V[0, 350, 3], V[0, 333, 0] = float("inf"), -float("inf"), -float("inf")
    got = nf.attention_prompt(Q, K, V, 1, S, 1).cpu()[0].float()
    assert torch.equal(got[:300], ok.cpu()[0, :300].float()) and torch.equal(got[:, 4:], ok.cpu()[0, :, 4:].float())
    assert (got[300:350, 3] == float("inf")).all() and got[350:, 3].isnan().all() and (got[333:, 0] == -float("inf")).all()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("slope, cap", ((1e6, 0.0), (1e12, 0.0), (1e6, 30.0)))
def test_prompt_steep_slopes(nf, dtype, causal, slope, cap):
    """Every other key weighs nothing: a row gives its own value.  (The weight may be rounded, and the result.)"""
    Q, K, V = rows(gen(9), 1, 2000, 2, 1, 64, dtype)
    got = nf.attention_prompt(Q, K, V, 1, 2000, 2, 1, causal=causal, cap=cap, slope=torch.full((1, 2), slope, device="cuda"))
    want = V.cpu().double().repeat(1, 1, 2)
    near(got, want, want.abs() * (2 * 2.0 ** -8 if dtype == BF else 4 * 2.0 ** -24), "O")


FORMS = {"plain": dict(), "biased": dict(slope=True), "capped": dict(cap=5.0), "capped and biased": dict(cap=5.0, slope=True), "negative scale": dict(scale=-0.1), "negative scale, biased": dict(scale=-0.1, slope=True)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 256), (F32, 64), (F32, 128), (F32, 256)], ids=str)
def test_prompt_forms_of_scores(nf, dtype, d, form):
    """Every form of the scores, over documents, with infinities in rows past the length and in keys that some rows see."""
    g, kw = gen(d), dict(FORMS[form])
    M, B, S, heads, kv = 2, 2, 140, 4, 2
    if kw.pop("slope", False):
        kw["slope"] = slopes(g, M, heads)
    kw.update(length=ints([[S, 99], [130, S]]), doc=ints((torch.arange(S) // 50).expand(M, B, S)))
    Q, K, V = (x.contiguous() for x in rows(g, M, B * S, heads, kv, d, dtype))
    want, tol = plain.prompt(Q, K, V, B, S, heads, kv, **kw)
    near(nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw), want, tol)
    V[0, S + 99:], K[0, S + 99:], V[1, 60, :d] = math.nan, math.inf, math.inf
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, **kw).cpu()
    sees = torch.zeros(want.shape, dtype=torch.bool)
    sees[1, 60:100, :heads // kv * d] = True                  # its own document's later rows, under the heads of the first key head
    assert (got[sees] == math.inf).all()
    near(torch.where(sees, 0.0, got.double()), torch.where(sees, 0.0, want), tol)


def test_prompt_far_rows(nf):
    """Rows more than 2^31 elements and 2^32 bytes into a buffer."""
    M, S, heads, d = 2, 100, 1, 64
    wide = torch.zeros(M * S, 12_000_000, dtype=BF, device="cuda").view(M, S, -1)     # 2.4e9 elements
    g = gen(7)
    x = torch.randn(M, S, 3 * d, generator=g).to(BF).cuda()
    wide[:, :, -3 * d:] = x
    Q, K, V = (wide[:, :, -3 * d + i * d: wide.shape[2] - 3 * d + (i + 1) * d] for i in range(3))
    near(nf.attention_prompt(Q, K, V, 1, S, heads), *plain.prompt(x[:, :, :d], x[:, :, d:2 * d], x[:, :, 2 * d:], 1, S, 1, 1))


def test_prompt_long_bias_and_sums(nf):
    """A long row in each type: the last 40 rows of 5000 against 64 bits."""
    g = gen(8)
    S = 5000
    for dtype in (BF, F32):
        Q, K, V = rows(g, 1, S, 1, 1, 64, dtype)
        s = torch.full((1, 1), 0.003, device="cuda")
        got = nf.attention_prompt(Q, K, V, 1, S, 1, slope=s, cap=20.0)
        at = torch.arange(S)
        i = at[-40:]
        q, k, v = (plain.heads_of(x, 1, S, 1)[0, 0, 0] for x in (Q, K, V))
        o, tol, _, _ = plain.attend(q[-40:], k, v, at[None] <= i[:, None], 64 ** -0.5, 20.0, float(s), (i[:, None] - at[None]).abs().double(), dtype)
        near(got[0, -40:], o, tol, str(dtype))


# ------------------------------------------------------------------------------------------------------------------------------ trees
def cache(g, M, B, kv, C, d, dtype):
    return torch.randn(M, B, kv, C, d, generator=g).to(dtype).cuda(), torch.randn(M, B, kv, C, d, generator=g).to(dtype).cuda()


def random_parents(g, M, B, T):
    p = (torch.rand(M, B, T, generator=g) * (torch.arange(T) + 1)).floor() - 1
    return ints(p)


def check_tree(nf, g, dtype, M, B, T, C, heads, kv, d, length, parent="random", nodes=None, start=None, pos=None, slope=False, cap=0.0):
    Q, K, V = rows(g, M, B * T, heads, kv, d, dtype)
    Kc, Vc = cache(g, M, B, kv, C, d, dtype)
    for m in range(M):                                        # what lies behind the entries is not read
        for b in range(B):
            Kc[m, b, :, max(0, int(length[m][b])):] = float("nan")
            Vc[m, b, :, max(0, int(length[m][b])):] = float("nan")
    kw = dict(start=None if start is None else ints(start), parent=random_parents(g, M, B, T) if parent == "random" else parent, nodes=None if nodes is None else ints(nodes),
              pos=pos, slope=slopes(g, M, heads) if slope else None, cap=cap)
    lse = torch.full((M, B * T, heads), 7.0, device="cuda")
    got = nf.attention_tree(Q, K, V, Kc, Vc, ints(length), lse=lse, **kw)
    o, tol, want, ltol = plain.tree(Q, K, V, Kc, Vc, ints(length), **kw)
    near(got, o, tol, "O")
    gone = want == -math.inf
    assert (lse.cpu()[gone] == -math.inf).all() and (got.cpu().view(M, B * T, heads, d)[gone] == 0).all()
    near(torch.where(gone, 0.0, lse.cpu().double()), torch.where(gone, 0.0, want), ltol.nan_to_num(posinf=1.0), "lse")
    assert torch.equal(nf.attention_tree(Q, K, V, Kc, Vc, ints(length), **kw), got)      # without lse the same bits, and twice the same
    return got


@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_nodes(nf, dtype, T):
    check_tree(nf, gen(T), dtype, 2, 2, T, 150, 4, 2, 64, [[150, 0], [64, 99]], slope=True, cap=4.0)


@pytest.mark.parametrize("C", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_cache_lengths(nf, dtype, C):
    check_tree(nf, gen(C), dtype, 1, 3, 3, C, 4, 1, 64, [[C, C - 1, C // 2]], slope=True)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 1), (64, 2), (40, 1)])
@pytest.mark.parametrize("T", [1, 7])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_heads(nf, dtype, T, heads, kv):
    check_tree(nf, gen(heads), dtype, 2, 1, T, 200, heads, kv, 64, [[200], [131]], slope=True)


@pytest.mark.parametrize("d", [1, 7, 8, 20, 32, 40, 64, 72, 80, 96, 100, 120, 128, 136, 192, 256])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_head_sizes(nf, dtype, d):
    check_tree(nf, gen(d), dtype, 1, 2, 4, 140, 4, 2, d, [[140, 77]], cap=3.0)


@pytest.mark.parametrize("T", [3, 6, 13, 20])
@pytest.mark.parametrize("form", [f for f in FORMS if "scale" not in f])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (BF, 256), (F32, 64), (F32, 128), (F32, 256)], ids=str)
def test_tree_forms_of_scores(nf, dtype, d, form, T):
    """Every form of the scores with rows of every kernel (12, 24, 52 and 80 to a key head)."""
    kw = dict(FORMS[form])
    check_tree(nf, gen(T), dtype, 1, 2, T, 1300, 8, 2, d, [[1300, 70]], **kw)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_parents_positions_and_empty_rows(nf, dtype):
    g = gen(9)
    M, B, T, C, heads, kv = 2, 3, 9, 90, 4, 2
    length, nodes = [[0, 90, 17], [64, -4, 200]], [[9, 0, 4], [-1, 20, 1]]
    for parent in (None, "random", ints(torch.full((M, B, T), -1)), ints(torch.full((M, B, T), 50)), ints(torch.arange(T).expand(M, B, T) // 2 - 1)):
        pos = ints(torch.randint(0, 5000, (M, B, kv, C), generator=g))
        check_tree(nf, g, dtype, M, B, T, C, heads, kv, 64, length, parent=parent, nodes=nodes, start=[[0, 5000, 17], [70, 3, 999]], pos=pos, slope=True)


@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("dtype,C", [(BF, 5000), (F32, 3000)], ids=str)
def test_tree_long_cache(nf, dtype, C, T):
    """Caches long enough to be shared out, sequences of very different lengths."""
    check_tree(nf, gen(10), dtype, 1, 3, T, C, 4, 1, 64, [[C, 130, 0]], slope=True, start=[[C + 5, 4000, 0]])
    check_tree(nf, gen(11), dtype, 1, 1, T, C, 2, 2, 128, [[C - 1]])


@pytest.mark.parametrize("T", [1, 6, 13, 26])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (BF, 256), (BF, 20)], ids=str)
def test_tree_bits_are_a_sequences_own(nf, dtype, d, T):
    """Models and sequences merged or alone, and caches of another capacity: the same bits, also where a cache is shared out."""
    g = gen(14)
    M, B, heads, kv, C = 2, 2, 4, 1, 2500
    Q, K, V = rows(g, M, B * T, heads, kv, d, dtype)
    Kc, Vc = cache(g, M, B, kv, C, d, dtype)
    length, parent, slope = ints([[2500, 700], [1, 1300]]), random_parents(g, M, B, T), slopes(g, M, heads) * 0.01
    want = nf.attention_tree(Q, K, V, Kc, Vc, length, parent=parent, slope=slope)
    wide = [torch.full((M, B, kv, 5000, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
    for w, x in zip(wide, (Kc, Vc)):
        w[:, :, :, :C] = x
    assert torch.equal(nf.attention_tree(Q, K, V, *wide, length, parent=parent, slope=slope), want)
    for m in range(M):
        for b in range(B):
            r = slice(b * T, b * T + T)
            one = nf.attention_tree(Q[m:m + 1, r].contiguous(), K[m:m + 1, r].contiguous(), V[m:m + 1, r].contiguous(), Kc[m:m + 1, b:b + 1].contiguous(), Vc[m:m + 1, b:b + 1].contiguous(),
                                    length[m:m + 1, b:b + 1].contiguous(), parent=parent[m:m + 1, b:b + 1].contiguous(), slope=slope[m:m + 1])
            assert torch.equal(one, want[m:m + 1, r])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (BF, 20)], ids=str)
def test_tree_what_is_not_seen_has_no_part(nf, dtype, d, bad):
    """A node that holds NaN or infinities reaches its descendants only; nodes past the number of them reach nobody."""
    g = gen(12)
    B, T, C, heads, kv = 2, 6, 70, 4, 2
    Q, K, V = (x.contiguous() for x in rows(g, 1, B * T, heads, kv, d, dtype))
    Kc, Vc = cache(g, 1, B, kv, C, d, dtype)
    kw = dict(parent=ints([[[-1, 0, 0, 1, 2, 2]] * B]), nodes=ints([[6, 3]]), slope=slopes(g, 1, heads))
    ok = nf.attention_tree(Q, K, V, Kc, Vc, ints([[70, 33]]), **kw)
    for x in (Q, K, V):
        x[0, 2] = bad                                         # node 2 of the first sequence: 4 and 5 see it
        x[0, T + 3:] = bad
    got = nf.attention_tree(Q, K, V, Kc, Vc, ints([[70, 33]]), **kw)
    same = torch.tensor([0, 1, 3, 6, 7, 8, 9, 10, 11])
    assert torch.equal(got.cpu()[0, same], ok.cpu()[0, same])


def test_tree_far_entries(nf):
    """A cache of more than 2^31 elements: the last sequences' entries lie past 2^32 bytes."""
    B, C, d = 3, 6_000_000, 128
    Kc = torch.zeros(1, B, 1, C, d, dtype=BF, device="cuda")
    Vc = torch.zeros(1, B, 1, C, d, dtype=BF, device="cuda")
    g = gen(13)
    k, v = torch.randn(40, d, generator=g).to(BF).cuda(), torch.randn(40, d, generator=g).to(BF).cuda()
    Kc[0, 2, 0, :40], Vc[0, 2, 0, :40] = k, v
    Q, K, V = rows(g, 1, B, 1, 1, d, BF)
    got = nf.attention_tree(Q, K, V, Kc, Vc, ints([[0, 0, 40]]))
    small = torch.zeros(1, B, 1, 40, d, dtype=BF), torch.zeros(1, B, 1, 40, d, dtype=BF)
    small[0][0, 2, 0], small[1][0, 2, 0] = k.cpu(), v.cpu()
    o, tol, _, _ = plain.tree(Q, K, V, *small, ints([[0, 0, 40]]))
    near(got, o, tol)
    # the same at the other end of one long cache: zero keys and values before the last 40
    Kc[0, 2, 0, -40:], Vc[0, 2, 0, -40:] = k, v
    Kc[0, 2, 0, :40] = 0
    Vc[0, 2, 0, :40] = 0
    got = nf.attention_tree(Q, K, V, Kc, Vc, ints([[0, 0, C]]), scale=40.0 * d ** -0.5).cpu().double()
    q, kd, vd = Q[0, 2].cpu().double(), torch.cat((k, K[0, 2:3])).cpu().double(), torch.cat((v, V[0, 2:3])).cpu().double()
    s = kd @ q * 40.0 * d ** -0.5
    assert float(s.max()) > 40                                # e^40 against 6e6 keys of score 0: they do not count
    p = torch.softmax(s, 0)
    near(got[0, 2], p @ vd, (2 * (d + 2) * 2.0 ** -24 * 40 * float((kd.abs() @ q.abs()).max()) * d ** -0.5 + 2.0 ** -7) * (p @ vd.abs()) + 2.0 ** -8 * (p @ vd).abs())


# ------------------------------------------------------------------------------------------------------------------------ the cache
@pytest.mark.parametrize("d", [3, 20, 64, 128])
@pytest.mark.parametrize("T,n", [(1, None), (7, None), (26, 5), (300, None)])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_append(nf, dtype, T, n, d):
    g = gen(T)
    M, B, kv, C = 2, 3, 3, 310
    _, K, V = rows(g, M, B * T, 1, kv, d, dtype)
    Kc, Vc = cache(g, M, B, kv, C, d, dtype)
    pos, weight = ints(torch.randint(0, 99, (M, B, kv, C), generator=g)), torch.rand(M, B, kv, C, generator=g).cuda()
    length, count = ints([[0, 3, 305], [310, -2, 9]]), ints([[1, 400, T], [4, 2, 0]])
    index = None if n is None else ints(torch.randint(-1, T + 1, (M, B, n), generator=g))
    for kw in (dict(), dict(count=count), dict(start=ints([[0, 9, 1000], [5, 6, 7]]), count=count)):
        a, b, p, w = Kc.clone(), Vc.clone(), pos.clone(), weight.clone()
        nf.cache_append(K, V, a, b, p, w, length, index=index, **kw)
        want = plain.append(K, V, Kc, Vc, pos, weight, length, index=index, **kw)
        for x, y in zip((a, b, p, w), want):
            assert torch.equal(x.cpu(), y)
    a, b = Kc.clone(), Vc.clone()
    nf.cache_append(K.contiguous(), V.contiguous(), a, b, None, None, length, index=index)
    want = plain.append(K, V, Kc, Vc, None, None, length, index=index)
    assert torch.equal(a.cpu(), want[0]) and torch.equal(b.cpu(), want[1])


@pytest.mark.parametrize("heads,kv,d,C,T,n", [(4, 2, 64, 200, 6, 4), (1, 1, 64, 65, 1, None), (8, 1, 128, 300, 3, None), (6, 2, 80, 129, 20, 9), (12, 12, 64, 64, 2, 2),
                                              (4, 4, 20, 70, 5, 5), (3, 1, 7, 33, 4, None), (16, 1, 256, 130, 33, 33), (64, 1, 32, 96, 64, 40)])
@pytest.mark.parametrize("cap", [0.0, 3.0])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_weigh(nf, dtype, cap, heads, kv, d, C, T, n):
    g = gen(C + T)
    M, B = 2, 2
    Q, K, V = rows(g, M, B * T, heads, kv, d, dtype)
    Kc, _ = cache(g, M, B, kv, C, d, dtype)
    rows_n = T if n is None else n
    length = [[C - rows_n, 0], [C // 2, C]]
    count = ints([[rows_n, rows_n], [max(1, rows_n - 1), 2]])
    for m in range(M):
        for b in range(B):
            Kc[m, b, :, length[m][b] + int(count[m, b]):] = float("nan")
    index = None if n is None else torch.stack([torch.randperm(T, generator=g)[:n].sort().values for _ in range(M * B)]).view(M, B, n)
    if n is not None and n > 3:
        index[0, 0, 1] = T                                    # no such row
    index = None if n is None else ints(index)
    pos = ints(torch.randint(0, 4000, (M, B, kv, C), generator=g))
    weight = torch.rand(M, B, kv, C, generator=g).cuda()
    lse = (torch.rand(M, B * T, heads, generator=g) * 3 + 5).cuda()
    lse[0, 0] = -math.inf                                     # a row that saw nothing
    for kw in (dict(), dict(pos=pos, start=ints([[3000, 10], [4000, 77]]), slope=slopes(g, M, heads) * 0.01), dict(slope=slopes(g, M, heads))):
        kw.update(index=index, count=count, cap=cap)
        got = nf.cache_weigh(Q, lse, Kc, weight, ints(length), **kw)
        near(got, *plain.weigh(Q, lse, Kc, weight, ints(length), **kw))
        inplace = weight.clone()
        assert nf.cache_weigh(Q, lse, Kc, inplace, ints(length), out=inplace, **kw) is inplace
        assert torch.equal(inplace, got)


@pytest.mark.parametrize("C,budget", [(1, 1), (2, 1), (65, 64), (100, 37), (1030, 1), (1030, 1029), (5000, 700), (9000, 8000)])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (F32, 20), (BF, 3)], ids=str)
def test_evict(nf, dtype, d, C, budget):
    g = gen(C)
    M, B, kv = 1, 3, 2
    Kc, Vc = cache(g, M, B, kv, C, d, dtype)
    weight = torch.rand(M, B, kv, C, generator=g).square()
    weight[torch.rand(M, B, kv, C, generator=g) < 0.3] = 0.0   # many ties
    weight[0, 0, 0, ::5] = -0.0
    weight = weight.cuda()
    pos = ints(torch.stack([torch.randperm(C, generator=g) for _ in range(M * B * kv)]).view(M, B, kv, C))
    length = ints([[C, max(budget - 1, 0), (C + budget) // 2]])
    for kw in (dict(), dict(recent=min(30, C)), dict(recent=C), dict(recent=5, start=ints([[C + 2, 7, C - 3]]))):
        want = plain.evict(Kc, Vc, pos, weight, length, budget, **kw)
        a, b, p, w = Kc.clone(), Vc.clone(), pos.clone(), weight.clone()
        nf.cache_evict(a, b, p, w, length, budget, **kw)
        for x, y in zip((a, b, p, w), want):
            assert torch.equal(x.cpu(), y)
        a, b, p, w = Kc.clone(), Vc.clone(), torch.full_like(pos, -7), torch.full_like(weight, -7.0)
        out = nf.cache_evict(a, b, pos, weight, length, budget, pos_out=p, weight_out=w, **kw)
        assert out[0] is p and out[1] is w
        held = torch.minimum(length.cpu(), torch.tensor(budget))
        stay = torch.arange(C) < held[..., None]
        for x, y, old in ((p, want[2], -7), (w, want[3], -7.0)):
            assert torch.equal(x.cpu(), torch.where(stay[:, :, None].expand(y.shape), y, torch.full_like(y, old)))
        assert torch.equal(a.cpu(), want[0]) and torch.equal(b.cpu(), want[1])
    a, b, w = Kc.clone(), Vc.clone(), weight.clone()
    nf.cache_evict(a, b, None, w, length, budget)             # without positions
    want = plain.evict(Kc, Vc, None, weight, length, budget)
    assert torch.equal(a.cpu(), want[0]) and torch.equal(b.cpu(), want[1]) and torch.equal(w.cpu(), want[3])


@pytest.mark.parametrize("C,budget", [(3000, 1000), (20000, 3000), (32769, 32000), (40001, 17)])
def test_evict_long(nf, C, budget):
    test_evict(nf, BF, 8, C, budget)


def test_evict_odd_weights(nf):
    """NaN counts as the largest, infinities and negative numbers in their order, equal ones by slot."""
    w = torch.tensor([math.nan, 1.0, -2.0, math.inf, 0.0, -0.0, 1e-40, -1e-40, 1.0, -math.inf, 5.0, -math.nan]).view(1, 1, 1, 12)
    K = torch.arange(12.0).view(1, 1, 1, 12, 1).repeat(1, 1, 1, 1, 4)
    for budget in range(1, 13):
        a, b, x = K.cuda(), (-K).cuda(), w.cuda()
        nf.cache_evict(a, b, None, x, ints([[12]]), budget)
        want = plain.evict(K, -K, None, w, ints([[12]]), budget)
        assert torch.equal(a.cpu(), want[0]) and torch.equal(b.cpu(), want[1])


# ------------------------------------------------------------------------------------------------------------------------- together
def decode(nf, g, dtype, steps, budget, stream=None):
    """Prompts, then steps of drafting, accepting, weighing and evicting; every result against the definitions on the same state."""
    M, B, S, heads, kv, d, C, T, n = 2, 2, 50, 4, 2, 64, 96, 6, 3
    slope, cap = slopes(g, M, heads) * 0.1, 6.0
    plens = ints([[50, 33], [1, 47]])
    Q, K, V = rows(g, M, B * S, heads, kv, d, dtype)
    got = nf.attention_prompt(Q, K, V, B, S, heads, kv, slope=slope, cap=cap, length=plens)
    near(got, *plain.prompt(Q, K, V, B, S, heads, kv, slope=slope, cap=cap, length=plens))
    Kc, Vc = torch.full((M, B, kv, C, d), math.nan, dtype=dtype, device="cuda"), torch.full((M, B, kv, C, d), math.nan, dtype=dtype, device="cuda")
    pos, weight = torch.full((M, B, kv, C), -1, dtype=torch.int32, device="cuda"), torch.full((M, B, kv, C), math.nan, device="cuda")
    length = torch.zeros_like(plens)
    start = length.clone()
    nf.cache_append(K, V, Kc, Vc, pos, weight, length, count=plens)
    length += plens
    start += plens
    for _ in range(steps):
        Q, K, V = rows(g, M, B * T, heads, kv, d, dtype)
        parent = ints([[[-1, 0, 0, 1, 3, 2], [-1, 0, 1, 2, 3, 4]]] * M)
        lse = torch.empty(M, B * T, heads, device="cuda")
        kw = dict(start=start, pos=pos, slope=slope, cap=cap)
        want = plain.tree(Q, K, V, Kc, Vc, length, parent=parent, **kw)
        got = nf.attention_tree(Q, K, V, Kc, Vc, length, parent=parent, lse=lse, **kw)
        near(got, want[0], want[1])
        near(lse, want[2], want[3])
        index, count = ints([[[0, 1, 3], [0, 1, 2]]] * M), ints([[3, 1], [2, 3]])
        after = plain.append(K, V, Kc, Vc, pos, weight, length, start=start, index=index, count=count)
        nf.cache_append(K, V, Kc, Vc, pos, weight, length, start=start, index=index, count=count)
        for x, y in zip((Kc, Vc, pos, weight), after):
            assert torch.equal(x.cpu().nan_to_num(-1.0), y.nan_to_num(-1.0))
        held = torch.arange(C)[None, None, None] < (length + count).cpu()[..., None, None].expand(M, B, kv, 1)
        w, tol = plain.weigh(Q, lse, Kc, weight, length, index=index, count=count, **kw)
        nf.cache_weigh(Q, lse, Kc, weight, length, index=index, count=count, out=weight, **kw)
        near(torch.where(held, weight.cpu(), 0.0), torch.where(held, w, 0.0), tol.nan_to_num(1.0))
        # an accepted row's weights over its path and the cache add up to 1 for each of its heads
        length += count
        start += count
        after = plain.evict(Kc, Vc, pos, weight, length, budget, start=start, recent=8)
        nf.cache_evict(Kc, Vc, pos, weight, length, budget, start=start, recent=8)
        for x, y in zip((Kc, Vc, pos, weight), after):
            assert torch.equal(x.cpu().nan_to_num(-1.0), y.nan_to_num(-1.0))
        length.clamp_(max=budget)
    for m in range(M):                                        # every entry is a different token that has been seen, the latest 8 among them
        for b in range(B):
            for h in range(kv):
                p = pos[m, b, h, :int(length[m, b])].tolist()
                assert len(set(p)) == len(p) and max(p) == int(start[m, b]) - 1
                assert set(range(max(0, int(start[m, b]) - 8), int(start[m, b]))) <= set(p)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_a_run_of_all_together(nf, dtype):
    decode(nf, gen(20), dtype, steps=4, budget=40)


def test_single_tokens_give_what_a_prompt_gives(nf):
    """The rows of a prompt one after the other over a cache, against the prompt's attention: both near the same exact rows."""
    g = gen(21)
    M, B, S, heads, kv, d = 2, 1, 70, 4, 2, 64
    Q, K, V = rows(g, M, B * S, heads, kv, d, F32)
    s = slopes(g, M, heads) * 0.2
    ref, tol = plain.prompt(Q, K, V, B, S, heads, kv, slope=s, cap=5.0)
    near(nf.attention_prompt(Q, K, V, B, S, heads, kv, slope=s, cap=5.0), ref, tol)
    Kc, Vc = torch.zeros(M, B, kv, S, d, device="cuda"), torch.zeros(M, B, kv, S, d, device="cuda")
    length = torch.zeros(M, B, dtype=torch.int32, device="cuda")
    for i in range(S):
        q, k, v = Q[:, i:i + 1], K[:, i:i + 1], V[:, i:i + 1]
        near(nf.attention_tree(q, k, v, Kc, Vc, length, slope=s, cap=5.0), ref[:, i:i + 1], tol[:, i:i + 1], "row %d" % i)
        nf.cache_append(k, v, Kc, Vc, None, None, length)
        length += 1


def test_last_rows_as_a_chain_weigh_the_prompt(nf):
    """The weights that a prompt's last rows give: those rows as a chain over the rows before them; each row's weights add up to 1 per head."""
    g = gen(22)
    S, W, heads, kv, d = 120, 10, 4, 2, 64
    Q, K, V = rows(g, 1, S, heads, kv, d, BF)
    Kc, Vc = torch.zeros(1, 1, kv, S, d, dtype=BF, device="cuda"), torch.zeros(1, 1, kv, S, d, dtype=BF, device="cuda")
    weight, length = torch.zeros(1, 1, kv, S, device="cuda"), ints([[S - W]])
    nf.cache_append(K[:, :S - W], V[:, :S - W], Kc, Vc, None, weight, ints([[0]]))
    lse = torch.empty(1, W, heads, device="cuda")
    last = Q[:, S - W:], K[:, S - W:], V[:, S - W:]
    o = nf.attention_tree(*last, Kc, Vc, length, lse=lse)
    want, tol = plain.prompt(Q, K, V, 1, S, heads, kv)
    near(o, want[:, S - W:], tol[:, S - W:])
    nf.cache_append(last[1], last[2], Kc, Vc, None, weight, length)
    nf.cache_weigh(last[0], lse, Kc, weight, length, out=weight)
    total = weight.cpu().double().sum(-1)
    assert ((total - W * heads / kv).abs() < W * heads / kv * 1e-4).all()


# ------------------------------------------------------------------------------------------------------------ streams, graphs, users
def step_calls(nf, s):
    o = nf.attention_tree(s["Q"], s["K"], s["V"], s["Kc"], s["Vc"], s["length"], parent=s["parent"], pos=s["pos"], slope=s["slope"], cap=5.0, lse=s["lse"], start=s["start"], out=s["O"])
    nf.cache_append(s["K"], s["V"], s["Kc"], s["Vc"], s["pos"], s["weight"], s["length"], start=s["start"], index=s["index"])
    nf.cache_weigh(s["Q"], s["lse"], s["Kc"], s["weight"], s["length"], start=s["start"], index=s["index"], pos=s["pos"], slope=s["slope"], cap=5.0, out=s["weight"])
    s["length"] += s["index"].shape[2]
    s["start"] += s["index"].shape[2]
    nf.cache_evict(s["Kc"], s["Vc"], s["pos"], s["weight"], s["length"], s["budget"], start=s["start"], recent=4)
    s["length"].clamp_(max=s["budget"])
    return o


def step_state(g, dtype=BF, C=3000, budget=2990, M=1, B=2, T=5):
    heads, kv, d = 4, 2, 64
    Q, K, V = rows(g, M, B * T, heads, kv, d, dtype)
    Kc, Vc = cache(g, M, B, kv, C, d, dtype)
    pos = ints(torch.arange(C).expand(M, B, kv, C).contiguous())
    return dict(Q=Q, K=K, V=V, Kc=Kc, Vc=Vc, pos=pos, weight=torch.rand(M, B, kv, C, generator=g).cuda(), length=ints([[budget, budget // 2]] * M), start=ints([[budget, budget // 2]] * M),
                parent=random_parents(g, M, B, T), slope=slopes(g, M, heads) * 0.01, lse=torch.empty(M, B * T, heads, device="cuda"), index=ints([[[0, 2], [1, 3]]] * M), budget=budget,
                O=torch.empty(M, B * T, heads * d, dtype=dtype, device="cuda"))


def copied(s):
    return {k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()}


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_captured_steps_replay_as_eager_ones(nf, dtype):
    """A captured step, replayed on the state that it changes, with eager steps of another state between the replays."""
    s = step_state(gen(30), dtype)
    eager, other = copied(s), copied(s)
    step_calls(nf, copied(s))                                 # what a first call does is done
    torch.cuda.synchronize()
    fresh, graph = copied(s), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_calls(nf, s)
    for k, v in fresh.items():
        if torch.is_tensor(v):
            s[k].copy_(v)
    for _ in range(4):
        q = torch.randn(s["Q"].shape, generator=gen(31)).to(dtype).cuda()
        s["Q"].copy_(q)
        eager["Q"].copy_(q)
        graph.replay()
        want = step_calls(nf, eager)
        step_calls(nf, other)
        torch.cuda.synchronize()
        assert torch.equal(s["O"], want)
        for k in ("Kc", "Vc", "pos", "weight", "length"):
            assert torch.equal(s[k], eager[k]), k


def test_two_streams_at_once(nf):
    """Two states on two streams, each call with a workspace of its own, against the same calls one after the other."""
    a, b = step_state(gen(32)), step_state(gen(33), F32)
    want = []
    for s in (copied(a), copied(b)):
        for _ in range(3):
            step_calls(nf, s)
        want.append(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                step_calls(nf, s)
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        for k in ("O", "Kc", "Vc", "pos", "weight"):
            assert torch.equal(s[k], w[k]), k


def test_a_given_stream(nf):
    """stream=: the call runs there, and so does what its results wait for."""
    s = step_state(gen(34))
    want = nf.attention_tree(s["Q"], s["K"], s["V"], s["Kc"], s["Vc"], s["length"])
    p = nf.attention_prompt(s["Q"], s["K"], s["V"], 2, 5, 4, 2)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = nf.attention_tree(s["Q"], s["K"], s["V"], s["Kc"], s["Vc"], s["length"], stream=st)
    pg = nf.attention_prompt(s["Q"], s["K"], s["V"], 2, 5, 4, 2, stream=st)
    st.synchronize()
    assert torch.equal(got, want) and torch.equal(pg, p)


def test_a_workspace_of_the_caller(nf):
    s = step_state(gen(35))
    need = nf.attention_tree_workspace(1, 2, 5, 3000, 4, 2, 64, BF)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    args = (s["Q"], s["K"], s["V"], s["Kc"], s["Vc"], s["length"])
    assert torch.equal(nf.attention_tree(*args, workspace=ws), nf.attention_tree(*args))
    if need > 16:
        with pytest.raises(nf.NetFuseError):
            nf.attention_tree(*args, workspace=ws[:16])
    need = nf.cache_evict_workspace(1, 2, 3000, 2, 2000)
    with pytest.raises(nf.NetFuseError):
        nf.cache_evict(s["Kc"], s["Vc"], s["pos"], s["weight"], s["length"], 2000, workspace=torch.empty(need - 4, dtype=torch.uint8, device="cuda"))
