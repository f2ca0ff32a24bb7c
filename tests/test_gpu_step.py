"""What surrounds the decoders' attention against plain 64-bit implementations: heads normed and rotated, caches of 4 bits written, read and attended to, log probabilities."""
import math

import pytest
import torch

import decoder_plain as DP
import step_plain as P

pytestmark = pytest.mark.gpu
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


# ------------------------------------------------------------------------------------------------------------------------------------ rotate
#       M  B  S  heads kv  d   rot  sections       inter  norm  positions   lengths
ROTATE = [
    (2, 2, 3, 4, 2, 64, 64, None, False, True, "start", False),
    (1, 1, 1, 1, 1, 128, 128, None, False, False, "none", False),
    (3, 2, 5, 12, 12, 64, 32, None, False, True, "start", True),
    (2, 1, 7, 8, 2, 128, 128, [16, 24, 24], False, True, "pos", True),
    (2, 3, 4, 3, 1, 128, 64, [0, 20, 12], True, False, "pos", False),
    (1, 2, 9, 32, 8, 128, 128, None, True, True, "pos", False),
    (2, 2, 3, 5, 3, 80, 80, [8, 16, 16], False, True, "pos", False),
    (2, 2, 3, 5, 3, 80, 40, None, False, True, "far", False),        # turned features that are no whole pieces
    (1, 2, 3, 2, 1, 256, 256, [32, 32, 32, 32], False, True, "pos", False),
    (1, 2, 3, 2, 2, 33, 32, None, True, True, "start", True),        # odd rows
    (1, 1, 2, 3, 3, 8, 8, None, True, False, "far", False),
    (2, 1, 3, 2, 1, 16, 0, None, False, True, "none", False),        # norms alone
    (1, 1, 4, 70, 3, 16, 16, None, False, True, "start", False),     # many small heads
    (1, 1, 3, 2, 2, 2, 2, None, False, True, "far", False),
    (2, 2, 3, 2, 0, 64, 64, None, False, True, "start", False),      # queries alone
    (1, 1, 2, 1, 1, 1, 0, None, False, True, "none", False),
]


def rotate_case(case, dtype, seed=0, packed=True):
    M, B, S, heads, kv, d, rot, sections, inter, norm, where, lengths = case
    g = gen(seed)
    x = (torch.randn(M, B * S, (heads + 2 * kv) * d + 8, generator=g) * 3).to(dtype).cuda()
    Q, K = x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d]
    if not packed:
        Q, K = Q.contiguous(), K.contiguous()
    freq = (10000.0 ** (-torch.arange(rot // 2).double() / max(1, rot // 2))).float().cuda() if rot else None
    gammas = [1 + 0.3 * torch.randn(M, d, generator=g).cuda() for _ in range(2)] if norm else [None, None]
    kw = dict(freq=freq, gamma_q=gammas[0], gamma_k=gammas[1], sections=sections, interleaved=inter)
    top = 2 ** 31 - 1 if where == "far" else 5000
    if where in ("pos", "far"):
        kw["pos"] = torch.randint(-top if where == "far" else 0, top, (M, B, S) + ((len(sections),) if sections else ()), generator=g, dtype=torch.int64).to(I32).cuda()
    if where == "start":
        kw["start"] = torch.randint(0, 100000, (M, B), generator=g).to(I32).cuda()
    if lengths:
        kw["length"] = torch.randint(0, S + 2, (M, B), generator=g).to(I32).cuda()
    return Q, (K if kv else None), B, S, heads, kv, kw


def check_rotate(case, dtype, Q, K, kw, got_q, got_k, before_q=None, before_k=None):
    M, B, S, heads, kv, d = case[:6]
    L = kw.get("length")
    there = torch.ones(M, B * S, 1, dtype=torch.bool) if L is None else (torch.arange(S) < L.cpu()[..., None]).view(M, B * S, 1)
    for x, n, gamma, got, before in ((Q, heads, kw["gamma_q"], got_q, before_q), (K, kv, kw["gamma_k"], got_k, before_k)):
        if x is None:
            assert got is None
            continue
        want, tol = P.rotate(x, B, S, n, kw["freq"], gamma, kw.get("pos"), kw.get("start"), kw["sections"], kw["interleaved"], 1e-6)
        rest = torch.zeros_like(want) if before is None else before.cpu().double()
        P.near(got, torch.where(there, want, rest), torch.where(there, tol, 0.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", ROTATE, ids=lambda c: "M%d-B%d-S%d-h%d-%d-d%d-r%d-%s-%d%d-%s%d" % c)
def test_rotate(nf, case, dtype):
    Q, K, B, S, heads, kv, kw = rotate_case(case, dtype)
    q, k = nf.rotate_heads(Q, K, B, S, heads, kv, **kw)
    check_rotate(case, dtype, Q, K, kw, q, k)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", [ROTATE[i] for i in (0, 2, 3, 5, 7, 9)], ids=lambda c: "d%d-r%d" % (c[5], c[6]))
def test_rotate_in_place(nf, case, dtype):
    """Queries and keys of one packed projection, turned where they are: the rest of it stays."""
    Q, K, B, S, heads, kv, kw = rotate_case(case, dtype, 1)
    whole = Q._base
    before = whole.clone()
    q, k = nf.rotate_heads(Q, K, B, S, heads, kv, out_q=Q, out_k=K, **kw)
    assert q is Q and k is K
    n, d = heads + kv, case[5]
    check_rotate(case, dtype, before[:, :, :heads * d], before[:, :, heads * d:n * d], kw, q, k, before[:, :, :heads * d], before[:, :, heads * d:n * d])
    assert torch.equal(whole[:, :, n * d:], before[:, :, n * d:])


@pytest.mark.parametrize("case", [ROTATE[i] for i in (0, 3, 7)], ids=lambda c: "d%d-r%d" % (c[5], c[6]))
def test_rotate_into_rows_of_a_larger_tensor(nf, case):
    Q, K, B, S, heads, kv, kw = rotate_case(case, BF, 2)
    M, d = case[0], case[5]
    into = torch.full((M, B * S, (heads + kv) * d + 5), 7.0, dtype=BF, device="cuda")
    oq, ok = into[:, :, 2:2 + heads * d], into[:, :, 2 + heads * d:2 + (heads + kv) * d]          # rows that start anywhere
    before = into.clone()
    nf.rotate_heads(Q, K, B, S, heads, kv, out_q=oq, out_k=ok, **kw)
    check_rotate(case, BF, Q, K, kw, oq, ok, before[:, :, 2:2 + heads * d], before[:, :, 2 + heads * d:2 + (heads + kv) * d])
    assert bool((into[:, :, :2] == 7).all()) and bool((into[:, :, 2 + (heads + kv) * d:] == 7).all())


def test_rotate_of_the_last_positions(nf):
    """A start so far that its rows' positions leave 32 bits goes on counting."""
    Q, freq = torch.randn(1, 4, 32, device="cuda"), torch.tensor([1.0] + [0.01] * 15, device="cuda")
    start = 2 ** 31 - 2
    q, _ = nf.rotate_heads(Q, None, 1, 4, 1, freq=freq, start=ints([[start]]))
    where = (start + torch.arange(4)).double()
    angle = where[:, None] * freq.cpu().double()
    a, b = Q[0].cpu().double().chunk(2, 1)
    want = torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), 1)
    room = (a.abs() + b.abs()) * (2.0 ** -21 + 2.0 ** -23 + 2.0 ** -51 * angle)
    P.near(q[0], want, torch.cat((room, room), 1) + 2.0 ** -24 * want.abs())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotate_of_large_results(nf, dtype):
    """Rows of more than 32 MB, which are stored past the caches, are those that calls of fewer tokens give; in place and into tensors of their own."""
    S, heads, kv, d, cut = 2100, 40, 24, 128, 1050
    Q, K, _, _, _, _, kw = rotate_case((2, 1, S, heads, kv, d, d, None, False, True, "start", False), dtype)
    Q, K = Q.contiguous(), K.contiguous()
    q, k = nf.rotate_heads(Q, K, 1, S, heads, kv, **kw)
    for at in (0, cut):
        part = dict(kw, start=kw["start"] + at)
        one = nf.rotate_heads(Q[:, at:at + cut], K[:, at:at + cut], 1, cut, heads, kv, **part)
        assert torch.equal(one[0], q[:, at:at + cut]) and torch.equal(one[1], k[:, at:at + cut])
    nf.rotate_heads(Q, K, 1, S, heads, kv, out_q=Q, out_k=K, **kw)
    assert torch.equal(Q, q) and torch.equal(K, k)


def test_rotate_keeps_rows_apart(nf):
    """Infinities and NaN in one head reach no other one; rows past the length are not read into anything."""
    case = (2, 2, 4, 4, 2, 64, 32, None, False, True, "start", True)
    Q, K, B, S, heads, kv, kw = rotate_case(case, F32, 3, packed=False)
    kw["length"] = ints([[2, 4], [0, 3]])
    want = nf.rotate_heads(Q, K, B, S, heads, kv, **kw)
    Q2, K2 = Q.clone(), K.clone()
    Q2[0, 0, :64] = math.nan                                          # head 0 of a row
    Q2[0, 2:4] = math.inf                                             # past a length
    K2[1, :4] = math.nan                                              # a sequence of no tokens
    got = nf.rotate_heads(Q2, K2, B, S, heads, kv, **kw)
    assert torch.isnan(got[0][0, 0, :64]).all()
    got[0][0, 0, :64] = want[0][0, 0, :64]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rotate_turns_nothing_past_rot(nf):
    """An infinity among the features that are not turned stays one and reaches no other feature."""
    Q = torch.randn(1, 3, 2 * 64, device="cuda")
    Q[0, :, 40] = math.inf
    freq = torch.rand(16, device="cuda")
    clean = Q.clone()
    clean[0, :, 40] = 0.0
    q, _ = nf.rotate_heads(Q, None, 1, 3, 2, freq=freq)
    want, _ = nf.rotate_heads(clean, None, 1, 3, 2, freq=freq)
    assert bool((q[0, :, 40] == math.inf).all())
    q[0, :, 40] = 0.0
    assert torch.equal(q, want)


def test_rotate_far_positions_agree_with_a_difference_of_angles(nf):
    """q . k after rotation depends on the distance alone, also where positions are far (float32 angles would be off by whole turns)."""
    d, freq = 64, (10000.0 ** (-torch.arange(32).double() / 32)).float().cuda()
    q, k = torch.randn(1, 1, d, device="cuda"), torch.randn(1, 1, d, device="cuda")
    score = lambda p, r: float((nf.rotate_heads(q, None, 1, 1, 1, freq=freq, start=ints([[p]]))[0].double() * nf.rotate_heads(k, None, 1, 1, 1, freq=freq, start=ints([[r]]))[0].double()).sum())  # noqa: E731
    room = 4 * 2.0 ** -20 * float(q.norm() * k.norm())                # both rows: cosines within 2^-21, angles of 2^24 within 2^-27
    for base in (0, 1 << 16, (1 << 24) + 1):
        assert abs(score(base + 9, base + 2) - score(9, 2)) <= room


# --------------------------------------------------------------------------------------------------------------------------------------- fp4
def spread(g, shape, dtype):
    """Values of many sizes: groups of all exponents, zeros, values halfway between codes, largest ones at 6 and 7 times a power of two."""
    x = torch.randn(shape, generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-6, 7, shape[:-1] + (1,), generator=g).double())
    edge = torch.tensor([0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -5.0, -2.5, 0.2490234375, 7.03125, -7.0], dtype=torch.float64)
    pick = torch.randint(0, 16, shape, generator=g)
    return torch.where(torch.rand(shape, generator=g, dtype=torch.float64) < 0.4, edge[pick], x).to(dtype)


#       M  B  T  n  C   kv d    index count weights lengths
APPEND = [
    (2, 2, 3, 3, 9, 2, 64, False, False, True, [[0, 4], [6, 9]]),
    (1, 1, 1, 1, 4, 1, 32, False, False, True, [[3]]),
    (2, 1, 5, 2, 8, 3, 128, True, True, True, [[1], [7]]),
    (1, 2, 4, 6, 40, 2, 80, True, True, False, [[0, 30]]),           # three groups, the last of them half, rows taken twice
    (2, 2, 7, 7, 30, 1, 33, False, True, True, [[2, 2], [29, 30]]),  # one feature in the last group
    (1, 1, 200, 200, 256, 4, 128, False, False, True, [[10]]),
    (1, 2, 3, 3, 5, 2, 256, False, False, True, [[1, 2]]),
    (1, 1, 3, 3, 5, 5, 1, False, False, True, [[1]]),
    (1, 1, 9, 9, 12, 1, 96, False, True, True, [[2]]),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", APPEND, ids=lambda c: "M%d-B%d-T%d-n%d-C%d-k%d-d%d" % c[:7])
def test_append_fp4(nf, case, dtype):
    M, B, T, n, C, kv, d, indexed, counted, weighed, lengths = case
    g = gen(sum(case[:7]))
    rows = spread(g, (M, B * T, 2 * kv * d), dtype).cuda()
    K, V = rows[:, :, :kv * d], rows[:, :, kv * d:]
    cache = [torch.randint(0, 256, t.shape, generator=g, dtype=torch.int64).to(U8).cuda() for t in nf.cache_fp4(M, B, kv, C, d)]
    pos = torch.randint(0, 99, (M, B, kv, C), generator=g).to(I32).cuda() if weighed else None
    w = torch.rand(M, B, kv, C, generator=g).cuda() if weighed else None
    L, start = ints(lengths), torch.randint(0, 1000, (M, B), generator=g).to(I32).cuda()
    index = torch.randint(-1, T + 1, (M, B, n), generator=g).to(I32).cuda() if indexed else None
    count = torch.randint(0, n + 2, (M, B), generator=g).to(I32).cuda() if counted else None
    want = [t.cpu().clone() for t in cache]
    want_pos, want_w = (pos.cpu().clone(), w.cpu().clone()) if weighed else (None, None)
    for m in range(M):
        for b in range(B):
            for i in range(n if count is None else min(int(count[m, b]), n)):
                r, slot = (i if index is None else int(index[m, b, i])), lengths[m][b] + i
                if not 0 <= r < T or slot >= C:
                    continue
                for x, codes, scales in ((K, 0, 1), (V, 2, 3)):
                    c, s = P.quantise(x[m, b * T + r].view(kv, d))
                    want[codes][m, b, :, slot], want[scales][m, b, :, slot] = c, s
                if weighed:
                    want_pos[m, b, :, slot], want_w[m, b, :, slot] = int(start[m, b]) + i, 0.0
    nf.cache_append_fp4(K, V, *cache, pos, w, L, start=start, index=index, count=count)
    for got, exact in zip(cache, want):
        assert torch.equal(got.cpu(), exact)
    if weighed:
        assert torch.equal(pos.cpu(), want_pos) and torch.equal(w.cpu(), want_w)
    k, v = nf.cache_read_fp4(*cache, d, dtype=dtype)
    for got, codes, scales in ((k, 0, 1), (v, 2, 3)):
        exact = P.dequantise(want[codes], want[scales], d).float().to(dtype)
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(exact)) and torch.equal(got.cpu().nan_to_num(), exact.nan_to_num())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_fp4_of_the_types_ends(nf, dtype):
    """Groups of the largest and the smallest numbers, denormal ones, infinities and NaN: each ends with its group."""
    big = torch.finfo(dtype).max
    groups = [[big], [-big, 1.0], [2.0 ** 127, 2.0 ** 125], [7 * 2.0 ** 125], [2.0 ** -126], [2.0 ** -127], [3 * 2.0 ** -127, 2.0 ** -128], [2.0 ** -133], [math.inf, 1.0], [math.nan], [-math.inf], [0.0], [-0.0],
              [1.75], [1.7578125], [3.5, 0.25], [2.0 ** -125, 2.0 ** -127]]
    x = torch.zeros(len(groups), 32, dtype=torch.float64)
    for i, v in enumerate(groups):
        x[i, 3 * i % 29:3 * i % 29 + len(v)] = torch.tensor(v, dtype=torch.float64)
    x[:, 31] = 2.0 ** -140
    rows = x.to(dtype).view(1, 1, -1).cuda()                          # a head of one group each
    kv = len(groups)
    cache = nf.cache_fp4(1, 1, kv, 1, 32)
    nf.cache_append_fp4(rows, rows, *cache, None, None, ints([[0]]))
    codes, scales = P.quantise(rows.cpu().view(kv, 32))
    assert torch.equal(cache[0].cpu().view(kv, 16), codes) and torch.equal(cache[1].cpu().view(kv, 2), scales)
    assert [int(s) for s in scales[8:11, 0]] == [255] * 3 and int(scales[0, 0]) == 252 and int(scales[11, 0]) == 2
    k, v = nf.cache_read_fp4(*cache, 32, dtype=dtype)
    assert torch.isnan(k[0, 0, 8:11]).all() and torch.isfinite(k[0, 0, :8]).all() and torch.equal(k.nan_to_num(), v.nan_to_num())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,n,C", [(64, None, 37), (80, 5, 9), (33, 50, 20), (256, 3, 3), (1, 2, 5), (128, 700, 600), (32, 1, 1)])
def test_read_fp4_of_any_bytes(nf, d, n, C, dtype):
    """Every code under every scale; ranges that begin before the cache and end past it."""
    M, B, kv = 2, 2, 3
    g = gen(d + C)
    cache = [torch.randint(0, 256, t.shape, generator=g, dtype=torch.int64).to(U8).cuda() for t in nf.cache_fp4(M, B, kv, C, d)]
    m = C if n is None else n
    for first, count in ((None, None), (ints([[0, C // 2], [C, -2]]), ints([[m, m // 2], [3, m + 7]])), (None, ints([[0, 1], [-5, m]]))):
        k, v = nf.cache_read_fp4(*cache, d, n=n, first=first, count=count, dtype=dtype)
        for got, codes, scales in ((k, 0, 1), (v, 2, 3)):
            all_of = P.dequantise(cache[codes], cache[scales], d).float().to(dtype)
            want = torch.zeros(M, B, kv, m, d, dtype=dtype)
            for a in range(M):
                for b in range(B):
                    for i in range(m if count is None else min(max(int(count[a, b]), 0), m)):
                        slot = i + (0 if first is None else int(first[a, b]))
                        if 0 <= slot < C:
                            want[a, b, :, i] = all_of[a, b, :, slot]
            assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want)) and torch.equal(got.cpu().nan_to_num(0.0), want.nan_to_num(0.0))
        only, none = nf.cache_read_fp4(cache[0], cache[1], None, None, d, n=n, first=first, count=count, dtype=dtype)
        assert none is None and torch.equal(only.view(I32 if dtype == F32 else torch.int16), k.view(I32 if dtype == F32 else torch.int16))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_read_fp4_of_large_results(nf, dtype):
    """Entries of more than 32 MB, which are stored past the caches, are those that calls of fewer entries give."""
    M, B, kv, C, d = 2, 2, 4, 2500, 128
    g = gen(8)
    cache = [torch.randint(0, 252, t.shape, generator=g, dtype=torch.int64).to(U8).cuda() for t in nf.cache_fp4(M, B, kv, C, d)]
    count = ints([[2500, 7], [0, 1999]])
    k, v = nf.cache_read_fp4(*cache, d, count=count, dtype=dtype)
    for at in range(0, C, 500):
        few = nf.cache_read_fp4(*cache, d, n=500, first=torch.full((M, B), at, dtype=I32, device="cuda"), count=(count - at).clamp(0, 500), dtype=dtype)
        for got, want in zip(few, (k, v)):
            assert torch.equal(got, want[:, :, :, at:at + 500])


def test_fp4_rows_past_four_gigabytes(nf):
    """A cache whose offsets pass 32 bits: entries at its end are written and read there."""
    M, B, kv, d = 1, 1, 1, 128
    C = (1 << 32) // 64 + 1000
    cache = [torch.empty(t, dtype=U8, device="cuda") for t in ((M, B, kv, C, 64), (M, B, kv, C, 4))]
    cache = cache + cache                                             # values where the keys are: the same rows
    x = torch.randn(1, 8, d, device="cuda")
    nf.cache_append_fp4(x, x, *cache, None, None, ints([[C - 8]]))
    k, _ = nf.cache_read_fp4(cache[0], cache[1], None, None, d, n=8, first=ints([[C - 8]]), dtype=F32)
    assert torch.equal(k.cpu().double().view(8, d), P.dequantise(*P.quantise(x[0]), d))


# -------------------------------------------------------------------------------------------------------------------------------------- tree
#       M  B  T  C    heads kv d  cap  slope pos   start nodes parent lengths
TREE = [
    (2, 2, 1, 40, 4, 2, 64, 0.0, False, False, False, False, "chain", [[40, 0], [1, 17]]),
    (1, 2, 5, 70, 8, 2, 128, 0.0, True, True, True, True, "tree", [[70, 33]]),
    (2, 1, 7, 130, 2, 2, 32, 20.0, False, False, True, False, "tree", [[129], [64]]),
    (1, 1, 26, 700, 8, 2, 128, 50.0, False, False, True, False, "tree", [[699]]),
    (1, 2, 64, 100, 2, 1, 64, 0.0, True, False, False, True, "tree", [[100, 31]]),
    (1, 1, 3, 90, 6, 3, 80, 15.0, True, True, True, False, "tree", [[77]]),
    (1, 1, 2, 33, 3, 3, 33, 0.0, True, False, False, False, "chain", [[20]]),       # rows of an odd size
    (1, 1, 4, 50, 4, 1, 256, 0.0, True, True, False, False, "tree", [[50]]),
    (1, 1, 13, 60, 8, 2, 256, 30.0, False, False, False, True, "tree", [[48]]),
    (1, 1, 1, 2100, 4, 1, 128, 0.0, True, False, False, False, "chain", [[2099]]),  # several chunks of a cache
    (2, 1, 1, 1500, 2, 2, 64, 10.0, False, True, True, False, "chain", [[1400], [3]]),
    (1, 1, 40, 2500, 4, 1, 128, 0.0, True, True, True, False, "tree", [[2500]]),
    (1, 1, 20, 1300, 4, 1, 64, 0.0, False, False, False, False, "roots", [[1111]]),
    (1, 1, 8, 1100, 8, 2, 128, 0.0, False, False, False, False, "chain", [[1100]]),
    (1, 1, 9, 600, 4, 2, 64, 5.0, True, False, False, True, "tree", [[600]]),
    (1, 1, 1, 64, 1, 1, 8, 0.0, False, False, False, False, "chain", [[0]]),         # the token alone
    (1, 1, 10, 300, 2, 2, 96, 0.0, False, False, False, False, "tree", [[257]]),
    (1, 1, 17, 1030, 8, 4, 40, 0.0, True, False, False, False, "tree", [[1030]]),
    (1, 1, 1, 90, 2, 2, 36, 0.0, True, False, False, False, "chain", [[88]]),       # features that are no whole pieces of bfloat16
    (1, 1, 6, 200, 4, 1, 132, 9.0, False, True, True, False, "tree", [[177]]),
    (1, 1, 3, 150, 2, 1, 200, 0.0, True, True, False, False, "tree", [[149]]),      # seven groups
    (1, 1, 30, 300, 4, 1, 168, 0.0, True, False, False, False, "tree", [[291]]),    # six groups, many rows
    (1, 1, 35, 1100, 2, 1, 64, 0.0, False, True, True, False, "tree", [[1029]]),
]


def tree_case(nf, case, dtype, seed=0, packed=True):
    M, B, T, C, heads, kv, d, cap, biased, posed, started, noded, parents, lengths = case
    g = gen(seed + sum(case[:7]))
    x = torch.randn(M, B * T, (heads + 2 * kv) * d, generator=g)
    x[:, :, :heads * d] *= 1.5
    x = x.to(dtype).cuda()
    rows = [x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d], x[:, :, (heads + kv) * d:]]
    if not packed:
        rows = [t.contiguous() for t in rows]
    cache = []
    for _ in range(2):
        codes, scales = P.quantise(torch.randn(M, B, kv, C, d, generator=g))
        cache += [codes.contiguous().cuda(), scales.contiguous().cuda()]
    kw = dict(cap=cap)
    if biased:
        kw["slope"] = (torch.rand(M, heads, generator=g) * 0.2).cuda()
    if posed:
        kw["pos"] = torch.randint(0, 3 * C, (M, B, kv, C), generator=g).to(I32).cuda()
    if started:
        kw["start"] = torch.randint(C, 4 * C, (M, B), generator=g).to(I32).cuda()
    if noded:
        kw["nodes"] = torch.randint(0, T + 1, (M, B), generator=g).to(I32).cuda()
    if parents != "chain":
        par = (torch.rand(M, B, T, generator=g) * torch.arange(T)).floor().to(I32) if parents == "tree" else torch.full((M, B, T), -1, dtype=I32)
        par[:, :, 0] = -1
        kw["parent"] = par.cuda()
    return rows, cache, ints(lengths), kw


def check_tree(case, dtype, rows, cache, L, kw, O, lse):
    d = case[6]
    dense = [P.dequantise(cache[i], cache[i + 1], d) for i in (0, 2)]
    want, tol, wl, tl = DP.tree(*rows, *dense, L, **kw)
    P.near(O, want, tol)
    P.near(lse, wl, tl)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", TREE, ids=lambda c: "M%d-B%d-T%d-C%d-h%d-%d-d%d-cap%g-%d%d%d%d-%s" % c[:13])
def test_tree_fp4(nf, case, dtype):
    rows, cache, L, kw = tree_case(nf, case, dtype)
    lse = torch.empty(case[0], case[1] * case[2], case[4], device="cuda")
    O = nf.attention_tree_fp4(*rows, *cache, L, lse=lse, **kw)
    check_tree(case, dtype, rows, cache, L, kw, O, lse)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", [TREE[i] for i in (1, 3, 5, 9, 11)], ids=lambda c: "T%d-C%d-d%d" % (c[2], c[3], c[6]))
def test_tree_fp4_general_kernel_agrees(nf, case, dtype):
    """Rows that start at any element take the general kernel: the same definition."""
    M, B, T, C, heads, kv, d = case[:7]
    rows, cache, L, kw = tree_case(nf, case, dtype, packed=False)
    odd = torch.zeros(M, B * T, (heads + 2 * kv) * d + 3, dtype=dtype, device="cuda")
    at = 1
    moved = []
    for t in rows:
        odd[:, :, at:at + t.shape[2]] = t
        moved.append(odd[:, :, at:at + t.shape[2]])
        at += t.shape[2]
    lse = torch.empty(M, B * T, heads, device="cuda")
    O = nf.attention_tree_fp4(*moved, *cache, L, lse=lse, **kw)
    check_tree(case, dtype, rows, cache, L, kw, O, lse)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 80, 40, 200])
def test_fp4_caches_of_single_models(nf, d, dtype):
    """Slices of a merged cache of odd capacity: each model's is a cache as good as any, and the merged calls are the models' own."""
    M, B, T, C, heads, kv = 3, 1, 2, 37, 4, 2
    case = (M, B, T, C, heads, kv, d, 0.0, True, False, False, False, "chain", [[30], [5], [37]])
    rows, cache, L, kw = tree_case(nf, case, dtype, packed=False)
    O = nf.attention_tree_fp4(*rows, *cache, L, **kw)
    k, v = nf.cache_read_fp4(*cache, d, dtype=dtype)
    after = [t.clone() for t in cache]
    nf.cache_append_fp4(rows[1], rows[2], *after, None, None, L)
    for m in range(M):
        one, held, l = [t[m:m + 1] for t in rows], [t[m:m + 1] for t in cache], L[m:m + 1].clone()
        assert torch.equal(nf.attention_tree_fp4(*one, *held, l, slope=kw["slope"][m:m + 1].clone()), O[m:m + 1])
        k1, v1 = nf.cache_read_fp4(*held, d, dtype=dtype)
        assert torch.equal(k1, k[m:m + 1]) and torch.equal(v1, v[m:m + 1])
    for m in range(M):
        nf.cache_append_fp4(*[t[m:m + 1] for t in rows[1:]], *[t[m:m + 1] for t in cache], None, None, L[m:m + 1].clone())
    for a, b in zip(cache, after):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 256, 80])
def test_tree_fp4_reads_nothing_past_the_length(nf, d, dtype):
    """What lies in other slots (NaN scales here), in nodes that are not there and in positions past the length has no part."""
    for T, C, n in ((1, 300, 130), (12, 700, 513), (30, 1500, 1025)):
        case = (1, 2, T, C, 4, 2, d, 0.0, True, True, True, T > 1, "tree" if T > 1 else "chain", [[n, 3]])
        rows, cache, L, kw = tree_case(nf, case, dtype, packed=False)
        if T > 1:
            kw["nodes"] = ints([[T - 1, 1]])
        want = nf.attention_tree_fp4(*rows, *cache, L, **kw)
        for i in (1, 3):
            cache[i][0, 0, :, n:], cache[i][0, 1, :, 3:] = 255, 255
        for i in (0, 2):
            cache[i][0, 0, :, n:] = 0x77
        kw["pos"][0, 0, :, n:] = -2 ** 31
        if T > 1:
            for t in rows[1:]:
                t[0, T - 1], t[0, T + 1:] = math.nan, math.inf
        assert torch.equal(nf.attention_tree_fp4(*rows, *cache, L, **kw), want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_tree_fp4_groups_that_read_as_nan(nf, dtype):
    """A cached key or value of NaN reaches the rows of its own head and sequence, and the value's NaN its own features alone."""
    case = (1, 2, 3, 200, 4, 2, 64, 0.0, False, False, False, False, "tree", [[200, 150]])
    rows, cache, L, kw = tree_case(nf, case, dtype)
    want = nf.attention_tree_fp4(*rows, *cache, L, **kw).view(1, 2, 3, 4, 64)
    cache[3][0, 1, 1, 149, 1] = 255                                   # a value's second group: features 32 on of heads 2 and 3
    got = nf.attention_tree_fp4(*rows, *cache, L, **kw).view(1, 2, 3, 4, 64)
    assert torch.isnan(got[0, 1, :, 2:, 32:]).all()
    got[0, 1, :, 2:, 32:] = want[0, 1, :, 2:, 32:]
    assert torch.equal(got, want)
    cache[3][0, 1, 1, 149, 1] = 127
    cache[1][0, 0, 0, 7, 0] = 255                                     # a key: rows of heads 0 and 1
    got = nf.attention_tree_fp4(*rows, *cache, L, **kw).view(1, 2, 3, 4, 64)
    assert torch.isnan(got[0, 0, :, :2]).all() and torch.isfinite(got[0, 0, :, 2:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,C,n,d", [(1, 600, 577, 64), (1, 3000, 2900, 128), (12, 1100, 1090, 128), (40, 1400, 1300, 64)])
def test_tree_fp4_bits_of_a_sequence_are_its_own(nf, T, C, n, d, dtype):
    """Neither other models and sequences nor the capacity change a bit."""
    case = (2, 2, T, C, 4, 2, d, 0.0, True, False, False, False, "tree" if T > 1 else "chain", [[n, 5], [C, n // 2]])
    rows, cache, L, kw = tree_case(nf, case, dtype, packed=False)
    all_of = nf.attention_tree_fp4(*rows, *cache, L, **kw).view(2, 2, T, -1)
    one = [t.view(2, 2, T, -1)[0, 0][None].contiguous() for t in rows]
    for room in (n, n + 900):
        mine = []
        for t in cache:
            x = torch.full((1, 1, 2, room, t.shape[-1]), 3, dtype=U8, device="cuda")
            x[:, :, :, :n] = t[0, 0, :, :n]
            mine.append(x)
        own = {k: v for k, v in kw.items() if k == "cap"}
        own["slope"] = kw["slope"][:1]
        if T > 1:
            own["parent"] = kw["parent"][:1, :1].contiguous()
        got = nf.attention_tree_fp4(*one, *mine, ints([[n]]), **own)
        assert torch.equal(got.view(T, -1), all_of[0, 0])


# ---------------------------------------------------------------------------------------------------------------------------------- logprobs
#          M  B  T  V      n  k   scale cap   vocab           nodes
LOGPROBS = [
    (2, 1, 1, 50, 1, 5, 1.0, 0.0, None, None),
    (1, 1, 3, 1, 2, 3, 1.0, 0.0, None, None),                          # one token
    (2, 2, 3, 4096, 1, 20, 0.7, 0.0, None, [[3, 0], [1, 2]]),
    (1, 1, 4, 4097, 3, 32, 1.25, 30.0, None, None),
    (3, 1, 2, 9001, 1, 8, 1.0, 0.0, [9001, 17, 0], None),
    (1, 1, 2, 50001, 4, 20, 1.0, 5.0, None, None),
    (1, 2, 2, 131071, 1, 8, 1.0, 0.0, [130000], [[2, 1]]),
    (1, 1, 5, 777, 0, 1, 1.0, 0.0, None, None),
    (1, 1, 2, 300, 70, 0, 3.0, 0.0, None, None),
    (1, 1, 1, 270001, 1, 32, 1.0, 0.0, None, None),                    # more chunks than lanes
    (1, 1, 1, 20, 0, 0, 1.0, 0.0, None, None),                         # the entropy alone
]


def logprob_case(case, dtype, seed=0):
    M, B, T, V, n, k, scale, cap, vocab, nodes = case
    g = gen(seed + V)
    x = torch.randn(M, B * T, V, generator=g) * 2.5
    x[:, :, V // 3] += 6
    token = torch.randint(-1, V + 1, (M, B * T, n), generator=g).to(I32) if n else None
    if n:
        token[:, :, 0] = V // 3
    return x.to(dtype).cuda(), (token.cuda() if n else None), dict(k=k, scale=scale, cap=cap, vocab=None if vocab is None else ints(vocab), nodes=None if nodes is None else ints(nodes))


def check_logprobs(got, x, token, kw):
    want = P.logprobs(x, token, kw["k"], kw["vocab"], kw["nodes"], kw["scale"], kw["cap"])
    logp, entropy, top, top_logp = got
    assert (logp is None) == (token is None) and (top is None) == (kw["k"] == 0) == (top_logp is None)
    if token is not None:
        P.near(logp, want[0], want[1])
    P.near(entropy, want[2], want[3])
    if kw["k"]:
        assert torch.equal(top.cpu(), want[4])
        P.near(top_logp, want[5], want[6])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", LOGPROBS, ids=lambda c: "M%d-B%d-T%d-V%d-n%d-k%d-s%g-cap%g" % c[:8])
def test_logprobs(nf, case, dtype):
    x, token, kw = logprob_case(case, dtype)
    check_logprobs(nf.token_logprobs(x, token, **kw), x, token, kw)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs_of_equal_logits(nf, dtype):
    """Every logit alike, and many alike at the border of the alternatives: the lower token first, over lanes, pieces and chunks."""
    for V in (33, 5000, 20000):
        x = torch.zeros(1, 3, V, dtype=dtype, device="cuda")
        x[0, 1, 7::5] = 1.0
        x[0, 2, V // 2:] = -0.0
        x[0, 2, V - 1] = 2.0
        token = ints([[[0], [1], [V - 1]]])
        kw = dict(k=20, vocab=None, nodes=None, scale=1.0, cap=0.0)
        check_logprobs(nf.token_logprobs(x, token, **kw), x, token, kw)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 4000])
def test_logprobs_of_floods(nf, dtype, rows):
    """More candidates than a wavefront's list holds, whether it takes one chunk (few rows) or several: equal ones past the border, a few masked rows' lowest values, and
    large ones that lie in a few lanes (those of the same 8 neighbouring tokens of each 512)."""
    V = 9000 if rows == 1 else 13000
    kinds = torch.zeros(4, V)
    kinds[0, ::3] = 1.0
    kinds[0, 4000:4010] = 2.0
    kinds[1] = torch.finfo(dtype).min
    kinds[1, [7, 4500, 8999]] = torch.tensor([1.0, 3.0, 2.0])
    lane = torch.arange(V) % 512 // 8
    kinds[2] = torch.where(lane < 3, 5.0 + torch.rand(V, generator=gen(1)), torch.rand(V, generator=gen(2)))
    kinds[3] = torch.where(lane < 3, 5.0, 1.0)
    x = kinds.to(dtype).cuda()[None].expand(rows, 4, V).reshape(1, 4 * rows, V)
    kw = dict(k=20, vocab=None, nodes=None, scale=1.0, cap=0.0)
    got = nf.token_logprobs(x, **kw)
    for r in (0, rows - 1):
        part = [None if t is None else t[:, 4 * r:4 * r + 4] for t in got]
        check_logprobs(part, x[:, 4 * r:4 * r + 4], None, kw)
    for t in got[1:]:
        assert torch.equal(t.view(rows, -1), t.view(rows, -1)[:1].expand(rows, -1))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 3000])
def test_logprobs_of_lists_that_fill(nf, dtype, rows):
    """The most alternatives that there are, of rows whose candidates fill a wavefront's list from chunk to chunk: random, rising and falling ones, steps of many equals, and those of a few lanes."""
    V = 13000
    j = torch.arange(V)
    g = gen(5)
    kinds = torch.stack([torch.randn(V, generator=g) * 3, j.float() / 256, -j.float() / 256, (j // 300).float(), -(j // 300).float(),
                         torch.where(j % 512 // 8 < 3, 5.0 + torch.rand(V, generator=g), torch.rand(V, generator=g)),
                         torch.where(j % 256 // 4 < 2, 5.0 + j / 4096, torch.rand(V, generator=g))])
    n = kinds.shape[0]
    x = kinds.to(dtype).cuda()[None].expand(rows, n, V).reshape(1, n * rows, V)
    for k in (17, 32):
        kw = dict(k=k, vocab=None, nodes=None, scale=1.0, cap=0.0)
        got = nf.token_logprobs(x, **kw)
        check_logprobs([None if t is None else t[:, :n] for t in got], x[:, :n], None, kw)
        for t in got[1:]:
            assert torch.equal(t.view(rows, -1), t.view(rows, -1)[:1].expand(rows, -1))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs_bits_do_not_depend_on_the_other_rows(nf, dtype):
    """Rows whose chunks are one wavefront's each give the bits that they give among thousands, several chunks to a wavefront."""
    V, g = 20011, gen(31)
    x = (torch.randn(1, 6000, V, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") * 3).to(dtype)
    for cap in (0.0, 25.0):
        kw = dict(k=12, cap=cap)
        token = torch.randint(0, V, (1, 6000, 2), generator=g).to(I32).cuda()
        many = nf.token_logprobs(x, token, **kw)
        for r in (0, 2999, 5999):
            for a, b in zip(many, nf.token_logprobs(x[:, r:r + 1], token[:, r:r + 1].contiguous(), **kw)):
                assert torch.equal(a[:, r:r + 1], b)
        check_logprobs([t[:, :2] for t in many], x[:, :2], token[:, :2], dict(kw, vocab=None, nodes=None, scale=1.0))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_logprobs_of_odd_logits(nf, dtype, cap):
    """Tokens that are masked with -infinity or the type's lowest value, rows of nothing else, +infinity, NaN; what lies past the vocabulary."""
    V = 9000
    x = torch.randn(1, 9, V, generator=gen(5)).to(dtype).cuda()
    x[0, 0, 10:] = -math.inf
    x[0, 1] = -math.inf
    x[0, 2, :8000] = torch.finfo(dtype).min
    x[0, 3, 100] = math.inf
    x[0, 4, 5000] = math.nan
    x[0, 5] = math.nan
    x[0, 6, ::2] = -math.inf
    x[0, 7] = torch.finfo(dtype).min
    x[0, 8, :4096] = -math.inf
    x[0, 4].view(torch.int16 if dtype == BF else I32)[6001] = 0x7f81 if dtype == BF else 0x7f800001      # a signalling NaN
    token = ints([[[3, 11, 100]] * 9])
    kw = dict(k=12, vocab=None, nodes=None, scale=1.0, cap=cap)
    check_logprobs(nf.token_logprobs(x, token, **kw), x, token, kw)
    y = x.clone()
    y[:, :, 6000:] = math.nan
    kw["vocab"] = ints([6000])
    for z in (x, y):
        check_logprobs(nf.token_logprobs(z, token, **kw), x[:, :, :6000], token, dict(kw, vocab=None))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shift", [-3e4, 1e4])
def test_logprobs_of_large_logits(nf, dtype, shift):
    """Logits that are large beside their differences: what is lost is their own rounding."""
    x = (torch.randn(1, 4, 3000, generator=gen(9)) * 400 + shift).to(dtype).cuda()
    token = ints([[[5, 2999]] * 4])
    kw = dict(k=4, vocab=None, nodes=None, scale=0.01, cap=0.0)
    check_logprobs(nf.token_logprobs(x, token, **kw), x, token, kw)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs_of_strided_rows(nf, dtype):
    """Columns of a larger tensor, rows that start at any element; a row's bits are its own."""
    V = 5003
    wide = torch.randn(3, 7, V + 6, generator=gen(11)).to(dtype).cuda()
    x, token = wide[1:, 2:6, 3:3 + V], ints([[[1]] * 4] * 2)
    kw = dict(k=6, vocab=None, nodes=None, scale=1.0, cap=0.0)
    got = nf.token_logprobs(x, token, **kw)
    check_logprobs(got, x, token, kw)
    for a, b in zip(got, nf.token_logprobs(x.contiguous(), token, **kw)):
        assert torch.equal(a, b)
    for a, b in zip(got, nf.token_logprobs(x[1:, 2:3].contiguous(), token[1:, 2:3].contiguous(), **kw)):
        assert torch.equal(a[1:, 2:3], b)


# ------------------------------------------------------------------------------------------------------------------------------ all together
def steps(nf, M, B, T, C, heads, kv, d, V, dtype, graph):
    """Steps of a decoder as they are used: turned queries and keys, attention over the cache of 4 bits, log probabilities, the accepted path appended."""
    g = gen(21)
    freq = (10000.0 ** (-torch.arange(d // 2).double() / (d // 2))).float().cuda()
    gq, gk = (1 + 0.1 * torch.randn(M, d, generator=g).cuda() for _ in range(2))
    W = (torch.randn(M, heads * d, V, generator=g) * 0.3).to(dtype).cuda()
    cache = list(nf.cache_fp4(M, B, kv, C, d))
    pos, w = torch.zeros(M, B, kv, C, dtype=I32, device="cuda"), torch.zeros(M, B, kv, C, device="cuda")
    L = torch.zeros(M, B, dtype=I32, device="cuda")
    first = torch.randn(M, B * 9, 2 * kv * d, generator=g).to(dtype).cuda()
    nf.cache_append_fp4(first[:, :, :kv * d], first[:, :, kv * d:], *cache, pos, w, L)
    L += 9
    parent, index, count = ints([[[-1, 0, 0, 1, 2]] * B] * M), ints([[[0, 2, 4]] * B] * M), ints([[3, 2]] * M)
    depth = ints([0, 1, 1, 2, 2])
    x = torch.randn(4, M, B * T, (heads + 2 * kv) * d, generator=g).to(dtype).cuda()
    qkv = torch.empty_like(x[0])
    out = []

    def step():
        Q, K, Vv = qkv[:, :, :heads * d], qkv[:, :, heads * d:(heads + kv) * d], qkv[:, :, (heads + kv) * d:]
        nf.rotate_heads(Q, K, B, T, heads, kv, freq=freq, gamma_q=gq, gamma_k=gk, pos=(L[..., None] + depth).contiguous(), out_q=Q, out_k=K)
        O = nf.attention_tree_fp4(Q, K, Vv, *cache, L, parent=parent)
        y = nf.linear(O, W)
        r = nf.token_logprobs(y, k=4)
        nf.cache_append_fp4(K, Vv, *cache, pos, w, L, index=index, count=count)
        L.add_(count)
        return (O, y) + tuple(t for t in r if t is not None)
    if graph:
        qkv.copy_(x[0])
        held = [t.clone() for t in cache + [pos, w, L]]
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            step()
        torch.cuda.current_stream().wait_stream(st)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            res = step()
        for t, o in zip(cache + [pos, w, L], held):
            t.copy_(o)
    for i in range(4):
        qkv.copy_(x[i])
        if graph:
            gr.replay()
            torch.cuda.synchronize()
        else:
            res = step()
        out.append([t.clone() for t in res])
        torch.ones(1000, device="cuda").sum().item()                  # the program's own work between the steps
    return out, [t.clone() for t in cache + [pos, w, L]]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("C", [40, 2000])
def test_steps_of_a_decoder(nf, dtype, C):
    """Eager and replayed steps give the same bits; the last state is what the definitions give."""
    shape = (2, 2, 5, C, 4, 2, 64, 520)
    out, state = steps(nf, *shape, dtype, False)
    again, state2 = steps(nf, *shape, dtype, True)
    for a, b in zip(out, again):
        for s, t in zip(a, b):
            assert torch.equal(s, t)
    for s, t in zip(state, state2):
        assert torch.equal(s, t)
    assert state[-1].cpu().tolist() == [[9 + 12, 9 + 8]] * 2
    y, entropy, top, top_logp = out[-1][1:]
    check_logprobs((None, entropy, top, top_logp), y, None, dict(k=4, vocab=None, nodes=None, scale=1.0, cap=0.0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_cache_of_4_bits_is_weighed_and_evicted(nf, dtype):
    """Keys read back are weighed as any others; two evictions from the same weights move codes and scales alike."""
    M, B, kv, C, d, T, heads, budget = 2, 2, 2, 60, 64, 2, 4, 37
    case = (M, B, T, C, heads, kv, d, 0.0, False, False, False, False, "chain", [[58, 44], [20, 37]])
    rows, cache, L, kw = tree_case(nf, case, dtype)
    g = gen(3)
    lse = torch.empty(M, B * T, heads, device="cuda")
    nf.attention_tree_fp4(*rows, *cache, L, lse=lse)
    pos, w = torch.arange(C, dtype=I32, device="cuda").expand(M, B, kv, C).contiguous(), torch.rand(M, B, kv, C, generator=g).cuda()
    nf.cache_append_fp4(rows[1], rows[2], *cache, pos, w, L)
    w = nf.cache_weigh(rows[0], lse, nf.cache_read_fp4(cache[0], cache[1], None, None, d, dtype=dtype)[0], w, L)
    L = (L + T).clamp(max=C)
    before = [t.clone() for t in cache]
    pos_out, w_out = torch.zeros_like(pos), torch.zeros_like(w)
    nf.cache_evict(cache[0].view(BF), cache[2].view(BF), pos, w, L, budget, recent=4, start=L, pos_out=pos_out, weight_out=w_out)
    nf.cache_evict(cache[1].view(BF), cache[3].view(BF), pos, w, L, budget, recent=4, start=L, pos_out=pos_out, weight_out=w_out)
    for m in range(M):
        for b in range(B):
            for h in range(kv):
                n = min(int(L[m, b]), budget)
                stay = pos_out[m, b, h, :n].long()                    # an entry's position is the slot that it came from
                assert stay.unique().numel() == n
                for t, o in zip(cache, before):
                    assert torch.equal(t[m, b, h, :n], o[m, b, h, stay])


def test_given_streams(nf):
    """Calls on a stream of the caller's give what the current stream's do."""
    case = (1, 2, 3, 900, 4, 2, 64, 0.0, True, False, False, False, "tree", [[900, 700]])
    rows, cache, L, kw = tree_case(nf, case, BF)
    Q, K, B, S, heads, kv, rkw = rotate_case(ROTATE[2], BF)
    x, token, lkw = logprob_case(LOGPROBS[2], BF)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def calls(stream):
        r = list(nf.rotate_heads(Q, K, B, S, heads, kv, stream=stream, **rkw))
        r += [nf.attention_tree_fp4(*rows, *cache, L, stream=stream, **kw)]
        r += list(nf.cache_read_fp4(*cache, 64, stream=stream))
        return r + list(nf.token_logprobs(x, token, stream=stream, **lkw))
    want = calls(None)
    got = calls(st)
    st.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,heads,kv,d", [(1, 4, 1, 64), (1, 3, 1, 128), (2, 2, 1, 96), (4, 2, 2, 64), (1, 5, 1, 128), (2, 4, 1, 32), (1, 1, 1, 128)])
def test_tree_fp4_of_few_rows(nf, T, heads, kv, d, dtype):
    """Up to four rows to a key head, whose scores several lanes share: every rest of a step, one step and several, caps, slopes and positions, the tree's own rows beside them."""
    for n in (0, 1, 15, 16, 17, 63, 64, 65, 200, 255, 256, 257, 700, 1024, 1025, 1300):
        case = (1, 1, T, n + 5, heads, kv, d, 12.0 if n % 2 else 0.0, n % 3 != 0, n % 4 == 1, False, T > 1 and n % 5 == 0, "tree" if T > 1 else "chain", [[n]])
        rows, cache, L, kw = tree_case(nf, case, dtype, seed=n)
        lse = torch.empty(1, T, heads, device="cuda")
        O = nf.attention_tree_fp4(*rows, *cache, L, lse=lse, **kw)
        check_tree(case, dtype, rows, cache, L, kw, O, lse)
