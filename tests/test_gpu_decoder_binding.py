"""The decoders' calls marshalled natively against the Python functions: the same outputs, and the same exception for what either
refuses (the native path hands what it does not take to the Python one)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    assert nf._native is not None, "the binding was not built, or for another torch"
    return nf


def _r(*s, dt=BF):
    return torch.randn(*s, device="cuda").to(dt)


def _i(x):
    return torch.tensor(x, dtype=I32, device="cuda")


def _cases(nf, dt):
    """(function, positional arguments, keywords); what a call writes is cloned before each run."""
    M, B, T, C, H, kv, d = 2, 2, 3, 40, 4, 2, 32
    x = _r(M, B * T, (H + 2 * kv) * d, dt=dt)
    Q, K, V = x[:, :, :H * d], x[:, :, H * d:(H + kv) * d], x[:, :, (H + kv) * d:]
    Kc, Vc = _r(M, B, kv, C, d, dt=dt), _r(M, B, kv, C, d, dt=dt)
    L, pos, w = _i([[30, 0], [7, 36]]), _i([0] * (M * B * kv * C)).view(M, B, kv, C), torch.rand(M, B, kv, C, device="cuda")
    slope, lse = torch.rand(M, H, device="cuda"), torch.rand(M, B * T, H, device="cuda") + 3
    idx, par = _i([[[0, 2]] * B] * M), _i([[[-1, 0, 0]] * B] * M)
    p, t, a, g, e = nf.attention_prompt, nf.attention_tree, nf.cache_append, nf.cache_weigh, nf.cache_evict
    step = (Q, K, V, Kc, Vc, L)
    return [
        (p, (Q, K, V, B, T, H, kv), {}), (p, (Q, K, V, B, T, H, kv), dict(cap=2.0, slope=slope, length=_i([[3, 2], [0, 1]]), prefix=_i([[1, 2], [0, 0]]))),
        (p, (Q, K, V, B, T, H, kv), dict(causal=False, doc=_i([[[0, 0, 1]] * B] * M), scale=0.5)), (p, (Q, K, V, B, T, H, kv), dict(out=torch.empty(M, B * T, H * d, device="cuda", dtype=dt))),
        (p, (Q, K, V, B, T, H, kv), dict(cap=2)), (p, (Q, K, V, B, T, H, kv), dict(causal=1)), (p, (Q, Q, Q, B, T, H), {}), (p, (Q, K, V, B, T, H), {}), (p, (Q, K, V, B, T + 1, H, kv), {}),
        (p, (Q, K, V, B, T, 3, kv), {}), (p, (Q, K, V, B, T, H, 0), {}), (p, (Q, K.contiguous(), V, B, T, H, kv), {}), (p, (Q.cpu(), K, V, B, T, H, kv), {}), (p, (Q.half(), K, V, B, T, H, kv), {}),
        (p, (Q, K, V, B, T, H, kv), dict(causal=False, prefix=_i([[1, 1], [1, 1]]))), (p, (Q, K, V, B, T, H, kv), dict(cap=-1.0)), (p, (Q, K, V, B, T, H, kv), dict(length=L.long())),
        (p, (Q, K, V, B, T, H, kv), dict(slope=slope.t())), (p, (Q[:, :, ::2], K, V, B, T, H, kv), {}), (p, (torch.nn.Parameter(Q), K, V, B, T, H, kv), {}), (p, (Q[0], K, V, B, T, H, kv), {}),
        (t, step, {}), (t, step, dict(start=_i([[50, 0], [9, 36]]), parent=par, nodes=_i([[3, 1], [0, 2]]), pos=pos, slope=slope, cap=3.0, lse=torch.empty(M, B * T, H, device="cuda"))),
        (t, step, dict(scale=0.25, out=torch.empty(M, B * T, H * d, device="cuda", dtype=dt), workspace=torch.empty(64, device="cuda"))), (t, step, dict(workspace=torch.empty(64))),
        (t, step[:5] + (None,), {}), (t, step[:5] + (L.view(-1),), {}), (t, (Q, K, V, Kc[:, :, :, :39], Vc, L), {}), (t, (Q, K, V, Kc, Vc[:, :, :, :39], L), {}), (t, (Q[:, :5], K, V, Kc, Vc, L), {}),
        (t, step, dict(parent=par[:, :, :2])), (t, step, dict(pos=pos.float())), (t, step, dict(lse=torch.empty(M, B * T, kv, device="cuda"))), (t, step, dict(cap=float("nan"))),
        (t, (Q, K, V, Kc.float() if dt == BF else Kc.bfloat16(), Vc, L), {}), (t, (Q, K, V, Kc[0], Vc, L), {}),
        (a, (K, V, Kc, Vc, pos, w, L), {}), (a, (K, V, Kc, Vc, None, None, L), dict(index=idx, count=_i([[2, 1], [0, 2]]), start=_i([[1, 2], [3, 4]]))), (a, (K, V, Kc, Vc, pos, w, None), {}),
        (a, (K, V, Kc, Vc, w, pos, L), {}), (a, (K, V, Kc, Vc, pos, w, L), dict(index=idx[0])), (a, (K, V.float() if dt == BF else V.bfloat16(), Kc, Vc, pos, w, L), {}), (a, (K, V[:, :5], Kc, Vc, pos, w, L), {}),
        (g, (Q, lse, Kc, w, L), {}), (g, (Q, lse, Kc, w, L), dict(index=idx, count=_i([[2, 1], [0, 2]]), pos=pos, slope=slope, start=L, cap=4.0, out=torch.empty_like(w))), (g, (Q, lse, Kc, w, L), dict(out=w)),
        (g, (Q, None, Kc, w, L), {}), (g, (Q, lse[:, :2], Kc, w, L), {}), (g, (Q, lse, Kc, w[:, :, :1], L), {}), (g, (Q, lse, Kc, w, L), dict(scale=float("inf"))), (g, (Q, lse, Kc, w, L), dict(out=w.double())),
        (e, (Kc, Vc, pos, w, L, 20), {}), (e, (Kc, Vc, pos, w, L, 20), dict(recent=4, start=_i([[50, 1], [2, 40]]), pos_out=torch.zeros_like(pos), weight_out=torch.zeros_like(w))), (e, (Kc, Vc, None, w, L, 5), {}),
        (e, (Kc, Vc, None, w, L, 5), dict(recent=3)), (e, (Kc, Vc, pos, w, L, 0), {}), (e, (Kc, Vc, pos, w, L, 41), {}), (e, (Kc, Vc, pos, None, L, 20), {}), (e, (Kc, Vc, pos, w, L, 20), dict(recent=-1)),
        (e, (Kc, Vc, pos, w, L, 20), dict(workspace=torch.empty(4096, device="cuda"))), (e, (Kc, Vc, pos, w, L, 20), dict(weight_out=pos)),
    ]


def _plain(x):
    return isinstance(x, torch.Tensor) and type(x) is torch.Tensor


def _outcome(call):
    fn, args, kw = call
    seen = {}
    def own(x):                                               # a copy of the same strides; one copy for one operand named twice
        if not _plain(x):
            return x
        if id(x) not in seen:
            seen[id(x)] = x.clone() if x.is_contiguous() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device).copy_(x)
        return seen[id(x)]
    args, kw = [own(x) for x in args], {k: own(v) for k, v in kw.items()}
    try:
        r = fn(*args, **kw)
    except Exception as e:                                    # compared below
        return type(e), str(e)
    torch.cuda.synchronize()
    keep = [x for x in (r if isinstance(r, tuple) else (r,)) if _plain(x)]
    return keep + [x for x in seen.values() if "workspace" not in kw or x is not kw["workspace"]]


@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_native_calls_are_the_python_ones(nf, monkeypatch, dt):
    torch.manual_seed(1)
    cases, native = _cases(nf, dt), nf._native
    taken = 0
    for k, call in enumerate(cases):
        got = _outcome(call)
        monkeypatch.setattr(nf, "_native", None)
        want = _outcome(call)
        monkeypatch.setattr(nf, "_native", native)
        what = "call %d, %s" % (k, call[0].__name__)
        if isinstance(want, tuple):
            assert got == want, what
        else:
            assert isinstance(got, list) and len(got) == len(want), what
            for x, y in zip(got, want):
                assert x.dtype == y.dtype and torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)), what
            taken += 1
    assert taken > 15


def test_the_common_calls_are_taken(nf, monkeypatch):
    """Without the checks of the Python functions: a call that came to them would fail."""
    import paper_2009_13062_amd.decoder as D
    monkeypatch.setattr(D, "_dense", None)
    monkeypatch.setattr(D, "_rows", None)
    cases = _cases(nf, BF)
    for k in (0, 1, 2, 3, 21, 22, 23, 36, 37, 43, 44, 45, 51, 52, 53):
        fn, args, kw = cases[k]
        fn(*args, **kw)
    torch.cuda.synchronize()
