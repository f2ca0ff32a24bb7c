"""The step's calls marshalled natively against the Python functions: the same outputs, and the same exception for what either refuses."""
import pytest
import torch

from test_gpu_decoder_binding import _i, _outcome, _r

pytestmark = pytest.mark.gpu
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    assert nf._native is not None, "the binding was not built, or for another torch"
    return nf


def _cases(nf, dt):
    """(function, positional arguments, keywords)"""
    M, B, T, C, H, kv, d, V = 2, 2, 3, 40, 4, 2, 32, 70
    x = _r(M, B * T, (H + 2 * kv) * d, dt=dt)
    Q, K, W = x[:, :, :H * d], x[:, :, H * d:(H + kv) * d], x[:, :, (H + kv) * d:]
    new = lambda n: torch.randint(0, 256, (M, B, kv, C, n), device="cuda", dtype=U8)  # noqa: E731
    cache = (new(16), new(2), new(16), new(2))
    cache[1].clamp_(2, 200), cache[3].clamp_(100, 130)
    L, pos, w = _i([[30, 0], [7, 36]]), _i([0] * (M * B * kv * C)).view(M, B, kv, C), torch.rand(M, B, kv, C, device="cuda")
    slope, par, idx = torch.rand(M, H, device="cuda"), _i([[[-1, 0, 0]] * B] * M), _i([[[0, 2]] * B] * M)
    freq, gq, gk = torch.rand(16, device="cuda"), torch.rand(M, d, device="cuda"), torch.rand(M, d, device="cuda")
    p1, p3 = _i([[[1, 2, 3]] * B] * M), _i([[[[1, 2, 3]] * T] * B] * M)
    z, tok = _r(M, B * T, V, dt=dt), _i([[[1]] * (B * T)] * M)
    r, a, e, t, g = nf.rotate_heads, nf.cache_append_fp4, nf.cache_read_fp4, nf.attention_tree_fp4, nf.token_logprobs
    rot, step = (Q, K, B, T, H, kv), (Q, K, W) + cache + (L,)
    full = lambda *s, like=dt: torch.zeros(*s, device="cuda", dtype=like)  # noqa: E731
    out = (full(M, B * T, 1, like=F32), full(M, B * T, like=F32), full(M, B * T, 2, like=I32), full(M, B * T, 2, like=F32))
    return [
        (r, rot, dict(freq=freq)), (r, rot, dict(freq=freq, gamma_q=gq, gamma_k=gk, pos=p1, interleaved=True)), (r, rot, dict(freq=freq, pos=p3, sections=[4, 6, 6], eps=1e-5)), (r, rot, dict(gamma_k=gk)),
        (r, rot, dict(freq=freq, start=L, length=_i([[2, 3], [0, 1]]))), (r, rot, dict(freq=freq, length=L, out_q=full(M, B * T, H * d), out_k=full(M, B * T, kv * d))), (r, (Q, None, B, T, H), dict(freq=freq)),
        (r, rot, dict(freq=freq, out_q=full(M, B * T, H * d))), (r, (Q, Q, B, T, H), dict(freq=freq)), (r, rot, dict(freq=freq, pos=p1[..., None].contiguous(), sections=[16])), (r, rot, dict(freq=freq, pos=p3)),
        (r, rot, dict(freq=freq, pos=p3, sections=[4, 6, 5])), (r, rot, dict(freq=freq, pos=p3, sections=(4, 6, 6))), (r, rot, dict(freq=freq, sections=[8, 8])), (r, rot, dict(freq=freq, sections=[])), (r, rot, dict(eps=-1.0)),
        (r, rot, dict(freq=freq.double())), (r, rot, dict(freq=torch.rand(17, device="cuda"))), (r, rot, dict(gamma_q=gq[:, :5])), (r, (Q, K, B, T + 1, H, kv), {}), (r, (Q, K, B, T, 3, kv), {}), (r, (Q, K, B, T, H, 0), {}),
        (r, (Q.cpu(), K, B, T, H, kv), {}), (r, (Q.half(), K, B, T, H, kv), {}), (r, (Q, K, B, T, H, kv), dict(length=L.long())), (r, (Q, None, B, T, H), dict(out_k=K)), (r, rot, dict(out_q=full(M, B * T, 5))),
        (r, rot, dict(freq=torch.empty(0, device="cuda"))), (r, rot, dict(freq=freq, interleaved=1)), (r, rot, dict(freq=freq, eps=1)),
        (a, (K, W) + cache + (pos, w, L), {}), (a, (K, W) + cache + (None, None, L), dict(index=idx, count=_i([[2, 1], [0, 2]]), start=L)), (a, (K, W) + cache + (pos, w, None), {}), (a, (K, W) + cache + (w, pos, L), {}),
        (a, (K, W, cache[0].float()) + cache[1:] + (pos, w, L), {}), (a, (K, W, cache[0][:, :, :, :, :8]) + cache[1:] + (pos, w, L), {}), (a, (K, W[:, :5]) + cache + (pos, w, L), {}), (a, (K, W) + cache[:2] + (None, None, pos, w, L), {}),
        (a, (Q, Q) + cache + (pos, w, L), {}), (a, (K[0], W) + cache + (pos, w, L), {}), (a, (K, W, cache[0][0]) + cache[1:] + (pos, w, L), {}),
        (e, cache + (d,), {}), (e, cache + (d,), dict(out_k=full(M, B, kv, C, d), out_v=full(M, B, kv, C, d), count=L)), (e, cache[:2] + (None, None, d), dict(out_k=full(M, B, kv, 5, d), n=5, first=L)), (e, cache + (d,), dict(dtype=dt, n=3)),
        (e, cache + (64,), {}), (e, cache + (d,), dict(n=0)), (e, cache[:3] + (None, d), {}), (e, cache[:2] + (None, None, d), dict(out_v=full(M, B, kv, C, d))), (e, cache + (d,), dict(out_k=full(M, B, kv, C, 5))),
        (e, cache + (d,), dict(dtype=torch.half)), (e, cache + (d,), dict(first=L.long())), (e, cache + (d,), dict(out_k=full(M, B, kv, C, d))),
        (t, step, {}), (t, step, dict(start=L, parent=par, nodes=_i([[3, 1], [0, 2]]), pos=pos, slope=slope, cap=3.0, lse=full(M, B * T, H, like=F32), out=full(M, B * T, H * d))), (t, step, dict(scale=0.25, workspace=full(64, like=F32))),
        (t, step, dict(workspace=torch.empty(64))), (t, step[:7] + (None,), {}), (t, step[:7] + (L.view(-1),), {}), (t, (Q[:, :5],) + step[1:], {}), (t, step, dict(parent=par[:, :, :2])), (t, step, dict(pos=pos.float())),
        (t, step, dict(cap=float("nan"))), (t, (Q.float() if dt == BF else Q.bfloat16(),) + step[1:], {}), (t, step, dict(lse=full(M, B * T, kv, like=F32))), (t, step[:4] + (cache[0],) + step[5:], {}),
        (g, (z,), {}), (g, (z, tok), dict(k=2, scale=0.5, cap=4.0, vocab=_i([70, 9]), nodes=_i([[3, 1], [0, 2]]))), (g, (z, tok), dict(k=2, out=out)), (g, (z[:, :, 1:], None), dict(k=32)), (g, (z, tok), dict(workspace=full(9000, like=F32))),
        (g, (z,), dict(k=33)), (g, (z,), dict(k=-1)), (g, (z,), dict(scale=0.0)), (g, (z,), dict(scale=float("nan"))), (g, (z, tok.long()), {}), (g, (z, tok[0]), {}), (g, (z, tok[:, :2]), {}), (g, (z,), dict(vocab=_i([1]))),
        (g, (z,), dict(nodes=_i([[1] * 4] * M))), (g, (z[0],), {}), (g, (z.half(),), {}), (g, (z, tok), dict(k=1, out=out)), (g, (z,), dict(workspace=full(2, like=F32))), (g, (z[:, :, ::2],), {}), (g, (z.cpu(),), {}),
    ]


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
                assert x.dtype == y.dtype and torch.equal(x.nan_to_num(7.0) if x.is_floating_point() else x, y.nan_to_num(7.0) if y.is_floating_point() else y), what
            taken += 1
    assert taken > 25


def test_the_common_calls_are_taken(nf, monkeypatch):
    """Without the checks of the Python functions: a call that came to them would fail."""
    import paper_2009_13062_amd.step as S
    monkeypatch.setattr(S, "_dense", None)
    monkeypatch.setattr(S, "_rows", None)
    cases = _cases(nf, BF)
    named = {}
    for fn, args, kw in cases:
        named.setdefault(fn.__name__, []).append((fn, args, kw))
    for name, which in (("rotate_heads", (0, 1, 2, 3, 5, 6, 7, 8, 9)), ("cache_append_fp4", (0, 1)), ("cache_read_fp4", (1, 2)), ("attention_tree_fp4", (0, 1, 2)), ("token_logprobs", (0, 1, 2, 3, 4))):
        for k in which:
            fn, args, kw = named[name][k]
            fn(*args, **kw)
    torch.cuda.synchronize()
