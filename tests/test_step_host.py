"""Refusals of the operators around the decoders' attention: on the host, before any HIP call."""
import ctypes
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2009_13062_amd", "libnetfuse.so")
OK, EINVAL, EUNSUPPORTED = 0, 1, 2
P = 1 << 20                                                # a well-aligned fake device address; never dereferenced on the host


@pytest.fixture(scope="module")
def nf():
    if not os.path.exists(LIB):
        sys.path.insert(0, ROOT)
        import __graft_entry__ as g
        g.build()
    import paper_2009_13062_amd as nf
    return nf


def caller(f, ok, wrap=lambda k, v: v):
    def call(**kw):
        a = dict(ok, **kw)
        return f(*[wrap(k, v) for k, v in a.items()], None)
    return call


def sections(*n):
    return (ctypes.c_int * len(n))(*n)


def test_rotate_refuses(nf):
    ok = dict(Q=P, K=P, gq=P, gk=P, freq=P, pos=P, start=P, length=P, sections=None, Qo=P, Ko=P, M=2, B=2, S=3, heads=4, kv=2, d=64, rot=64, axes=1, qm=6 * 256, qr=256, km=6 * 128, kr=128,
              qom=6 * 256, qor=256, kom=6 * 128, kor=128, eps=1e-6, inter=0, dt=1)
    call = caller(nf.lib.netfuse_rotate_heads, ok)
    for bad in (dict(Q=None), dict(Qo=None), dict(K=None), dict(Ko=None), dict(K=None, Ko=None), dict(kv=0), dict(kv=-1), dict(M=0), dict(B=0), dict(S=-1), dict(heads=0), dict(d=0), dict(dt=2), dict(rot=-2), dict(rot=63),
                dict(rot=66), dict(freq=None), dict(axes=0), dict(axes=5), dict(axes=3), dict(axes=2, sections=sections(16, 16), pos=None), dict(axes=2, sections=sections(16, 15)),
                dict(axes=2, sections=sections(33, -1)), dict(sections=sections(31)), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(qr=255), dict(kr=127), dict(qm=100), dict(kom=1),
                dict(qor=100), dict(qm=7 * 256), dict(kr=130, km=6 * 130), dict(Q=P + 1), dict(Ko=P + 1), dict(gq=P + 2), dict(pos=P + 1), dict(M=2 ** 31 - 1, B=2 ** 31 - 1),
                dict(B=2 ** 30, S=2 ** 30), dict(qm=-5)):
        assert call(**bad) == EINVAL, bad
    assert call(d=258, rot=64, qr=4 * 258, qor=4 * 258, kr=2 * 258, kor=2 * 258, qm=6 * 4 * 258, qom=6 * 4 * 258, km=6 * 2 * 258, kom=6 * 2 * 258) == EUNSUPPORTED
    big = dict(M=1, B=2 ** 15, S=2 ** 14, qm=0, km=0, qom=0, kom=0)
    assert call(**big) == EUNSUPPORTED                     # 2^29 wavefronts


def test_append_fp4_refuses(nf):
    ok = dict(K=P, V=P, index=P, count=P, length=P, start=P, Kc=P, Ks=P, Vc=P, Vs=P, pos=P, weight=P, M=2, B=2, T=3, n=2, C=8, kv=2, d=64, sm=6 * 128, sr=128, dt=1)
    call = caller(nf.lib.netfuse_cache_append_fp4, ok)
    for bad in [dict([(k, None)]) for k in ("K", "V", "length", "Kc", "Ks", "Vc", "Vs")] + [
            dict(M=0), dict(B=-1), dict(T=0), dict(n=0), dict(C=0), dict(C=2 ** 30 + 1), dict(kv=0), dict(d=0), dict(dt=-1), dict(index=None), dict(sr=100), dict(sm=100), dict(K=P + 1), dict(Kc=P + 8),
            dict(Ks=P + 1), dict(Vc=P + 1), dict(Vs=P + 1), dict(pos=P + 2), dict(weight=P + 1), dict(B=2 ** 30, T=2 ** 30)]:
        assert call(**bad) == EINVAL, bad
    assert call(d=288, sr=2 * 288, sm=6 * 2 * 288) == EUNSUPPORTED


def test_read_fp4_refuses(nf):
    ok = dict(Kc=P, Ks=P, Vc=P, Vs=P, first=P, count=P, K=P, V=P, M=2, B=2, n=5, C=8, kv=2, d=64, dt=1)
    call = caller(nf.lib.netfuse_cache_read_fp4, ok)
    for bad in [dict([(k, None)]) for k in ("Kc", "Ks", "Vc", "Vs", "K", "V")] + [
            dict(Vc=None, V=None), dict(Vc=None, Vs=None), dict(M=0), dict(B=0), dict(n=0), dict(n=2 ** 30 + 1), dict(C=0), dict(kv=0), dict(d=-1), dict(dt=9), dict(Kc=P + 4), dict(Vs=P + 3), dict(d=128, Ks=P + 2), dict(K=P + 1), dict(V=P + 1),
            dict(first=P + 2), dict(count=P + 1), dict(M=2 ** 31 - 1, B=2 ** 31 - 1)]:
        assert call(**bad) == EINVAL, bad
    assert call(d=257) == EUNSUPPORTED


def test_tree_fp4_refuses(nf):
    ok = dict(Q=P, K=P, V=P, Kc=P, Ks=P, Vc=P, Vs=P, pos=P, length=P, start=P, parent=P, nodes=P, slope=P, O=P, lse=P, ws=P, bytes=1 << 40, M=2, B=2, T=3, C=8, heads=4, kv=2, d=64, qm=6 * 256, qr=256,
              km=6 * 128, kr=128, scale=0.125, cap=0.0, dt=1)
    call = caller(nf.lib.netfuse_attention_tree_fp4, ok)
    for bad in [dict([(k, None)]) for k in ("Q", "K", "V", "Kc", "Ks", "Vc", "Vs", "length", "O")] + [
            dict(M=0), dict(B=0), dict(T=0), dict(C=0), dict(C=2 ** 30 + 1), dict(heads=3), dict(kv=0), dict(d=0), dict(dt=4), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(qr=255),
            dict(kr=100), dict(qm=7), dict(Kc=P + 2), dict(Ks=P + 3), dict(O=P + 1), dict(lse=P + 2), dict(ws=P + 4), dict(slope=P + 1)]:
        assert call(**bad) == EINVAL, bad
    assert call(T=65, qm=130 * 256, km=130 * 128) == EUNSUPPORTED and call(d=260, qr=1040, kr=520, qm=6 * 1040, km=6 * 520) == EUNSUPPORTED
    size = nf.lib.netfuse_attention_tree_fp4_workspace
    assert size(0, 1, 1, 8, 4, 2, 64, 1) == -1 and size(1, 1, 65, 8, 4, 2, 64, 1) == -1 and size(1, 1, 1, 8, 4, 3, 64, 1) == -1 and size(1, 1, 1, 8, 4, 2, 300, 1) == -1
    assert size(1, 1, 1, 8, 4, 2, 64, 7) == -1 and size(1, 1, 1, 8, 4, 2, 64, 1) == 0
    need = size(1, 2, 1, 100003, 32, 8, 128, 1)
    if need > 0:                                           # a long cache is shared out
        long = dict(M=1, B=2, T=1, C=100003, heads=32, kv=8, d=128, qm=0, qr=4096, km=0, kr=1024)
        assert call(**long, ws=None) == EINVAL and call(**long, bytes=need - 1) == EINVAL


def test_logprobs_refuse(nf):
    ok = dict(logits=P, token=P, vocab=P, nodes=P, logp=P, entropy=P, top=P, top_logp=P, ws=P, bytes=1 << 40, M=2, B=2, T=3, V=100, n=1, k=5, sm=600, sr=100, scale=1.0, cap=0.0, dt=1)
    call = caller(nf.lib.netfuse_token_logprobs, ok)
    for bad in [dict([(k, None)]) for k in ("logits", "token", "logp", "entropy", "top", "top_logp", "ws")] + [
            dict(M=0), dict(B=0), dict(T=-1), dict(V=0), dict(V=2 ** 30 + 1), dict(n=-1), dict(k=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(cap=-2.0), dict(sr=99), dict(sm=1), dict(dt=3),
            dict(bytes=16), dict(logits=P + 1), dict(top=P + 2), dict(ws=P + 8), dict(M=2 ** 20, B=2 ** 12, T=1, sm=600)]:
        assert call(**bad) == EINVAL, bad
    assert call(k=33) == EUNSUPPORTED
    size = nf.lib.netfuse_token_logprobs_workspace
    assert size(1, 1, 1, 100, 33) == -1 and size(0, 1, 1, 100, 1) == -1 and size(1, 1, 1, 0, 1) == -1 and size(2, 2, 3, 100, 5) > 0


def test_python_refuses(nf):
    """Tensors on the host, and what would not fit: an exception that says what."""
    x, i = torch.zeros(1, 2, 64), torch.zeros(1, 1, dtype=torch.int32)
    u = [torch.zeros(1, 1, 1, 4, n, dtype=torch.uint8) for n in (32, 2)]
    for f in (lambda: nf.rotate_heads(x, x, 1, 2, 1), lambda: nf.cache_append_fp4(x, x, *u, *u, None, None, i), lambda: nf.cache_read_fp4(*u, *u, 64),
              lambda: nf.attention_tree_fp4(x, x, x, *u, *u, i), lambda: nf.token_logprobs(x)):
        with pytest.raises(ValueError, match="CUDA|cuda"):
            f()
    with pytest.raises(ValueError, match="make 3 heads"):
        nf.rotate_heads(x, x, 1, 2, 3)
    with pytest.raises(TypeError):
        nf.token_logprobs(x.half())
    with pytest.raises(ValueError):
        nf.rotate_heads(x[0], x, 1, 2, 1)
    with pytest.raises(ValueError, match="codes"):
        nf.cache_read_fp4(u[0][0], u[1], *u, 64)
    assert [t.shape[-1] for t in nf.cache_fp4(1, 2, 3, 4, 80, device="cpu")] == [48, 4, 48, 4]
