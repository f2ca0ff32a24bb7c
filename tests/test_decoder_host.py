"""What the decoders' entry points refuse before any HIP call, and what the binding refuses; no GPU needed."""
import pytest
import torch

OK, EINVAL, EUNSUPPORTED = 0, 1, 2
P = 4096          # a non-null, well-aligned fake device address; never dereferenced on the host
BIG = 2 ** 31 - 1


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def caller(f, names, ok):
    def call(**kw):
        a = dict(ok, **kw)
        assert set(a) == set(names)
        return f(*[a[n] for n in names])
    return call


def test_prompt_refuses(nf):
    names = "Q K V slope len prefix doc O M B S heads kv d qm qr km kr causal scale cap dt stream".split()
    ok = dict(Q=P, K=P, V=P, slope=P, len=P, prefix=P, doc=P, O=P, M=2, B=1, S=8, heads=4, kv=2, d=64, qm=8 * 256, qr=256, km=8 * 128, kr=128, causal=1, scale=0.125, cap=0.0, dt=1, stream=None)
    call = caller(nf.lib.netfuse_attention_prompt, names, ok)
    inf, nan = float("inf"), float("nan")
    for bad in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(M=0), dict(B=-1), dict(S=0), dict(heads=0), dict(kv=0), dict(d=0), dict(heads=3), dict(qr=255), dict(kr=127),
                dict(qm=100), dict(km=100), dict(qm=-1), dict(scale=nan), dict(scale=inf), dict(cap=-1.0), dict(cap=nan), dict(cap=inf), dict(cap=1e-31), dict(cap=1e31), dict(dt=2), dict(causal=0),
                dict(Q=P + 1), dict(K=P + 1), dict(V=P + 1), dict(O=P + 1), dict(slope=P + 2), dict(len=P + 1), dict(prefix=P + 2), dict(doc=P + 3), dict(B=BIG, S=BIG), dict(M=BIG, qm=2 ** 60),
                dict(heads=BIG, kv=1, d=256)):
        assert call(**bad) == EINVAL, bad
    assert call(d=257, qr=2048, qm=2048 * 8, kr=1024, km=1024 * 8) == EUNSUPPORTED


def test_tree_refuses(nf):
    names = "Q K V Kc Vc pos len start parent nodes slope O lse ws wsb M B T C heads kv d qm qr km kr scale cap dt stream".split()
    ok = dict(Q=P, K=P, V=P, Kc=P, Vc=P, pos=P, len=P, start=P, parent=P, nodes=P, slope=P, O=P, lse=P, ws=P, wsb=1 << 40, M=2, B=1, T=8, C=100, heads=4, kv=2, d=64, qm=8 * 256, qr=256, km=8 * 128,
              kr=128, scale=0.125, cap=0.0, dt=1, stream=None)
    call = caller(nf.lib.netfuse_attention_tree, names, ok)
    for bad in (dict(Q=None), dict(K=None), dict(V=None), dict(Kc=None), dict(Vc=None), dict(len=None), dict(O=None), dict(M=0), dict(B=0), dict(T=0), dict(C=0), dict(heads=3), dict(kv=0), dict(d=-1),
                dict(qr=255), dict(kr=1), dict(qm=1), dict(km=1), dict(scale=float("nan")), dict(cap=-2.0), dict(dt=5), dict(Q=P + 1), dict(Kc=P + 1), dict(Vc=P + 1), dict(pos=P + 1), dict(len=P + 1),
                dict(start=P + 1), dict(parent=P + 2), dict(nodes=P + 1), dict(slope=P + 1), dict(lse=P + 2), dict(ws=P + 8), dict(M=BIG, B=BIG, kv=BIG, heads=BIG, C=BIG), dict(C=(1 << 30) + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(T=65, qm=65 * 256, km=65 * 128) == EUNSUPPORTED
    assert call(d=257, qr=2048, qm=2048 * 8, kr=1024, km=1024 * 8) == EUNSUPPORTED
    size = nf.lib.netfuse_attention_tree_workspace
    for bad in ((0, 1, 8, 100, 4, 2, 64, 1), (2, 0, 8, 100, 4, 2, 64, 1), (2, 1, 0, 100, 4, 2, 64, 1), (2, 1, 65, 100, 4, 2, 64, 1), (2, 1, 8, 0, 4, 2, 64, 1), (2, 1, 8, 100, 3, 2, 64, 1),
                (2, 1, 8, 100, 4, 2, 257, 1), (2, 1, 8, 100, 4, 2, 64, 9), (1, 1, 1, (1 << 30) + 1, 1, 1, 8, 1)):
        assert size(*bad) == -1, bad
    for dt in (0, 1):
        need = size(1, 1, 1, 1 << 20, 8, 1, 128, dt)
        assert need >= 0
        if need > 0:
            one = dict(M=1, B=1, T=1, C=1 << 20, heads=8, kv=1, d=128, qm=0, qr=1024, km=0, kr=128, dt=dt)
            assert call(ws=None, **one) == EINVAL and call(wsb=need - 1, **one) == EINVAL


def test_cache_calls_refuse(nf):
    names = "K V index count len start Kc Vc pos weight M B T n C kv d km kr dt stream".split()
    call = caller(nf.lib.netfuse_cache_append, names, dict(K=P, V=P, index=P, count=P, len=P, start=P, Kc=P, Vc=P, pos=P, weight=P, M=2, B=1, T=8, n=3, C=100, kv=2, d=64, km=8 * 128, kr=128, dt=1, stream=None))
    for bad in (dict(K=None), dict(V=None), dict(Kc=None), dict(Vc=None), dict(len=None), dict(M=0), dict(B=0), dict(T=0), dict(n=0), dict(C=0), dict(kv=0), dict(d=0), dict(index=None), dict(kr=127), dict(km=5),
                dict(dt=-1), dict(K=P + 1), dict(Kc=P + 1), dict(index=P + 1), dict(count=P + 2), dict(pos=P + 1), dict(weight=P + 2), dict(start=P + 1), dict(len=P + 1), dict(B=BIG, n=BIG), dict(B=BIG, T=BIG), dict(C=(1 << 30) + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(d=257, kr=1024, km=8 * 1024) == EUNSUPPORTED

    names = "Q lse index count Kc pos len start slope weight out M B T n C heads kv d qm qr scale cap dt stream".split()
    call = caller(nf.lib.netfuse_cache_weigh, names, dict(Q=P, lse=P, index=P, count=P, Kc=P, pos=P, len=P, start=P, slope=P, weight=P, out=P, M=2, B=1, T=8, n=3, C=100, heads=4, kv=2, d=64, qm=8 * 256, qr=256,
                                                          scale=0.125, cap=0.0, dt=1, stream=None))
    for bad in (dict(Q=None), dict(lse=None), dict(Kc=None), dict(len=None), dict(weight=None), dict(out=None), dict(M=0), dict(T=0), dict(n=-1), dict(C=0), dict(heads=5), dict(index=None), dict(qr=9), dict(qm=9),
                dict(scale=float("inf")), dict(cap=-1.0), dict(dt=3), dict(Q=P + 1), dict(lse=P + 1), dict(weight=P + 1), dict(out=P + 2), dict(slope=P + 1), dict(pos=P + 1), dict(C=(1 << 30) + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(d=257, qr=2048, qm=8 * 2048) == EUNSUPPORTED

    names = "Kc Vc pos weight len start pos_out weight_out ws wsb M B C kv d budget recent dt stream".split()
    call = caller(nf.lib.netfuse_cache_evict, names, dict(Kc=P, Vc=P, pos=P, weight=P, len=P, start=P, pos_out=P, weight_out=P, ws=P, wsb=1 << 40, M=2, B=1, C=100, kv=2, d=64, budget=60, recent=4, dt=1, stream=None))
    for bad in (dict(Kc=None), dict(Vc=None), dict(weight=None), dict(len=None), dict(weight_out=None), dict(ws=None), dict(wsb=16), dict(pos=None), dict(pos_out=None), dict(pos=None, pos_out=None), dict(M=0),
                dict(C=0), dict(kv=0), dict(d=0), dict(budget=0), dict(budget=101), dict(recent=-1), dict(dt=2), dict(Kc=P + 1), dict(weight=P + 1), dict(ws=P + 4), dict(weight_out=P + 1), dict(C=(1 << 30) + 1)):
        assert call(**bad) == EINVAL, bad
    assert call(d=257) == EUNSUPPORTED
    size = nf.lib.netfuse_cache_evict_workspace
    for bad in ((0, 1, 100, 2, 60), (2, 0, 100, 2, 60), (2, 1, 0, 2, 60), (2, 1, 100, 0, 60), (2, 1, 100, 2, 0), (2, 1, 100, 2, 101), (1, 1, (1 << 30) + 1, 1, 5), (BIG, BIG, BIG, BIG, 2 ** 30)):
        assert size(*bad) == -1, bad
    assert size(2, 1, 100, 2, 100) >= 4


class Placed(torch.Tensor):
    """A host tensor that says it lies on a device: what the binding's checks see, up to the first address."""
    device_index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.device_index))


def placed(*shape, dtype=torch.bfloat16, index=0):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Placed)
    t.device_index = index
    return t


@pytest.fixture
def device0(nf, monkeypatch):
    monkeypatch.setattr(nf, "_device", lambda: 0)
    monkeypatch.setattr(nf, "_raw_stream", lambda d: 0)


def prompt_args(**kw):
    a = dict(Q=placed(2, 6, 256), K=placed(2, 6, 128), V=placed(2, 6, 128), B=2, S=3, heads=4, kv_heads=2, out=placed(2, 6, 256))
    a.update(kw)
    return a


@pytest.mark.parametrize("bad,error", [
    (dict(Q=torch.zeros(2, 6, 256, dtype=torch.bfloat16)), ValueError), (dict(Q=placed(2, 6, 256, dtype=torch.float16)), TypeError), (dict(K=placed(2, 6, 128, dtype=torch.float32)), TypeError),
    (dict(K=placed(2, 6, 64)), ValueError), (dict(V=placed(2, 5, 128)), ValueError), (dict(heads=3), ValueError), (dict(heads=0), ValueError), (dict(S=4), ValueError), (dict(Q=placed(6, 256)), ValueError),
    (dict(Q=placed(2, 256, 6).transpose(1, 2)), ValueError), (dict(K=placed(2, 6, 256)[:, :, :128]), ValueError), (dict(length=placed(2, 2, dtype=torch.int64)), TypeError),
    (dict(length=placed(2, 3, dtype=torch.int32)), ValueError), (dict(slope=placed(4, 2, dtype=torch.float32)), ValueError), (dict(slope=placed(4, 2, dtype=torch.float32).t()), ValueError),
    (dict(doc=placed(2, 2, 4, dtype=torch.int32)), ValueError), (dict(prefix=torch.zeros(2, 2, dtype=torch.int32)), ValueError), (dict(out=placed(2, 6, 128)), ValueError),
    (dict(out=placed(2, 6, 256, dtype=torch.float32)), TypeError), (dict(Q=placed(2, 6, 256, index=1)), ValueError), (dict(length=placed(2, 2, dtype=torch.int32, index=1)), ValueError)], ids=str)
def test_binding_refuses_prompts(nf, device0, monkeypatch, bad, error):
    monkeypatch.setattr(nf.lib, "netfuse_attention_prompt", lambda *a: pytest.fail("the call was made"))
    with pytest.raises(error):
        nf.attention_prompt(**prompt_args(**bad))


def test_binding_passes_strides_and_sizes(nf, device0, monkeypatch):
    """Column blocks of a packed projection go as they are; dimensions of one element say nothing about strides."""
    seen = []
    monkeypatch.setattr(nf.lib, "netfuse_attention_prompt", lambda *a: seen.append(a) or 0)
    x = placed(2, 6, 512)
    nf.attention_prompt(**prompt_args(Q=x[:, :, :256], K=x[:, :, 256:384], V=x[:, :, 384:]))
    assert seen[-1][8:19] == (2, 2, 3, 4, 2, 64, 6 * 512, 512, 6 * 512, 512, 1)
    one = placed(1, 1, 512)
    nf.attention_prompt(**prompt_args(Q=one[:, :, :256], K=one[:, :, 256:384], V=one[:, :, 384:], B=1, S=1, out=placed(1, 1, 256)))
    assert seen[-1][8:19] == (1, 1, 1, 4, 2, 64, 256, 256, 128, 128, 1)
    # K and V of another stride each are refused
    with pytest.raises(ValueError):
        nf.attention_prompt(**prompt_args(K=x[:, :, 256:384]))


def step_args(C=10, T=3):
    i32 = torch.int32
    return dict(Q=placed(2, 2 * T, 256), K=placed(2, 2 * T, 128), V=placed(2, 2 * T, 128), Kc=placed(2, 2, 2, C, 64), Vc=placed(2, 2, 2, C, 64), length=placed(2, 2, dtype=i32)), placed(2, 2 * T, 256)


@pytest.mark.parametrize("bad,error", [
    (dict(Kc=placed(2, 2, 2, 10)), ValueError), (dict(Vc=placed(2, 2, 2, 9, 64)), ValueError), (dict(Kc=placed(2, 2, 2, 10, 64, dtype=torch.float32)), TypeError), (dict(Q=placed(2, 7, 256)), ValueError),
    (dict(Q=placed(2, 6, 250)), ValueError), (dict(length=None), ValueError), (dict(length=placed(2, 2, dtype=torch.int64)), TypeError), (dict(pos=placed(2, 2, 10, dtype=torch.int32)), ValueError),
    (dict(parent=placed(2, 2, 4, dtype=torch.int32)), ValueError), (dict(nodes=placed(2, 3, dtype=torch.int32)), ValueError), (dict(lse=placed(2, 6, 2, dtype=torch.float32)), ValueError),
    (dict(Kc=placed(2, 2, 2, 10, 64, index=1)), ValueError), (dict(Kc=placed(2, 2, 10, 2, 64).transpose(2, 3)), ValueError), (dict(workspace=torch.zeros(64, dtype=torch.uint8)), ValueError)], ids=str)
def test_binding_refuses_trees(nf, device0, monkeypatch, bad, error):
    monkeypatch.setattr(nf.lib, "netfuse_attention_tree", lambda *a: pytest.fail("the call was made"))
    args, out = step_args()
    args.update(bad)
    with pytest.raises(error):
        nf.attention_tree(out=out, **args)


def test_binding_refuses_cache_calls(nf, device0, monkeypatch):
    for name in ("netfuse_cache_append", "netfuse_cache_weigh", "netfuse_cache_evict"):
        monkeypatch.setattr(nf.lib, name, lambda *a: pytest.fail("the call was made"))
    s, _ = step_args()
    i32, f32 = torch.int32, torch.float32
    pos, w, lse = placed(2, 2, 2, 10, dtype=i32), placed(2, 2, 2, 10, dtype=f32), placed(2, 6, 4, dtype=f32)
    append = dict(K=s["K"], V=s["V"], Kc=s["Kc"], Vc=s["Vc"], pos=pos, weight=w, length=s["length"])
    for bad in (dict(K=placed(2, 5, 128)), dict(V=placed(2, 6, 128, dtype=f32)), dict(pos=w), dict(weight=pos), dict(length=None), dict(index=placed(2, 2, 3, dtype=torch.int64)), dict(index=placed(2, 3, dtype=i32)),
                dict(count=placed(2, dtype=i32)), dict(start=placed(2, 2, dtype=f32)), dict(Kc=placed(2, 2, 2, 10, 64, index=1))):
        with pytest.raises((ValueError, TypeError)):
            nf.cache_append(**dict(append, **bad))
    weigh = dict(Q=s["Q"], lse=lse, Kc=s["Kc"], weight=w, length=s["length"])
    for bad in (dict(lse=None), dict(weight=None), dict(length=None), dict(lse=placed(2, 6, 2, dtype=f32)), dict(weight=placed(2, 2, 2, 9, dtype=f32)), dict(Q=placed(2, 6, 255)), dict(out=placed(2, 2, 2, 9, dtype=f32)),
                dict(Kc=placed(2, 2, 2, 10, 64, dtype=f32)), dict(slope=placed(2, 2, dtype=f32)), dict(Kc=placed(2, 2, 2, 640))):
        with pytest.raises((ValueError, TypeError)):
            nf.cache_weigh(**dict(weigh, **bad))
    evict = dict(Kc=s["Kc"], Vc=s["Vc"], pos=pos, weight=w, length=s["length"], budget=5)
    for bad in (dict(weight=None), dict(length=None), dict(pos=placed(2, 2, 2, 9, dtype=i32)), dict(weight_out=pos), dict(Vc=placed(2, 2, 2, 10, 32)), dict(workspace=torch.zeros(999, dtype=torch.uint8))):
        with pytest.raises((ValueError, TypeError)):
            nf.cache_evict(**dict(evict, **bad))
