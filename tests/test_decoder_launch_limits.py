"""Sizes whose launches would have 2^32 threads or more, which HIP does not take: refused as unsupported before anything is enqueued, in every
kernel choice of the decoders' calls.  No GPU needed: the addresses are never used."""
import pytest

EUNSUPPORTED = 2
P, ROOM = 4096, 1 << 61
T24 = 1 << 24                                                 # workgroups of 256 threads


@pytest.fixture(scope="module")
def lib():
    import paper_2009_13062_amd as nf
    return nf.lib


@pytest.mark.parametrize("sizes", [
    dict(M=32, B=8, S=8192, heads=32, kv=32, d=20, dt=1), dict(M=1, B=T24, S=4, heads=1, kv=1, d=3, dt=0),                     # one wavefront per row
    dict(M=1, B=T24, S=1, heads=1, kv=1, d=64, dt=1), dict(M=2, B=T24 // 4, S=129, heads=1, kv=1, d=128, dt=1),              # bfloat16 tiles
    dict(M=16, B=T24 // 16, S=1, heads=3, kv=1, d=64, dt=0), dict(M=1, B=T24 // 16, S=256, heads=1, kv=1, d=256, dt=0)], ids=str)
def test_prompts(lib, sizes):
    s = sizes
    q, k = s["heads"] * s["d"], s["kv"] * s["d"]
    n = s["B"] * s["S"]
    assert lib.netfuse_attention_prompt(P, P, P, None, None, None, None, P, s["M"], s["B"], s["S"], s["heads"], s["kv"], s["d"], n * q, q, n * k, k, 1, 0.125, 0.0, s["dt"], None) == EUNSUPPORTED


@pytest.mark.parametrize("sizes", [
    dict(M=1, B=T24, T=1, C=8, heads=4, kv=1, d=20, dt=1), dict(M=1, B=T24, T=1, C=8, heads=1, kv=1, d=64, dt=1), dict(M=1, B=T24, T=1, C=8, heads=1, kv=1, d=64, dt=0),
    dict(M=1, B=T24 // 8, T=64, C=8 * 1024, heads=2, kv=1, d=128, dt=1),                                                     # rows of 8 chunks each
    # the attention fits, and what joins its chunks does not: a workgroup per row, a group of lanes per row
    dict(M=1, B=512, T=64, C=9 * 1024, heads=512, kv=1, d=64, dt=1), dict(M=2, B=256, T=64, C=9 * 1024, heads=512, kv=1, d=256, dt=0),
    dict(M=1, B=8192, T=64, C=2 * 1024, heads=512, kv=1, d=64, dt=1), dict(M=1, B=2048, T=64, C=2 * 1024, heads=512, kv=1, d=256, dt=0)], ids=str)
def test_trees(lib, sizes):
    s = sizes
    q, k = s["heads"] * s["d"], s["kv"] * s["d"]
    n = s["B"] * s["T"]
    assert lib.netfuse_attention_tree(P, P, P, P, P, None, P, None, None, None, None, P, None, P, ROOM, s["M"], s["B"], s["T"], s["C"], s["heads"], s["kv"], s["d"], n * q, q, n * k, k, 0.125, 0.0,
                                      s["dt"], None) == EUNSUPPORTED


@pytest.mark.parametrize("d,dt", [(64, 1), (64, 0), (3, 0), (3, 1)])
def test_caches(lib, d, dt):
    n, k = 2 * T24, d
    assert lib.netfuse_cache_append(P, P, None, None, P, None, P, P, None, None, 1, n, 1, 1, 8, 1, d, n * k, k, dt, None) == EUNSUPPORTED
    assert lib.netfuse_cache_weigh(P, P, None, None, P, None, P, None, None, P, P, 1, n, 1, 1, 8, 1, 1, d, n * k, k, 0.125, 0.0, dt, None) == EUNSUPPORTED
    evict = lambda B, C, budget: lib.netfuse_cache_evict(P, P, None, P, P, None, None, P, P, ROOM, 1, B, C, 1, d, budget, 0, dt, None)  # noqa: E731
    assert evict(T24, 8, 4) == EUNSUPPORTED                                                                    # workgroups of 256 threads per head
    assert evict(T24 // 4, 9000, 8999) == EUNSUPPORTED and evict(T24 // 4, 40000, 39999) == EUNSUPPORTED        # of 1024
    assert evict(T24 // 16, 8192, 4096) == EUNSUPPORTED                                                        # those that move the rows
