"""Workspace of the operators around the decoders' attention: a cache that is shared out needs some, and a call without it is refused on the host."""
from test_step_host import EINVAL, P, caller, nf  # noqa: F401


def test_a_shared_cache_needs_room(nf):                                # noqa: F811
    size = nf.lib.netfuse_attention_tree_fp4_workspace
    for T, dt in ((1, 0), (1, 1), (26, 0), (26, 1), (64, 1)):
        need = size(1, 2, T, 100003, 32, 8, 128, dt)
        assert need > 0
        ok = dict(Q=P, K=P, V=P, Kc=P, Ks=P, Vc=P, Vs=P, pos=P, length=P, start=P, parent=P, nodes=P, slope=P, O=P, lse=P, ws=P, bytes=need, M=1, B=2, T=T, C=100003, heads=32, kv=8, d=128, qm=0, qr=4096,
                  km=0, kr=1024, scale=0.125, cap=0.0, dt=dt)
        call = caller(nf.lib.netfuse_attention_tree_fp4, ok)
        for bad in (dict(ws=None), dict(bytes=need - 1), dict(bytes=0), dict(ws=P + 8)):
            assert call(**bad) == EINVAL, (T, dt, bad)


def test_log_probabilities_need_room(nf):                              # noqa: F811
    for V, k in ((1, 0), (100, 5), (50001, 32), (131071, 8)):
        need = nf.lib.netfuse_token_logprobs_workspace(2, 2, 3, V, k)
        assert need > 0
        ok = dict(logits=P, token=P, vocab=P, nodes=P, logp=P, entropy=P, top=P, top_logp=P, ws=P, bytes=need, M=2, B=2, T=3, V=V, n=1, k=k, sm=6 * V, sr=V, scale=1.0, cap=0.0, dt=1)
        call = caller(nf.lib.netfuse_token_logprobs, ok)
        for bad in (dict(ws=None), dict(bytes=need - 1), dict(bytes=0), dict(ws=P + 4)):
            assert call(**bad) == EINVAL, (V, k, bad)
