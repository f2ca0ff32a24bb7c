"""What a decoder call on a given stream allocates comes from that stream's pool: memory of the current stream's may still be in use there."""
import contextlib

import pytest
import torch

from test_decoder_host import placed

I32, F32 = torch.int32, torch.float32


class Given:
    cuda_stream = 4096


class Made(torch.Tensor):
    """Memory that a call allocated: the stream whose pool it is from, and the streams that its end waits for."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 0))

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.fixture
def made(monkeypatch):
    import paper_2009_13062_amd as nf
    at, out, now = ["current"], [], "current"
    empty = torch.empty

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    def allocate(shape, dtype=None, device=None):
        t = empty(shape, dtype=dtype).as_subclass(Made)
        t.pool, t.recorded = at[-1], []
        out.append(t)
        return t
    monkeypatch.setattr(nf, "_device", lambda: 0)
    monkeypatch.setattr(nf, "_raw_stream", lambda d: 0)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(torch, "empty_like", lambda x: allocate(x.shape, x.dtype))
    for name in ("attention_prompt", "attention_tree", "cache_weigh", "cache_evict"):
        monkeypatch.setattr(nf.lib, "netfuse_" + name, lambda *a: 0)
    return nf, out


@pytest.mark.parametrize("stream", [None, Given()], ids=["current", "given"])
def test_memory_of_a_call_is_its_streams(made, stream):
    nf, out = made
    M, B, T, C, heads, kv, d = 1, 2, 3, 5000, 4, 2, 64
    Q, K = placed(M, B * T, heads * d), placed(M, B * T, kv * d)
    Kc, L = placed(M, B, kv, C, d), placed(M, B, dtype=I32)
    pos, w = placed(M, B, kv, C, dtype=I32), placed(M, B, kv, C, dtype=F32)
    results = [nf.attention_prompt(Q, K, K, B, T, heads, kv, stream=stream), nf.attention_tree(Q, K, K, Kc, Kc, L, stream=stream),
               nf.cache_weigh(Q, placed(M, B * T, heads, dtype=F32), Kc, w, L, stream=stream)]
    nf.cache_evict(Kc, Kc, pos, w, L, 100, stream=stream)
    assert len(out) == 5                                      # three results, two workspaces
    assert all(t.pool == ("current" if stream is None else stream) for t in out)
    for t in out:                                             # results are used on the current stream, workspaces nowhere else
        assert t.recorded == (["current"] if stream is not None and any(t is r for r in results) else [])
