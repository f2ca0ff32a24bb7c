"""Calls on a given stream while the current one is busy: nothing that is queued there reaches their memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def busy_blocks(sizes, value):
    """Blocks of these bytes that the current stream will still write, behind some milliseconds of other work, and that are free for the next call."""
    big = torch.ones(4096, 4096, device="cuda")
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    for _ in range(12):
        big = torch.mm(big, big).mul_(1e-4)
    for x in blocks:
        x.fill_(value)


def test_results_of_a_given_stream_are_not_written_by_the_current_one(nf):
    g = torch.Generator().manual_seed(1)
    M, B, T, C, heads, kv, d = 2, 4, 5, 4000, 8, 2, 64
    x = torch.randn(M, B * T, (heads + 2 * kv) * d, generator=g).to(BF).cuda()
    Q, K, V = x[:, :, :heads * d], x[:, :, heads * d:(heads + kv) * d], x[:, :, (heads + kv) * d:]
    Kc, Vc = (torch.randn(M, B, kv, C, d, generator=g).to(BF).cuda() for _ in range(2))
    L = torch.full((M, B), C - T, dtype=torch.int32).cuda()
    w, lse = torch.rand(M, B, kv, C, generator=g).cuda(), torch.empty(M, B * T, heads, device="cuda")
    st = torch.cuda.Stream()

    def calls(stream):
        o = nf.attention_prompt(Q, K, V, B, T, heads, kv, stream=stream)
        p = nf.attention_tree(Q, K, V, Kc, Vc, L, lse=lse, stream=stream)
        return o, p, nf.cache_weigh(Q, lse, Kc, w, L, stream=stream)
    want = [t.clone() for t in calls(None)]
    sizes = [t.numel() * t.element_size() for t in want] + [nf.attention_tree_workspace(M, B, T, C, heads, kv, d, BF)]
    torch.cuda.synchronize()
    for _ in range(3):
        busy_blocks(sizes, 255)                               # NaN in either type
        got = calls(st)
        st.synchronize()
        early = [t.clone() for t in got]
        torch.cuda.synchronize()
        for a, b, c in zip(got, early, want):
            assert torch.equal(a, c) and torch.equal(b, c)


def test_evictions_of_a_given_stream_keep_their_lists(nf):
    """The lists that say which entries move lie in memory of the call's stream."""
    g = torch.Generator().manual_seed(2)
    M, B, kv, C, d, budget = 2, 4, 2, 6000, 64, 2500
    Kc, Vc = (torch.randn(M, B, kv, C, d, generator=g).to(BF).cuda() for _ in range(2))
    pos, w = torch.arange(C, dtype=torch.int32).expand(M, B, kv, C).contiguous().cuda(), torch.rand(M, B, kv, C, generator=g).cuda()
    L = torch.full((M, B), C, dtype=torch.int32).cuda()
    want = [t.clone() for t in (Kc, Vc, pos, w)]
    nf.cache_evict(*want, L, budget)
    st = torch.cuda.Stream()
    for _ in range(3):
        got = [t.clone() for t in (Kc, Vc, pos, w)]
        torch.cuda.synchronize()
        busy_blocks([nf.cache_evict_workspace(M, B, C, kv, budget)], 0)
        nf.cache_evict(*got, L, budget, stream=st)
        st.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
