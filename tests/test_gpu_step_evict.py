"""Caches of 4 bits cut back by netfuse_cache_evict, as the header says: codes, then scales, as bfloat16 rows of half as many bytes; any byte, any number of groups, small and large caches."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C,budget", [(60, 37), (3000, 2048), (20000, 999)])
@pytest.mark.parametrize("d", [8, 32, 64, 96, 128, 200, 256])
def test_any_bytes_are_moved(d, C, budget):
    import paper_2009_13062_amd as nf
    M, B, kv = 2, 1, 2
    g = torch.Generator().manual_seed(d + C)
    cache = [torch.randint(0, 256, t.shape, generator=g, dtype=torch.int64).to(torch.uint8).cuda() for t in nf.cache_fp4(M, B, kv, C, d)]
    before = [t.clone() for t in cache]
    pos = torch.arange(C, dtype=torch.int32, device="cuda").expand(M, B, kv, C).contiguous()
    w = torch.rand(M, B, kv, C, generator=g).cuda()
    L = torch.tensor([[C], [max(1, C - 13)]], dtype=torch.int32, device="cuda")
    pos_out, w_out = torch.full_like(pos, -7), torch.zeros_like(w)
    for keys, values in ((0, 2), (1, 3)):
        nf.cache_evict(cache[keys].view(torch.bfloat16), cache[values].view(torch.bfloat16), pos, w, L, budget, recent=4, start=L, pos_out=pos_out, weight_out=w_out)
    for m in range(M):
        n = min(int(L[m, 0]), budget)
        for h in range(kv):
            stay = pos_out[m, 0, h, :n].long()                        # an entry's position is the slot that it came from
            alive = w[m, 0, h, :int(L[m, 0])].clone()
            alive[-4:] = 2.0                                          # the recent ones stay
            best = alive.sort(descending=True, stable=True).indices[:n]
            assert torch.equal(stay.sort().values, best.sort().values)
            assert torch.equal(w_out[m, 0, h, :n], w[m, 0, h, stay])
            for t, o in zip(cache, before):
                assert torch.equal(t[m, 0, h, :n], o[m, 0, h, stay])
