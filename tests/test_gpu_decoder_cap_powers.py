"""Caps and scales whose quotient float32 holds, but not its powers times the scale: rows of zero scores give the mean of what they see, over caches of bfloat16 and of 4 bits."""
import pytest
import torch

import decoder_plain as plain
import step_plain

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("scale,cap", [(1e16, 1.1e12), (1e30, 1.1e26), (1e33, 1e30), (1e20, 1e17), (1e-20, 9e-17)], ids=str)
@pytest.mark.parametrize("biased", [False, True], ids=["", "biased"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_powers_of_scale_over_cap(nf, d, biased, scale, cap):
    """Every second query is 0.  The others' scores are decided by an overflow or the cap's size: finite results."""
    g = torch.Generator().manual_seed(d)
    heads, kv, C, T = 4, 1, 150, 26
    zero = torch.arange(T) % 2 == 0
    Q = torch.randn(1, T, heads * d, generator=g) * (0.1 * cap / scale / d ** 0.5)
    Q[:, zero] = 0
    Q, K, V = (x.to(BF).cuda() for x in (Q, torch.randn(1, T, kv * d, generator=g), torch.randn(1, T, kv * d, generator=g)))
    kw = dict(scale=scale, cap=cap, slope=(torch.rand(1, heads, generator=g) * 0.1).cuda() if biased else None)

    def check(got, want, tol):
        assert got.isfinite().all()
        off = (got.cpu().double() - want).abs()[0, zero]
        assert (off <= tol[0, zero]).all()
    check(nf.attention_prompt(Q, K, V, 1, T, heads, kv, **kw), *plain.prompt(Q, K, V, 1, T, heads, kv, **kw))
    L = ints([[C - 3]])
    dense = [torch.randn(1, 1, kv, C, d, generator=g) for _ in range(2)]
    held = [t.to(BF).cuda() for t in dense]
    check(nf.attention_tree(Q, K, V, *held, L, **kw), *plain.tree(Q, K, V, *held, L, **kw)[:2])
    codes = [t.cuda() for x in dense for t in step_plain.quantise(x)]
    opened = [step_plain.dequantise(codes[i], codes[i + 1], d) for i in (0, 2)]
    check(nf.attention_tree_fp4(Q, K, V, *codes, L, **kw), *plain.tree(Q, K, V, *opened, L, **kw)[:2])
