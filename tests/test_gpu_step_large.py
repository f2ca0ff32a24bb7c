"""Rotated rows that the last cache does not hold, and rows that it does: the same bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_of_more_than_the_last_cache(dtype):
    """More than 256 MB of results are stored past the caches.  Prompt by prompt, and in two halves, they are stored through them."""
    import paper_2009_13062_amd as nf
    B, heads, kv, d = 6, 24, 8, 128
    S = (280 << 20) // (B * (heads + kv) * d * (2 if dtype == torch.bfloat16 else 4)) + 1
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(1, B * S, (heads + kv) * d, generator=g, device="cuda").to(dtype)
    Q, K = x[:, :, :heads * d], x[:, :, heads * d:]
    gamma = torch.rand(1, d, generator=g, device="cuda") + 0.5
    freq = torch.rand(d // 2, generator=g, device="cuda")
    start = torch.randint(0, 9000, (1, B), generator=g, device="cuda", dtype=torch.int32)
    q, k = nf.rotate_heads(Q, K, B, S, heads, kv, freq=freq, gamma_q=gamma, gamma_k=gamma, start=start)
    for n in (1, 3):
        for b in range(0, B, n):
            rows = slice(b * S, (b + n) * S)
            one = nf.rotate_heads(Q[:, rows], K[:, rows], n, S, heads, kv, freq=freq, gamma_q=gamma, gamma_k=gamma, start=start[:, b:b + n].contiguous())
            assert torch.equal(one[0], q[:, rows]) and torch.equal(one[1], k[:, rows])
    inplace = nf.rotate_heads(Q, K, B, S, heads, kv, freq=freq, gamma_q=gamma, gamma_k=gamma, start=start, out_q=Q, out_k=K)
    assert torch.equal(inplace[0], q) and torch.equal(inplace[1], k)
