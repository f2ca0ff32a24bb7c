"""Log probabilities under caps and scales of any size: quotients and powers of them that are no float32 number, and caps so large that tanh's error is large."""
import pytest
import torch

import step_plain as P

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


def check(nf, x, scale, cap, k=4):
    x = x.cuda()
    token = torch.randint(0, x.shape[2], (*x.shape[:2], 3), generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    want = P.logprobs(x, token, k, None, None, scale, cap)
    logp, entropy, top, top_logp = nf.token_logprobs(x, token, k=k, scale=scale, cap=cap)
    P.near(logp, want[0], want[1])
    P.near(entropy, want[2], want[3])
    assert torch.equal(top.cpu(), want[4])
    P.near(top_logp, want[5], want[6])


# scale / cap: infinite, largest, smallest, 0 in float32.  `size` is that of the logits, so that scale * logit is about 3 or the cap decides.
RATIOS = [(1e20, 1e-20, 1.0), (1e10, 1e-30, 3.0), (1e30, 1e-30, 1e-30), (1e-20, 1e30, 3e20), (1e-30, 1e30, 3e30), (1e-8, 1e30, 3e8), (1e-30, 1e-30, 1.0)]


@pytest.mark.parametrize("scale,cap,size", RATIOS, ids=str)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_scale_over_cap_of_any_size(nf, dtype, scale, cap, size):
    """Every third logit is 0, and so is what it stands for."""
    x = torch.randn(1, 3, 4500, generator=torch.Generator().manual_seed(2)) * size
    x[:, :, ::3] = 0
    x[0, 2] = 0
    check(nf, x.to(dtype), scale, cap)


# Powers of scale / cap times scale that float32 does not hold, too small (the first four) and too large ones.
POWERS = [(1e-3, 9.9), (0.01, 90.0), (0.003, 28.0), (1e-4, 0.9), (100.0, 0.02), (9000.0, 1.0), (1e5, 30.0), (1e10, 1e7)]


@pytest.mark.parametrize("reach", [0.3, 0.7])
@pytest.mark.parametrize("scale,cap", POWERS, ids=str)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_powers_that_leave_float32(nf, dtype, scale, cap, reach):
    """Logits up to `reach` caps, of either sign and all negative, in a row of a few whole chunks."""
    x = (torch.rand(1, 2, 8192, generator=torch.Generator().manual_seed(3)) * 2 - 1) * (reach * cap / scale)
    x[0, 1] = -x[0, 1].abs()
    check(nf, x.to(dtype), scale, cap)


@pytest.mark.parametrize("reach", [0.3, 0.7, 3.0])
@pytest.mark.parametrize("cap", [1e6, 1e9, 1e30])
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_caps_whose_error_is_large(nf, dtype, cap, reach):
    """The largest logit has the largest x, whatever the errors of tanh are: half a million of units of a cap of 1e12, say.  No probability is above 1."""
    x = (torch.rand(1, 40, 4500, generator=torch.Generator().manual_seed(4)) * 2 - 1) * reach
    x[0, 20:, 1::2] = 0.2499                                          # on either side of where the form of tanh changes
    x[0, 20:, 0] = torch.linspace(0.2501, 0.26, 20)
    check(nf, x.to(dtype), min(cap, 1e30), cap)
    logp = nf.token_logprobs(x.to(dtype).cuda(), k=8, scale=cap, cap=cap)[3]
    assert (logp <= 0).all()


@pytest.mark.parametrize("c,t", [(30.0, 0.7), (15.0, 2.5), (50.0, 1.0)])
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_temperature_after_a_cap(nf, dtype, c, t):
    """Logits capped by the model and divided by a temperature afterwards are scale 1 / t under the cap c / t; under the cap c they are another distribution."""
    x = (torch.randn(1, 3, 5000, generator=torch.Generator().manual_seed(6)) * 8).to(dtype)
    z = (c * torch.tanh(x.double() / c) / t)
    want = torch.log_softmax(z, -1)
    token = z.topk(5, -1).indices.to(torch.int32)
    room = P.logprobs(x, token, 0, None, None, 1 / t, c / t)[1]      # the operator's own bound of its own definition
    logp = nf.token_logprobs(x.cuda(), token.cuda(), scale=1 / t, cap=c / t)[0]
    # 1 / t and c / t are rounded to float32: the quotient by 2^-23, the factor outside by 2^-24, of x and of the largest x
    P.near(logp, want.gather(-1, token.long()), room + 2.0 ** -22 * 2 * z.abs().amax())
    if t != 1:
        other = nf.token_logprobs(x.cuda(), token.cuda(), scale=1 / t, cap=c)[0].cpu().double()
        assert ((other - want.gather(-1, token.long())).abs() > 100 * room).any()


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 0.25, 0.5])
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_largest_and_lowest_logits_in_a_row(nf, dtype, scale):
    """Their difference leaves float32, times the scale it does not."""
    x = torch.randn(1, 3, 2600, generator=torch.Generator().manual_seed(7)).to(dtype)
    x[0, :, 100], x[0, 0, 200:], x[0, 1, 2500] = torch.finfo(dtype).max, torch.finfo(dtype).min, torch.finfo(dtype).min
    token = torch.tensor([100, 250, 2500, 7], dtype=torch.int32).expand(1, 3, 4).contiguous()
    want = P.logprobs(x, token, 3, None, None, scale, 0.0)
    logp, entropy, top, top_logp = nf.token_logprobs(x.cuda(), token.cuda(), k=3, scale=scale)
    P.near(logp, want[0], want[1])
    P.near(entropy, want[2], want[3])
    assert torch.equal(top.cpu(), want[4])
    P.near(top_logp, want[5], want[6])
