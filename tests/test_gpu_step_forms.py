"""Every form of the kernels around the decoders' attention that a call's sizes choose: trees over a cache of 4 bits by rows, features, cap and bias, and rotations whose turned features are no
whole pieces."""
import pytest
import torch

import test_gpu_step as S

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def nf():
    import paper_2009_13062_amd as nf
    return nf


# tokens, query heads of a key head: 3 to 80 rows, on both sides of where the kernel or its shares of keys change for 64 (16), 128 (32) and 256 features (64), and 4, 16 and 32 in float32
ROWS = [(1, 3), (4, 1), (5, 1), (4, 4), (17, 1), (12, 2), (32, 1), (11, 3), (24, 2), (64, 1), (13, 5), (40, 2)]


@pytest.mark.parametrize("cap,biased", [(0.0, False), (0.0, True), (20.0, False), (20.0, True)], ids=["raw", "biased", "capped", "capped-biased"])
@pytest.mark.parametrize("T,group", ROWS, ids=lambda x: str(x))
@pytest.mark.parametrize("d", [64, 40, 128, 104, 256, 232])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_tree_fp4_forms(nf, dtype, d, T, group, cap, biased):
    """Two chunks of a cache, the second one's last tile and step cut short, and a cache of less than one tile."""
    case = (1, 2, T, 1100, group, 1, d, cap, biased, T % 2 == 0, False, False, "tree" if T > 1 else "chain", [[1061, 37]])
    rows, cache, L, kw = S.tree_case(nf, case, dtype)
    lse = torch.empty(1, 2 * T, group, device="cuda")
    O = nf.attention_tree_fp4(*rows, *cache, L, lse=lse, **kw)
    S.check_tree(case, dtype, rows, cache, L, kw, O, lse)


#       M  B  S  heads kv  d   rot  sections      inter  norm  positions  lengths: features that turn, or a row of them, which are no whole pieces of the lanes
TURNS = [(2, 2, 3, 5, 3, d, rot, None, inter, norm, "start", False)
         for d, rot in ((64, 36), (64, 20), (80, 20), (80, 44), (128, 4), (128, 124), (256, 12), (256, 252), (4, 4), (12, 8), (70, 32), (255, 128)) for inter in (False, True) for norm in (False, True)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", TURNS, ids=lambda c: "d%d-rot%d-%d%d" % (c[5], c[6], c[8], c[9]))
def test_rotations_of_odd_parts(nf, case, dtype):
    Q, K, B, T, heads, kv, kw = S.rotate_case(case, dtype)
    S.check_rotate(case, dtype, Q, K, kw, *nf.rotate_heads(Q, K, B, T, heads, kv, **kw))
    q, k = Q.contiguous(), K.contiguous()
    S.check_rotate(case, dtype, Q, K, kw, *nf.rotate_heads(q, k, B, T, heads, kv, out_q=q, out_k=k, **kw))          # in place
