"""Queries that are no numbers: they spoil what they give weight to, in every kernel, and nothing else."""
import pytest
import torch

import paper_2405_03917_b200 as cq
from tests import bounded as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5


@pytest.mark.parametrize("variant", [0, 1, 2, 3])
@pytest.mark.parametrize("c,Hq,Hkv,n_q,lens", [(8, 8, 2, 20, [300, 90]), (4, 8, 1, 3, [70, 64]), (2, 4, 2, 150, [500, 151]), (8, 4, 1, 150, [400, 149])])
def test_masses_of_tokens_that_the_query_does_not_see(variant, c, Hq, Hkv, n_q, lens):
    # a query in the middle of the new tokens: those behind it get weight from the later queries alone
    cap, i = 512, n_q // 2
    case = B.Case(c + n_q, c, 8, Hq, Hkv, lens, cap)
    q = case.queries(2, n_q)
    k, _ = case.contiguous()
    call = lambda x: cq.cq_attn_mass(x, k, case.kcb, case.seq_lens(), SCALE, c, 8, cap, variant=variant)
    want = call(q)
    bad = q.clone()
    bad[0, i, Hq - 1, 7], bad[1, i, 0, 100] = float("nan"), float("nan")
    got = call(bad)
    for s, h in ((0, Hkv - 1), (1, 0)):
        seen = lens[s] - n_q + i + 1
        assert torch.isnan(got[s, h, :seen]).all()
        assert torch.equal(got[s, h, seen:], want[s, h, seen:])
        others = [j for j in range(Hkv) if j != h]
        assert torch.equal(got[s, others], want[s, others])
