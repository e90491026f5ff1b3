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


@pytest.mark.parametrize("scale", [0.0, -0.0])
@pytest.mark.parametrize("value", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("variant", [1, 2, 3])
@pytest.mark.parametrize("c,Hq,Hkv,n_q", [(8, 8, 2, 20), (4, 8, 1, 1), (2, 4, 2, 2)])
def test_a_scale_of_zero_hides_no_query(variant, value, scale, c, Hq, Hkv, n_q):
    lens, cap = [300, 90], 304
    case = B.Case(c + n_q, c, 8, Hq, Hkv, lens, cap)
    q = case.queries(2, n_q)
    k, v = case.contiguous()
    bad = q.clone()
    bad[0, n_q - 1, Hq - 1, 5], bad[1, 0, 1, 127] = float(value), float(value)
    hit = torch.zeros(2, n_q, Hq, dtype=torch.bool, device=DEV)
    hit[0, n_q - 1, Hq - 1] = hit[1, 0, 1] = True
    out = cq.cq_window_attn(bad, k, v, case.kcb, case.vcb, case.seq_lens(), scale, c, 8, cap, 0, variant=variant)
    assert torch.isnan(out[hit]).all()
    for s in range(2):
        want, tol, p = B.attend(case, s, q[s], lens[s], 0.0)
        B.check(out[s][~hit[s]], want[~hit[s]], tol[~hit[s]], f"seq {s}")
    mass = cq.cq_attn_mass(bad, k, case.kcb, case.seq_lens(), scale, c, 8, cap, variant=variant)
    for s, h in ((0, Hkv - 1), (1, 1 // (Hq // Hkv))):
        n = lens[s]
        seen = n if s == 0 else n - n_q + 1                              # tokens that the query sees
        assert torch.isnan(mass[s, h, :seen]).all()
        assert torch.isfinite(mass[s, h, seen:]).all()
        others = [i for i in range(Hkv) if i != h]
        assert torch.isfinite(mass[s, others]).all()


@pytest.mark.parametrize("variant", [1, 2, 3])
def test_a_scale_of_zero_weighs_all_visible_tokens_alike(variant):
    case = B.Case(3, 8, 8, 8, 2, [300, 90], 304)
    q = case.queries(2, 20)
    k, v = case.contiguous()
    mass = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), 0.0, 8, 8, 304, variant=variant)
    for s, n in enumerate(case.lens):
        t = torch.arange(n, device=DEV)
        pos = torch.arange(n - 20, n, device=DEV)[:, None]
        want = 4 * ((t[None] <= pos).double() / (pos + 1)).sum(0)
        # a normaliser that is a sum of ones is exact; the weight 2^(0 - log2 n): log2 (two steps of 2^-23 x 9), the exponential (2^-22), and 80 additions
        assert ((mass[s, :, :n].double() - want).abs() <= want * (2 * 9 * 2.0 ** -23 + 2.0 ** -22 + 80 * 2.0 ** -23)).all()
