"""cq_paged_attn writes nothing behind a workspace of exactly the size it asks for: the workspace is the front of a larger buffer, whose rest has to
keep its pattern, and the results are those of the 64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2405_03917_b200 as cq
from tests import bounded as B
from tests.test_workspace_plans import SERVED, mix

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5
BEHIND = 24 << 20                                    # more than all partial sums that a call can lay out (148 slots of 133 KB)


@pytest.mark.parametrize("variant", [0, 2, 3])
@pytest.mark.parametrize("m", SERVED + [mix([1] * 20 + [300, 40], 8, 2, 2048, c=4, page=48, window=700, sinks=5)], ids=lambda m: f"{len(m['new'])}x{m['rows']}on{m['hkv']}")
def test_nothing_is_written_behind_the_workspace(m, variant):
    new, cap = m["new"], m["per_seq"] * m["page"]
    g = np.random.default_rng(m["rows"])
    lens = [int(x) for x in g.integers(1, 1500, len(new))]
    lens = [cap - 3 if x == max(new) else max(n, x) for n, x in zip(lens, new)]
    offsets = np.concatenate([[0], np.cumsum(new)]).tolist()
    case = B.Case(m["rows"], m["c"], 8, m["hq"], m["hkv"], lens, cap)
    k, v, table = case.paged(m["page"])
    q = case.queries(offsets[-1])
    size = cq.cq_paged_attn_workspace_bytes(len(new), offsets[-1], m["max_q"], m["hq"], m["hkv"], 128, m["c"], 8, m["page"], m["per_seq"], m["window"],
                                            m["sinks"])
    buffer = torch.full((size + BEHIND,), 0x5A, dtype=torch.uint8, device=DEV)
    out = cq.cq_paged_attn(q, torch.tensor(offsets, dtype=torch.int32, device=DEV), k, v, case.kcb, case.vcb, table, case.seq_lens(), SCALE, m["c"], 8,
                           m["page"], m["max_q"], m["window"], m["sinks"], workspace=buffer[:size], variant=variant)
    assert (buffer[size:] == 0x5A).all()
    for s in range(len(new)):
        lo, hi = offsets[s], offsets[s + 1]
        want, tol, _ = B.attend(case, s, q[lo:hi], lens[s], SCALE, m["window"], m["sinks"])
        B.check(out[lo:hi], want, tol, f"seq {s} of {lens[s]} with {new[s]} new")


def test_a_workspace_one_byte_short_is_refused():
    m = SERVED[0]
    case = B.Case(1, 8, 8, 32, 32, [64] * 4, m["per_seq"] * m["page"])
    k, v, table = case.paged(m["page"])
    size = cq.cq_paged_attn_workspace_bytes(4, 23, 20, 32, 32, 128, 8, 8, m["page"], m["per_seq"])
    out = torch.full((23, 32, 128), 3.0, dtype=torch.float16, device=DEV)
    with pytest.raises(cq.CQError) as e:
        cq.cq_paged_attn(case.queries(23), torch.tensor([0, 1, 2, 3, 23], dtype=torch.int32, device=DEV), k, v, case.kcb, case.vcb, table, case.seq_lens(),
                         SCALE, 8, 8, m["page"], 20, out=out, workspace=torch.empty(size - 1, dtype=torch.uint8, device=DEV))
    assert e.value.status == -5 and (out == 3.0).all()
