"""The operators on bounded caches at their edges: batches of many ragged sequences, windows and chunks as long as the cache, shared pages,
caches beyond 4 GiB, queries that are no numbers, captured and concurrent calls."""
import numpy as np
import pytest
import torch

import paper_2405_03917_b200 as cq
from tests import bounded as B
from tests.test_gpu_bounded_evict import check_evict, mass_tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("variant", [0, 2, 3])
@pytest.mark.parametrize("n_seq", [33, 64, 65, 150])
def test_many_ragged_sequences(variant, n_seq):
    # up to 64 sequences are taken by length, more in their order; some have no new tokens, some see nothing
    g = np.random.default_rng(n_seq)
    lens = [int(x) for x in g.integers(0, 300, n_seq)]
    new = [int(min(n, g.integers(0, 40))) for n in lens]
    lens[3], new[3] = 2, 5                                              # more new tokens than cached ones: three rows see nothing
    offsets = np.concatenate([[0], np.cumsum(new)])
    case = B.Case(n_seq, 8, 8, 8, 2, lens, 304)
    q = case.queries(int(offsets[-1]))
    k, v, table = case.paged(16)
    out = torch.full_like(q, 9.0)
    cq.cq_paged_attn(q, ints(offsets), k, v, case.kcb, case.vcb, table, case.seq_lens(), SCALE, 8, 8, 16, 40, out=out, variant=variant)
    for s in range(n_seq):
        lo, hi = int(offsets[s]), int(offsets[s + 1])
        if hi > lo:
            want, tol, _ = B.attend(case, s, q[lo:hi], lens[s], SCALE)
            B.check(out[lo:hi], want, tol, f"variant {variant} seq {s} of {lens[s]} with {new[s]} new")


@pytest.mark.parametrize("n_q", [1, 30])
def test_a_window_as_wide_as_the_cache(n_q):
    case = B.Case(3, 8, 8, 8, 2, [400, 30], 400)
    q = case.queries(2, n_q)
    k, v = case.contiguous()
    call = lambda window, sinks: cq.cq_window_attn(q, k, v, case.kcb, case.vcb, case.seq_lens(), SCALE, 8, 8, 400, window, sinks)
    want = call(0, 0)
    assert torch.equal(call(400, 7), want) and torch.equal(call(1 << 40, 1 << 40), want) and torch.equal(call(0, 9), want)
    want, tol, _ = B.attend(case, 0, q[0], 400, SCALE, 399, 0)
    B.check(call(399, 0)[0], want, tol)
    want, tol, _ = B.attend(case, 0, q[0], 400, SCALE)
    B.check(call(5, 400)[0], want, tol)                                 # sinks as many as there is room: everything is seen


@pytest.mark.parametrize("variant", [0, 1, 2, 3])
def test_a_chunk_as_long_as_the_cache(variant):
    case = B.Case(4, 4, 8, 4, 2, [176, 50, 1, 0], 176)
    q = case.queries(4, 176)
    k, v = case.contiguous()
    out = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, case.seq_lens(), SCALE, 4, 8, 176, 60, 2, variant=variant)
    mass = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 4, 8, 176, variant=variant)
    for s, n in enumerate(case.lens):
        want, tol, _ = B.attend(case, s, q[s, 176 - n:], n, SCALE, 60, 2)
        B.check(out[s, 176 - n:], want, tol, f"seq {s}")
        assert (out[s, :176 - n] == 0).all()                            # queries before the first token see nothing
        if n:
            _, _, p = B.attend(case, s, q[s, 176 - n:], n, SCALE)
            # (the rows that see nothing add nothing: the tolerance of the rows that do)
            tol = mass_tolerance(case, s, q[s, 176 - n:], n, p)
            assert ((mass[s, :, :n].double() - p.view(2, -1, n).sum(1)).abs() <= tol).all(), s


@pytest.mark.parametrize("variant", [0, 1, 2, 3])
def test_sequences_that_share_pages(variant):
    # a common beginning held once; a page twice in one sequence
    case = B.Case(5, 8, 8, 8, 2, [128, 128], 128)
    for rm in (case.kc, case.vc):
        rm[1, :64] = rm[0, :64]
        rm[1, 96:128] = rm[1, 64:96]
    k, v, table = case.paged(32)
    table = table.clone()
    table[1, :2] = table[0, :2]
    table[1, 3] = table[1, 2]
    q = case.queries(41)
    out = cq.cq_paged_attn(q, ints([0, 1, 41]), k, v, case.kcb, case.vcb, table, case.seq_lens(), SCALE, 8, 8, 32, 40, variant=variant)
    for s, (lo, hi) in enumerate([(0, 1), (1, 41)]):
        want, tol, _ = B.attend(case, s, q[lo:hi], 128, SCALE)
        B.check(out[lo:hi], want, tol, f"seq {s}")


def test_caches_beyond_four_gib():
    # the last of nine sequences of 2^20 tokens, 8 heads, 64 groups: 4.5 GiB of codes per tensor
    H, cap, n = 8, 1 << 20, 100
    case = B.Case(6, 2, 8, H, H, [n], 112)
    bufs = []
    for rm in (case.kc, case.vc):
        buf = torch.zeros(cq.cq_codes_bytes(9, cap, H, 128, 2, 8), dtype=torch.uint8, device=DEV)
        buf.view(9, H, cap // 16, 64 * 16)[8, :, :7] = case.codes(rm).view(H, 7, 64 * 16)
        bufs.append(buf)
    lens = ints([0] * 8 + [n])
    for n_q, variants in ((1, (0, 1, 2)), (40, (0, 3))):
        q = case.queries(9, n_q)
        want, tol, p = B.attend(case, 0, q[8], n, SCALE, 70, 3)
        _, _, p = B.attend(case, 0, q[8], n, SCALE)
        for variant in variants:
            out = cq.cq_window_attn(q, *bufs, case.kcb, case.vcb, lens, SCALE, 2, 8, cap, 70, 3, variant=variant)
            B.check(out[8], want, tol, f"variant {variant}")
            assert (out[:8] == 0).all()
            mass = cq.cq_attn_mass(q, bufs[0], case.kcb, lens, SCALE, 2, 8, cap, variant=variant)
            assert ((mass[8, :, :n].double() - p.view(H, -1, n).sum(1)).abs() <= mass_tolerance(case, 0, q[8], n, p)).all(), variant
            assert (mass[:8] == 0).all() and (mass[8, :, n:] == 0).all()
    weights = torch.rand(9, H, cap, device=DEV)
    out_codes = [torch.zeros(cq.cq_codes_bytes(9, 48, H, 128, 2, 8), dtype=torch.uint8, device=DEV) for _ in range(2)]
    kept, left = cq.cq_evict(weights, *bufs, lens, 128, 2, 8, cap, 48, 4, 10, k_codes_out=out_codes[0], v_codes_out=out_codes[1],
                             mass_out=torch.zeros(9, H, 48, device=DEV), out_max_tokens=48)
    assert left.tolist() == [0] * 8 + [48]
    for x, rm in zip(out_codes, (case.kc, case.vc)):
        got = case.rowmajor(x, 9, 48)
        for h in range(H):
            at = B.evict_plain(weights[8, h, :n].cpu().numpy(), n, 48, 4, 10)
            np.testing.assert_array_equal(kept[8, h].cpu().numpy(), at)
            np.testing.assert_array_equal(got[8, :, h], rm[0, at, h])


@pytest.mark.parametrize("variant", [1, 2, 3])
def test_a_query_that_is_no_number_spoils_its_own_rows_alone(variant):
    case = B.Case(7, 8, 8, 8, 2, [300, 90], 304)
    q = case.queries(2, 20)
    k, v = case.contiguous()
    call = lambda x: cq.cq_window_attn(x, k, v, case.kcb, case.vcb, case.seq_lens(), SCALE, 8, 8, 304, 0, variant=variant)
    want = call(q)
    bad = q.clone()
    bad[0, 7, 5], bad[1, 0, 2, 3] = float("nan"), float("nan")
    got = call(bad)
    assert torch.isnan(got[0, 7, 5]).all() and torch.isnan(got[1, 0, 2]).all()
    keep = torch.ones(2, 20, 8, dtype=torch.bool, device=DEV)
    keep[0, 7, 5] = keep[1, 0, 2] = False
    for s in range(2):
        ref, tol, _ = B.attend(case, s, q[s], case.lens[s], SCALE)
        B.check(got[s][keep[s]], ref[keep[s]], tol[keep[s]], f"seq {s}")
    assert torch.isfinite(want).all()
    # masses: the KV head's of that sequence are no numbers, the others as they were
    mass = lambda x: cq.cq_attn_mass(x, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 304, variant=variant)
    first, second = mass(q), mass(bad)
    assert torch.isnan(second[0, 1, :288]).all() and torch.isnan(second[1, 0, :71]).all()      # the tokens that the query sees
    assert torch.equal(second[0, 0], first[0, 0]) and torch.equal(second[1, 1], first[1, 1])


def test_captured_steps_over_pages():
    # append and attention in one graph, replayed with other lengths, offsets, tables and inputs in the same buffers
    H, Hq, page, n_pages = 2, 8, 16, 40
    case = B.Case(8, 8, 8, Hq, H, [0, 0, 0], 160)
    g = torch.Generator().manual_seed(8)
    books = [case.kcb.float(), case.vcb.float()]
    rows = 50
    new_pools = lambda: [torch.zeros(cq.cq_codes_bytes(n_pages, page, H, 128, 8, 8), dtype=torch.uint8, device=DEV) for _ in range(2)]
    k, v = (torch.randn(rows, H, 128, generator=g).half().to(DEV) for _ in range(2))
    q = case.queries(rows)
    perm = np.random.default_rng(8).permutation(n_pages)[:30].reshape(3, 10)
    offsets, table, lens = ints([0, 1, 40, 50]), ints(perm), ints([1, 39, 10])
    pools, out = new_pools(), torch.zeros_like(q)
    ws_a = torch.empty(cq.cq_paged_append_workspace_bytes(rows, H, 128, 8, 8), dtype=torch.uint8, device=DEV)
    ws_b = torch.empty(cq.cq_paged_attn_workspace_bytes(3, rows, 40, Hq, H, 128, 8, 8, page, 10), dtype=torch.uint8, device=DEV)

    def step(pools, out, ws_a, ws_b):
        cq.cq_paged_append(k, v, offsets, *books, table, lens, 8, 8, page, 40, *pools, workspace=ws_a)
        cq.cq_paged_attn(q, offsets, *pools, case.kcb, case.vcb, table, lens, SCALE, 8, 8, page, 40, out=out, workspace=ws_b)

    step(pools, out, ws_a, ws_b)
    for p in pools:
        p.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pools, out, ws_a, ws_b)
    other, want = new_pools(), torch.zeros_like(q)
    for off, at, n in (([0, 1, 40, 50], perm, [1, 39, 10]), ([0, 20, 20, 22], perm[:, ::-1], [25, 39, 100]), ([0, 40, 41, 50], perm, [140, 40, 19])):
        offsets.copy_(ints(off))
        table.copy_(ints(at.copy()))
        lens.copy_(ints(n))
        q.copy_(q.flip(0))
        k.copy_(k.flip(0))
        out.zero_()
        want.zero_()
        ws_b.fill_(255)
        graph.replay()
        step(other, want, torch.empty_like(ws_a), torch.empty_like(ws_b))
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isfinite(out).all()
        assert torch.equal(pools[0], other[0]) and torch.equal(pools[1], other[1])


@pytest.mark.parametrize("n_q", [1, 3, 90])
def test_captured_masses(n_q):
    case = B.Case(9, 8, 8, 8, 2, [900, 200], 912)
    q = case.queries(2, n_q)
    k, _ = case.contiguous()
    lens = case.seq_lens()
    mass = torch.zeros(2, 2, 912, device=DEV)
    ws = torch.empty(cq.cq_attn_mass_workspace_bytes(2, n_q, 8, 2, 128, 8, 8, 912), dtype=torch.uint8, device=DEV)
    call = lambda x: cq.cq_attn_mass(q, k, case.kcb, lens, SCALE, 8, 8, 912, x, x, workspace=ws)
    call(mass)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(mass)
        call(mass)
    for n in ([900, 200], [n_q, 912], [0, 100]):
        lens.copy_(ints(n))
        mass.fill_(0.5)
        want = mass.clone()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for _ in range(2):
            call(want)
        torch.cuda.synchronize()
        assert torch.equal(mass, want)


def test_calls_at_once_on_two_streams():
    # each with a workspace of its own
    case = B.Case(10, 8, 8, 8, 2, [3000, 1200, 600], 3008)
    k, v = case.contiguous()
    pk, pv, table = case.paged(64)
    lens, offsets = case.seq_lens(), ints([0, 1, 300, 302])
    q, one = case.queries(302), case.queries(3, 1)
    many = case.queries(3, 100)

    def all_of_them():
        return [cq.cq_paged_attn(q, offsets, pk, pv, case.kcb, case.vcb, table, lens, SCALE, 8, 8, 64, 299),
                cq.cq_window_attn(one, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 3008, 1000, 4),
                cq.cq_attn_mass(one, k, case.kcb, lens, SCALE, 8, 8, 3008), cq.cq_attn_mass(many, k, case.kcb, lens, SCALE, 8, 8, 3008)]
    want = all_of_them()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(all_of_them())
    torch.cuda.synchronize()
    for one_call in got:
        for a, b_ in zip(one_call, want):
            assert torch.equal(a, b_)


def test_masses_that_are_no_numbers_of_either_sign_stay():
    case = B.Case(11, 8, 8, 2, 2, [500], 512)
    mass = np.random.default_rng(11).standard_normal((1, 2, 512)).astype(np.float32)
    bits = mass.view(np.uint32)
    bits[0, 0, [20, 30, 400]] = [0xffc00000, 0xff800001, 0x7f800001]
    mass[0, 1, :] = -np.inf                                             # all alike, the lowest there is
    check_evict(case, mass, 100, 2, 8, 128)
    check_evict(case, mass, 100, 2, 8)


@pytest.mark.parametrize("keep,sinks,recent", [(512, 0, 0), (511, 511, 0), (511, 0, 511), (16, 8, 8)])
def test_evictions_that_leave_no_choice(keep, sinks, recent):
    case = B.Case(12, 4, 8, 2, 2, [512, 511, 17], 512)
    mass = np.random.default_rng(12).exponential(1.0, (3, 2, 512)).astype(np.float32)
    check_evict(case, mass, keep, sinks, recent, keep)
    check_evict(case, mass, keep, sinks, recent)


def test_the_learner_and_the_masses_in_one_process():
    # every call site opts in to its own shared memory
    g = torch.Generator().manual_seed(13)
    x = torch.randn(600, 1, 128, generator=g).half().to(DEV)
    for c in (8, 4):
        u = torch.rand(1, 128 // c, 256, generator=g, dtype=torch.float64).to(DEV)
        assert torch.isfinite(cq.cq_learn_centroids(x, None, u, c, 8, 3)[0]).all()
    for c in (8, 4, 2):
        case = B.Case(13 + c, c, 8, 8, 2, [300, 90], 304)
        k, _ = case.contiguous()
        for n_q, variant in ((1, 2), (2, 2), (40, 3)):
            q = case.queries(2, n_q)
            got = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, c, 8, 304, variant=variant)
            _, _, p = B.attend(case, 0, q[0], 300, SCALE)
            assert ((got[0, :, :300].double() - p.view(2, -1, 300).sum(1)).abs() <= mass_tolerance(case, 0, q[0], 300, p)).all()
