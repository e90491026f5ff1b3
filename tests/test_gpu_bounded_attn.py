"""GPU parity of cq_window_attn and cq_paged_attn with the 64-bit definition: every kernel, windows and sinks that end anywhere, ragged
chunks, queries that see nothing, pages in any order, absent pages, rows of no sequence, streams and captured graphs."""
import numpy as np
import pytest
import torch

import paper_2405_03917_b200 as cq
from tests import bounded as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5


def run_window(case, q, window, sinks, variant, scale=SCALE, lens=None, **kw):
    k, v = case.contiguous()
    return cq.cq_window_attn(q, k, v, case.kcb, case.vcb, case.seq_lens(lens), scale, case.c, case.b, case.cap, window, sinks, variant=variant, **kw)


def check_window(case, q, window, sinks, variant, scale=SCALE):
    out = run_window(case, q, window, sinks, variant, scale)
    for s, n in enumerate(case.lens):
        want, tol, _ = B.attend(case, s, q[s], min(n, case.cap), scale, window, sinks)
        B.check(out[s], want, tol, f"variant {variant} seq {s} of {n} window {window} sinks {sinks}")


VARIANTS = [1, 2, 3]


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("c,Hq,Hkv,n_q", [(8, 8, 2, 1), (8, 4, 4, 1), (4, 8, 2, 3), (2, 4, 2, 2), (8, 8, 1, 5), (4, 6, 2, 4), (8, 4, 1, 70), (4, 3, 1, 99),
                                          (2, 2, 2, 140), (8, 40, 1, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 0), (64, 4), (1, 0), (17, 40), (500, 3)])
def test_window(variant, c, Hq, Hkv, n_q, window, sinks):
    lens = [700, n_q, 333, 1, 0, 65 + n_q]
    case = B.Case(c * 100 + Hq + n_q, c, 8, Hq, Hkv, lens, 704)
    check_window(case, case.queries(len(lens), n_q), window, sinks, variant)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 2000])
def test_every_length(variant, n):
    case = B.Case(n, 8, 8, 8, 2, [n, max(1, n - 1)], n + 5)
    check_window(case, case.queries(2, 1), 0, 0, variant)
    check_window(case, case.queries(2, 1), 30, 2, variant)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("scale", [-0.07, 0.0, 1.5])
def test_scales(variant, scale):
    # large scores move the softmax's reference often; a negative scale turns their order around
    case = B.Case(5, 8, 8, 8, 2, [900, 130], 900, spread=2.0)
    q = case.queries(2, 3)
    check_window(case, q, 400, 5, variant, scale)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("b", [1, 5, 7])
def test_fewer_than_256_centroids(variant, b):
    case = B.Case(b, 8, b, 4, 2, [300, 77], 300)
    check_window(case, case.queries(2, 6), 120, 3, variant)


@pytest.mark.parametrize("c,b,D,Hq,Hkv", [(8, 10, 128, 4, 2), (4, 8, 64, 4, 1), (3, 4, 96, 2, 2), (8, 9, 256, 4, 4), (1, 6, 40, 3, 1)])
def test_other_shapes_take_the_plain_kernel(c, b, D, Hq, Hkv):
    case = B.Case(c + b, c, b, Hq, Hkv, [150, 9, 0], 160, D=D)
    q = case.queries(3, 4)
    check_window(case, q, 50, 2, 0, D ** -0.5)


def test_many_short_and_few_long_contexts():
    # more items than CTAs, and a context that many CTAs share
    case = B.Case(3, 8, 8, 8, 2, [int(x) for x in np.random.default_rng(0).integers(0, 90, 200)], 96)
    check_window(case, case.queries(200, 1), 0, 0, 0)
    long = B.Case(4, 8, 8, 8, 2, [30001], 30016)
    check_window(long, long.queries(1, 1), 0, 0, 0)
    check_window(long, long.queries(1, 20), 0, 0, 0)
    check_window(long, long.queries(1, 20), 7777, 100, 0)


def test_lengths_outside_of_the_capacity_are_clamped():
    case = B.Case(6, 8, 8, 4, 1, [200, 0], 200)
    q = case.queries(2, 2)
    out = run_window(case, q, 64, 1, 0, lens=[100000, -5])
    want, tol, _ = B.attend(case, 0, q[0], 200, SCALE, 64, 1)
    B.check(out[0], want, tol)
    assert (out[1] == 0).all()


def test_codes_behind_the_length_do_not_matter():
    case = B.Case(8, 8, 8, 8, 2, [37, 100], 112)
    q = case.queries(2, 1)
    k, v = case.contiguous()
    first = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, case.seq_lens(), SCALE, 8, 8, 112, 20, 3)
    other = B.Case(9, 8, 8, 8, 2, [37, 100], 112)
    for a, b_ in ((case.kc, other.kc), (case.vc, other.vc)):
        b_[0, :37], b_[1, :100] = a[0, :37], a[1, :100]
    k2, v2 = other.contiguous()
    second = cq.cq_window_attn(q, k2, v2, case.kcb, case.vcb, case.seq_lens(), SCALE, 8, 8, 112, 20, 3)
    assert torch.equal(first, second)


# ------------------------------------------------------------------------------------------ pages

def run_paged(case, q, offsets, page, max_q, variant=0, window=0, sinks=0, seed=0, out=None, table=None, lens=None, **kw):
    k, v, t = case.paged(page, seed)
    offs = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    return cq.cq_paged_attn(q, offs, k, v, case.kcb, case.vcb, t if table is None else table, case.seq_lens(lens), SCALE, case.c, case.b, page, max_q,
                            window, sinks, out=out, variant=variant, **kw)


@pytest.mark.parametrize("variant", [0] + VARIANTS)
@pytest.mark.parametrize("page", [16, 48, 64, 256])
@pytest.mark.parametrize("c,Hq,Hkv,window,sinks", [(8, 8, 2, 0, 0), (4, 4, 4, 90, 5), (2, 6, 2, 0, 0)])
def test_paged_ragged(variant, page, c, Hq, Hkv, window, sinks):
    lens, new = [517, 64, 1, 300, 0, 33], [1, 40, 1, 0, 0, 33]
    offsets = np.concatenate([[0], np.cumsum(new)])
    case = B.Case(page + c, c, 8, Hq, Hkv, lens, 528)
    q = case.queries(int(offsets[-1]) + 3)                          # three rows of no sequence at the end
    out = torch.full((q.shape[0], Hq, 128), 7.0, dtype=torch.float16, device=DEV)
    run_paged(case, q, offsets.tolist(), page, max(new), variant, window, sinks, out=out)
    for s in range(len(lens)):
        lo, hi = int(offsets[s]), int(offsets[s + 1])
        want, tol, _ = B.attend(case, s, q[lo:hi], lens[s], SCALE, window, sinks)
        B.check(out[lo:hi], want, tol, f"variant {variant} seq {s} page {page}")
    assert (out[int(offsets[-1]):] == 7.0).all()


@pytest.mark.parametrize("variant", [0] + VARIANTS)
def test_absent_pages(variant):
    # entries outside of the pool: their tokens are absent; a sequence without any page gets zero rows
    lens, new = [200, 130, 90], [3, 20, 2]
    offsets = [0, 3, 23, 25]
    case = B.Case(21, 8, 8, 8, 2, lens, 256)
    q = case.queries(25)
    k, v, t = case.paged(32)
    t = t.clone()
    t[0, 2], t[1, 0], t[2, :] = -1, 1 << 30, -7
    out = cq.cq_paged_attn(q, torch.tensor(offsets, dtype=torch.int32, device=DEV), k, v, case.kcb, case.vcb, t, case.seq_lens(), SCALE, 8, 8, 32, 20,
                           variant=variant)
    for s in range(3):
        absent = torch.zeros(256, dtype=torch.bool, device=DEV)
        for j in range(8):
            if not 0 <= int(t[s, j]) < k.numel() // (32 * 2 * 16):
                absent[j * 32:(j + 1) * 32] = True
        want, tol, _ = B.attend(case, s, q[offsets[s]:offsets[s + 1]], lens[s], SCALE, absent=absent)
        B.check(out[offsets[s]:offsets[s + 1]], want, tol, f"variant {variant} seq {s}")
    assert (out[23:] == 0).all()


@pytest.mark.parametrize("variant", [0] + VARIANTS)
def test_counts_above_max_q_and_wild_offsets(variant):
    lens = [100, 80]
    case = B.Case(22, 8, 8, 4, 2, lens, 112)
    q = case.queries(30)
    out = torch.full_like(q, 3.0)
    # sequence 0 claims 25 rows with max_q 20; sequence 1 the rows from 25 to far beyond the end
    run_paged(case, q, [0, 25, 1 << 29], 16, 20, variant, out=out)
    want, tol, _ = B.attend(case, 0, q[:20], 100, SCALE)
    B.check(out[:20], want, tol)
    assert (out[20:25] == 3.0).all()
    want, tol, _ = B.attend(case, 1, q[25:30], 80, SCALE)
    B.check(out[25:30], want, tol)
    out.fill_(3.0)
    run_paged(case, q, [-9, -4, -20], 16, 20, variant, out=out)
    assert (out == 3.0).all()


def test_pages_far_into_a_large_pool():
    # byte offsets beyond 32 bits: 2^18 pages of 16 tokens, 8 heads, 32 groups are 2^30 * 4 bytes
    n_pages, H, G = (1 << 18) + 64, 8, 32
    case = B.Case(23, 4, 8, 8, H, [64], 64)
    pools = []
    for rm in (case.kc, case.vc):
        pool = torch.zeros(n_pages * H * G * 16, dtype=torch.uint8, device=DEV)
        codes = case.codes(rm).view(H, 4, G * 16)
        for j in range(4):
            page = n_pages - 1 - 5 * j
            pool.view(n_pages, H, G * 16)[page] = codes[:, j]
        pools.append(pool)
    table = torch.tensor([[n_pages - 1, n_pages - 6, n_pages - 11, n_pages - 16]], dtype=torch.int32, device=DEV)
    for n_q, variant in ((1, 0), (20, 0), (2, 1)):
        q = case.queries(n_q)
        out = cq.cq_paged_attn(q, torch.tensor([0, n_q], dtype=torch.int32, device=DEV), *pools, case.kcb, case.vcb, table, case.seq_lens(), SCALE, 4, 8,
                               16, n_q, variant=variant)
        want, tol, _ = B.attend(case, 0, q, 64, SCALE)
        B.check(out, want, tol, f"variant {variant}")


# ------------------------------------------------------------------------------------------ streams, graphs, workspaces

def test_other_streams_and_captured_graphs():
    case = B.Case(31, 8, 8, 8, 2, [900, 40, 333], 912)
    k, v = case.contiguous()
    lens = case.seq_lens()
    for n_q in (1, 40):
        q = case.queries(3, n_q)
        eager = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 912, 300, 4)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            there = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 912, 300, 4)
        side.synchronize()
        assert torch.equal(there, eager)
        size = cq.cq_window_attn_workspace_bytes(3, n_q, 8, 2, 128, 8, 8, 912, 300, 4)
        ws = torch.empty(size, dtype=torch.uint8, device=DEV)
        out = torch.zeros_like(eager)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 912, 300, 4, out=out, workspace=ws)
            cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 912, 300, 4, out=out, workspace=ws)
        for fill in (0, 255):
            ws.fill_(fill)                                              # what a workspace holds before does not matter
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
        # the same graph with other lengths and queries in the same buffers
        lens2 = torch.tensor([500, 41, 1], dtype=torch.int32, device=DEV)
        q.copy_(torch.flip(q, [0]))
        keep = lens.clone()
        lens.copy_(lens2)
        graph.replay()
        again = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens2, SCALE, 8, 8, 912, 300, 4)
        assert torch.equal(out, again)
        lens.copy_(keep)


def test_calls_back_to_back_on_two_streams():
    case = B.Case(32, 8, 8, 8, 2, [3000, 2500], 3008)
    k, v = case.contiguous()
    lens = case.seq_lens()
    qs = [case.queries(2, 1) for _ in range(6)]
    want = [cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 3008, 0) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i, q in enumerate(qs):
        with torch.cuda.stream(streams[i % 2]):
            got.append(cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, 8, 8, 3008, 0))
    torch.cuda.synchronize()
    for a, b_ in zip(got, want):
        assert torch.equal(a, b_)


def test_workspace_too_small_is_refused():
    case = B.Case(33, 8, 8, 8, 2, [3000], 3008)
    k, v = case.contiguous()
    q = case.queries(1, 1)
    size = cq.cq_window_attn_workspace_bytes(1, 1, 8, 2, 128, 8, 8, 3008, 0)
    with pytest.raises(cq.CQError) as e:
        cq.cq_window_attn(q, k, v, case.kcb, case.vcb, case.seq_lens(), SCALE, 8, 8, 3008, 0, workspace=torch.empty(size - 16, dtype=torch.uint8, device=DEV))
    assert e.value.status == -5


# ------------------------------------------------------------------------------------------ the way into the pages, and a run of all

@pytest.mark.parametrize("c,b", [(8, 8), (4, 8), (8, 10), (2, 8), (8, 9)])
def test_append_writes_the_codes_of_encode(c, b):
    H, D, page = 2, 128, 32
    g = torch.Generator().manual_seed(c * b)
    new, before = [37, 1, 0, 16], [5, 63, 10, 32]
    lens = [a + m for a, m in zip(before, new)]
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
    rows = sum(new)
    k, v = (torch.randn(rows, H, D, generator=g).half().to(DEV) for _ in range(2))
    books = [torch.randn(H, D // c, 1 << b, c, generator=g).half().float().to(DEV) for _ in range(2)]
    n_pages = 12
    bytes_ = cq.cq_codes_bytes(n_pages, page, H, D, c, b)
    pools = [torch.full((bytes_,), 0x5a, dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.tensor([[7, 2, -1, -1], [3, 11, -1, -1], [0, -1, -1, -1], [9, 1, -1, -1]], dtype=torch.int32, device=DEV)
    old = [cq.cq_codes_to_rowmajor(p, n_pages, page, H, D, c, b).clone() for p in pools]
    cq.cq_paged_append(k, v, offsets, *books, table, torch.tensor(lens, dtype=torch.int32, device=DEV), c, b, page, 37, *pools)
    for x, book, pool, was in zip((k, v), books, pools, old):
        buf = torch.zeros(cq.cq_codes_bytes(1, rows, H, D, c, b), dtype=torch.uint8, device=DEV)
        cq.cq_encode(x[None], book, c, b, buf, rows)
        codes = cq.cq_codes_to_rowmajor(buf, 1, rows, H, D, c, b)[0]
        want = was.clone()
        for s in range(4):
            for i in range(new[s]):
                t = before[s] + i
                want[int(table[s, t // page]), t % page] = codes[int(offsets[s]) + i]
        assert torch.equal(cq.cq_codes_to_rowmajor(pool, n_pages, page, H, D, c, b), want)


def test_append_skips_what_has_no_place():
    H, D, c, b, page = 1, 128, 8, 8, 16
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(20, H, D, generator=g).half().to(DEV) for _ in range(2))
    books = [torch.randn(H, 16, 256, c, generator=g).to(DEV) for _ in range(2)]
    pools = [torch.zeros(cq.cq_codes_bytes(4, page, H, D, c, b), dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.tensor([[0, 99], [1, 2]], dtype=torch.int32, device=DEV)
    # sequence 0: its second page is outside of the pool; sequence 1: its last tokens lie behind the capacity
    cq.cq_paged_append(k, v, torch.tensor([0, 10, 20], dtype=torch.int32, device=DEV), *books, table, torch.tensor([20, 37], dtype=torch.int32, device=DEV),
                       c, b, page, 10, *pools)
    buf = torch.zeros(cq.cq_codes_bytes(1, 20, H, D, c, b), dtype=torch.uint8, device=DEV)
    cq.cq_encode(k[None], books[0], c, b, buf, 20)
    codes = cq.cq_codes_to_rowmajor(buf, 1, 20, H, D, c, b)[0]
    got = cq.cq_codes_to_rowmajor(pools[0], 4, page, H, D, c, b)
    want = torch.zeros_like(got)
    want[0, 10:16] = codes[0:6]                                          # positions 10 ... 15 of 10 ... 19
    want[2, 11:16] = codes[10:15]                                        # positions 27 ... 31 of 27 ... 36
    assert torch.equal(got, want)


def test_a_served_batch_over_pages():
    # two prompts and two running conversations: append, attend, then three more steps of one token each
    H, Hq, D, c, b, page = 2, 8, 128, 8, 8, 32
    case = B.Case(41, c, b, Hq, H, [0, 0, 0], 256)
    g = torch.Generator().manual_seed(41)
    books = [case.kcb.float(), case.vcb.float()]
    pools = [torch.zeros(cq.cq_codes_bytes(30, page, H, D, c, b), dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.tensor(np.random.default_rng(1).permutation(30)[:24].reshape(3, 8), dtype=torch.int32, device=DEV)
    lens = [0, 0, 0]
    for new in ([50, 7, 100], [1, 1, 1], [1, 30, 1], [1, 1, 1]):
        rows = sum(new)
        offsets = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
        x = [torch.randn(rows, H, D, generator=g).half().to(DEV) for _ in range(2)]
        lens_before, lens = lens, [a + m for a, m in zip(lens, new)]
        sl = torch.tensor(lens, dtype=torch.int32, device=DEV)
        cq.cq_paged_append(*x, offsets, *books, table, sl, c, b, page, max(new), *pools)
        for rm, xx, book in zip((case.kc, case.vc), x, books):
            buf = torch.zeros(cq.cq_codes_bytes(1, rows, H, D, c, b), dtype=torch.uint8, device=DEV)
            cq.cq_encode(xx[None], book, c, b, buf, rows)
            codes = cq.cq_codes_to_rowmajor(buf, 1, rows, H, D, c, b)[0].cpu().numpy()
            at = 0
            for s in range(3):
                rm[s, lens_before[s]:lens[s]] = codes[at:at + new[s]]
                at += new[s]
        q = case.queries(rows)
        out = cq.cq_paged_attn(q, offsets, *pools, case.kcb, case.vcb, table, sl, SCALE, c, b, page, max(new), 64, 4)
        at = 0
        for s in range(3):
            want, tol, _ = B.attend(case, s, q[at:at + new[s]], lens[s], SCALE, 64, 4)
            B.check(out[at:at + new[s]], want, tol, f"seq {s} at {lens[s]}")
            at += new[s]
