"""GPU parity of cq_attn_mass with the 64-bit definition and of cq_evict with a plain selection: exact positions, codes and masses."""
import numpy as np
import pytest
import torch

import paper_2405_03917_b200 as cq
from tests import bounded as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5
VARIANTS = [0, 1, 2, 3]


def mass_tolerance(case, s, q, n, p):
    """A weight's relative error: 4 e_s as in tests/bounded.py (score, scaling and exponential, of the weight and of the normaliser), n 2^-23
    for the normaliser's sum; (rows) 2^-23 for the sum over rows, and a rounding of the sum with what was there (up to 1 here)."""
    R = case.Hq // case.Hkv
    K = case.vectors("k", s, n).repeat_interleave(R, 0)
    e_s = 130 * 2.0 ** -23 * SCALE * (q.double().abs().transpose(0, 1) @ K.abs().transpose(1, 2)).amax() + 2.0 ** -22
    got = p.view(case.Hkv, R * q.shape[0], n).sum(1)
    return got * (4 * e_s + n * 2.0 ** -23 + R * q.shape[0] * 2.0 ** -23) + 2.0 ** -23 * (1 + got)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("c,Hq,Hkv,n_q", [(8, 8, 2, 1), (4, 4, 4, 1), (2, 6, 2, 5), (8, 8, 1, 32), (8, 20, 1, 3), (4, 3, 3, 70), (8, 4, 1, 150), (2, 6, 2, 200)])
def test_mass(variant, c, Hq, Hkv, n_q):
    lens = [700, n_q, 1, 0, 333, 64 + n_q]
    cap = 709
    case = B.Case(c + Hq + n_q, c, 8, Hq, Hkv, lens, cap)
    q = case.queries(len(lens), n_q)
    k, _ = case.contiguous()
    g = torch.Generator(device=DEV).manual_seed(5)
    mass = torch.rand(len(lens), Hkv, cap, generator=g, device=DEV)
    fresh = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, c, 8, cap, variant=variant)
    out = torch.full_like(mass, -1.0)
    cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, c, 8, cap, mass, out, variant=variant)
    inplace = mass.clone()
    cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, c, 8, cap, inplace, inplace, variant=variant)
    for s, n in enumerate(lens):
        assert (out[s, :, n:] == -1.0).all() and (fresh[s, :, n:] == 0).all() and torch.equal(inplace[s, :, n:], mass[s, :, n:])
        if n == 0:
            continue
        _, _, p = B.attend(case, s, q[s], n, SCALE)
        want = p.view(Hkv, -1, n).sum(1)
        tol = mass_tolerance(case, s, q[s], n, p)
        for what, base, got in (("fresh", 0.0, fresh), ("out", mass[s, :, :n].double(), out), ("in place", mass[s, :, :n].double(), inplace)):
            bad = (got[s, :, :n].double() - want - base).abs() > tol
            assert not bad.any(), f"variant {variant} seq {s} {what}: {int(bad.sum())} off"
    assert torch.equal(out[0, :, :700], inplace[0, :, :700])


@pytest.mark.parametrize("variant", VARIANTS)
def test_mass_of_long_contexts_and_many_sequences(variant):
    case = B.Case(2, 8, 8, 8, 2, [20001], 20016)
    q = case.queries(1, 2)
    k, _ = case.contiguous()
    got = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 20016, variant=variant)
    _, _, p = B.attend(case, 0, q[0], 20001, SCALE)
    want = p.view(2, -1, 20001).sum(1)
    assert ((got[0, :, :20001].double() - want).abs() <= mass_tolerance(case, 0, q[0], 20001, p)).all()
    case = B.Case(3, 8, 8, 4, 2, [int(x) for x in np.random.default_rng(0).integers(0, 70, 300)], 80)
    q = case.queries(300, 1)
    k, _ = case.contiguous()
    got = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 80, variant=variant)
    for s in range(0, 300, 7):
        n = case.lens[s]
        if n:
            _, _, p = B.attend(case, s, q[s], n, SCALE)
            assert ((got[s, :, :n].double() - p.view(2, -1, n).sum(1)).abs() <= mass_tolerance(case, s, q[s], n, p)).all(), s


@pytest.mark.parametrize("n_q", [1, 3, 70, 300])
def test_mass_repeats_bit_by_bit(n_q):
    case = B.Case(9, 8, 8, 8, 2, [5000, 700], 5008)
    q = case.queries(2, n_q)
    k, _ = case.contiguous()
    first = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 5008)
    for _ in range(3):
        assert torch.equal(cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 5008), first)


def test_mass_shapes_of_the_plain_kernel():
    case = B.Case(4, 8, 10, 4, 2, [150, 33], 160)
    q = case.queries(2, 3)
    k, _ = case.contiguous()
    got = cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 10, 160)
    for s, n in enumerate(case.lens):
        _, _, p = B.attend(case, s, q[s], n, SCALE)
        assert ((got[s, :, :n].double() - p.view(2, -1, n).sum(1)).abs() <= mass_tolerance(case, s, q[s], n, p)).all()


# ------------------------------------------------------------------------------------------ eviction

def check_evict(case, mass, keep, sinks, recent, room=None):
    n_seq, H, cap = mass.shape
    k, v = case.contiguous()
    m = torch.from_numpy(mass).to(DEV)
    where = {}
    if room is not None:
        fill = lambda: torch.full((cq.cq_codes_bytes(n_seq, room, H, case.D, case.c, case.b),), 0xAB, dtype=torch.uint8, device=DEV)
        where = dict(k_codes_out=fill(), v_codes_out=fill(), mass_out=torch.full((n_seq, H, room), -5.0, device=DEV), out_max_tokens=room)
    kept, lens = cq.cq_evict(m, k, v, case.seq_lens(), case.D, case.c, case.b, cap, keep, sinks, recent, **where)
    ko, vo, mo = (where["k_codes_out"], where["v_codes_out"], where["mass_out"]) if room is not None else (k, v, m)
    out_cap = room if room is not None else cap
    krm, vrm = case.rowmajor(ko, n_seq, out_cap), case.rowmajor(vo, n_seq, out_cap)
    mo, kept, lens = mo.cpu().numpy(), kept.cpu().numpy(), lens.cpu().numpy()
    for s, n in enumerate(case.lens):
        left = min(n, keep)
        assert lens[s] == left
        for h in range(H):
            want = B.evict_plain(mass[s, h], n, keep, sinks, recent)
            np.testing.assert_array_equal(kept[s, h, :left], want)
            assert (kept[s, h, left:] == -1).all()
            np.testing.assert_array_equal(krm[s, :left, h], case.kc[s, want, h])
            np.testing.assert_array_equal(vrm[s, :left, h], case.vc[s, want, h])
            np.testing.assert_array_equal(mo[s, h, :left], mass[s, h, want])
            pad = -(-left // 16) * 16
            assert (krm[s, left:min(pad, out_cap), h] == 0).all() and (vrm[s, left:min(pad, out_cap), h] == 0).all()
            if room is None:
                np.testing.assert_array_equal(krm[s, pad:, h], case.kc[s, pad:, h])
                np.testing.assert_array_equal(mo[s, h, left:], mass[s, h, left:])
            else:
                assert (mo[s, h, left:] == -5.0).all()


@pytest.mark.parametrize("room", [None, 128])
@pytest.mark.parametrize("c,b", [(8, 8), (4, 8), (2, 8), (8, 10), (8, 16), (16, 9), (128, 9)])
@pytest.mark.parametrize("keep,sinks,recent", [(64, 4, 16), (1, 0, 0), (100, 0, 100), (33, 33, 0), (128, 5, 0)])
def test_evict(room, c, b, keep, sinks, recent):
    lens = [300, keep, keep + 1, 0, 1, 150]
    case = B.Case(c + b + keep, c, b, 2, 2, lens, 304)
    mass = np.random.default_rng(keep).exponential(1.0, (6, 2, 304)).astype(np.float32)
    check_evict(case, mass, keep, sinks, recent, room)


@pytest.mark.parametrize("room", [None, 512])
def test_ties_zeros_and_values_that_are_no_numbers(room):
    case = B.Case(1, 8, 8, 3, 3, [900, 700, 333], 912)
    g = np.random.default_rng(2)
    mass = g.integers(0, 4, (3, 3, 912)).astype(np.float32)             # many alike
    mass[1] = 0.0                                                       # all alike
    mass[1, :, ::2] = -0.0
    mass[2] = g.standard_normal((3, 912)).astype(np.float32)            # of both signs, with infinities and NaN
    mass[2, 0, 50], mass[2, 0, 60], mass[2, 0, 70], mass[2, 1, 100] = np.inf, -np.inf, np.nan, np.nan
    check_evict(case, mass, 200, 4, 32, room)


@pytest.mark.parametrize("n", [4096, 4097, 16384, 16385, 32768, 32769, 70001])
def test_every_length_class(n):
    case = B.Case(n, 8, 8, 1, 1, [n, n - 1, n // 2], n + 3)
    mass = np.random.default_rng(n).exponential(1.0, (3, 1, n + 3)).astype(np.float32)
    mass[1] = np.round(mass[1] * 8) / 8                                 # ties at the threshold
    check_evict(case, mass, n // 3, 4, 100, room=n // 3 + 10)
    check_evict(case, mass, n // 3, 4, 100)


def test_masses_that_share_all_but_the_last_bits():
    # the three histograms must all be needed
    case = B.Case(7, 8, 8, 1, 1, [3000], 3008)
    bits = (0x3f800000 + np.random.default_rng(3).permutation(3008)).astype(np.uint32)
    check_evict(case, bits.view(np.float32).reshape(1, 1, 3008), 1000, 0, 0, 1008)


def test_a_cache_cut_down_between_steps():
    # attention masses over some steps, eviction in place, and the next step's attention over what stays
    H, Hq, c, b, cap = 2, 8, 8, 8, 256
    case = B.Case(51, c, b, Hq, H, [200, 90], cap)
    k, v = case.contiguous()
    mass = torch.zeros(2, H, cap, device=DEV)
    for _ in range(3):
        q = case.queries(2, 1)
        cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, c, b, cap, mass, mass)
    assert abs(mass.sum().item() - 3 * 2 * Hq) < 1e-3                   # every query head hands out a weight of one
    kept, lens = cq.cq_evict(mass, k, v, case.seq_lens(), 128, c, b, cap, 96, 4, 16)
    assert lens.tolist() == [96, 90]
    q = case.queries(2, 1)
    out = cq.cq_window_attn(q, k, v, case.kcb, case.vcb, lens, SCALE, c, b, cap, 0)
    for s, n in enumerate([96, 90]):
        for h in range(H):
            at = kept[s, h, :n].long()
            r = slice(h * 4, h * 4 + 4)
            K, V = case.vectors("k", s, case.lens[s])[h][at], case.vectors("v", s, case.lens[s])[h][at]
            p = torch.softmax(q[s, 0, r].double() @ K.T * SCALE, -1)
            want = p @ V
            # (the bound of tests/bounded.py at its largest score error here, 130 2^-23 * |q||K| <= 2e-3)
            tol = 2.0 ** -11 * want.abs() + 2.0 ** -25 + (2 * 2.0 ** -11 + 8e-3 + n * 2.0 ** -23) * (p @ V.abs())
            B.check(out[s, 0, r], want, tol)


def test_evict_in_a_graph_and_on_another_stream():
    case = B.Case(61, 8, 8, 2, 2, [500, 77], 512)
    k, v = case.contiguous()
    mass = torch.rand(2, 2, 512, device=DEV)
    size = cq.cq_codes_bytes(2, 128, 2, 128, 8, 8)
    new = lambda: dict(k_codes_out=torch.zeros(size, dtype=torch.uint8, device=DEV), v_codes_out=torch.zeros(size, dtype=torch.uint8, device=DEV),
                       mass_out=torch.zeros(2, 2, 128, device=DEV), out_max_tokens=128)
    a, b_ = new(), new()
    lens = case.seq_lens()
    kept, left = cq.cq_evict(mass, k, v, lens, 128, 8, 8, 512, 128, 4, 20, **a)
    kept2, left2 = torch.zeros_like(kept), torch.zeros_like(left)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cq.cq_evict(mass, k, v, lens, 128, 8, 8, 512, 128, 4, 20, kept=kept2, seq_lens_out=left2, **b_)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kept, kept2) and torch.equal(left, left2)
    for name in ("k_codes_out", "v_codes_out", "mass_out"):
        assert torch.equal(a[name], b_[name])


def test_mass_with_less_workspace():
    # without room for the scores the second pass works them out again: the same masses up to the order of a few additions
    case = B.Case(12, 8, 8, 8, 2, [1500, 33, 700], 1504)
    q = case.queries(3, 1)
    k, _ = case.contiguous()
    full = cq.cq_attn_mass_workspace_bytes(3, 1, 8, 2, 128, 8, 8, 1504)
    least = cq.cq_attn_mass_workspace_bytes(3, 1, 8, 2, 128, 8, 8, 1)
    assert least < full
    call = lambda size: cq.cq_attn_mass(q, k, case.kcb, case.seq_lens(), SCALE, 8, 8, 1504, workspace=torch.empty(size, dtype=torch.uint8, device=DEV))
    for got in (call(full), call(least)):
        for s, n in enumerate(case.lens):
            _, _, p = B.attend(case, s, q[s], n, SCALE)
            assert ((got[s, :, :n].double() - p.view(2, -1, n).sum(1)).abs() <= mass_tolerance(case, s, q[s], n, p)).all()


# ------------------------------------------------------------------------------------------ more (sequence, head) pairs than two per SM

MANY = dict(n_seq=50, H=6)


@pytest.mark.parametrize("room", [None, 128])
@pytest.mark.parametrize("c,b", [(8, 8), (2, 8), (8, 10), (128, 9)])
@pytest.mark.parametrize("keep,sinks,recent", [(64, 4, 16), (100, 0, 100), (128, 5, 0)])
def test_evict_of_many_heads(room, c, b, keep, sinks, recent):
    g = np.random.default_rng(keep + c)
    lens = [int(x) for x in g.integers(0, 300, MANY["n_seq"])]
    lens[:4] = [keep, keep + 1, 0, 300]
    case = B.Case(c + b + keep, c, b, MANY["H"], MANY["H"], lens, 304)
    mass = g.exponential(1.0, (MANY["n_seq"], MANY["H"], 304)).astype(np.float32)
    check_evict(case, mass, keep, sinks, recent, room)


@pytest.mark.parametrize("room", [None, 512])
def test_ties_and_values_that_are_no_numbers_of_many_heads(room):
    g = np.random.default_rng(5)
    n = MANY["n_seq"]
    case = B.Case(15, 16, 8, MANY["H"], MANY["H"], [int(x) for x in g.integers(1, 2500, n)], 2512)
    mass = g.exponential(1.0, (n, MANY["H"], 2512)).astype(np.float32)
    mass[:10] = g.integers(0, 4, mass[:10].shape)                       # many alike: more than are ranked against each other
    mass[10:14] = 0.0
    mass[12, :, ::2] = -0.0
    mass[14:18] = g.standard_normal(mass[14:18].shape)
    mass[14, :, ::7], mass[15, :, 1::5], mass[16, :, 3::11] = np.inf, -np.inf, np.nan
    mass[18] = -np.inf
    mass.view(np.uint32)[19, :, ::13] = 0xffc00001                      # NaN of the other sign
    bits = 0x3f800000 + np.stack([g.permutation(2512) for _ in range(10 * MANY["H"])]).reshape(10, MANY["H"], 2512)
    mass[20:30] = bits.astype(np.uint32).view(np.float32)               # alike but for the last bits
    check_evict(case, mass, 200, 4, 32, room)


def test_many_heads_at_the_longest_capacities_of_a_kernel():
    n = 38                                                              # x 8 heads = 304
    for cap in (32768, 32769):
        g = np.random.default_rng(cap)
        lens = [cap, cap - 1, 5, 20000] + [int(x) for x in g.integers(0, 200, n - 4)]
        case = B.Case(16, 128, 8, 8, 8, lens, cap)
        mass = g.exponential(1.0, (n, 8, cap)).astype(np.float32)
        check_evict(case, mass, 1000, 4, 100, 1008)
