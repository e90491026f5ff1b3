"""Plain implementations, in 64 bits, of the operators on bounded caches, and the tolerances of their tests.

Tolerance of an attention output (fp16), per element, with A = sum_t p_t |Vhat_t| and e_s the error of a score:
  * rounding of the output: 2^-11 |out|, and half of fp16's smallest step, 2^-25;
  * every softmax weight is rounded to fp16 before the second product: 2^-11 A, and as much for a normaliser that was summed from
    unrounded weights (|out| <= A);
  * weights below 2^-14 of the reference (whose weight is at least 1) have fp16's smallest step: n 2^-25 max|Vhat| for n tokens;
  * a score is a sum of 128 exact products in fp32, e_s <= 130 * 2^-23 * |scale| max_t sum_c |q_c Khat_tc| (each addition off by at
    most a step: tensor cores may truncate), and as much again for its scaling and the exponential (2^-22); numerator and denominator: 4 e_s A;
  * sums over tokens in fp32: 2^-17 A covers thousands of additions (they round to nearest or truncate: n 2^-23 at worst, n <= 64).
Sums over more tokens are pairwise or in registers of one warp's tokens; n 2^-23 A is added in full for them.
"""
from __future__ import annotations

import numpy as np
import torch

import paper_2405_03917_b200 as cq

DEV = "cuda"



class Case:
    """A cache of random codes: row-major codes on the host, library layout on the device, fp16 codebooks."""

    def __init__(self, seed, c, b, Hq, Hkv, lens, cap, D=128, spread=1.0):
        g = np.random.default_rng(seed)
        self.c, self.b, self.Hq, self.Hkv, self.D, self.G, self.cap, self.lens = c, b, Hq, Hkv, D, D // c, cap, list(lens)
        self.n = len(self.lens)
        kcb = (g.standard_normal((Hkv, self.G, 1 << b, c)) * spread).astype(np.float16)
        vcb = g.standard_normal((Hkv, self.G, 1 << b, c)).astype(np.float16)
        self.kc = g.integers(0, 1 << b, size=(self.n, cap, Hkv, self.G)).astype(np.int32)
        self.vc = g.integers(0, 1 << b, size=(self.n, cap, Hkv, self.G)).astype(np.int32)
        self.kcb, self.vcb = torch.from_numpy(kcb).to(DEV), torch.from_numpy(vcb).to(DEV)
        self.g = g

    def codes(self, rm):
        t = torch.from_numpy(rm.astype(np.uint8)) if self.b <= 8 else torch.from_numpy(rm.astype(np.uint16).view(np.int16))
        return cq.cq_codes_from_rowmajor(t.to(DEV), self.D, self.c, self.b)

    def rowmajor(self, codes, n, cap):
        rm = cq.cq_codes_to_rowmajor(codes, n, cap, self.Hkv, self.D, self.c, self.b).cpu().numpy()
        return rm.astype(np.int32) & ((1 << self.b) - 1)

    def contiguous(self):
        return self.codes(self.kc), self.codes(self.vc)

    def seq_lens(self, lens=None):
        return torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device=DEV)

    def queries(self, *shape):
        return torch.from_numpy(self.g.standard_normal((*shape, self.Hq, self.D)).astype(np.float16)).to(DEV)

    def vectors(self, which, s, n):
        """Reconstructions of the first n tokens of sequence s: float64 (Hkv, n, D)."""
        rm = torch.from_numpy((self.kc if which == "k" else self.vc)[s, :n]).to(DEV).long()        # (n, Hkv, G)
        book = (self.kcb if which == "k" else self.vcb).double()
        h = torch.arange(self.Hkv, device=DEV)[None, :, None]
        g = torch.arange(self.G, device=DEV)[None, None, :]
        return book[h, g, rm].reshape(n, self.Hkv, self.D).transpose(0, 1)

    def paged(self, page, seed=0, spare=3):
        """The same cache in pages: (k_pages, v_pages, page_table, order of the pages)."""
        g = np.random.default_rng(seed)
        per = -(-self.cap // page)
        used = [-(-x // page) for x in self.lens]
        total = sum(used) + spare
        order = g.permutation(total)
        table = np.full((self.n, per), -1, np.int32)
        pools = [g.integers(0, 1 << self.b, size=(total, page, self.Hkv, self.G)).astype(np.int32) for _ in range(2)]
        at = 0
        for s in range(self.n):
            for j in range(used[s]):
                p = int(order[at])
                at += 1
                table[s, j] = p
                for pool, rm in zip(pools, (self.kc, self.vc)):
                    part = rm[s, j * page:(j + 1) * page]
                    pool[p, :part.shape[0]] = part
        return self.codes(pools[0]), self.codes(pools[1]), torch.from_numpy(table).to(DEV)


def seen(n, m, window, sinks):
    """Tokens of 0 ... n - 1 that each of the m newest sees: (m, n) bool."""
    t = torch.arange(n, device=DEV)[None]
    pos = torch.arange(n - m, n, device=DEV)[:, None]
    ok = t <= pos
    if window:
        ok = ok & ((t < sinks) | (t > pos - window))
    return ok


def attend(case, s, q, n, scale, window=0, sinks=0, absent=None):
    """q (m, Hq, D) of sequence s with n cached tokens -> (out, tolerance, weights), float64; weights (Hq, m, n)."""
    m = q.shape[0]
    R = case.Hq // case.Hkv
    if n == 0:
        z = torch.zeros(m, case.Hq, case.D, dtype=torch.float64, device=DEV)
        return z, z + 1e-12, torch.zeros(case.Hq, m, 0, dtype=torch.float64, device=DEV)
    K = case.vectors("k", s, n).repeat_interleave(R, 0)
    V = case.vectors("v", s, n).repeat_interleave(R, 0)
    ok = seen(n, m, window, sinks)
    if absent is not None:
        ok = ok & ~absent[None, :n]
    x = q.double().transpose(0, 1) @ K.transpose(1, 2) * scale
    x = x.masked_fill(~ok, float("-inf"))
    some = ok.any(-1)
    p = torch.where(some[None, :, None], torch.softmax(x, -1), torch.zeros_like(x))
    out = (p @ V).transpose(0, 1)
    A = (p @ V.abs()).transpose(0, 1)
    e_s = 130 * 2.0 ** -23 * abs(scale) * (q.double().abs().transpose(0, 1) @ K.abs().transpose(1, 2)).amax(-1).transpose(0, 1)[..., None] + 2.0 ** -22
    tol = 2.0 ** -11 * out.abs() + 2.0 ** -25 + (2 * 2.0 ** -11 + 4 * e_s + n * 2.0 ** -23) * A + n * 2.0 ** -25 * V.abs().max()
    tol = torch.where(some[:, None, None], tol, torch.zeros_like(tol))
    return out, tol, p


def check(got, want, tol, what=""):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: non-finite output"
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off; worst {((got - want).abs() / tol.clamp_min(1e-30)).max().item():.2f} tolerances"


def evict_plain(mass, n, keep, sinks, recent):
    """Positions that stay of n tokens with these masses (float64 or float32 numpy), ascending."""
    if n <= keep:
        return np.arange(n)
    order = np.where(np.isnan(mass[:n]), np.inf, mass[:n].astype(np.float64))
    nan = np.isnan(mass[:n])
    forced = np.zeros(n, bool)
    forced[:sinks] = True
    forced[n - recent:] = True
    # forced first, then NaN, then by mass, then by position
    rank = np.lexsort((np.arange(n), -order, ~nan, ~forced))
    return np.sort(rank[:keep])
