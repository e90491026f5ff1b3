"""The workspace that a call asks for holds what its kernels lay out in it, whatever the mix of sequences: checked on the host, with the launches
of every call recorded and nothing run."""
import random

import pytest

import paper_2405_03917_b200 as cq
from paper_2405_03917_b200 import build
from tests.host_launches import Recorder

P = 0x10000          # a made-up, aligned, non-NULL address
ROWS, ROW_BYTES = 256, (128 + 2) * 4                 # a slot of the tensor-core kernel: 256 rows' reference, sum and accumulators
CHUNK_THREADS, MERGE_THREADS = 704, 256
SMS = 148                                            # as the recorder's device has them
SIZE = ("cq_paged_attn_workspace_bytes", "z", "iliiiiiillll")
CALL = ("cq_paged_attn_variant", "i", "p" * 8 + "fll" + "iliiiiii" + "lll" + "ppzip")


@pytest.fixture(scope="module")
def recorder():
    build.build()
    r = Recorder(cq.library_path())
    yield r
    r.close()


def size_of(m):
    return (*SIZE, [m["n_seq"], m["rows"], m["max_q"], m["hq"], m["hkv"], 128, m["c"], 8, m["page"], m["per_seq"], m["window"], m["sinks"]])


def call_of(m, ws_bytes, variant=0):
    return (*CALL, [P] * 8 + [1.0, m["window"], m["sinks"], m["n_seq"], m["rows"], m["max_q"], m["hq"], m["hkv"], 128, m["c"], 8, 9, m["page"], m["per_seq"],
                              P, P, ws_bytes, variant, None])


def laid_out(launches):
    """Bytes of the partial sums that the launches of a call lay out."""
    most = 0
    for (grid, threads), behind in zip(launches, launches[1:] + [(0, 0)]):
        if threads == CHUNK_THREADS and behind[1] == MERGE_THREADS:          # (without a merge behind it the kernel writes no partial sums)
            most = max(most, grid * ROWS * ROW_BYTES)
    return most


def mix(new, hq, hkv, capacity, c=8, page=64, window=0, sinks=0, max_q=None):
    return dict(new=new, n_seq=len(new), rows=sum(new), max_q=max_q or max(new), hq=hq, hkv=hkv, c=c, page=page, per_seq=-(-capacity // page), window=window,
                sinks=sinks)


def check(recorder, mixes, variants=(0, 3)):
    asked = [got for got, _ in recorder.record([size_of(m) for m in mixes])]
    split = 0
    for variant in variants:
        for m, size, (st, launches) in zip(mixes, asked, recorder.record([call_of(m, size, variant) for m, size in zip(mixes, asked)])):
            assert 0 < size <= SMS * ROWS * ROW_BYTES and st == 0, (m, variant, st)
            assert any(threads == CHUNK_THREADS for _, threads in launches) or m["max_q"] * m["hq"] // m["hkv"] <= 16
            assert laid_out(launches) <= size, f"variant {variant}: {laid_out(launches)} bytes laid out, {size} asked for: {m}"
            split += laid_out(launches) > 0
        for m, (st, launches) in zip(mixes, recorder.record([call_of(m, size - 1, variant) for m, size in zip(mixes, asked)])):
            assert st == -5 and not launches, m
    return split


# conversations that take one token each, next to one or two short chunks
SERVED = [mix([1] * 3 + [20], 32, 32, 4096), mix([1] * 15 + [8], 32, 8, 9216), mix([1] * 8 + [8] * 2, 32, 8, 9216), mix([1] * 15 + [9], 32, 8, 9216),
          mix([1] * 11 + [24], 32, 8, 4096, page=16)]


def test_conversations_next_to_a_chunk(recorder):
    assert check(recorder, SERVED) > 0


@pytest.mark.parametrize("R,n_q", [(1, 256), (1, 257), (3, 85), (3, 86), (4, 200), (100, 2), (100, 3), (100, 9)])
def test_masses_of_several_row_tiles_hold_their_sums(R, n_q):
    # floor(256 / R) query tokens to a row tile; above one, 4 bytes per cached token and KV head for each
    n_seq, hkv, tiles = 64, 4, -(-n_q // (256 // R))
    size = lambda cap: cq.cq_attn_mass_workspace_bytes(n_seq, n_q, R * hkv, hkv, 128, 8, 8, cap)
    assert size(4096) - size(2048) == (4 * n_seq * hkv * 2048 * tiles if tiles > 1 else 0)


def test_random_mixes(recorder):
    rng = random.Random(7)
    mixes = []
    for _ in range(1500):
        hq, hkv = rng.choice([(32, 8), (32, 32), (40, 40), (8, 1), (12, 4), (1, 1), (64, 8), (8, 2), (30, 10), (100, 1), (17, 17)])
        n = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 20, 33, 64, 65, 100])
        chunks = rng.randint(0, min(n, 4))
        new = [rng.randint(2, rng.choice([4, 16, 64, 600])) for _ in range(chunks)] + [rng.choice([0, 1, 1, 1]) for _ in range(n - chunks)]
        if sum(new) == 0:
            new[0] = 1
        bounded = rng.random() < 0.3
        mixes.append(mix(new, hq, hkv, rng.choice([640, 1000, 4096, 9216, 32768, 1 << 20]), rng.choice([2, 4, 8]), rng.choice([16, 48, 64, 256]),
                         rng.randint(1, 4096) if bounded else 0, rng.randint(0, 70) if bounded else 0, max(new) + rng.choice([0, 0, 3])))
    assert check(recorder, mixes) > 100
