"""cq_evict refuses buffers that overlap otherwise than in place, on the host: launches are recorded and nothing runs."""
import pytest

import paper_2405_03917_b200 as cq
from paper_2405_03917_b200 import build
from tests.host_launches import Recorder

SHAPE = -2
TYPES = ("cq_evict", "i", "pppp" + "iiiii" + "lllll" + "pppppp")
N_SEQ, HEADS, D, C, B_, CAP, KEEP, ROOM = 2, 3, 128, 8, 8, 300, 64, 100
CODES, CODES_OUT = N_SEQ * HEADS * 19 * 256, N_SEQ * HEADS * 7 * 256          # 19 and 7 blocks of 16 tokens, 16 groups
MASS, MASS_OUT, KEPT, LENS = N_SEQ * HEADS * CAP * 4, N_SEQ * HEADS * ROOM * 4, N_SEQ * HEADS * KEEP * 4, N_SEQ * 4
SIZES = dict(mass=MASS, kc=CODES, vc=CODES, lens=LENS, mo=MASS_OUT, ko=CODES_OUT, vo=CODES_OUT, kept=KEPT, left=LENS)
INPUTS, OUTPUTS = ("mass", "kc", "vc", "lens"), ("mo", "ko", "vo", "kept", "left")


def up(n):
    return -(-n // 16) * 16


def side_by_side():
    """Every buffer right behind the one before (at the next 16 bytes)."""
    at, p = {}, 1 << 20
    for name, size in SIZES.items():
        at[name] = p
        p += up(size)
    return at


@pytest.fixture(scope="module")
def status():
    build.build()
    r = Recorder(cq.library_path())

    def of(cases):
        calls = [(*TYPES, [a["mass"], a["kc"], a["vc"], a["lens"], N_SEQ, HEADS, D, C, B_, CAP, KEEP, 4, 16, room, a["mo"], a["ko"], a["vo"], a["kept"], a["left"], None])
                 for a, room in cases]
        got = r.record(calls)
        assert all(bool(launches) == (st == 0) for st, launches in got)
        return [st for st, _ in got]
    yield of
    r.close()


def test_buffers_side_by_side_are_taken(status):
    assert status([(side_by_side(), ROOM)]) == [0]


@pytest.mark.parametrize("out", OUTPUTS)
def test_an_output_that_overlaps_anything(status, out):
    cases = []
    for other in INPUTS + OUTPUTS:
        if other != out:
            at = side_by_side()
            # the same place, the last 16 bytes (4 for the lengths), and from before its beginning
            places = {at[other], at[other] + up(max(SIZES[other] - 16, 0)) - (16 if SIZES[other] % 16 and SIZES[other] > 16 else 0)}
            for p in places | ({at[other] - up(SIZES[out]) + 16} if SIZES[out] > 16 else set()):
                cases.append(({**at, out: p}, ROOM))
    assert set(status(cases)) == {SHAPE}


def test_in_place(status):
    at = side_by_side()
    # (the cache's capacity is the output's then; kept and the lengths lie behind everything else)
    here = {**at, "mo": at["mass"], "ko": at["kc"], "vo": at["vc"]}
    assert status([(here, CAP)]) == [0]
    wrong = [{**here, "kept": at["mass"] + MASS - 16}, {**here, "kept": at["kc"]}, {**here, "left": at["vc"] + 64}, {**here, "left": at["lens"] + 4},
             {**here, "ko": at["kc"] + 256}, {**here, "mo": at["mass"] + 16}, {**here, "vc": at["kc"] + 4096, "vo": at["kc"] + 4096},
             {**here, "kept": at["left"] + LENS - 4}]
    assert set(status([(w, CAP) for w in wrong])) == {SHAPE}
