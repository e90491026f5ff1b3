"""The operators on bounded caches refuse, on the host and before anything is launched, what they do not support: no GPU needed."""
import pytest
import torch

import paper_2405_03917_b200 as cq

P = 0x10000          # a fake, aligned, non-NULL address: every call here fails before it is touched
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


def caller(name, fields):
    def call(**kw):
        assert not set(kw) - {k for k, _ in fields}, kw
        return getattr(cq.lib(), name)(*[kw.get(k, d) for k, d in fields])
    return call


WINDOW = [("q", P), ("kc", P), ("vc", P), ("kcb", P), ("vcb", P), ("lens", P), ("scale", 1.0), ("window", 64), ("sinks", 4), ("n_seq", 2),
          ("n_q", 1), ("hq", 8), ("hkv", 2), ("D", 128), ("c", 8), ("b", 8), ("cap", 256), ("out", P), ("ws", P), ("ws_bytes", 1 << 40),
          ("variant", 0), ("stream", None)]
PAGED = [("q", P), ("offsets", P), ("kc", P), ("vc", P), ("kcb", P), ("vcb", P), ("table", P), ("lens", P), ("scale", 1.0), ("window", 0), ("sinks", 0),
         ("n_seq", 2), ("rows", 5), ("max_q", 4), ("hq", 8), ("hkv", 2), ("D", 128), ("c", 8), ("b", 8), ("n_pages", 9), ("page", 64), ("per_seq", 4),
         ("out", P), ("ws", P), ("ws_bytes", 1 << 40), ("variant", 0), ("stream", None)]
APPEND = [("k", P), ("v", P), ("offsets", P), ("kcb", P), ("vcb", P), ("table", P), ("lens", P), ("n_seq", 2), ("rows", 5), ("max_q", 4), ("heads", 2),
          ("D", 128), ("c", 8), ("b", 8), ("n_pages", 9), ("page", 64), ("per_seq", 4), ("kp", P), ("vp", P + 4096), ("ws", P), ("ws_bytes", 1 << 40),
          ("stream", None)]
MASS = [("q", P), ("kc", P), ("kcb", P), ("lens", P), ("scale", 1.0), ("mass_in", P), ("n_seq", 2), ("n_q", 1), ("hq", 8), ("hkv", 2), ("D", 128),
        ("c", 8), ("b", 8), ("cap", 256), ("mass_out", P), ("ws", P), ("ws_bytes", 1 << 40), ("variant", 0), ("stream", None)]
EVICT = [("mass", P), ("kc", P + 4096), ("vc", P + 8192), ("lens", P), ("n_seq", 2), ("heads", 2), ("D", 128), ("c", 8), ("b", 8), ("cap", 256),
         ("keep", 64), ("sinks", 4), ("recent", 16), ("out_cap", 128), ("mass_out", P + 64), ("ko", P + 12288), ("vo", P + 16384), ("kept", P),
         ("lens_out", P + 64), ("stream", None)]
CALLS = {"cq_window_attn_variant": WINDOW, "cq_paged_attn_variant": PAGED, "cq_paged_append": APPEND, "cq_attn_mass_variant": MASS, "cq_evict": EVICT}


@pytest.mark.parametrize("name", list(CALLS))
def test_null_pointers(name):
    call = caller(name, CALLS[name])
    optional = {"stream", "mass_in"}
    for k, d in CALLS[name]:
        if k not in optional and isinstance(d, int) and d >= P and d < 1 << 20:
            assert call(**{k: None}) == NULL, k


@pytest.mark.parametrize("name", list(CALLS))
def test_alignment(name):
    call = caller(name, CALLS[name])
    for k in ("q", "k", "kc", "vc", "kp", "kcb", "ko", "ws"):
        if k in dict(CALLS[name]):
            assert call(**{k: dict(CALLS[name])[k] + 8}) == ALIGN, k
    for k in ("lens", "offsets", "table", "mass_out"):
        if k in dict(CALLS[name]):
            assert call(**{k: dict(CALLS[name])[k] + 2}) == ALIGN, k


@pytest.mark.parametrize("name", list(CALLS))
def test_quantiser_shapes(name):
    call = caller(name, CALLS[name])
    assert call(c=3) == SHAPE
    assert call(n_seq=0) == SHAPE
    assert call(D=512) == UNSUPPORTED
    assert call(b=11) == UNSUPPORTED
    if "hkv" in dict(CALLS[name]):
        assert call(hkv=3) == SHAPE


def test_window_and_mass_arguments():
    for name in ("cq_window_attn_variant", "cq_attn_mass_variant"):
        call = caller(name, CALLS[name])
        assert call(n_q=0) == SHAPE
        assert call(n_q=257) == SHAPE            # more new tokens than the cache has room for
        assert call(variant=9) == SHAPE
        assert call(variant=-1) == SHAPE
        assert call(cap=(1 << 30) + 16) == UNSUPPORTED
        assert call(ws_bytes=0) == WORKSPACE
    call = caller("cq_window_attn_variant", WINDOW)
    assert call(window=-1) == SHAPE
    assert call(sinks=-1) == SHAPE


def test_paged_arguments():
    for name in ("cq_paged_attn_variant", "cq_paged_append"):
        call = caller(name, CALLS[name])
        assert call(page=24) == SHAPE            # not whole blocks of 16 tokens
        assert call(page=0) == SHAPE
        assert call(n_pages=0) == SHAPE
        assert call(per_seq=0) == SHAPE
        assert call(max_q=0) == SHAPE
        assert call(max_q=257) == SHAPE
        assert call(rows=-1) == SHAPE
        assert call(per_seq=(1 << 30) // 64 + 1) == UNSUPPORTED
        assert call(ws_bytes=0) == WORKSPACE
    assert caller("cq_paged_attn_variant", PAGED)(rows=0, ws_bytes=1 << 40) == 0          # nothing to do is no error
    assert caller("cq_paged_append", APPEND)(rows=0) == 0
    assert caller("cq_paged_append", APPEND)(vp=P) == SHAPE


def test_evict_arguments():
    call = caller("cq_evict", EVICT)
    assert call(keep=0) == SHAPE
    assert call(keep=129) == SHAPE               # more than the output cache holds
    assert call(sinks=-1) == SHAPE
    assert call(recent=61) == SHAPE              # sinks and recent tokens beyond n_keep
    assert call(ko=P + 4096) == SHAPE            # one buffer in place, the others not
    assert call(ko=P + 4096, vo=P + 8192, mass_out=P) == SHAPE          # in place at another capacity
    assert call(ko=P + 16384) == SHAPE           # one buffer for both outputs
    assert call(lens_out=P) == SHAPE             # the lengths are read by every head
    assert call(cap=(1 << 30) + 16) == UNSUPPORTED


def test_workspace_sizes():
    assert cq.cq_window_attn_workspace_bytes(2, 1, 8, 2, 128, 8, 8, 256, 64, 4) > 0
    assert cq.cq_window_attn_workspace_bytes(2, 1, 8, 3, 128, 8, 8, 256, 64, 4) == 0
    assert cq.cq_paged_attn_workspace_bytes(2, 5, 4, 8, 2, 128, 8, 8, 64, 4) > 0
    assert cq.cq_paged_attn_workspace_bytes(2, 5, 4, 8, 2, 128, 8, 8, 24, 4) == 0
    assert cq.cq_attn_mass_workspace_bytes(2, 1, 8, 2, 128, 8, 8, 256) > 0
    assert cq.cq_paged_append_workspace_bytes(5, 2, 128, 8, 8) >= 2 * 2 * 16 * 16


def test_the_binding_names_what_is_wrong():
    q = torch.zeros(2, 1, 8, 128, dtype=torch.float16)
    codes = torch.zeros(2 * 2 * 16 * 16 * 16, dtype=torch.uint8)
    book = torch.zeros(2, 16, 256, 8, dtype=torch.float16)
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="k_codes holds"):
        cq.cq_window_attn(q, codes[:-1], codes, book, book, lens, 1.0, 8, 8, 256, 64)
    with pytest.raises(ValueError, match="come together"):
        cq.cq_evict(torch.zeros(2, 2, 256), codes, codes, lens, 128, 8, 8, 256, 16, k_codes_out=codes)


@pytest.mark.parametrize("name", ["cq_window_attn_variant", "cq_paged_attn_variant", "cq_attn_mass_variant"])
def test_kernels_that_a_caller_names(name):
    call = caller(name, CALLS[name])
    for variant in (2, 3):                                               # of shapes that are not theirs
        for D, c, b in ((64, 8, 8), (128, 8, 10), (128, 16, 8), (256, 8, 8), (96, 3, 4)):
            assert call(variant=variant, D=D, c=c, b=b) == UNSUPPORTED, (variant, D, c, b)
    for variant in (-1, 4):
        assert call(variant=variant) == SHAPE
