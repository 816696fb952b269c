"""Arguments that the calls on ragged chunks refuse beside those of their sizes, on the host and before any launch (no GPU needed)."""
import ctypes

import pytest

import paper_2509_15763_b200 as ug
from paper_2509_15763_b200 import binding, build

INVALID, ALIGN = 1, 3
MB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def refused(call, code):
    before = ug.unigist_launch_count()
    assert call() == code, ug.unigist_last_error_string()
    assert ug.unigist_last_error_string() and ug.unigist_launch_count() == before


# Addresses that only the host's checks see: every argument in a megabyte of its own.
HALF = (ctypes.c_uint8 * 64)(*([0] * 64))


def at(i):
    return (i + 16) * MB


def rope(**kw):
    a = dict(n=4, heads=2, D=64, src=at(0), ss=128, dst=at(1), ds=128, pos=at(2), axes=1, fa=HALF, base=10000.0, flags=0)
    a.update(kw)
    return binding.lib().unigist_rope_axes(*a.values(), None)


def append(**kw):
    a = dict(S=2, Hkv=2, D=64, n=3, k=at(0), ks=128, v=at(1), vs=128, cu=at(2), pos=at(3), axes=1, fa=HALF, base=10000.0, kc=at(4), vc=at(5), w=at(6), blocks=4,
             table=at(7), width=2, lens=at(8), new=at(9))
    a.update(kw)
    return binding.lib().unigist_chunk_append(*a.values(), None)


def attn(**kw):
    a = dict(S=2, Hq=4, Hkv=2, D=64, scale=0.0, n=3, q=at(0), qs=256, cu=at(1), kc=at(2), vc=at(3), blocks=4, table=at(4), width=2, lens=at(5), o=at(6), lse=at(7),
             ws=at(8), ws_bytes=MB)
    a.update(kw)
    return binding.lib().unigist_chunk_attn(*a.values(), None)


def weigh(**kw):
    a = dict(S=2, Hq=4, Hkv=2, D=64, scale=0.0, n=3, q=at(0), qs=256, cu=at(1), lse=at(2), kc=at(3), blocks=4, table=at(4), width=2, lens=at(5), w_in=at(6), decay=1.0,
             w_out=at(7))
    a.update(kw)
    return binding.lib().unigist_cache_weigh(*a.values(), None)


def evict(**kw):
    a = dict(S=2, Hkv=2, D=64, keep=10, first=2, last=3, kc=at(0), vc=at(1), w=at(2), blocks=4, table=at(3), width=2, lens=at(4), to=at(5), to_width=2, new=at(6),
             kept=at(7))
    a.update(kw)
    return binding.lib().unigist_cache_evict(*a.values(), None)


@pytest.mark.parametrize("call,name", [(rope, "pos"), (append, "cu"), (append, "pos"), (append, "w"), (append, "table"), (append, "lens"), (append, "new"),
                                       (attn, "cu"), (attn, "table"), (attn, "lens"), (attn, "lse"), (weigh, "cu"), (weigh, "lse"), (weigh, "table"),
                                       (weigh, "lens"), (weigh, "w_in"), (weigh, "w_out"), (evict, "table"), (evict, "lens"), (evict, "to"), (evict, "new"),
                                       (evict, "kept")])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_numbers_that_are_not_aligned(call, name, off):
    """A 32-bit number at an odd address is a fault on the device."""
    refused(lambda: call(**{name: at(30) + off}), ALIGN)


# (S 2, Hq 4, Hkv 2, D 64, 3 rows, 4 pages of 64: what each argument spans)
O_BYTES, CACHE, SMALL = 3 * 4 * 64 * 2, 4 * 2 * 64 * 64 * 2, 8


@pytest.mark.parametrize("name,bytes_", [("q", (2 * 256 + 4 * 64) * 2), ("cu", 12), ("kc", CACHE), ("vc", CACHE), ("table", 16), ("lens", 8), ("lse", 3 * 4 * 4)])
@pytest.mark.parametrize("where", ["start", "end", "inside"])
def test_an_output_of_the_attention_over_one_of_its_inputs(name, bytes_, where):
    place = at(30)
    o = {"start": place + (bytes_ - 1) // 16 * 16, "end": place - O_BYTES + 16, "inside": place}[where]
    refused(lambda: attn(**{name: place, "o": o}), INVALID)


def test_an_output_of_the_attention_over_its_workspace():
    need = ug.unigist_chunk_attn_workspace_bytes(2, 3, 4, 2, 64, 2)
    refused(lambda: attn(ws=at(30), o=at(30) + need - 16, ws_bytes=need), INVALID)
    refused(lambda: attn(ws=at(30), o=at(30) - O_BYTES + 16, ws_bytes=need), INVALID)
    refused(lambda: attn(ws=at(30), lse=at(30) + need - 16, ws_bytes=need), INVALID)
