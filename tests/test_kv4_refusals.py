"""What the page calls of the 4-bit cache refuse on the host (no GPU needed: nothing is dereferenced)."""
import ctypes

import pytest

import paper_2412_07174_amd as scap
from paper_2412_07174_amd.binding import KV4CacheArg

FAKE = 0x7F0000001000


def cache():
    return ctypes.byref(KV4CacheArg(pool=FAKE, refs=FAKE, pages=100, kv_heads=8, head_dim=128, page_tokens=64, layers=2))


# Arrays of a fork of 6 rows of 5 pages into 4: their sizes in words
SIZES = {"table": 30, "lens": 6, "parents": 4, "table_out": 20, "lens_out": 4}


@pytest.mark.parametrize("out,other", [("table_out", "table"), ("table_out", "lens"), ("table_out", "parents"), ("lens_out", "table"),
                                       ("lens_out", "lens"), ("lens_out", "parents"), ("table_out", "lens_out")])
@pytest.mark.parametrize("where", ["same", "first word", "last word"])
def test_a_fork_writes_nothing_that_it_reads(out, other, where):
    """Rows are written while other rows' lengths, pages and parents are still being read."""
    at = {name: FAKE + 4096 * i for i, name in enumerate(SIZES)}
    at[out] = at[other] + {"same": 0, "first word": -4 * (SIZES[out] - 1), "last word": 4 * (SIZES[other] - 1)}[where]
    lib = scap.load_library()
    assert lib.scap_kv4_fork(cache(), at["table"], at["lens"], 6, at["parents"], 4, at["table_out"], at["lens_out"], 5, None) == -5


@pytest.mark.parametrize("what,n", enumerate([16, 12, 22, 10, 10, 7, 10]))
def test_a_packed_call_of_another_number_of_words_reads_none(what, n):
    """A number that is not the call's is refused before the array is touched (its address here is nowhere); the call's own goes on to
    the cache, which is missing."""
    lib = scap.load_library()
    for wrong in (1, n - 1, n + 1, 255, 1 << 20):
        assert lib.scap_kv4_call(what | wrong << 8, ctypes.c_char_p(8)) == -5
    assert lib.scap_kv4_call(what | n << 8, bytes(8 * n)) == -1
    assert lib.scap_kv4_call(7 | n << 8, ctypes.c_char_p(8)) == -5 and lib.scap_kv4_call(what - (1 << 8), ctypes.c_char_p(8)) == -5
