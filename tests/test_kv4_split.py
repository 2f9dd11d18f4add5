"""How an attention call over the 4-bit cache cuts the key axis, on the host: csrc/scap_kv4_split.hpp, compiled as it is, over sizes up to the ends
of the documented ranges.  What has to hold is the room that a workspace has for partial results and arrival counters, and the grid."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

import paper_2412_07174_amd as scap
from paper_2412_07174_amd.binding import KV4CacheArg

CSRC = os.path.join(os.path.dirname(os.path.abspath(scap.__file__)), "csrc")
MOST = 1 << 30   # tokens of a sequence

SOURCE = """
#include "scap_kv4_split.hpp"
// out: chunk, workgroups, partial results, row blocks that are cut, row blocks, longest sequence that is cut and shorter than a chunk
extern "C" void split(int places, int min_chunk, int slot_rows, int64_t B, const int* range, const int* rows, const int* blocks, int64_t* out) {
    float total = 0.f;
    int n = 0;
    for (int64_t base = 0; base < B; base += 64) {   // 64 sequences at a time, as a wavefront adds them up
        float sum = 0.f;
        for (int64_t b = base; b < base + 64 && b < B; ++b) sum += (float)blocks[b] * (float)range[b], n += blocks[b];
        total += sum;
    }
    float inv = 0.f;
    const auto cut = [&](int64_t b, int chunk, float inv) { return scap::kv4_cut(range[b], rows[b], chunk, inv, places, slot_rows); };
    const int chunk = scap::kv4_choose_chunk(total, n, places, min_chunk, inv, [&](int chunk, float inv) {
        int64_t items = 0;
        for (int64_t b = 0; b < B; ++b) items += blocks[b] * cut(b, chunk, inv);
        return items;
    });
    for (int i = 0; i < 6; ++i) out[i] = 0;
    out[0] = chunk, out[4] = n;
    for (int64_t b = 0; b < B; ++b) {
        const int c = cut(b, chunk, inv);
        out[1] += (int64_t)blocks[b] * c;
        if (c > 1) out[2] += (int64_t)blocks[b] * c, out[3] += blocks[b];
        if (c > 1 && range[b] <= chunk && range[b] > out[5]) out[5] = range[b];
        if ((int64_t)c * chunk < range[b] && c > 1) out[5] = -range[b];   // chunks that do not cover it
    }
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    (d / "split.cpp").write_text(SOURCE)
    lib = str(d / "split.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, str(d / "split.cpp"), "-o", lib],
                   check=True)
    f = ctypes.CDLL(lib).split
    ints, p = np.ctypeslib.ndpointer(np.int32, flags="C"), np.ctypeslib.ndpointer(np.int64, flags="C")
    f.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64, ints, ints, ints, p]
    f.restype = None

    def run(places, min_chunk, slot_rows, ranges, rows, blocks):
        out = np.zeros(6, dtype=np.int64)
        a = [np.ascontiguousarray(x, dtype=np.int32) for x in (ranges, rows, blocks)]
        f(places, min_chunk, slot_rows, len(ranges), *a, out)
        return dict(zip(("chunk", "items", "slots", "cuts", "n", "odd"), out.tolist()))

    return run


def holds(r, places, what):
    assert r["slots"] <= 2 * (places + 2) and r["cuts"] <= places + 2, (what, r)
    assert r["items"] <= r["n"] + places + 2, (what, r)
    assert r["odd"] == 0, (what, r)


@pytest.mark.parametrize("places", [1, 2, 3, 16, 64, 128, 256, 512, 1024])
@pytest.mark.parametrize("length", [MOST, MOST - 1, 1000000001, 999999999, (1 << 24) + 1, 1 << 20, 4097, 129, 1, 0])
@pytest.mark.parametrize("seqs", [1, 140, 1024, 5000])
def test_equal_sequences(split, places, length, seqs):
    for blocks in (1, 2, 7, 4096):
        r = split(places, 128, 1 << 30, [length] * seqs, [blocks] * seqs, [blocks] * seqs)
        holds(r, places, blocks)
        if seqs * blocks >= places:
            assert r["slots"] == 0, "enough rows' blocks for every place: nothing is cut"


def test_ragged_sequences(split):
    rng = random.Random(5)
    for _ in range(400):
        places = rng.choice([1, 2, 5, 32, 64, 128, 512, 1024])
        top = rng.choice([300, 5000, 1 << 20, 1 << 26, MOST])
        B = rng.choice([1, 2, 16, 65, 300, 3000])
        lens = [int(top * rng.random() ** rng.choice([1, 4])) for _ in range(B)]
        lens[rng.randrange(B)] = top
        blocks = [rng.choice([1, 1, 2, 40]) for _ in range(B)] if rng.random() < 0.5 else [1] * B
        rows = [16 * b for b in blocks]
        slot_rows = rng.choice([16, 1 << 30])
        r = split(places, rng.choice([128, 256]), slot_rows, lens, rows, blocks)
        holds(r, places, (places, top, B))


def test_as_many_sequences_as_a_call_takes(split):
    """Their ranges' sum in fp32 is some 2^14 roundings off."""
    rng = np.random.default_rng(6)
    for most in (3, 4097, 1 << 24, MOST):
        lens = rng.integers(0, most, 1 << 20)
        lens[77] = MOST
        for places in (2, 128, 1024):
            holds(split(places, 128, 1 << 30, lens, np.ones_like(lens), np.ones_like(lens)), places, (most, places))


@pytest.mark.parametrize("D,heads,tokens,seqs,waves", [(64, 1, 131072, 1, 8), (128, 8, 140, 140, 4), (64, 8, 129, 129, 4), (128, 8, 1024, 1024, 4)])
def test_the_workspace_has_room_for_the_longest_sequences(split, D, heads, tokens, seqs, waves):
    """By what the library asks for: one query head a kv head, tokens / seqs new ones a sequence, as long as a sequence may be."""
    c = KV4CacheArg(pool=1 << 20, refs=0, pages=100, kv_heads=heads, head_dim=D, page_tokens=64, layers=1)
    new = tokens // seqs
    room = scap.load_library().scap_kv4_workspace_bytes(ctypes.byref(c), seqs, tokens, heads, new) - (1 << 20)
    if new == 1:
        places, blocks, slot = 4096 // waves // heads, 1, 2 * (D + 2) * 4
    else:   # blocks of 256 rows
        places, blocks, slot = 2048 // waves // heads, new // 256, 256 * (D + 2) * 4
    r = split(places, 128 if new == 1 else 256, new, [MOST] * seqs, [new] * seqs, [blocks] * seqs)
    holds(r, places, "")
    assert r["slots"] * heads * slot <= room
