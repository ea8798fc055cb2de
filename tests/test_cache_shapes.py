"""How calls of attention over a cache are cut, on the CPU: the header's rule,
compiled here, and what it and the kernel's choice by lengths make of the calls
that the GPU tests make, so that no arrangement is left without one."""
import ctypes
import subprocess

import numpy as np
import pytest

import test_gpu_decoder as D
from paper_2605_01060_amd import build as B

CUS = 256
WRAPPER = r"""
#include "cache_shape.h"
using namespace surge;
extern "C" void shape(int64_t n_seqs, int64_t max_rows, int hk, int group, int dh, int64_t max_length,
                      int cus, int64_t* out) {
  const CacheShape s = cache_attention_shape(n_seqs, max_rows, hk, group, dh, max_length, cus);
  out[0] = s.tile_rows, out[1] = s.block_shift, out[2] = s.tiles, out[3] = s.units, out[4] = s.workers;
  out[5] = s.least_share, out[6] = s.wave_units;
  out[7] = s.workers ? cache_attention_join(s, max_length) : -1, out[8] = s.workspace_bytes(dh);
}
"""


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    d = tmp_path_factory.mktemp("cache_shape")
    src, so = d / "wrapper.cpp", d / "wrapper.so"
    src.write_text(WRAPPER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{B.CSRC}", str(src), "-o", str(so)],
                   check=True)
    lib = ctypes.CDLL(str(so))
    lib.shape.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 3 + [ctypes.c_int64, ctypes.c_int, ctypes.c_void_p]

    def of(n_seqs, max_rows, hk, group, dh, max_length):
        out = np.zeros(9, np.int64)
        lib.shape(n_seqs, max_rows, hk, group, dh, max_length, CUS, out.ctypes.data)
        names = ("tile_rows", "block_shift", "tiles", "units", "workers", "least_share", "wave_units", "join",
                 "workspace")
        return dict(zip(names, out.tolist()))

    return of


def arrangement(shape, lengths, rows, hk, group, dh, max_length, causal):
    """(rows of a tile, who has a unit, join's waves, whether a unit was cut,
    whether a thread has several (sequence, tile) pairs that begin inside a
    sequence).  Who: a "unit" a workgroup, a "wave" each, or of a call that is
    shared out, equal "parts", "whole" units or equal "shares", as
    shared_units chooses by the lengths."""
    lengths, rows = np.asarray(lengths, np.int64), np.asarray(rows, np.int64)
    s = shape(len(lengths), int(rows.max()), hk, group, dh, max_length)
    if not s["workers"]:
        return s["tile_rows"], "wave" if s["wave_units"] else "unit", -1, False, False
    blocks = []
    for n, r in zip(lengths.tolist(), rows.tolist()):
        for t in range(s["tiles"]):
            first = t * s["tile_rows"]
            if first >= r * group:
                blocks.append(0)
                continue
            last = min(first + s["tile_rows"], r * group) - 1
            sees = max(n - r + last // group + 1, 0) if causal else n
            blocks.append(max(-(-sees // (1 << s["block_shift"])), 1))
    blocks = np.array(blocks)
    total, most = int(blocks.sum()) * hk, int(blocks.max())
    workers, units = s["workers"], s["units"]
    share = max(-(-total // workers), s["least_share"])
    per = -(-len(blocks) // 256)
    if units <= workers // 4 and per == 1:
        who, cut = "parts", share
        if int((-(-blocks // cut)).sum()) * hk > workers:
            cut = max((total + workers - units - 1) // (workers - units), s["least_share"])
        cut = most > cut
    elif units <= workers and s["tile_rows"] < 64 and most <= share * (2 if s["tile_rows"] == 16 else 1) + 6:
        who, cut = "whole", False
    else:
        ends = np.cumsum(np.repeat(blocks[blocks > 0], hk))
        who, cut = "shares", bool((((ends[:-1] % share) != 0) | (np.diff(ends) > share)).any())
    return s["tile_rows"], who, s["join"], cut, s["tiles"] > 1 and per > 1 and per % s["tiles"] != 0


def batch_call(seqs, rows, length):
    """As test_attention_of_batches makes it."""
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(1, length, seqs)
    lengths[rng.random(seqs) < 0.1] = 0
    lengths[seqs // 2], lengths[-1] = length, 0
    counts = rng.integers(1, rows + 1, seqs)
    counts[rng.random(seqs) < 0.1] = 0
    counts[seqs // 2] = rows
    return lengths, counts


def many_call(seqs, rows, length):
    """As test_attention_of_many_units makes it."""
    rng = np.random.default_rng(seqs + rows)
    lengths = rng.integers(0, length, seqs)
    lengths[seqs // 2] = length
    counts = rng.integers(0, rows + 1, seqs)
    counts[seqs // 2] = rows
    return lengths, counts


def calls():
    """(lengths, rows, heads, key heads, d_head) of the GPU tests' attention."""
    for lengths, rows, _, heads, hk, dh in D.LONG:
        yield lengths, rows, heads, hk, dh
    yield from D.SHAPES
    for _, heads, hk, dh in D.HEADS:
        yield [n for n, _ in D.MIX], [r for _, r in D.MIX], heads, hk, dh
        for rows in (1, 2, 3, 5, 9, 20):  # test_attention_of_steps
            yield [1, 90, 0, 17, 64, 33, 500, 2, 130], [rows] * 9, heads, hk, dh
    for seqs, rows, length, _, heads, hk, dh in D.BATCHES:
        yield *batch_call(seqs, rows, length), heads, hk, dh
    for seqs, rows, length, _, heads, hk, dh in D.MANY:
        yield *many_call(seqs, rows, length), heads, hk, dh
    for seqs, rows, shortest, length, _, heads, hk, dh in D.SHARED:
        yield *D.shared_call(seqs, rows, shortest, length), heads, hk, dh


def taken(shape, lengths, rows, heads, hk, dh, causal=True):
    return arrangement(shape, lengths, rows, hk, heads // hk, dh, int(max(lengths)), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_every_arrangement_has_a_call_on_the_gpu(shape, dh, causal):
    found = {taken(shape, *c, causal) for c in calls() if c[-1] == dh}
    who = {(tile, w) for tile, w, *_ in found}
    assert who >= {(tile, w) for tile in (16, 32) for w in ("unit", "wave", "parts", "whole", "shares")}
    assert who >= {(tile, w) for tile in (64, 128) for w in ("unit", "parts", "shares")}
    cuts = {(tile, w) for tile, w, _, cut, _ in found if cut}
    assert cuts >= {(tile, w) for tile in (16, 32, 64, 128) for w in ("parts", "shares")}
    assert any(inside for *_, inside in found)  # a thread's pairs that begin inside a sequence


def test_every_join_has_a_call_on_the_gpu(shape):
    found = {(dh, join) for *c, dh in calls() for _, _, join, cut, _ in [taken(shape, *c, dh)] if cut}
    assert found >= {(dh, join) for dh in (32, 64, 128) for join in (0, 1, 4, 16)}


@pytest.mark.parametrize("call", D.MANY)
def test_calls_of_many_units(shape, call):
    """Short units are a wave's; those of tiles that stay tiles a workgroup's."""
    seqs, rows, length, _, heads, hk, dh = call
    tile, who, *_ = taken(shape, *many_call(seqs, rows, length), heads, hk, dh)
    assert (tile < 64) == (who == "wave")


@pytest.mark.parametrize("rows,hk,group,dh", [(1, 8, 4, 128), (8, 8, 4, 128), (1, 12, 1, 64), (30, 8, 1, 64),
                                              (1, 12, 1, 32), (20, 12, 1, 32)])
def test_no_wave_has_a_long_unit_to_itself(shape, rows, hk, group, dh):
    """One sequence's keys may be as many as max_length says, however short the
    others are: beyond 1024 a unit has a workgroup, however many units there are."""
    for seqs in (2000, 20_000):
        for length in (1025, 2048, 8192, 100_003, 1 << 30):
            assert not shape(seqs, rows, hk, group, dh, length)["wave_units"], (seqs, length)
        for length in (1, 128, 240, 1024):
            assert shape(seqs, rows, hk, group, dh, length)["wave_units"], (seqs, length)


@pytest.mark.parametrize("seqs,rows,longest,page,heads,hk,dh", D.TAILS)
def test_calls_of_one_long_sequence_among_many(shape, seqs, rows, longest, page, heads, hk, dh):
    s = shape(seqs, rows, hk, heads // hk, dh, longest)
    places = {16: {32: 7, 64: 4, 128: 3}, 32: {32: 5, 64: 3, 128: 2}}[s["tile_rows"]][dh]
    assert s["units"] >= 8 * CUS * places
    assert s["workers"] == 0 and s["wave_units"] == (longest <= 1024)


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_workspaces_stay_within_what_is_documented(shape, dh):
    most = 0
    for seqs in (1, 2, 5, 16, 48, 64, 96, 97, 128, 192, 256, 500, 700, 1000, 2048):
        for hk in (1, 2, 4, 8, 12, 64):
            for rows in (1, 4, 8, 16, 60, 128, 500, 5000, 1 << 20):
                for length in (100, 900, 1100, 2000, 3000, 100_003, 1 << 30):
                    most = max(most, shape(seqs, rows, hk, 4, dh, length)["workspace"])
    assert 0 < most <= 68_200_000
    # More sequences may need less: 96 of 8 key heads are shared out, 97 are not.
    if dh == 128:
        assert shape(96, 1, 8, 4, dh, 8000)["workspace"] > 0 == shape(97, 1, 8, 4, dh, 8000)["workspace"]
