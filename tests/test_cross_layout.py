"""Cross attention on the CPU: its LDS swizzles from the expressions of the
source file, and the work list that the host builds."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

from paper_2605_01060_amd import build as B

with open(os.path.join(B.CSRC, "cross_attention.hip")) as _f:
    SRC = _f.read()

# Lanes of a half wave that a 16-byte read is served for at once.
FIRST = [*range(0, 4), *range(12, 16), *range(20, 28)]
GROUPS = [FIRST, [lane for lane in range(32) if lane not in FIRST]]


def _expression(function, cpr):
    body = SRC[SRC.index(function):]
    return re.search(rf"if constexpr \(CPR == {cpr}\) return (.*?);", body).group(1)


def slot(cpr, row, chunk):
    return eval(_expression("int kv_slot", cpr), {"row": row, "chunk": chunk})


@pytest.mark.parametrize("cpr", [8, 16])
def test_reads_of_keys_have_no_bank_conflicts(cpr):
    """One chunk of 32 rows, 16 lanes at a time, over 16 slots of 16 bytes."""
    for chunk in range(cpr):
        for lanes in GROUPS:
            assert len({slot(cpr, lane, chunk) % 16 for lane in lanes}) == 16


@pytest.mark.parametrize("cpr", [8, 16])
def test_transposing_reads_of_values_have_no_bank_conflicts(cpr):
    """32 lanes of 8 bytes: 4 chunks of each of 4 consecutive rows."""
    for row0 in range(0, 64, 4):
        for chunk0 in range(0, cpr, 4):
            slots = {slot(cpr, row0 + r, chunk0 + c) % 16 for r in range(4) for c in range(4)}
            assert len(slots) == 16


@pytest.mark.parametrize("cpr", [8, 16])
def test_a_copy_puts_each_chunk_where_it_is_read(cpr):
    rows = 64 // cpr  # that a copy fills
    for copy in range(64 // rows):
        for lane in range(64):
            chunk = eval(_expression("int kv_copy_chunk", cpr), {"lane": lane, "copy": copy})
            assert slot(cpr, copy * rows + lane // cpr, chunk) == 64 * copy + lane


@pytest.mark.parametrize("cpr", [8, 16])
def test_addresses_by_exclusive_or(cpr):
    """The kernel takes K's chunk 2 kk + half at the address of chunk half ^ 32
    kk, and V's chunk 4 dt + c of key + 8 h at that of chunk c of the key ^ (64
    dt ^ 32 h)."""
    swz = int(re.search(r"H_SWZ = CPR == 4 \? 16 : (\d+);", SRC).group(1))
    for row in range(32):
        for half in range(2):
            for kk in range(cpr // 2):
                assert slot(cpr, row, 2 * kk + half) * 16 == (slot(cpr, row, half) * 16) ^ (32 * kk)
    for key in range(8):
        for c in range(4):
            for dt in range(cpr // 4):
                for h in range(2):
                    at = (slot(cpr, key, c) * 16 ^ (64 * dt ^ swz * h)) + 8 * h * cpr * 16
                    assert slot(cpr, key + 8 * h, 4 * dt + c) * 16 == at


WRAPPER = r"""
#include "cross_list.h"
using namespace surge;
static CrossList list;
extern "C" void build(int64_t n, const int64_t* q, const int64_t* kv, int h, int g, int dh, int cus,
                      int64_t* sizes) {
  list = CrossList();
  build_cross_list(n, q, kv, h, g, dh, cus, &list);
  for (int c = 0; c < CROSS_CLASSES; ++c) sizes[c] = (int64_t)list.items[c].size();
  sizes[3] = (int64_t)list.joins.size();
  sizes[4] = list.n_parts;
  sizes[5] = list.max_parts;
}
extern "C" int short_blocks() { return list.short_blocks; }
extern "C" const void* items(int c) { return list.items[c].data(); }
extern "C" const void* joins() { return list.joins.data(); }
"""


@pytest.fixture(scope="module")
def lists(tmp_path_factory):
    d = tmp_path_factory.mktemp("cross")
    src, so = d / "wrapper.cpp", d / "wrapper.so"
    src.write_text(WRAPPER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", f"-I{B.CSRC}", str(src),
                    os.path.join(B.CSRC, "cross.cpp"), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.build.argtypes = [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int] * 4 + \
        [ctypes.c_void_p]
    for f, args in ((lib.items, [ctypes.c_int]), (lib.joins, [])):
        f.argtypes, f.restype = args, ctypes.c_void_p

    def build(q, kv, heads, group, dh, cus):
        cu = [np.concatenate([[0], np.cumsum(x)]).astype(np.int64) for x in (q, kv)]
        sizes = np.zeros(6, np.int64)
        lib.build(len(q), cu[0].ctypes.data, cu[1].ctypes.data, heads, group, dh, cus, sizes.ctypes.data)

        def array(ptr, n, width):
            if n == 0:
                return np.zeros((0, width), np.int32)
            return np.ctypeslib.as_array(ctypes.cast(ptr, ctypes.POINTER(ctypes.c_int32)), (n, width)).copy()

        return [array(lib.items(c), int(sizes[c]), 8) for c in range(3)], \
            array(lib.joins(), int(sizes[3]), 6), int(sizes[4]), int(sizes[5]), cu

    build.short_blocks = lambda: bool(lib.short_blocks())
    return build


ROWS = (128, 64, 32)


def check_list(q, kv, group, items, joins, n_parts, max_parts, cu):
    """Every row of 32 meets every key of its text once, in order of its
    parts, and what is split is joined."""
    seen, slots = {}, {}
    for c, step in enumerate(ROWS):
        lengths = items[c][:, 5] - items[c][:, 4]
        assert (np.diff(lengths) <= 0).all()  # longest first
        for q_beg, row0, rows, kv_beg, k0, k1, part, _ in items[c].tolist():
            assert 0 <= row0 < rows and row0 % step == 0
            for b in range(row0, min(rows, row0 + step), 32):
                seen.setdefault((q_beg, kv_beg, rows, b), []).append((k0, k1))
                if part >= 0:
                    s = part + (b - row0) // 32
                    assert s not in slots
                    slots[s] = (q_beg, b, k0)
    assert sorted(slots) == list(range(n_parts))
    want = {(int(cu[0][i]), int(cu[1][i]), q[i] * group, b): kv[i]
            for i in range(len(q)) for b in range(0, q[i] * group, 32)}
    assert set(seen) == set(want)
    for key, parts in seen.items():
        parts.sort()
        assert parts[0][0] == 0 and parts[-1][1] == want[key]
        assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
    joined = 0
    for q_beg, row0, rows, part0, parts, stride in joins.tolist():
        assert 1 <= rows <= 32 and 2 <= parts <= max_parts
        got = [slots[part0 + p * stride] for p in range(parts)]
        assert all(g[:2] == (q_beg, row0) for g in got) and got == sorted(got)
        joined += parts
    assert joined == n_parts


@settings(max_examples=150, deadline=None)
@given(seqs=st.lists(st.tuples(st.sampled_from([0, 1, 1, 2, 7, 33, 64, 65, 129, 700]),
                               st.sampled_from([0, 1, 31, 32, 33, 64, 257, 1000, 9001, 50_000])),
                     min_size=1, max_size=12),
       heads=st.sampled_from([1, 4, 12]), group=st.sampled_from([1, 3, 8]),
       dh=st.sampled_from([32, 64, 128]), cus=st.sampled_from([1, 8, 256]))
def test_lists_cover_every_row_and_key_once(lists, seqs, heads, group, dh, cus):
    # Sequences of no query share their first token with the next one: keep
    # the texts apart by a state each.
    q, kv = [s[0] for s in seqs], [s[1] + (i % 2) for i, s in enumerate(seqs)]
    items, joins, n_parts, max_parts, cu = lists(q, kv, heads, group, dh, cus)
    check_list(q, kv, group, items, joins, n_parts, max_parts, cu)


def test_few_rows_over_a_long_text_are_split_over_the_chip(lists):
    items, joins, n_parts, max_parts, _ = lists([1], [100_000], 8, 4, 128, 256)
    assert n_parts == max_parts == len(items[2]) and 4 * 256 * 0.9 <= 8 * n_parts <= 4 * 256
    items, joins, n_parts, _, _ = lists([1] * 2000, [48] * 2000, 12, 1, 64, 256)
    assert n_parts == 0 and len(joins) == 0 and len(items[2]) == 2000


def test_short_blocks_of_keys_where_the_third_unit_of_a_cu_is_filled(lists):
    def short(n, q, kv, heads, dh):
        lists([q] * n, [kv] * n, heads, 1, dh, 256)
        return lists.short_blocks()

    assert short(96, 128, 1000, 8, 128)       # 768 units: 3 a CU
    assert not short(128, 128, 1000, 8, 128)  # 1024: twice 2 a CU
    assert not short(1, 128, 256, 12, 128)
    assert short(300, 128, 512, 8, 128)       # many units
    assert not short(300, 128, 256, 8, 128)   # of few blocks
    for dh in (32, 64):
        assert not short(96, 128, 1000, 8, dh) and not short(300, 128, 512, 8, dh)


@pytest.mark.parametrize("n", [1, 20, 399, 3000])
@pytest.mark.parametrize("heads,group,dh", [(12, 1, 64), (2, 4, 128)])
def test_lists_of_queries_without_states_beside_states_without_queries(lists, n, heads, group, dh):
    """Few units and, from 399 texts on 12 key heads, more than eight a CU: no text
    that is read has a key, and one that is not read has some."""
    q, kv = [1] * n + [0], [0] * n + [100]
    items, joins, n_parts, max_parts, cu = lists(q, kv, heads, group, dh, 256)
    check_list(q, kv, group, items, joins, n_parts, max_parts, cu)
    assert n_parts == 0 and len(items[2]) == n


@settings(max_examples=100, deadline=None)
@given(kinds=st.lists(st.tuples(st.sampled_from([0, 0, 1, 33, 130]), st.sampled_from([0, 0, 1, 100, 3000])),
                      min_size=1, max_size=6),
       times=st.sampled_from([1, 40, 300]), heads=st.sampled_from([1, 12]),
       dh=st.sampled_from([64, 128]))
def test_lists_of_many_texts(lists, kinds, times, heads, dh):
    """The same, up to 1,800 texts: either length is 0 as often as not."""
    q, kv = [k[0] for k in kinds] * times, [k[1] for k in kinds] * times
    items, joins, n_parts, max_parts, cu = lists(q, kv, heads, 2, dh, 64)
    seen = {}
    for c, step in enumerate(ROWS):
        for q_beg, row0, rows, kv_beg, k0, k1, part, _ in items[c].tolist():
            assert 0 <= row0 < rows and row0 % step == 0 and k1 >= k0
            seen.setdefault((q_beg, row0), []).append((k0, k1))
    keys = {int(cu[0][i]): kv[i] for i in range(len(q)) if q[i]}
    assert {b for b, _ in seen} == set(keys)
    for (q_beg, _), parts in seen.items():
        parts.sort()
        assert parts[0][0] == 0 and parts[-1][1] == keys[q_beg]
        assert all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
    assert sum(j[4] for j in joins.tolist()) == n_parts and 2 * len(joins) <= n_parts
