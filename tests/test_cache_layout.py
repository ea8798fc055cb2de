"""Where the cache's attention puts keys and values in LDS, from its source: the
bank conflicts that its comments rule out, and the addresses that its kernels
derive from each other by an exclusive or."""
import os
import re

import pytest

from paper_2605_01060_amd import build as B

with open(os.path.join(B.CSRC, "cache_attention.hip")) as _f:
    SOURCE = _f.read()

# Lanes that the LDS serves together in a 16-byte read, of each half wave.
READ_SETS = ([0, 1, 2, 3, 12, 13, 14, 15, 20, 21, 22, 23, 24, 25, 26, 27],
             [4, 5, 6, 7, 8, 9, 10, 11, 16, 17, 18, 19, 28, 29, 30, 31])


def slots(name, cpr):
    """Slot (16 bytes) of a chunk of a row, as the function `name` gives it."""
    body = SOURCE[SOURCE.index(f"uint32_t {name}("):]
    body = body[:body.index("\n}")]
    rule = re.search(rf"if constexpr \(CPR == {cpr}\)\s+return (.*?);", body, re.S)
    rule = rule or re.search(r"\n  return (.*?);", body, re.S)
    code = compile(" ".join(rule.group(1).split()), name, "eval")
    return lambda row, chunk: eval(code, {"row": row, "key": row, "chunk": chunk})


@pytest.mark.parametrize("cpr", [4, 8, 16])
@pytest.mark.parametrize("name", ["v_slot", "kv_position"])
def test_rows_keep_their_place(name, cpr):
    at = slots(name, cpr)
    for row in range(64):
        assert {at(row, c) for c in range(cpr)} == set(range(row * cpr, (row + 1) * cpr))


@pytest.mark.parametrize("cpr", [4, 8, 16])
@pytest.mark.parametrize("name", ["v_slot", "kv_position"])
def test_writes_of_a_chunk_of_eight_rows(name, cpr):
    """32 banks: eight slots."""
    at = slots(name, cpr)
    for row in range(0, 64, 8):
        for c in range(cpr):
            assert len({at(row + i, c) % 8 for i in range(8)}) == 8


@pytest.mark.parametrize("cpr", [4, 8, 16])
def test_few_rows_reads_of_values(cpr):
    """32 bytes of eight consecutive rows on 64 banks."""
    at = slots("v_slot", cpr)
    for row in range(0, 32, 8):
        for c in range(0, cpr, 2):
            assert len({at(row + i, c + j) % 16 for i in range(8) for j in range(2)}) == 16


@pytest.mark.parametrize("cpr", [4, 8, 16])
def test_tile_reads(cpr):
    """A chunk of the rows that are served together, and 64 bytes of four
    consecutive rows, on 64 banks."""
    at = slots("kv_position", cpr)
    for row in (0, 32):
        for group in READ_SETS:
            for c in range(cpr):
                assert len({at(row + r, c) % 16 for r in group}) == 16
    for row in range(0, 64, 4):
        for c in range(0, cpr, 4):
            assert len({at(row + i, c + j) % 16 for i in range(4) for j in range(4)}) == 16


@pytest.mark.parametrize("cpr", [4, 8, 16])
def test_tile_addresses(cpr):
    """Chunks and rows 8, 16 and 32 further on by an exclusive or of the address."""
    at = slots("kv_position", cpr)
    swz = re.search(r"H_SWZ = CPR == 16 \? (\d+) : (\d+);", SOURCE)
    swz = int(swz.group(1 if cpr == 16 else 2)) // 16
    for row in range(32):
        for c in range(cpr):
            assert at(row, c) == (at(row, 0) ^ c)
            assert at(row + 32, c) == at(row, c) + 32 * cpr
            assert at(row % 8 + 16, c) == at(row % 8, c) + 16 * cpr
            assert at(row % 8 + 8, c) == (at(row % 8, c) ^ swz) + 8 * cpr
