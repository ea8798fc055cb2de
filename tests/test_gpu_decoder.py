"""The decoder's operators on the GPU against their definitions in 64 bits:
keys and values written to a cache in 4 bits and read back, attention over it,
the check of drafted tokens, and the three together.

What a cache holds is compared bit by bit.  Attention's tolerance counts
roundings: one to bf16 is off by at most BF16 = 2^-8 of the value, one in fp32
by F32 = 2^-24.
"""
import math

import numpy as np
import pytest

from gpu_util import torch_cuda
from paper_2605_01060_amd import surge as S
from test_gpu_reader import (BF16, EPS, F32, check_i8, gen, linear_reference, norm_reference, quantized32, randn,
                             strided, within)

pytestmark = pytest.mark.gpu

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TINY = 2.0 ** -100


def dev(x, dtype=np.int32):
    return torch_cuda().from_numpy(np.ascontiguousarray(x, dtype)).cuda()


def cu_of(counts):
    return dev(np.concatenate([[0], np.cumsum(counts)]))


def quantized(x):
    """Codes [T, w] 0..15 and scale bytes [T, w / 32] of bf16 rows, in 64 bits."""
    torch = torch_cuda()
    x = x.double().view(len(x), -1, 32)
    a = x.abs().amax(2, keepdim=True)
    marked = ~torch.isfinite(a)
    a = torch.where(marked, 1.0, a.clamp_min(TINY))
    e = torch.ceil(torch.log2(a / 7)).clamp_max(125)
    y = x.abs() / torch.exp2(e)
    code = torch.zeros(x.shape, dtype=torch.int64, device=x.device)
    for i in range(7):  # nearest, ties to the even code
        middle = (VALUES[i] + VALUES[i + 1]) / 2
        code += (y > middle) | ((y == middle) & (i % 2 == 1))
    code += 8 * torch.signbit(x)
    byte = torch.where(marked, 255, e.long() + 127)
    return code.flatten(1), byte[..., 0]


def values(code, byte):
    """What codes [.., w] and scale bytes [.., w / 32] stand for, in 64 bits."""
    torch = torch_cuda()
    v = torch.tensor(VALUES + [-x for x in VALUES], dtype=torch.float64, device=code.device)[code]
    scale = torch.where(byte == 255, math.nan, torch.exp2(byte.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


class Cache:
    """Pages with random places for sequences of the given lengths, filled with
    bytes that stand for NaN (or `fill`) until something is written."""

    def __init__(self, lengths, page, hk, dh, seed, fill=255, room=0, spare=3):
        torch = torch_cuda()
        self.lengths_np, self.page, self.hk, self.dh = np.asarray(lengths, np.int64), page, hk, dh
        need = -(-(self.lengths_np + room) // page)
        total = int(need.sum())
        self.n_pages = total + spare
        rng = np.random.default_rng(seed)
        perm = rng.permutation(self.n_pages)[:total]
        self.width = max(int(need.max(initial=0)), 1) + 2
        self.table_np = np.full((len(need), self.width), -7, np.int64)
        self.table_np[np.arange(self.width) < need[:, None]] = perm
        self.bytes = S.surge_cache_page_bytes(page, hk, dh)
        self.pages = torch.full((self.n_pages, self.bytes), fill, dtype=torch.uint8, device="cuda")
        self.table, self.lengths = dev(self.table_np), dev(self.lengths_np)
        self.max_length = int((self.lengths_np + room).max(initial=0))
        self.desc = S.KVCache(self.pages, self.n_pages, page, hk, dh, self.table, self.width, len(need),
                              self.lengths, self.max_length)

    def fields(self, pages=None):
        """Codes of keys, of values, scales of keys, of values, as views."""
        body = (self.pages if pages is None else pages).view(self.n_pages, self.hk, -1)
        out, at = [], 0
        for width in (self.dh // 2, self.dh // 2, self.dh // 32, self.dh // 32):
            out.append(body[:, :, at:at + self.page * width].unflatten(2, (self.page, width)))
            at += self.page * width
        assert at == body.shape[2]
        return out

    def put(self, seq, pos, k, v, pages=None):
        """Rows of keys and values [T, hk dh] at positions, by the definition."""
        torch = torch_cuda()
        page = torch.from_numpy(self.table_np[seq, np.asarray(pos) // self.page]).cuda()
        slot = torch.from_numpy(np.asarray(pos) % self.page).cuda()
        f = self.fields(pages)
        for w, x in enumerate((k, v)):
            code, byte = quantized(x)
            code = code.view(len(x), self.hk, self.dh)
            f[w][page, :, slot] = (code[..., ::2] + 16 * code[..., 1::2]).to(torch.uint8)
            f[w + 2][page, :, slot] = byte.view(len(x), self.hk, -1).to(torch.uint8)

    def fill(self, seed, scale=1.0):
        """Every sequence's positions, and the values that they stand for."""
        torch = torch_cuda()
        g = gen(seed)
        self.held = []
        for i, n in enumerate(self.lengths_np):
            k, v = ((scale * randn(g, int(n), self.hk * self.dh)).bfloat16() for _ in range(2))
            if n:
                self.put(i, np.arange(n), k, v)
            self.held.append([values(*quantized(x)).view(int(n), self.hk, self.dh) if n else
                              torch.zeros(0, self.hk, self.dh, dtype=torch.float64, device="cuda")
                              for x in (k, v)])
        return self


def places(lengths, rows):
    """Sequence and position of each row, some of them negative."""
    seq = np.repeat(np.arange(len(rows)), rows)
    pos = np.concatenate([np.arange(n - r, n) for n, r in zip(lengths, rows)]) if len(rows) else seq
    return seq, pos.astype(np.int64)


# ---------------------------------------------------------------------------
# Written and read back
# ---------------------------------------------------------------------------

LENGTHS = [5, 0, 1, 16, 17, 40, 3, 64, 100, 33, 0, 2, 300, 15]
ROWS = [5, 0, 1, 3, 17, 1, 7, 40, 0, 33, 2, 0, 129, 1]  # two sequences have more rows than positions


@pytest.mark.parametrize("page,hk,dh", [(16, 1, 32), (16, 16, 64), (32, 3, 64), (64, 2, 128), (128, 5, 32),
                                        (256, 1, 128), (32, 12, 64), (64, 8, 128)])
@pytest.mark.parametrize("uniform", [0, 1, 3])
def test_write_and_read(page, hk, dh, uniform):
    torch = torch_cuda()
    rows = [uniform] * len(LENGTHS) if uniform else ROWS
    c = Cache(LENGTHS, page, hk, dh, page + hk, fill=0xAB)
    g, n, w = gen(dh + uniform), sum(rows), hk * dh
    k, v = ((randn(g, n + 2, w) * torch.exp2(6 * randn(g, n + 2, 1))).bfloat16() for _ in range(2))
    (ks, _), (vs, _) = strided(k, 8), strided(v, 24)
    cu = None if uniform else cu_of(rows)
    want = c.pages.clone()
    seq, pos = places(LENGTHS, rows)
    on = pos >= 0
    c.put(seq[on], pos[on], k[:n][torch.from_numpy(on).cuda()], v[:n][torch.from_numpy(on).cuda()], want)
    stream = torch.cuda.current_stream()
    S.surge_op_cache_write(c.desc, n, cu, ks, w + 8, vs, w + 24, stream)
    assert torch.equal(c.pages, want)  # and nothing beside the rows' places
    out = [torch.full((n + 2, w + 16), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    S.surge_op_cache_read(c.desc, n, cu, out[0], w + 16, out[1], w + 16, stream)
    for x, o in ((k, out[0]), (v, out[1])):
        ref = values(*quantized(x[:n]))
        ref[torch.from_numpy(~on).cuda()] = 0
        assert torch.equal(o[:n, :w].double(), ref)
        assert (o[n:] == 7).all() and (o[:, w:] == 7).all()


def test_write_of_rows_behind_the_last_sequence():
    """Offsets that end before n_rows: the rows behind stay as they were."""
    torch = torch_cuda()
    c = Cache([40, 50], 16, 2, 64, 1, fill=0xAB)
    g = gen(1)
    k, v = (randn(g, 90, 128).bfloat16() for _ in range(2))
    cu = dev([0, 10, 31])
    want = c.pages.clone()
    seq, pos = places([40, 50], [10, 21])
    c.put(seq, pos, k[:31], v[:31], want)
    S.surge_op_cache_write(c.desc, 90, cu, k, 128, v, 128)
    assert torch.equal(c.pages, want)
    out = [torch.full((90, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    S.surge_op_cache_read(c.desc, 90, cu, out[0], 128, out[1], 128)
    assert torch.equal(out[0][:31].double(), values(*quantized(k[:31])))
    assert (out[0][31:] == 7).all() and (out[1][31:] == 7).all()


@pytest.mark.parametrize("seqs,empty", [(3000, False), (5000, True), (64, False), (65, True), (1, False)])
def test_write_and_read_of_many_sequences(seqs, empty):
    """Rows find their sequence among many, hundreds of empty ones between."""
    torch = torch_cuda()
    rng = np.random.default_rng(seqs)
    rows = rng.integers(0, 9, seqs)
    if empty:
        rows[rng.random(seqs) < 0.9] = 0
        rows[10:min(seqs, 400)] = 0
    rows[-1] = 3
    lengths = rows + rng.integers(0, 20, seqs)
    c = Cache(lengths, 16, 1, 32, seqs, fill=0xAB)
    g, n = gen(seqs), int(rows.sum())
    k, v = (randn(g, n, 32).bfloat16() for _ in range(2))
    want = c.pages.clone()
    c.put(*places(lengths, rows), k, v, want)
    S.surge_op_cache_write(c.desc, n, cu_of(rows), k, 32, v, 32)
    assert torch.equal(c.pages, want)
    out = [torch.empty_like(k) for _ in range(2)]
    S.surge_op_cache_read(c.desc, n, cu_of(rows), out[0], 32, out[1], 32)
    assert torch.equal(out[0].double(), values(*quantized(k)))
    assert torch.equal(out[1].double(), values(*quantized(v)))


def test_write_of_every_bf16():
    """Every finite bf16 as the largest of its 32 and beside larger ones."""
    torch = torch_cuda()
    bits = torch.arange(65536, device="cuda").to(torch.int16).view(torch.bfloat16)
    x = bits[torch.isfinite(bits)]
    rows = x[:, None].repeat(1, 32)
    rows[:, 1:] *= torch.rand(31, generator=gen(1), device="cuda").bfloat16()
    rows[::2, 7] = (rows[::2, 0].float() * 13).clamp(-3e38, 3e38).bfloat16()
    n = len(rows) // 16 * 16
    k, v = rows[:n].view(n // 16, 512), rows[:n].flip(0).view(n // 16, 512)
    c = Cache([len(k)], 64, 16, 32, 1)
    S.surge_op_cache_write(c.desc, len(k), None, k, 512, v, 512)
    out = [torch.empty_like(k) for _ in range(2)]
    S.surge_op_cache_read(c.desc, len(k), None, out[0], 512, out[1], 512)
    for a, o in ((k, out[0]), (v, out[1])):
        ref = values(*quantized(a))
        assert torch.equal(o.double(), ref) and torch.isfinite(o).all()
        # As documented: off by the scale at most.
        b = a.double().view(-1, 32)
        assert ((ref.view(-1, 32) - b).abs() <= b.abs().amax(1, keepdim=True).clamp_min(TINY) * (2 / 7)).all()


def test_write_marks_what_is_not_finite():
    torch = torch_cuda()
    c = Cache([4], 16, 1, 64, 1, fill=0)
    k = torch.ones(4, 64, device="cuda").bfloat16()
    k[0, 3], k[1, 40], k[2, 63] = math.nan, math.inf, -math.inf
    S.surge_op_cache_write(c.desc, 4, None, k, 64, k, 64)
    out = [torch.empty_like(k) for _ in range(2)]
    S.surge_op_cache_read(c.desc, 4, None, out[0], 64, out[1], 64)
    for o in out:
        nan = o.isnan()
        assert nan[0, :32].all() and nan[1, 32:].all() and nan[2, 32:].all() and int(nan.sum()) == 96
        assert (o[~nan] == 1).all()


def test_entries_that_are_no_pages():
    """Not written; read as NaN; lengths out of range are clamped."""
    torch = torch_cuda()
    c = Cache([40, 40, 40], 16, 1, 32, 1, fill=0xAB)
    good = c.table_np.copy()
    c.table_np[0, 1], c.table_np[1, 0], c.table_np[2, 2] = -1, c.n_pages, 1 << 30
    c.table.copy_(dev(c.table_np))
    k = randn(gen(1), 120, 32).bfloat16()
    want = c.pages.clone()
    seq, pos = places([40] * 3, [40] * 3)
    on = (c.table_np == good)[seq, pos // 16]
    on_t = torch.from_numpy(on).cuda()
    c.put(seq[on], pos[on], k[on_t], k[on_t], want)
    S.surge_op_cache_write(c.desc, 120, None, k, 32, k, 32)
    assert torch.equal(c.pages, want)
    out = [torch.empty_like(k) for _ in range(2)]
    S.surge_op_cache_read(c.desc, 120, None, out[0], 32, out[1], 32)
    assert torch.equal(out[0][on_t].double(), values(*quantized(k[on_t]))) and out[0][~on_t].isnan().all()
    c.lengths.copy_(dev([-5, 1 << 30, 0]))
    S.surge_op_cache_write(c.desc, 120, None, torch.zeros_like(k), 32, k, 32)
    seq, pos = places([0, 40, 0], [40] * 3)
    on = (pos >= 0) & (c.table_np == good)[seq, np.maximum(pos, 0) // 16]
    c.put(seq[on], pos[on], torch.zeros_like(k)[:on.sum()], k[torch.from_numpy(on).cuda()], want)
    assert torch.equal(c.pages, want)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def attend(c, q, rows, heads, causal, out, workspace=None, stream=None, cu=None, max_rows=None):
    torch = torch_cuda()
    max_rows = max(max(rows), 1) if max_rows is None else max_rows
    need = S.surge_cache_attention_workspace(c.desc, max_rows, heads)
    if workspace is None and need:
        workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    S.surge_op_cache_attention(c.desc, sum(rows), cu_of(rows) if cu is None else cu, max_rows, heads,
                               causal, c.dh ** -0.5, q, q.stride(0), workspace, out, out.stride(0),
                               stream or torch.cuda.current_stream())
    return need


def reference(c, q, rows, heads, causal):
    """Output and tolerance.  A probability is off by its rounding to bf16 and
    by its score's fp32 error (dh + 2 roundings of the sum of magnitudes, as a
    relative error, plus 8 roundings around the exponential); the sums add a
    rounding per 32-key step and part."""
    torch = torch_cuda()
    hk, dh = c.hk, c.dh
    G = heads // hk
    ref = torch.zeros(sum(rows), heads * dh, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(ref)
    at = 0
    for i, r in enumerate(rows):
        n = int(c.lengths_np[i])
        if r and n:
            k, v = (x.permute(1, 0, 2).contiguous() for x in c.held[i])
            x = q[at:at + r].double().view(r, hk, G, dh).permute(1, 0, 2, 3).reshape(hk, r * G, dh)
            kt = k.transpose(1, 2).contiguous()
            s = torch.bmm(x, kt) * dh ** -0.5
            pos = torch.arange(n - r, n, device="cuda").repeat_interleave(G)
            hidden = torch.arange(n, device="cuda") > pos[:, None] if causal else \
                torch.zeros(r * G, n, dtype=torch.bool, device="cuda")
            s = torch.where(hidden, -math.inf, s)
            none = hidden.all(1)
            s[:, none] = 0.0
            p = torch.softmax(s, 2)
            p[:, none] = 0.0
            o, o_abs = torch.bmm(p, v), torch.bmm(p, v.abs())
            size = torch.where(hidden, 0.0, torch.bmm(x.abs(), kt.abs())).amax(2, keepdim=True) * dh ** -0.5
            rel = BF16 + 2 * (dh + 2) * F32 * size + (16 + 2 * (n // 32 + 1)) * F32
            t = BF16 * o.abs() + 1.01 * rel * o_abs
            for y, to in ((o, ref), (t, tol)):
                to[at:at + r] = y.view(hk, r, G, dh).permute(1, 0, 2, 3).reshape(r, -1)
        at += r
    return ref, tol


MIX = [(40, 5), (33, 3), (70, 2), (1, 1), (31, 31), (32, 0), (33, 32), (0, 4), (64, 1), (65, 64), (127, 65),
       (128, 7), (2, 9), (500, 1), (3, 1), (257, 129), (1000, 16), (16, 17), (15, 1), (1500, 40)]


def check(c, rows, heads, causal, seed, pad=8):
    torch = torch_cuda()
    n, w = sum(rows), heads * c.dh
    q, _ = strided(randn(gen(seed), n, w).bfloat16(), pad)
    out = torch.full((n + 2, w + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    need = attend(c, q, rows, heads, causal, out)
    ref, tol = reference(c, q, rows, heads, causal)
    within(out[:n, :w], ref, tol)
    assert (out[n:] == 7).all() and (out[:, w:] == 7).all()
    return need, out


HEADS = [(16, 1, 1, 32), (32, 12, 12, 64), (16, 6, 2, 32), (64, 8, 1, 128), (128, 9, 3, 64), (256, 4, 2, 128),
         (32, 16, 4, 128), (64, 40, 1, 64), (16, 5, 5, 128), (16, 32, 8, 32)]


@pytest.mark.parametrize("page,heads,hk,dh", HEADS)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(page, heads, hk, dh, causal):
    """All together: the lengths and row counts of MIX, unwritten places NaN."""
    c = Cache([n for n, _ in MIX], page, hk, dh, heads, room=9).fill(page)
    check(c, [r for _, r in MIX], heads, causal, dh)


@pytest.mark.parametrize("page,heads,hk,dh", HEADS)
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 9, 20])
def test_attention_of_steps(page, heads, hk, dh, rows):
    """A few rows for each of several sequences, without offsets."""
    torch = torch_cuda()
    lengths = [1, 90, 0, 17, 64, 33, 500, 2, 130]
    c = Cache(lengths, page, hk, dh, heads + rows).fill(page + 1)
    for causal in (True, False):
        q = randn(gen(rows), rows * len(lengths), heads * dh).bfloat16()
        out = torch.full_like(q, math.nan)
        need = S.surge_cache_attention_workspace(c.desc, rows, heads)
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        S.surge_op_cache_attention(c.desc, len(q), None, rows, heads, causal, dh ** -0.5, q, heads * dh,
                                   ws, out, heads * dh, torch.cuda.current_stream())
        within(out, *reference(c, q, [rows] * len(lengths), heads, causal))


# Keys split over units: ends inside a block and a page, parts of one key.
LONG = [([5000], [1], 64, 4, 4, 64), ([20_011], [1], 16, 32, 8, 128), ([8193, 5], [3, 5], 32, 2, 2, 32),
        ([3001], [40], 64, 2, 1, 64), ([70_001], [1], 128, 1, 1, 128), ([2049, 100], [200, 3], 32, 2, 2, 128),
        ([4097], [150], 16, 8, 2, 64), ([257], [1], 256, 1, 1, 64), ([9000, 3, 0, 40_000, 777], [2, 1, 1, 5, 4], 32, 8, 2, 128),
        ([6000], [700], 64, 4, 1, 128), ([4100, 1030], [33, 5], 64, 8, 1, 128), ([2600], [9], 64, 16, 2, 128)]


@pytest.mark.parametrize("lengths,rows,page,heads,hk,dh", LONG)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_over_long_sequences(lengths, rows, page, heads, hk, dh, causal):
    torch = torch_cuda()
    c = Cache(lengths, page, hk, dh, sum(lengths)).fill(1)
    _, out = check(c, rows, heads, causal, 2)
    again = check(c, rows, heads, causal, 2)[1]
    assert torch.equal(out, again)  # no order of arrival in the result


# Calls whose units are shared out with cuts anywhere, a thread's (sequence, tile)
# pairs one or several, and calls of a unit a workgroup; lengths that differ, some
# sequences without rows or keys.
BATCHES = [(60, 1, 3000, 64, 32, 8, 128), (300, 1, 2500, 32, 4, 1, 64), (700, 2, 1400, 16, 2, 1, 32),
           (40, 7, 2200, 64, 12, 4, 128), (90, 9, 1500, 32, 6, 2, 64), (7, 350, 3000, 64, 8, 4, 128),
           (30, 12, 2600, 64, 16, 4, 64), (400, 1, 2100, 32, 2, 1, 32), (200, 4, 1800, 64, 4, 2, 128), (500, 1, 1300, 128, 8, 8, 32), (6, 260, 2500, 16, 9, 9, 32)]


@pytest.mark.parametrize("seqs,rows,length,page,heads,hk,dh", BATCHES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_batches(seqs, rows, length, page, heads, hk, dh, causal):
    torch = torch_cuda()
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(1, length, seqs)
    lengths[rng.random(seqs) < 0.1] = 0
    lengths[seqs // 2], lengths[-1] = length, 0
    counts = rng.integers(1, rows + 1, seqs)
    counts[rng.random(seqs) < 0.1] = 0
    counts[seqs // 2] = rows
    c = Cache(lengths, page, hk, dh, seqs).fill(2)
    check(c, [int(r) for r in counts], heads, causal, 3)


# Every arrangement of units that are shared out, for each kind of tile and size of
# heads (tests/test_cache_shapes.py states which a call takes): sequences, rows,
# shortest and longest length, page, heads.
SHARED = [
    # 16 and 32 rows: whole units (even lengths), equal shares, equal parts.
    (64, 4, 1200, 1500, 32, 32, 8, 128), (130, 4, 1200, 1500, 64, 16, 4, 64), (150, 8, 1200, 1500, 16, 6, 3, 32),
    (64, 8, 1250, 1500, 32, 32, 8, 128), (130, 7, 1250, 1500, 64, 16, 4, 64), (400, 10, 1250, 1500, 128, 6, 2, 32),
    (50, 3, 0, 4000, 16, 20, 4, 128), (70, 16, 0, 3000, 64, 4, 4, 64), (45, 5, 0, 3500, 32, 33, 11, 32),
    (40, 20, 0, 3100, 32, 4, 4, 128), (60, 9, 0, 2500, 64, 12, 4, 64), (50, 16, 0, 2700, 16, 16, 8, 32),
    (6, 1, 0, 3001, 16, 16, 2, 64), (6, 31, 0, 3001, 64, 2, 2, 128), (9, 17, 0, 2500, 16, 6, 6, 32),
    # 64 and 128 rows: equal shares, several units a workgroup; equal parts.
    (64, 16, 0, 2300, 64, 16, 4, 128), (20, 60, 0, 2400, 32, 16, 16, 64), (30, 30, 0, 2500, 16, 24, 12, 32),
    (5, 50, 0, 2300, 64, 4, 4, 128), (7, 16, 0, 2200, 64, 12, 3, 64), (6, 64, 0, 2100, 32, 4, 4, 32),
    (20, 70, 0, 2300, 64, 16, 8, 128), (9, 300, 0, 2400, 32, 16, 8, 64), (16, 200, 0, 2500, 16, 9, 9, 32),
    # Threads whose (sequence, tile) pairs begin inside a sequence.
    (5, 1000, 1000, 2600, 64, 8, 1, 128), (9, 900, 0, 2500, 32, 4, 1, 64), (3, 2000, 2000, 2700, 32, 6, 1, 32),
]


def shared_call(seqs, rows, shortest, length):
    """Lengths and rows of a call of SHARED: some sequences without keys, some
    without rows, the longest in the middle with the most rows."""
    rng = np.random.default_rng(seqs * rows)
    lengths = rng.integers(shortest, length + 1, seqs)
    lengths[rng.random(seqs) < 0.1] = 0
    counts = rng.integers(max(rows // 2, 1), rows + 1, seqs)
    counts[rng.random(seqs) < 0.1] = 0
    lengths[seqs // 2], counts[seqs // 2] = length, rows
    return lengths, [int(r) for r in counts]


@pytest.mark.parametrize("seqs,rows,shortest,length,page,heads,hk,dh", SHARED)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_shared_units(seqs, rows, shortest, length, page, heads, hk, dh, causal):
    torch = torch_cuda()
    lengths, counts = shared_call(seqs, rows, shortest, length)
    c = Cache(lengths, page, hk, dh, seqs).fill(2)
    need, out = check(c, counts, heads, causal, 3)
    assert need > 0
    assert torch.equal(out, check(c, counts, heads, causal, 3)[1])


# One long sequence, the last, among very many short ones: a wave has a unit up to 1024
# keys, a workgroup beyond.
TAILS = [(800, 1, 1024, 16, 16, 8, 128), (800, 1, 1025, 16, 16, 8, 128), (800, 3, 9001, 64, 16, 8, 128),
         (700, 1, 1024, 32, 12, 12, 64), (700, 16, 5003, 32, 12, 12, 64), (1200, 2, 1000, 16, 24, 12, 32),
         (1200, 1, 20_011, 128, 12, 12, 32), (900, 8, 1024, 16, 32, 8, 128), (900, 7, 3001, 64, 32, 8, 128)]


@pytest.mark.parametrize("seqs,rows,longest,page,heads,hk,dh", TAILS)
def test_attention_of_one_long_sequence_among_many(seqs, rows, longest, page, heads, hk, dh):
    lengths = np.random.default_rng(seqs + rows).integers(0, 70, seqs)
    lengths[-1] = longest
    c = Cache(lengths, page, hk, dh, seqs).fill(2)
    check(c, [rows] * seqs, heads, True, 3)


def test_attention_of_prompts_without_a_cache_before():
    """Rows for every position of sequences, one tile and more."""
    lengths = [130, 64, 1, 257, 640]
    c = Cache(lengths, 16, 2, 64, 1).fill(3)
    check(c, lengths, 4, True, 4)


def test_attention_leaves_rows_beyond_max_rows():
    torch = torch_cuda()
    c = Cache([50, 40], 16, 2, 64, 1).fill(3)
    q = randn(gen(1), 12, 128).bfloat16()
    full, out = (torch.full((12, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    attend(c, q, [9, 3], 2, True, full)
    attend(c, q, [9, 3], 2, True, out, max_rows=4)  # 4 rows of 2 heads' groups are in one tile of 16
    assert torch.equal(out[:4], full[:4]) and torch.equal(out[9:], full[9:])
    assert (out[4:9] == 7).all()


SHAPES = [([50], [1], 4, 2, 64), ([130, 40], [3, 1], 2, 2, 32), ([77], [9], 8, 2, 128), ([300], [50], 2, 2, 64),
          ([90], [33], 2, 1, 128), ([300], [70], 4, 4, 32), ([9000], [1], 4, 2, 64), ([20_011], [1], 32, 8, 128),
          ([3001], [40], 2, 2, 64), ([2049], [200], 2, 2, 128)]


def agrees(got, ref, tol):
    torch = torch_cuda()
    bad = ref.isnan()
    assert torch.equal(got.isnan(), bad), (int(got.isnan().sum()), int(bad.sum()))
    if not bad.all():
        within(got[~bad], ref[~bad], tol[~bad])


@pytest.mark.parametrize("lengths,rows,heads,hk,dh", SHAPES)
@pytest.mark.parametrize("which", ["k", "v"])
def test_attention_of_marked_keys(lengths, rows, heads, hk, dh, which):
    """A key or value marked NaN at the last position of a sequence, in one key
    head: the last row of that head's group is NaN, and none before it."""
    torch = torch_cuda()
    c = Cache(lengths, 16, hk, dh, 1).fill(5)
    q = randn(gen(6), sum(rows), heads * dh).bfloat16()
    ref, tol = reference(c, q, rows, heads, True)
    n, G = lengths[0], heads // hk
    f = c.fields()
    f["kv".index(which) + 2][c.table_np[0, (n - 1) // 16], hk - 1, (n - 1) % 16, dh // 32 - 1] = 255
    ref[rows[0] - 1, (hk - 1) * G * dh:] = math.nan
    out = torch.full_like(q, 7.0)
    attend(c, q, rows, heads, True, out)
    agrees(out, ref, tol)
    attend(c, q, rows, heads, False, out)
    nan = out.isnan()
    assert nan[:rows[0], (hk - 1) * G * dh:].all() and int(nan.sum()) == rows[0] * G * dh


# Many units, of a few rows each and short, or so many that each is a wave's.
MANY = [(500, 1, 100, 16, 4, 4, 32), (400, 6, 128, 32, 16, 4, 32), (300, 1, 90, 16, 8, 4, 64), (300, 7, 60, 64, 12, 3, 64),
        (200, 1, 33, 16, 32, 8, 128), (150, 5, 128, 32, 16, 4, 128), (800, 1, 230, 32, 8, 8, 128),
        (520, 17, 300, 16, 8, 8, 128), (400, 50, 64, 16, 4, 4, 64), (150, 90, 96, 16, 2, 2, 128), (60, 148, 90, 32, 2, 2, 128),
        (300, 20, 70, 32, 12, 3, 32)]


@pytest.mark.parametrize("seqs,rows,length,page,heads,hk,dh", MANY)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_many_units(seqs, rows, length, page, heads, hk, dh, causal):
    """And with a page that is missing, which some rows of one sequence see."""
    torch = torch_cuda()
    rng = np.random.default_rng(seqs + rows)
    lengths = rng.integers(0, length, seqs)
    lengths[seqs // 2] = length
    counts = rng.integers(0, rows + 1, seqs)
    counts[seqs // 2] = rows
    counts = [int(r) for r in counts]
    c = Cache(lengths, page, hk, dh, seqs).fill(2)
    n, w = sum(counts), heads * dh
    q, _ = strided(randn(gen(3), n, w).bfloat16(), 8)
    ref, tol = reference(c, q, counts, heads, causal)
    out = torch.full((n + 2, w + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    assert attend(c, q, counts, heads, causal, out) == 0  # not shared out
    within(out[:n, :w], ref, tol)
    assert (out[n:] == 7).all() and (out[:, w:] == 7).all()
    i, entry = seqs // 2, (length - 1) // page
    c.table[i, entry] = -1
    at = sum(counts[:i])
    sees = [at + j for j in range(rows) if not causal or length - rows + j >= entry * page]
    ref[sees] = math.nan
    attend(c, q, counts, heads, causal, out)
    agrees(out[:n, :w], ref, tol)


@pytest.mark.parametrize("lengths,rows,heads,hk,dh", SHAPES)
def test_attention_of_missing_pages_and_nan_queries(lengths, rows, heads, hk, dh):
    torch = torch_cuda()
    c = Cache(lengths, 16, hk, dh, 1).fill(5)
    q = randn(gen(6), sum(rows), heads * dh).bfloat16()
    out = torch.full_like(q, 7.0)
    ref, tol = reference(c, q, rows, heads, True)
    q[0, 5] = math.nan
    ref[0, :dh] = math.nan
    attend(c, q, rows, heads, True, out)
    agrees(out, ref, tol)
    entry = (lengths[0] - 1) // 16
    c.table[0, entry] = c.n_pages
    first = lengths[0] - rows[0]
    sees = [j for j in range(rows[0]) if first + j >= entry * 16]
    ref[sees] = math.nan
    attend(c, q, rows, heads, True, out)
    agrees(out, ref, tol)


@pytest.mark.parametrize("lengths,rows,heads,hk,dh", SHAPES)
def test_attention_of_scores_past_the_largest_float(lengths, rows, heads, hk, dh):
    """A row whose scores are all -inf, and one whose largest is +inf: NaN."""
    torch = torch_cuda()
    c = Cache(lengths, 16, hk, dh, 1)
    for i, n in enumerate(lengths):
        k = torch.full((n, hk * dh), 2.0 ** 120, device="cuda").bfloat16()
        c.put(i, np.arange(n), k, torch.ones_like(k))
    for sign in (1, -1):
        q = torch.full((sum(rows), heads * dh), sign * 2.0 ** 100, device="cuda").bfloat16()
        q[-1] = 0
        out = torch.full_like(q, 7.0)
        attend(c, q, rows, heads, True, out)
        assert out[:-1].isnan().all()
        assert (out[-1] == 1).all()  # every score 0: the mean of the values


@pytest.mark.parametrize("up", [True, False])
def test_attention_of_scores_that_rise_and_fall(up):
    """Scores that grow or fall by hundreds along the keys: the running maximum
    moves in every block, or all but the first keys vanish."""
    torch = torch_cuda()
    n, dh = 3000, 64
    c = Cache([n], 32, 1, dh, 1)
    ramp = torch.linspace(-400 if up else 400, 400 if up else -400, n, device="cuda")
    k = torch.zeros(n, dh, device="cuda")
    k[:, 0] = ramp
    v = randn(gen(1), n, dh).bfloat16()
    c.put(0, np.arange(n), k.bfloat16(), v)
    c.held = [[values(*quantized(x)).view(n, 1, dh) for x in (k.bfloat16(), v)]]
    q = torch.zeros(20, dh, device="cuda")
    q[:, 0] = torch.linspace(0.1, 30, 20, device="cuda")
    q = q.bfloat16()
    out = torch.empty_like(q)
    attend(c, q, [20], 1, True, out)
    within(out, *reference(c, q, [20], 1, True))


def test_pages_past_32_bits():
    """Pages whose addresses pass 2^32 bytes."""
    torch = torch_cuda()
    page, hk, dh = 256, 8, 128
    size = S.surge_cache_page_bytes(page, hk, dh)
    n_pages = (1 << 32) // size + 40
    pages = torch.full((n_pages, size), 255, dtype=torch.uint8, device="cuda")
    c = Cache([700, 300], page, hk, dh, 1)
    far = n_pages - 1 - np.arange(5)
    c.table_np[0, :3], c.table_np[1, :2] = far[:3], [0, far[4]]
    c.pages, c.n_pages = pages, n_pages
    c.table = dev(c.table_np)
    c.desc = S.KVCache(pages, n_pages, page, hk, dh, c.table, c.width, 2, c.lengths, 700)
    g = gen(1)
    k, v = (randn(g, 1000, hk * dh).bfloat16() for _ in range(2))
    cu = dev([0, 700, 1000])
    S.surge_op_cache_write(c.desc, 1000, cu, k, hk * dh, v, hk * dh)
    out = [torch.empty_like(k) for _ in range(2)]
    S.surge_op_cache_read(c.desc, 1000, cu, out[0], hk * dh, out[1], hk * dh)
    assert torch.equal(out[0].double(), values(*quantized(k)))
    assert torch.equal(out[1].double(), values(*quantized(v)))
    held = [values(*quantized(x)).view(1000, hk, dh) for x in (k, v)]
    c.held = [[x[:700] for x in held], [x[700:] for x in held]]
    for rows in ([2, 1], [100, 80]):
        check(c, rows, 16, True, 3)


def test_refused_workspaces():
    torch = torch_cuda()
    c = Cache([9000], 64, 2, 64, 1).fill(1)
    q = randn(gen(1), 1, 128).bfloat16()
    out = torch.full_like(q, 7.0)
    need = S.surge_cache_attention_workspace(c.desc, 1, 2)
    assert need > 0
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    for bad in (None, ws[:need - 1], ws[8:]):
        with pytest.raises(S.SurgeError) as e:
            S.surge_op_cache_attention(c.desc, 1, None, 1, 2, True, 0.125, q, 128, bad, out, 128)
        assert e.value.status in (S.SURGE_ERR_INVALID_ARGUMENT, S.SURGE_ERR_CAPACITY)
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_attention_on_two_streams():
    """One cache, two streams, a workspace each."""
    torch = torch_cuda()
    c = Cache([9000, 12_000], 64, 2, 128, 5).fill(1)
    q = [randn(gen(i), 3, 1024).bfloat16() for i in (1, 2)]
    want = [torch.empty_like(x) for x in q]
    for x, o in zip(q, want):
        need = attend(c, x, [1, 2], 8, True, o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty_like(o) for o in want]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cu = cu_of([1, 2])
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, s, w in zip(q, got, streams, spaces):
            attend(c, x, [1, 2], 8, True, o, w, s, cu)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---------------------------------------------------------------------------
# Drafts
# ---------------------------------------------------------------------------

def verified(p, q, drafts, counts, u):
    """Tokens and counts by the definition, in 64 bits on the host."""
    p = p.double().cpu().numpy()
    q = None if q is None else q.double().cpu().numpy()
    x, u = drafts.cpu().numpy(), u.double().cpu().numpy()
    n, k1, vocab = p.shape
    tokens, accepted = np.full((n, k1), -1, np.int32), np.zeros(n, np.int32)
    for i in range(n):
        c = min(max(int(counts[i]), 0), k1 - 1)
        a = 0
        while a < c and 0 <= x[i, a] < vocab and \
                u[i, a] * (1.0 if q is None else q[i, a, x[i, a]]) < p[i, a, x[i, a]]:
            tokens[i, a] = x[i, a]
            a += 1
        accepted[i] = a
        target = np.where(p[i, a] > 0, p[i, a], 0.0)
        r = target
        if a < c:
            if q is not None:
                with np.errstate(invalid="ignore"):
                    d = p[i, a] - q[i, a]
                r = np.where(d > 0, d, 0.0)
            elif 0 <= x[i, a] < vocab:
                r = target.copy()
                r[x[i, a]] = 0
            if not r.sum() > 0:
                r = target
        total = r.sum()
        if total > 0 and np.isfinite(total):
            over = np.flatnonzero((np.cumsum(r) > u[i, -1] * total) & (r > 0))
            tokens[i, a] = over[0] if len(over) else np.flatnonzero(r > 0)[-1]
    return tokens, accepted


def verify(p, q, drafts, counts, u, n_drafts="given", pad=0, stream=None):
    torch = torch_cuda()
    n, k1, vocab = p.shape
    if pad:
        p = torch.nn.functional.pad(p, (0, pad), value=1e30)
        q = None if q is None else torch.nn.functional.pad(q, (0, pad), value=-1e30)
    tokens = torch.full((n, k1), 77, dtype=torch.int32, device="cuda")
    accepted = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    need = S.surge_verify_workspace(n, vocab)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    S.surge_op_verify_drafts(n, k1 - 1, vocab, None if n_drafts is None else dev(counts), drafts, p,
                             vocab + pad, q, vocab + pad, u, ws, tokens, accepted,
                             stream or torch.cuda.current_stream())
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def draft_inputs(n, k, vocab, seed, sharp=3.0, near=1.0):
    torch = torch_cuda()
    g = gen(seed)
    logits = sharp * randn(g, n, k + 1, vocab)
    p = torch.softmax(logits, 2)
    q = torch.softmax(logits[:, :k] + near * randn(g, n, k, vocab), 2)
    noise = torch.rand(n, k, vocab, generator=g, device="cuda").clamp_min(1e-30)
    drafts = (q / -torch.log(noise)).argmax(2).int() if k else torch.zeros(n, 0, dtype=torch.int32, device="cuda")
    return p, q, drafts, torch.rand(n, k + 1, generator=g, device="cuda")


VERIFY = [(1, 1, 1), (3, 2, 2), (5, 4, 63), (40, 3, 100), (9, 7, 1000), (2, 4, 4095), (2, 4, 4096), (3, 4, 4097),
          (64, 4, 30_522), (1, 4, 30_522), (300, 1, 257), (5, 70, 500), (4, 6, 100_003), (1, 2, 262_145),
          (600, 2, 5000), (3, 0, 777), (2, 130, 64), (1, 1, 1 << 22)]


@pytest.mark.parametrize("n,k,vocab", VERIFY)
@pytest.mark.parametrize("probs", [True, False])
def test_verify_drafts(n, k, vocab, probs):
    p, q, drafts, u = draft_inputs(n, k, vocab, n + k + vocab)
    if not k:
        probs = False
    counts = np.random.default_rng(n).integers(-1, k + 2, n)
    counts[0] = k
    for c, given in ((counts, "given"), (np.full(n, k), None)):
        want = verified(p, q if probs else None, drafts, c, u)
        got = verify(p, q if probs else None, drafts, c, u, given, pad=5 if n % 2 else 0)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_verify_draws_from_the_target():
    """Drafts drawn from q and u even: the first token has the target's
    distribution (mean of 40,000 draws, five standard deviations)."""
    torch = torch_cuda()
    n, vocab = 40_000, 12
    p, q, _, _ = draft_inputs(1, 1, vocab, 3, sharp=1.0, near=1.5)
    g = gen(9)
    drafts = torch.multinomial(q[0, 0].expand(n, vocab), 1, generator=g).int()
    u = torch.rand(n, 2, generator=g, device="cuda")
    tokens, _ = verify(p.expand(n, 2, vocab).contiguous(), q.expand(n, 1, vocab).contiguous(), drafts,
                       np.ones(n), u)
    share = np.bincount(tokens[:, 0], minlength=vocab) / n
    want = p[0, 0].double().cpu().numpy()
    assert (np.abs(share - want) <= 5 * np.sqrt(want * (1 - want) / n) + 1e-9).all()


def test_verify_at_the_edges():
    """Drafts outside the vocabulary, rows that are not finite or nothing, q that
    leaves nothing over, u at 0, next to 1 and beyond."""
    torch = torch_cuda()
    n, k, vocab = 14, 2, 5000
    p, q, drafts, u = draft_inputs(n, k, vocab, 1)
    drafts[0, 0], drafts[1, 0], drafts[2, 1] = -1, vocab, 1 << 30
    p[3] = 0                       # nothing to draw: -1
    p[4, 0, 7] = math.inf          # infinite: -1
    drafts[4, 0] = 3
    u[4, 0] = 0.999999
    p[5, :, ::2] = math.nan        # counts as 0
    p[6, 0] = q[6, 0]              # rejected by u beyond 1, nothing left over: the target's own
    u[6, 0] = 2.0
    u[7] = 0.0
    u[8] = 1 - 2.0 ** -24
    u[9, k] = 1.0                  # beyond every sum: the last token that weighs anything
    p[9, :, vocab - 900:] = 0
    u[10] = math.nan
    q[11] = math.nan
    p[12, :, :4500] = 0            # the first tokens weigh nothing, u 0
    u[12, k] = 0.0
    p[13] = -p[13]
    counts = np.full(n, k)
    for x in (q, None):
        want = verified(p, x, drafts, counts, u)
        got = verify(p, x, drafts, counts, u)
        assert np.array_equal(got[0], want[0]), (got[0], want[0])
        assert np.array_equal(got[1], want[1])
    assert got[0][3, 0] == -1 and got[0][13, 0] == -1


@pytest.mark.parametrize("vocab,pad", [(5000, 0), (40_001, 3), (100_003, 0), (300_007, 1)])
def test_verify_at_the_edges_of_large_vocabularies(vocab, pad):
    """One launch and two, more tiles than a wave has lanes: what leaves nothing
    over, is not finite or nothing at all, tokens in the first and last tile."""
    torch = torch_cuda()
    n, k = 18, 2
    p, q, drafts, u = draft_inputs(n, k, vocab, 1)
    drafts[0, 0], drafts[1, 0], drafts[2, 1] = -1, vocab, 1 << 30
    p[3] = 0                                     # nothing to draw: -1
    p[4, 0, vocab - 7] = math.inf                # infinite: -1
    drafts[4, 0], u[4, 0] = 3, 0.999999
    p[5, :, ::2] = math.nan                      # counts as 0
    p[6, 0], u[6, 0] = q[6, 0], 2.0              # nothing left over: the target's own
    u[7] = 0.0
    u[8] = 1 - 2.0 ** -24
    p[9, :, vocab - 900:], u[9, k] = 0, 2.0      # beyond every sum: the last that weighs anything
    u[10] = math.nan
    q[11] = math.nan
    p[12, :, :4500], u[12, k] = 0, 0.0           # the first tokens weigh nothing
    p[13] = -p[13]
    p[14, 0], drafts[14, 0], u[14, 0] = 0, vocab - 1, 2.0
    p[14, 0, vocab - 1] = 1                      # a draft with all of the target's mass, rejected
    q[14, 0] = p[14, 0]
    p[15, 0], u[15, 0] = q[15, 0], 2.0
    p[15, 0, vocab // 2] += 2.0 ** -10           # one token left over
    q[16], u[16] = 1.0, 0.999                    # less than q everywhere
    p[17, 0], p[17, 0, 5], u[17, 0] = 0, math.inf, 2.0
    q[17, 0], drafts[17, 0] = math.inf, 5        # inf - inf: the target's own, infinite: -1
    counts = np.full(n, k)
    for x in (q, None):
        want = verified(p, x, drafts, counts, u)
        got = verify(p, x, drafts, counts, u, pad=pad)
        assert np.array_equal(got[0], want[0]), (got[0], want[0])
        assert np.array_equal(got[1], want[1])
        assert (got[0][[3, 13], 0] == -1).all() and got[0][14, 0] == vocab - 1
        again = verify(p, x, drafts, counts, u, pad=pad)
        assert np.array_equal(got[0], again[0])
    assert verified(p, q, drafts, counts, u)[0][15, 0] == vocab // 2


def test_verify_takes_the_token_on_either_side_of_a_border():
    """Sums that are exact: u at a border takes the next token."""
    torch = torch_cuda()
    vocab = 1 << 14
    u = torch.tensor([[0.0], [0.25], [0.5], [0.5 - 2.0 ** -25], [1 - 2.0 ** -24], [3 * 2.0 ** -14]], device="cuda")
    p = torch.full((len(u), 1, vocab), 1.0 / vocab, device="cuda")
    none = torch.zeros(len(u), 0, dtype=torch.int32, device="cuda")
    got, _ = verify(p, None, none, np.zeros(len(u)), u)
    assert got[:, 0].tolist() == [0, vocab // 4, vocab // 2, vocab // 2 - 1, vocab - 1, 3]


# ---------------------------------------------------------------------------
# Far ends of what may be asked for
# ---------------------------------------------------------------------------

def test_rows_whose_offsets_pass_32_bits():
    """Five column ranges of one matrix of the widest rows: written, read, attended."""
    torch = torch_cuda()
    n, ld, w = 1100, 1 << 22, 128
    big = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda").view(n, ld)
    k, v, q, out, back = (big[:, i * 256:i * 256 + w] for i in range(5))
    g = gen(1)
    for x in (k, v, q):
        x.copy_(randn(g, n, w).bfloat16())
    c = Cache([1200, 30], 32, 2, 64, 3, fill=0)
    rows, cu = [1080, 20], dev([0, 1080, 1100])
    c.fill(5)
    seq, pos = places(c.lengths_np, rows)
    S.surge_op_cache_write(c.desc, n, cu, k, ld, v, ld)
    S.surge_op_cache_read(c.desc, n, cu, out, ld, back, ld)
    assert torch.equal(out.double(), values(*quantized(k)))
    assert torch.equal(back.double(), values(*quantized(v)))
    for i, (first, size) in enumerate(((0, 1080), (1080, 20))):
        for t, x in enumerate((k, v)):
            c.held[i][t][-size:] = values(*quantized(x[first:first + size])).view(size, 2, 64)
    for wide in (rows, [1, 20]):
        m = sum(wide)
        at = big[n - m:]
        q, out = at[:, 512:512 + w], at[:, 768:768 + w]
        attend(c, q, wide, 2, True, out)
        within(out, *reference(c, q.contiguous(), wide, 2, True))


def test_verify_rows_whose_offsets_pass_32_bits():
    torch = torch_cuda()
    n, k, ld = 2, 1, 1 << 30
    for vocab in (100, 40_000):  # one launch and two
        p, q, drafts, u = draft_inputs(n, k, vocab, vocab)
        far = torch.empty(((k + 1) * n - 1) * ld + vocab, device="cuda")
        far_p = far.as_strided((n, k + 1, vocab), ((k + 1) * ld, ld, 1))
        far_p.copy_(p)
        far_q = far.as_strided((n, k, vocab), (k * ld, ld, 1), 1 << 29)
        far_q.copy_(q)
        for probs in (far_q, None):
            for u0 in (0.0, 1.0):  # accepted, rejected
                u[:, 0] = u0
                want = verified(p, None if probs is None else q, drafts, [k] * n, u)
                tokens = torch.empty(n, k + 1, dtype=torch.int32, device="cuda")
                accepted = torch.empty(n, dtype=torch.int32, device="cuda")
                ws = torch.empty(max(16, S.surge_verify_workspace(n, vocab)), dtype=torch.uint8, device="cuda")
                S.surge_op_verify_drafts(n, k, vocab, None, drafts, far_p, ld, probs, ld, u, ws, tokens, accepted)
                assert np.array_equal(tokens.cpu().numpy(), want[0])
                assert np.array_equal(accepted.cpu().numpy(), want[1])


def test_attention_of_a_hundred_thousand_sequences():
    """Of length 0, zeros, or 1: the value itself, whatever the score."""
    torch = torch_cuda()
    n, hk, dh = 100_003, 2, 32
    lengths = np.random.default_rng(1).integers(0, 2, n)
    c = Cache(lengths, 16, hk, dh, 1)
    g = gen(1)
    k, v, q = (randn(g, n, w).bfloat16() for w in (hk * dh, hk * dh, 2 * hk * dh))
    S.surge_op_cache_write(c.desc, n, None, k, hk * dh, v, hk * dh)
    out = torch.empty_like(q)
    attend(c, q, [1] * n, 2 * hk, True, out)
    held = values(*quantized(v)) * torch.from_numpy(lengths).cuda()[:, None]
    assert torch.equal(out.double().view(n, hk, 2, dh), held.view(n, hk, 1, dh).expand(n, hk, 2, dh))


def test_attention_of_a_million_sequences():
    """2^20 sequences of 8 key heads, as many as a call takes: a wave each."""
    torch = torch_cuda()
    n, hk, dh = 1 << 20, 8, 32
    lengths = np.random.default_rng(1).integers(0, 2, n)
    c = Cache(lengths, 16, hk, dh, 1)
    g = gen(1)
    k, v, q = (torch.randn(n, hk * dh, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    S.surge_op_cache_write(c.desc, n, None, k, hk * dh, v, hk * dh)
    out = torch.empty_like(q)
    attend(c, q, [1] * n, hk, True, out)
    on = torch.from_numpy(lengths).cuda()
    for i in range(0, n, 1 << 17):
        at = slice(i, i + (1 << 17))
        assert torch.equal(out[at].double(), values(*quantized(v[at])) * on[at, None])


@pytest.mark.parametrize("n,hk", [((1 << 27) + 1024, 4), (1 << 29, 1)])
def test_rows_that_need_a_launch_of_the_largest_size(n, hk):
    """More than 2^29 rows times key heads, a wave's four heads together, and 2^29
    rows of one: rows of negative positions but for the last ones."""
    torch = torch_cuda()
    dh, m = 32, 40
    w = hk * dh
    x = torch.empty(n, 2 * w, dtype=torch.bfloat16, device="cuda")
    last = randn(gen(1), m, 2 * w).bfloat16()
    x[-m:] = last
    c = Cache([m], 16, hk, dh, 1, fill=0xAB)
    want = c.pages.clone()
    c.put(0, np.arange(m), last[:, :w], last[:, w:], want)
    S.surge_op_cache_write(c.desc, n, None, x, 2 * w, x[:, w:], 2 * w)
    assert torch.equal(c.pages, want)
    x[::1 << 20] = 7.0
    S.surge_op_cache_read(c.desc, n, None, x, 2 * w, x[:, w:], 2 * w)
    assert torch.equal(x[-m:].double(), values(*quantized(last)))
    assert not x[:-m].view(torch.int16)[::1 << 10].any() and not x[:-m][::1 << 20].any()


@pytest.mark.parametrize("rows", [[2, 3], [60, 70]])
def test_attention_with_pages_shared_by_sequences(rows):
    """Two sequences that begin alike, with the same pages."""
    c = Cache([700, 900], 64, 2, 64, 1)
    c.table_np[1, :9] = c.table_np[0, :9]
    c.table.copy_(dev(c.table_np))
    c.fill(3)
    for w in range(2):
        c.held[0][w][:9 * 64] = c.held[1][w][:9 * 64]  # written last
    check(c, rows, 8, True, 4)


@pytest.mark.parametrize("rows", [[1, 1, 2], [40, 40, 40], [100, 3, 100]])
def test_attention_of_lengths_out_of_range(rows):
    """Below 0 is 0, beyond max_length is max_length."""
    torch = torch_cuda()
    c = Cache([0, 5000, 100], 16, 2, 64, 1).fill(2)
    c.lengths.copy_(dev([-5, (1 << 31) - 1, 100]))
    check(c, rows, 2, True, 4)
    check(c, rows, 2, False, 4)


def test_attention_over_caches_of_no_length():
    """max_length 0: a table without entries, every row zeros."""
    torch = torch_cuda()
    pages = torch.zeros(1, S.surge_cache_page_bytes(16, 2, 64), dtype=torch.uint8, device="cuda")
    c = S.KVCache(pages, 1, 16, 2, 64, dev([0]), 0, 3, dev([0, 7, -1]), 0)
    for rows in (1, 200):
        assert S.surge_cache_attention_workspace(c, rows, 4) == 0
        q = randn(gen(1), 3 * rows, 256).bfloat16()
        out = torch.full_like(q, 7.0)
        S.surge_op_cache_attention(c, 3 * rows, None, rows, 4, True, 0.125, q, 256, None, out, 256)
        assert (out == 0).all()
        S.surge_op_cache_write(c, 3 * rows, None, q, 256, q[:, 128:], 256)
        back = torch.full_like(q, 7.0)
        S.surge_op_cache_read(c, 3 * rows, None, back, 256, back[:, 128:], 256)
        assert (back == 0).all() and (pages == 0).all()


# ---------------------------------------------------------------------------
# The operators together: a step of a decoder
# ---------------------------------------------------------------------------

class Decoder:
    """Steps of a batch of answers: the drafts' and the last token's keys and
    values go into the cache, their queries attend, the logits of the attended
    rows are the target's, the drafts are checked, and the lengths go back to
    what was accepted."""

    def __init__(self, lengths, drafts, page, heads, hk, dh, vocab, seed):
        torch = torch_cuda()
        self.n, self.k, self.heads, self.vocab = len(lengths), drafts, heads, vocab
        rows = self.n * (drafts + 1)
        self.c = c = Cache(lengths, page, hk, dh, seed, room=64).fill(seed)
        g = gen(seed)
        self.head = randn(g, heads * dh, vocab) / math.sqrt(heads * dh)
        self.x = randn(g, rows, (heads + 2 * hk) * dh).bfloat16()  # Q | K | V of the step's rows
        self.q_probs = torch.softmax(randn(g, self.n, drafts, vocab), 2)
        self.drafts = torch.randint(0, vocab, (self.n, drafts), generator=g, device="cuda", dtype=torch.int32)
        self.u = torch.rand(self.n, drafts + 1, generator=g, device="cuda")
        self.out = torch.empty(rows, heads * dh, dtype=torch.bfloat16, device="cuda")
        self.p = torch.empty(self.n, drafts + 1, vocab, device="cuda")
        self.tokens = torch.empty(self.n, drafts + 1, dtype=torch.int32, device="cuda")
        self.accepted = torch.empty(self.n, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(max(16, S.surge_cache_attention_workspace(c.desc, drafts + 1, heads)),
                              dtype=torch.uint8, device="cuda")
        self.vws = torch.empty(max(16, S.surge_verify_workspace(self.n, vocab)), dtype=torch.uint8, device="cuda")

    def step(self, stream):
        torch = torch_cuda()
        c, m = self.c, self.k + 1
        rows, ld, qd = self.n * m, self.x.shape[1], self.heads * self.c.dh
        kd = c.hk * c.dh
        c.lengths.add_(m)
        S.surge_op_cache_write(c.desc, rows, None, self.x[:, qd:], ld, self.x[:, qd + kd:], ld, stream)
        S.surge_op_cache_attention(c.desc, rows, None, m, self.heads, True, c.dh ** -0.5, self.x, ld, self.ws,
                                   self.out, qd, stream)
        torch.softmax((self.out.float() @ self.head).view(self.n, m, -1), 2, out=self.p)
        S.surge_op_verify_drafts(self.n, self.k, self.vocab, None, self.drafts, self.p, self.vocab,
                                 self.q_probs, self.vocab, self.u, self.vws, self.tokens, self.accepted, stream)
        c.lengths.sub_(self.k - self.accepted)


def test_decoder_steps():
    """Each step against the definitions, positions overwritten after rejections."""
    torch = torch_cuda()
    d = Decoder([90, 1, 33, 0, 700, 3000], 3, 16, 8, 2, 64, 500, 1)
    c, g = d.c, gen(2)
    for _ in range(5):
        d.x.copy_(randn(g, *d.x.shape))
        d.u.copy_(torch.rand(d.u.shape, generator=g, device="cuda"))
        before = c.lengths.cpu().numpy().astype(np.int64)
        d.step(torch.cuda.current_stream())
        qd, kd, m = d.heads * c.dh, c.hk * c.dh, d.k + 1
        for i in range(d.n):
            for w in range(2):
                new = d.x[i * m:(i + 1) * m, qd + w * kd:qd + (w + 1) * kd]
                c.held[i][w] = torch.cat([c.held[i][w][:before[i]], values(*quantized(new)).view(m, c.hk, c.dh)])
        c.lengths_np = before + m
        within(d.out, *reference(c, d.x[:, :qd], [m] * d.n, d.heads, True))
        want = verified(d.p, d.q_probs, d.drafts, np.full(d.n, d.k), d.u)
        assert np.array_equal(d.tokens.cpu().numpy(), want[0]) and np.array_equal(d.accepted.cpu().numpy(), want[1])
        assert np.array_equal(c.lengths.cpu().numpy(), before + 1 + want[1])


def test_decoder_steps_captured_and_replayed():
    """Two decoders in a graph each, replayed as their answers grow, with new
    inputs, eager work and synchronisations between: the eager step's bits."""
    torch = torch_cuda()
    make = [lambda: Decoder([90, 1, 33, 0, 700, 5000], 3, 16, 8, 2, 64, 500, 1),
            lambda: Decoder([2000] * 3, 0, 32, 32, 8, 128, 3001, 2)]
    eager, replayed = [f() for f in make], [f() for f in make]
    stream = torch.cuda.Stream()
    graphs = []
    for d in replayed:
        start = d.c.lengths.clone()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):  # once before, for what torch's own product sets up
            d.step(stream)
        torch.cuda.synchronize()
        d.c.lengths.copy_(start)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            d.step(torch.cuda.current_stream())
        graphs.append(graph)
    g = gen(3)
    for step in range(6):
        for d, r in zip(eager, replayed):
            d.x.copy_(randn(g, *d.x.shape))
            d.u.copy_(torch.rand(d.u.shape, generator=g, device="cuda"))
            r.x.copy_(d.x)
            r.u.copy_(d.u)
        for d, r, graph in zip(eager, replayed, graphs):
            graph.replay()
            if step % 2:
                torch.cuda.synchronize()
            d.step(torch.cuda.current_stream())
        for d, r in zip(eager, replayed):
            assert torch.equal(d.out, r.out) and torch.equal(d.tokens, r.tokens)
            assert torch.equal(d.accepted, r.accepted) and torch.equal(d.c.lengths, r.c.lengths)
    for r, graph in zip(replayed, graphs):  # both at the same time, on a stream each
        r.start = r.c.lengths.clone()
        graph.replay()
        torch.cuda.synchronize()
        r.want = r.out.clone()
        r.c.lengths.copy_(r.start)
    streams = [torch.cuda.Stream() for _ in replayed]
    torch.cuda.synchronize()
    for graph, s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for r in replayed:
        assert torch.equal(r.out, r.want)


class Block:
    """A decoder's block of the library's operators alone: n = RMS(x) in int8;
    Q | K | V = n W in one matrix; K and V's columns to the cache; A = attention of
    Q's columns; y = x + A Wo."""

    def __init__(self, lengths, d, page, heads, hk, dh, seed):
        torch = torch_cuda()
        self.d, self.heads, self.c = d, heads, Cache(lengths, page, hk, dh, seed, room=200).fill(seed)
        g, self.wide = gen(seed), (heads + 2 * hk) * dh
        self.w, self.ws, self.bias = {}, {}, {}
        for name, n, k in (("qkv", self.wide, d), ("o", d, heads * dh)):
            q, s = quantized32(randn(g, n, k) / math.sqrt(k))
            self.w[name], self.ws[name], self.bias[name] = q.cuda(), s.contiguous().cuda(), 0.1 * randn(g, n)
        self.gamma = 1 + 0.1 * randn(g, d)

    def rows(self, rows, seed):
        """Room and inputs for a call of these rows."""
        torch = torch_cuda()
        c, m, qd = self.c, sum(rows), self.heads * self.c.dh
        self.given, self.cu, self.more = rows, cu_of(rows), dev(rows)
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.x = randn(gen(seed), m, self.d).bfloat16()
        self.n8, self.ns = torch.empty(m, self.d, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
        self.a8, self.as_ = torch.empty(m, qd, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
        self.qkv, self.a, self.y = (torch.empty(m, w, **bf16) for w in (self.wide, qd, self.d))
        need = S.surge_cache_attention_workspace(c.desc, max(rows), self.heads)
        self.space = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        return self

    def run(self, stream):
        c, d, m = self.c, self.d, sum(self.given)
        wide, qd, kd = self.wide, self.heads * self.c.dh, self.c.hk * self.c.dh
        c.lengths.add_(self.more)
        S.surge_op_block_norm(m, d, S.NORM_RMS, self.x, d, None, 0, None, None, None, None, 0, 1.0, self.gamma,
                              None, EPS, None, 0, None, 0, self.n8, d, self.ns, stream)
        S.surge_op_linear_i8(m, wide, d, self.n8, d, self.ns, self.w["qkv"], self.ws["qkv"], self.bias["qkv"],
                             None, 0, 0, self.qkv, wide, stream)
        S.surge_op_cache_write(c.desc, m, self.cu, self.qkv[:, qd:], wide, self.qkv[:, qd + kd:], wide, stream)
        S.surge_op_cache_attention(c.desc, m, self.cu, max(self.given), self.heads, True, c.dh ** -0.5, self.qkv,
                                   wide, self.space, self.a, qd, stream)
        S.surge_op_quantize_rows(m, qd, self.a, qd, self.a8, qd, self.as_, stream)
        S.surge_op_linear_i8(m, d, qd, self.a8, qd, self.as_, self.w["o"], self.ws["o"], self.bias["o"], self.x, d,
                             2, self.y, d, stream)

    def check(self):
        """Each operator against its definition of what the one before it gave."""
        torch = torch_cuda()
        c, qd, kd = self.c, self.heads * self.c.dh, self.c.hk * self.c.dh
        p = dict(x=self.x, block=None, post_gamma=None, gate=None, gate_rows=None, pre_gamma=self.gamma, pre_beta=None)
        check_i8(self.n8, self.ns, *norm_reference(p, False, 1.0, self.d)[2:], self.d)
        layer = lambda x, xs, name: dict(x=x, xs=xs, w=self.w[name], ws=self.ws[name],  # noqa: E731
                                         bias=self.bias[name], res=self.x)
        within(self.qkv, *linear_reference({**layer(self.n8, self.ns, "qkv"), "res": self.qkv}, 0))
        at = 0
        for i, r in enumerate(self.given):
            for w in range(2):
                new = self.qkv[at:at + r, qd + w * kd:qd + (w + 1) * kd]
                if r:
                    c.held[i][w] = torch.cat([c.held[i][w], values(*quantized(new)).view(r, c.hk, c.dh)])
            at += r
        c.lengths_np = c.lengths_np + np.array(self.given)
        assert np.array_equal(c.lengths.cpu().numpy(), c.lengths_np)
        within(self.a, *reference(c, self.qkv[:, :qd].contiguous(), self.given, self.heads, True))
        q, s = quantized32(self.a)
        assert torch.equal(self.a8.cpu(), q) and torch.equal(self.as_.cpu(), s)
        within(self.y, *linear_reference(layer(self.a8, self.as_, "o"), 2))


BLOCKS = [([0, 40, 3, 0, 700], 384, 16, 6, 3, 64), ([2000, 0, 5000], 256, 64, 16, 4, 128), ([5, 90], 128, 32, 8, 8, 32)]


@pytest.mark.parametrize("lengths,d,page,heads,hk,dh", BLOCKS)
def test_block_of_a_decoder(lengths, d, page, heads, hk, dh):
    """Prompts, then single tokens, then drafts, one sequence without any."""
    torch = torch_cuda()
    b, n = Block(lengths, d, page, heads, hk, dh, d), len(lengths)
    for i, rows in enumerate(([70] + [130] * (n - 1), [1] * n, [5] * (n - 1) + [0])):
        b.rows(rows, i).run(torch.cuda.current_stream())
        b.check()


def test_block_of_a_decoder_captured_and_replayed():
    """Replayed as its answers grow, with eager work between: the eager block's bits."""
    torch = torch_cuda()
    eager, replayed = (Block(*BLOCKS[1], 3).rows([2, 1, 2], 1) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        replayed.run(torch.cuda.current_stream())
    for step in range(5):
        eager.x.copy_(randn(gen(step), *eager.x.shape))
        replayed.x.copy_(eager.x)
        graph.replay()
        eager.run(torch.cuda.current_stream())
        if step % 2:
            torch.cuda.synchronize()
        assert torch.equal(eager.y, replayed.y) and torch.equal(eager.c.lengths, replayed.c.lengths)
    assert eager.c.lengths.cpu().tolist() == [2010, 5, 5010]


@pytest.mark.parametrize("heads,hk,dh", [(12, 12, 64), (8, 2, 128), (16, 4, 32)])
def test_states_of_an_encoder_kept_in_4_bits(heads, hk, dh):
    """Keys and values projected from texts' states by the library's layer, kept in
    the cache, read by latent queries of each text without a mask."""
    torch = torch_cuda()
    texts, d, latents = [48, 3, 200, 64, 1, 130, 17], 384, 9
    t, w = sum(texts), 2 * hk * dh
    g = gen(heads)
    x = randn(g, t, d).bfloat16()
    wt, bias = (randn(g, w, d) / math.sqrt(d)).bfloat16(), 0.1 * randn(g, w)
    kv = torch.empty(t, w, dtype=torch.bfloat16, device="cuda")
    S.surge_op_linear(t, w, d, x, wt, bias, None, 0, kv)
    ref = x.double() @ wt.double().t().contiguous() + bias.double()
    size = x.double().abs() @ wt.double().abs().t().contiguous() + bias.double().abs()
    within(kv, ref, BF16 * ref.abs() + 1.01 * (d + 2) * F32 * size)
    c = Cache(texts, 32, hk, dh, 1)
    S.surge_op_cache_write(c.desc, t, cu_of(texts), kv, w, kv[:, w // 2:], w, torch.cuda.current_stream())
    ends = np.cumsum([0] + texts)
    c.held = [[values(*quantized(y[a:b])).view(b - a, hk, dh) for y in (kv[:, :w // 2], kv[:, w // 2:])]
              for a, b in zip(ends, ends[1:])]
    check(c, [latents] * len(texts), heads, False, 2)
