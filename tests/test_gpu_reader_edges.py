"""The reader's operators at the edges of their ranges: texts that nobody
reads, rows that are not finite, scores that rise from block to block."""
import math

import pytest

from gpu_util import torch_cuda
from paper_2605_01060_amd import surge as S
from test_gpu_reader import (BF16, F32, block_norm, cross_call, cross_inputs,
                             cross_reference, cu_of, gen, norm64, norm_inputs, norm_reference, within)

pytestmark = pytest.mark.gpu


def test_cross_attention_of_many_queries_without_states_beside_states_without_queries():
    torch = torch_cuda()
    p = cross_inputs([1] * 399 + [0], [0] * 399 + [100], 12, 12, 64, 31)
    out = torch.full((400, 12 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    assert (out[:399] == 0).all() and (out[399] == 7).all()


def agrees(got, ref, tol):
    """NaN where the reference has it and nowhere else, and the rest within tol."""
    torch = torch_cuda()
    bad = ref.isnan()
    assert torch.equal(got.isnan(), bad), (int(got.isnan().sum()), int(bad.sum()))
    if not bad.all():
        within(got[~bad], ref[~bad], tol[~bad])


# Sequences of one unit or more per key head, of every height, whole and with
# their keys split: queries, states, heads, key heads, d_head, split.
SHAPES = [([1], [50], 4, 2, 64, False), ([3, 1], [130, 40], 2, 2, 32, False), ([9], [77], 8, 2, 128, False),
          ([50], [300], 2, 2, 64, True), ([33], [90], 2, 1, 128, False), ([70], [300], 4, 4, 32, False),
          ([40] * 6, [90, 60, 70, 100, 33, 50], 2, 2, 64, False), ([40] * 60, [100] * 60, 8, 8, 64, False),
          ([200, 1], [200, 9], 2, 2, 128, False), ([1], [9000], 4, 2, 64, True), ([1], [20_011], 32, 8, 128, True),
          ([3], [8193], 2, 2, 32, True), ([40], [3001], 2, 2, 64, True), ([200], [2049], 2, 2, 128, True),
          ([150], [4097], 8, 2, 64, True), ([1], [70_001], 1, 1, 128, True)]


def cross_out(p, split):
    torch = torch_cuda()
    out = torch.full((p["q"].shape[0], p["heads"] * p["dh"]), 7.0, dtype=torch.bfloat16, device="cuda")
    plan, _ = cross_call(p, out)
    assert (plan.n_parts > 0) == split
    return out


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
@pytest.mark.parametrize("mask", [None, 0.3])
def test_cross_attention_of_a_nan_query(q, kv, heads, kv_heads, dh, split, mask):
    """NaN in one head of a query: that head's output, and no other, is NaN."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv), mask)
    t, h = sum(q) // 2, heads - 1
    p["q"][t, h * dh + 5] = math.nan
    ref, tol = cross_reference(p)
    assert int(ref.isnan().sum()) == dh
    agrees(cross_out(p, split), ref, tol)


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
def test_cross_attention_of_nan_states(q, kv, heads, kv_heads, dh, split):
    """NaN in a state's key: all rows that read it; in all keys: all rows; in a
    state's value: that feature."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv))
    clean, w = p["kv"].clone(), kv_heads * dh
    for rows, col in ((kv[0] - 1, 3), (slice(0, kv[0]), 3), (kv[0] // 2, w + dh - 1)):
        p["kv"].copy_(clean)
        p["kv"][rows, col] = math.nan
        ref, tol = cross_reference(p)
        assert ref.isnan().any() and (len(q) == kv_heads == 1 or not ref.isnan().all())
        agrees(cross_out(p, split), ref, tol)


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_cross_attention_of_scores_past_the_largest_float(q, kv, heads, kv_heads, dh, split, sign):
    """scale q . k overflows at every state of the first text: NaN, not the
    zeros of a text without states."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv))
    p["scale"] = 1e38
    p["q"][:] = 1.0
    p["kv"][:kv[0], :kv_heads * dh] = sign
    p["kv"][kv[0]:, :kv_heads * dh] = 0
    out = cross_out(p, split)
    assert out[:q[0]].isnan().all()
    assert torch.isfinite(out[q[0]:]).all()


def lowest_keys(p, rows):
    """Scores of -inf at these states, for every row: 1 times -inf in one feature."""
    torch = torch_cuda()
    dh = p["dh"]
    p["q"][:, 0::dh] = 1.0
    p["kv"][rows, 0:p["kv_heads"] * dh:dh] = -math.inf
    seen = torch.ones(p["kv"].shape[0], dtype=torch.uint8, device="cuda")
    seen[rows] = 0
    return {**p, "mask": seen if p["mask"] is None else p["mask"] * seen}


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
@pytest.mark.parametrize("mask", [None, 0.3])
def test_cross_attention_of_scores_of_minus_infinity(q, kv, heads, kv_heads, dh, split, mask):
    """A text's first half (whole blocks and parts) scores -inf: its
    probabilities are 0, as if it were masked."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv), mask)
    ref, tol = cross_reference(lowest_keys(p, slice(0, (kv[0] + 1) // 2)))
    agrees(cross_out(p, split), ref, tol)


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
def test_cross_attention_of_rows_without_a_finite_score(q, kv, heads, kv_heads, dh, split):
    """All of a text's scores are -inf, or its masked rest is all that is not:
    0 / 0, which is not the zeros of a text without states."""
    torch = torch_cuda()
    for mask in (None, 0.3):
        p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv), mask)
        lowest_keys(p, slice(0, kv[0]))
        if mask is not None:
            p["mask"][:kv[0]] = 0
            p["mask"][kv[0] // 3] = 1
        out = cross_out(p, split)
        assert out[:q[0]].isnan().all()
        assert torch.isfinite(out[q[0]:]).all()


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_cross_attention_of_scores_whose_float_steps_are_large(q, kv, heads, kv_heads, dh, split, sign):
    """Scores of 2^20 to 2^100 and their multiples by 1 to 50: the states of the
    largest share a row, in equal parts, whatever a step of a float is there."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv))
    w, tk = kv_heads * dh, sum(kv)
    level = sign * (torch.randperm(tk, generator=gen(sum(kv)), device="cuda") % 50 + 1)
    p["q"].zero_()
    p["kv"][:, :w] = 0
    p["kv"][:, 0:w:dh] = level[:, None].bfloat16()
    want = []
    for i, n in enumerate(q):
        at = slice(int(p["cu_kv"][i]), int(p["cu_kv"][i + 1]))
        top = p["kv"][at, w:][level[at] == level[at].max()].double().view(-1, kv_heads, dh)
        want.append(torch.stack([top.mean(0), top.abs().mean(0)])[:, None].repeat_interleave(heads // kv_heads, 2)
                    .expand(2, n, heads, dh).reshape(2, n, heads * dh))
    ref, size = torch.cat(want, 1)
    for e in (20, 28, 33, 40, 100):
        p["q"][:, 0::dh] = 2.0 ** e
        # Equal probabilities, up to a rounding to bf16, and the sums.
        within(cross_out(p, split), ref, BF16 * ref.abs() + (1.01 * BF16 + tk * F32) * size, e)


def test_cross_plan_counts_the_units_that_hold_a_part():
    """Units of 128 and of 64 rows, all split, beside whole ones of a short text."""
    for q, rows in ((200, 128), (50, 64), (1, 32)):
        alone = S.CrossPlan(cu_of([q]), cu_of([40_000]), 2, 2, 64)
        assert alone.n_units == alone.n_parts > 2 * -(-q // rows)
        both = S.CrossPlan(cu_of([q, 130]), cu_of([40_000, 7]), 2, 2, 64)
        assert both.n_units - both.n_parts == 2 * 2
        whole = S.CrossPlan(cu_of([q]), cu_of([20]), 2, 2, 64)
        assert whole.n_parts == 0 and whole.n_units == 2 * -(-q // rows)


@pytest.mark.parametrize("kind", [S.NORM_LAYER, S.NORM_RMS])
@pytest.mark.parametrize("d", [40, 768, 2056, 8192])
@pytest.mark.parametrize("post", [False, True])
def test_block_norm_of_an_infinite_gate(kind, d, post):
    """An infinity of the gate's sign and the block's, without a beta that it
    could meet as 0 times infinity."""
    torch = torch_cuda()
    M = 7
    p = norm_inputs(M, d, False, post, "vector", True, d + kind)
    p["gate"][d // 3], p["gate"][d - 1] = math.inf, -math.inf
    y = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    block_norm(p, M, d, kind, 0.7, y)
    ry, ey, _, _ = norm_reference(p, kind == S.NORM_LAYER, 0.7, d)
    inf = ry.isinf()
    assert inf.sum() == 2 * M and torch.equal(y.double()[inf], ry[inf])
    within(y[~inf], ry[~inf], (BF16 * ry.abs() + 1.01 * ey)[~inf])


def underflowed(p):
    """What the keys add whose probability is below 2^-118 of their row's
    largest.  The reference of the exponentials is at most 2^8 below the largest
    score, so the others stay above the least normal float 2^-126 wherever they
    are formed (of a unit's keys, or as a part's weight times one of at most
    2^8); these may be flushed to 0, and lose what they add at the most."""
    torch = torch_cuda()
    heads, kv_heads, dh = p["heads"], p["kv_heads"], p["dh"]
    group, w = heads // kv_heads, kv_heads * dh
    lost = torch.zeros(p["q"].shape, dtype=torch.float64, device="cuda")
    for i in range(len(p["cu_q"]) - 1):
        r, c = (slice(int(cu[i]), int(cu[i + 1])) for cu in (p["cu_q"], p["cu_kv"]))
        k = p["kv"][c, :w].double().view(-1, kv_heads, dh).permute(1, 2, 0).contiguous()
        v = p["kv"][c, w:].double().view(-1, kv_heads, dh).permute(1, 0, 2).contiguous()
        q = p["q"][r].double().view(-1, kv_heads, group, dh).permute(1, 0, 2, 3).reshape(kv_heads, -1, dh)
        prob = torch.softmax(torch.bmm(q, k) * p["scale"], 2)
        prob = torch.where(prob < 2.0 ** -118 * prob.amax(2, keepdim=True), prob, 0.0)
        lost[r] = torch.bmm(prob, v.abs()).view(kv_heads, -1, group, dh).permute(1, 0, 2, 3) \
            .reshape(-1, heads * dh)
    return lost


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh,split", SHAPES)
@pytest.mark.parametrize("nats", [5.0, 7.0, 12.0])
@pytest.mark.parametrize("rows", ["rise", "fall", "both"])
def test_cross_attention_of_scores_that_rise_from_block_to_block(q, kv, heads, kv_heads, dh, split, nats, rows):
    """Eight stretches of a text whose scores differ by `nats` from one to the
    next, up or down or, in rows beside each other, both, and values that make
    up for it: every stretch counts in the output (of rows of one sign), so
    each rescaling of the sums is seen.  Scores of up to 100: the tolerance has
    them in it."""
    torch = torch_cuda()
    p = cross_inputs(q, kv, heads, kv_heads, dh, sum(kv) + int(nats))
    w = kv_heads * dh
    up = torch.ones(sum(q), device="cuda")
    if rows == "fall":
        up = -up
    if rows == "both":
        up[1::2] = -1
    for i, (a, n) in enumerate(zip(p["cu_kv"], kv)):
        level = torch.arange(n, device="cuda") * 8 // n - 3.5
        p["kv"][a:a + n, 0:w:dh] = (level * nats * math.sqrt(dh) / 8)[:, None].bfloat16()
        sign = -1.0 if rows == "fall" else 1.0
        p["kv"][a:a + n, w:] *= torch.exp(-sign * level * nats)[:, None]
    p["q"][:, 0::dh] = (8 * up)[:, None].bfloat16()
    ref, tol = cross_reference(p)
    within(cross_out(p, split), ref, tol + underflowed(p))


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_cross_attention_of_large_scores(dh):
    """Scores of hundreds and thousands against the definition."""
    torch = torch_cuda()
    p = cross_inputs([40, 1, 200, 2], [300, 4000, 500, 0], 2, 2, dh, 3)
    p["q"] *= 100
    p["kv"][:, :2 * dh] *= 10
    ref, tol = cross_reference(p)
    out = torch.empty_like(p["q"])
    cross_call(p, out)
    within(out, ref, tol)


@pytest.mark.parametrize("d", [40, 768, 2056, 8192])
def test_block_norm_of_an_infinite_gate_over_a_beta_of_0(d):
    torch = torch_cuda()
    M = 7
    p = norm_inputs(M, d, True, True, "vector", True, d)
    for i, gate in ((d // 3, math.inf), (d - 1, -math.inf)):
        p["gate"][i], p["post_beta"][i] = gate, 0.0
    y = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    block_norm(p, M, d, S.NORM_LAYER, 0.7, y)
    ry, ey, _, _ = norm_reference(p, True, 0.7, d)
    inf = ry.isinf()
    assert inf.sum() == 2 * M and torch.equal(y.double()[inf], ry[inf])
    within(y[~inf], ry[~inf], (BF16 * ry.abs() + 1.01 * ey)[~inf])


@pytest.mark.parametrize("kind", [S.NORM_LAYER, S.NORM_RMS])
@pytest.mark.parametrize("d", [8, 200, 384, 768, 2048, 3592, 8192])
@pytest.mark.parametrize("power,eps", [(64, 1e-5), (100, 1e-5), (100, 0.0), (30, 0.0), (-40, 0.0), (-64, 0.0),
                                       (-100, 0.0), (-120, 0.0)])
def test_block_norm_of_rows_whose_squares_leave_the_floats(kind, d, power, eps):
    """A norm without an eps that counts is the same of a row times a power of 2,
    though the squares of some rows here are above the largest or below the
    least float.  Rows of ordinary size beside them."""
    torch = torch_cuda()
    M, layer = 9, kind == S.NORM_LAYER
    p = norm_inputs(M, d, layer, True, "none", True, d + kind)
    by = torch.ones(M, 1, device="cuda")
    by[::3], by[1::3] = 2.0 ** power, 2.0 ** (power // 2)
    # (Times a power of 2 rounded again where a bf16 has fewer bits, below 2^-126.)
    x, block = ((p[k].float() * by).bfloat16() for k in ("x", "block"))
    far = torch.zeros_like(x)
    exact = torch.zeros(M, d, dtype=torch.float64, device="cuda")
    big = 2.0 ** 40  # the reference's eps counts for nothing here
    z, n = (torch.empty(M, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    block_norm({**p, "x": x, "block": None, "post_gamma": None, "post_beta": None}, M, d, kind, 1.0, None, z,
               eps=eps)
    ref, tol = norm64(x.double() / by.double() * big, exact, layer, p["pre_gamma"], p["pre_beta"], d)
    within(z, ref, BF16 * ref.abs() + 1.01 * tol)
    block_norm({**p, "x": far, "block": block}, M, d, kind, 1.0, n, None, eps=eps)
    ref, tol = norm64(block.double() / by.double() * big, exact, layer, p["post_gamma"], p["post_beta"], d)
    within(n, ref, BF16 * ref.abs() + 1.01 * tol)
