"""The reader's operators on the GPU against their definitions in 64 bits.

Inputs are rounded to their types first, so what is left is the kernels' own
arithmetic.  Tolerances count roundings: one to bf16 is off by at most
BF16 = 2^-8 of the value, one in fp32 by F32 = 2^-24.
"""
import math

import numpy as np
import pytest

from gpu_util import torch_cuda
from paper_2605_01060_amd import surge as S

pytestmark = pytest.mark.gpu

BF16, F32 = 2.0 ** -8, 2.0 ** -24
EPS = 1e-5


def gen(seed):
    return torch_cuda().Generator(device="cuda").manual_seed(seed)


def randn(g, *dims):
    return torch_cuda().randn(dims, generator=g, device="cuda")


def strided(t, extra, fill=7.0):
    """A copy of `t` as the left columns of a wider buffer, and that buffer."""
    torch = torch_cuda()
    big = torch.full((t.shape[0], t.shape[1] + extra), fill, device="cuda").to(t.dtype)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]], big


def within(got, ref, tol, what=""):
    torch = torch_cuda()
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - tol
    assert over.max() <= 0, (what, float((got - ref).abs().max()), float(over.max()))


# ---------------------------------------------------------------------------
# int8: quantizer and linear layer
# ---------------------------------------------------------------------------

def quantized32(x):
    """The quantizer's definition, operation by operation in fp32 on the CPU."""
    torch = torch_cuda()
    x = x.float().cpu()
    a = x.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
    inv = torch.full_like(a, 127.0) / a  # (a number over a tensor is a reciprocal and a product)
    return torch.round(x * inv).to(torch.int8), (a / 127.0)[:, 0]


@pytest.mark.parametrize("M,K", [(1, 8), (3, 64), (5, 136), (70, 384), (9, 632), (33, 768),
                                 (17, 1024), (6, 1032), (5, 2048), (4, 4096), (3, 8192), (2, 8200),
                                 (2, 16384), (20_001, 128)])
def test_quantize_rows(M, K):
    torch = torch_cuda()
    g = gen(M + K)
    x = (randn(g, M, K) * torch.exp2(20 * randn(g, M, 1))).bfloat16()
    x[M // 2] = 0
    xs, _ = strided(x, 24)
    cols = -(-K // 128) * 128
    big = torch.full((M + 1, cols + 32), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((M + 1,), -1.0, device="cuda")
    S.surge_op_quantize_rows(M, K, xs, K + 24, big, cols + 32, scale, torch.cuda.current_stream())
    q, s = quantized32(x)
    assert torch.equal(big[:M, :K].cpu(), q)
    assert torch.equal(scale[:M].cpu(), s)
    assert (big[:M, K:cols] == 0).all()  # the padding
    assert (big[:M, cols:] == 99).all() and (big[M] == 99).all() and scale[M] == -1.0


def test_quantize_rows_of_small_large_and_no_values():
    torch = torch_cuda()
    x = torch.zeros(6, 128, device="cuda").bfloat16()
    x[0, 3] = 1e-38
    x[1] = torch.finfo(torch.bfloat16).max
    x[1, 5] = -x[1, 5]
    x[2, 1], x[3, 2], x[4, 9] = math.nan, math.inf, -math.inf
    x[2:5, 77] = 1.0
    q = torch.full((6, 128), 99, dtype=torch.int8, device="cuda")
    scale = torch.zeros(6, device="cuda")
    S.surge_op_quantize_rows(6, 128, x, 128, q, 128, scale, torch.cuda.current_stream())
    torch.cuda.synchronize()
    fine = [0, 1, 5]
    rq, rs = quantized32(x[fine])
    assert torch.equal(q[fine].cpu(), rq) and torch.equal(scale[fine].cpu(), rs)
    assert (q[2:5] == 0).all() and scale[2:5].isnan().all()


def linear_inputs(M, N, K, seed, pad_x=0):
    torch = torch_cuda()
    g = gen(seed)

    def i8(*dims):
        return torch.randint(-127, 128, dims, generator=g, device="cuda", dtype=torch.int8)

    x = i8(M, K)
    if pad_x:
        x, _ = strided(x, pad_x)
    return dict(x=x, xs=torch.exp2(randn(g, M)) / 127, w=i8(N, K), ws=torch.exp2(randn(g, N)) / 2000,
                bias=randn(g, N), res=randn(g, M, N).bfloat16())


def linear_reference(p, epi, rows=None):
    torch = torch_cuda()
    r = slice(None) if rows is None else rows
    lin = (p["x"][r].double() @ p["w"].double().t().contiguous()) * p["xs"][r].double()[:, None] \
        * p["ws"].double()
    bias, res = p["bias"].double(), p["res"][r].double()
    v = lin + bias
    # Conversion, two products, the bias and the residual: five roundings.
    tol = 5 * F32 * (lin.abs() + bias.abs() + (res.abs() if epi == 2 else 0))
    if epi == 1:
        # GELU's slope is below 1.13, its fit within 3e-7.
        v = v * torch.special.erfc(-v / math.sqrt(2.0)) / 2
        tol = 1.13 * tol + 4e-7
    if epi == 2:
        v = v + res
    return v, BF16 * v.abs() + 1.01 * tol


LINEAR = [
    (1, 8, 128), (1, 768, 768), (2, 1000, 256), (3, 2304, 384), (7, 128, 4096), (16, 1024, 1024),
    (17, 136, 640), (33, 264, 128), (64, 4096, 128), (100, 24, 2048), (129, 1152, 384),
    (257, 1000, 768), (777, 1536, 384), (1000, 2304, 896), (1500, 504, 16384), (2049, 768, 768),
    (4100, 1032, 256), (8200, 256, 128), (13_579, 2304, 768), (20_000, 1024, 512), (9000, 2056, 1152),
]


@pytest.mark.parametrize("M,N,K", LINEAR)
@pytest.mark.parametrize("epi", [0, 1, 2])
def test_linear_i8(M, N, K, epi):
    torch = torch_cuda()
    pad = 16 if M % 2 else 0
    p = linear_inputs(M, N, K, M + N + K + epi, pad)
    big = torch.full((M + 1, N + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    S.surge_op_linear_i8(M, N, K, p["x"], K + pad, p["xs"], p["w"], p["ws"], p["bias"],
                         p["res"] if epi == 2 else None, N, epi, big, N + 8,
                         torch.cuda.current_stream())
    ref, tol = linear_reference(p, epi)
    within(big[:M, :N], ref, tol)
    assert (big[:M, N:] == 7).all() and (big[M] == 7).all()


# (rows, channels) of the tile, and shapes that take it on 256 compute units;
# the last two leave channels over for a second launch.
TILES = [((16, 16), 33, 1000, 768), ((64, 64), 300, 1000, 384), ((64, 64), 700, 520, 4096),
         ((64, 128), 777, 1536, 384),
         ((128, 128), 4100, 1032, 256), ((192, 256), 13_579, 768, 768), ((256, 256), 6000, 2304, 768),
         ((192, 256), 20_000, 1032, 1024), ((256, 256), 30_000, 1288, 2048)]


@pytest.mark.parametrize("tile,M,N,K", TILES)
@pytest.mark.parametrize("epi", [0, 1, 2])
def test_linear_i8_tiles(tile, M, N, K, epi):
    """Each kernel, and the bits of its rows in calls of a few rows."""
    torch = torch_cuda()
    assert S.surge_op_linear_i8_tile(M, N, K) == tile
    p = linear_inputs(M, N, K, M + epi)
    stream = torch.cuda.current_stream()

    def call(rows):
        y = torch.empty(len(rows), N, dtype=torch.bfloat16, device="cuda")
        res = p["res"][rows].contiguous() if epi == 2 else None
        S.surge_op_linear_i8(len(rows), N, K, p["x"][rows].contiguous(), K,
                             p["xs"][rows].contiguous(), p["w"], p["ws"], p["bias"], res, N, epi, y, N,
                             stream)
        return y

    y = call(torch.arange(M).cuda())
    rows = torch.unique(torch.cat([torch.arange(0, M, 97), torch.tensor([1, 255, 256, M - 2, M - 1])])).cuda()
    rows = rows[rows < M]
    ref, tol = linear_reference(p, epi, rows)
    within(y[rows], ref, tol)
    few = rows[:: max(1, len(rows) // 7)][:7]
    assert torch.equal(call(few), y[few])


def test_linear_i8_sums_exactly():
    """Sums that need all of 31 bits, the extreme values of int8 among them."""
    torch = torch_cuda()
    K, N = 65536, 16
    x = torch.full((2, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    x[1, 1::2] = 127
    one, zero = torch.ones(N, device="cuda"), torch.zeros(N, device="cuda")
    y = torch.empty(2, N, dtype=torch.bfloat16, device="cuda")
    S.surge_op_linear_i8(2, N, K, x, K, one, w, one, zero, None, 0, 0, y, N,
                         torch.cuda.current_stream())
    ref = x.double() @ w.double().t().contiguous()
    assert torch.equal(y, ref.bfloat16())


def test_linear_i8_large_and_in_place():
    """A SuperBatch's rows, the output over the residual, sampled rows."""
    torch = torch_cuda()
    M, N, K = 150_003, 1024, 4096
    p = linear_inputs(M, N, K, 5)
    y = p["res"].clone()
    S.surge_op_linear_i8(M, N, K, p["x"], K, p["xs"], p["w"], p["ws"], p["bias"], y, N, 2, y, N,
                         torch.cuda.current_stream())
    rows = torch.unique(torch.cat([torch.arange(0, M, 211), torch.tensor([1, 255, 256, M - 2, M - 1])])).cuda()
    ref, tol = linear_reference(p, 2, rows)
    within(y[rows], ref, tol)


def test_linear_i8_strides_past_32_bits():
    """Rows whose byte offsets pass 2^32 in the input and the output."""
    torch = torch_cuda()
    M, N, K, ld = 1100, 136, 256, 1 << 22
    p = linear_inputs(M, N, K, 6)
    x = torch.empty(M, ld, dtype=torch.int8, device="cuda")
    x[:, :K] = p["x"]
    y = torch.empty(M, ld, dtype=torch.bfloat16, device="cuda")
    S.surge_op_linear_i8(M, N, K, x, ld, p["xs"], p["w"], p["ws"], p["bias"], None, 0, 0, y, ld,
                         torch.cuda.current_stream())
    ref, tol = linear_reference(p, 0)
    within(y[:, :N], ref, tol)


def test_linear_i8_of_a_row_that_could_not_be_quantized():
    torch = torch_cuda()
    p = linear_inputs(40, 64, 128, 9)
    p["xs"][7] = math.nan
    y = torch.empty(40, 64, dtype=torch.bfloat16, device="cuda")
    S.surge_op_linear_i8(40, 64, 128, p["x"], 128, p["xs"], p["w"], p["ws"], p["bias"], None, 0, 1, y,
                         64, torch.cuda.current_stream())
    assert y[7].isnan().all()
    y[7] = 0
    assert torch.isfinite(y).all()


def test_linear_i8_of_more_rows_than_a_launch_takes():
    torch = torch_cuda()
    M, N, K = (1 << 24) + 37, 8, 128
    p = linear_inputs(M, N, K, 21)
    y = p["res"].clone()
    S.surge_op_linear_i8(M, N, K, p["x"], K, p["xs"], p["w"], p["ws"], p["bias"], y, N, 2, y, N,
                         torch.cuda.current_stream())
    rows = torch.cat([torch.arange(0, M, 50_021), torch.arange((1 << 24) - 300, M)]).cuda()
    ref, tol = linear_reference(p, 2, rows)
    within(y[rows], ref, tol)


def test_quantize_rows_and_norms_of_more_rows_than_a_grid_takes():
    """Rows of 8 features: 2^22 workgroups of 16 rows, the norm's four times over."""
    torch = torch_cuda()
    M = (1 << 26) + 21
    g = gen(22)
    x = torch.empty(M, 8, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    rows = torch.cat([torch.arange(0, M, 1_000_003), torch.arange((1 << 26) - 40, M)]).cuda()
    q = torch.empty(M, 128, dtype=torch.int8, device="cuda")
    scale = torch.empty(M, device="cuda")
    S.surge_op_quantize_rows(M, 8, x, 8, q, 128, scale, torch.cuda.current_stream())
    rq, rs = quantized32(x[rows])
    assert torch.equal(q[rows][:, :8].cpu(), rq) and torch.equal(scale[rows].cpu(), rs)
    del q, scale
    M = (1 << 28) + 21
    rows = torch.cat([torch.arange(0, M, 4_000_037), torch.arange((1 << 28) - 40, M)]).cuda()
    x = torch.empty(M, 8, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    p = norm_inputs(1, 8, True, False, "none", False, 22)
    z = torch.empty(M, 8, dtype=torch.bfloat16, device="cuda")
    block_norm({**p, "x": x}, M, 8, S.NORM_LAYER, 1.0, None, z)
    _, _, rz, ez = norm_reference({**p, "x": x[rows]}, True, 1.0, 8)
    within(z[rows], rz, BF16 * rz.abs() + 1.01 * ez)


# ---------------------------------------------------------------------------
# Block norm
# ---------------------------------------------------------------------------

def norm64(v, err, layer, gamma, beta, d):
    """The norm of v, known to `err`, and how far fp32 may be from it: a sum of
    d terms over at most 32 chunks' worth of adds in a lane and 8 joining
    steps is 40 roundings of the sum of magnitudes."""
    c = v - v.mean(1, keepdim=True) if layer else v
    rstd = 1 / (c.pow(2).mean(1, keepdim=True) + EPS).sqrt()
    n = c * rstd
    off = err + (44 * F32 * v.abs().mean(1, keepdim=True) + err.mean(1, keepdim=True) if layer else 0)
    # The variance's relative error is twice the mean error of c over its size.
    spread = 50 * F32 + (off * n.abs()).mean(1, keepdim=True) * rstd
    g = gamma.double()
    b = beta.double() if beta is not None else 0.0
    out = n * g + b
    tol = g.abs() * (off * rstd + n.abs() * spread * 2) + 4 * F32 * ((n * g).abs() + out.abs())
    return out, tol


def norm_reference(p, layer, res_scale, d):
    torch = torch_cuda()
    v = p["block"].double() if p["block"] is not None else torch.zeros_like(p["x"]).double()
    err = torch.zeros_like(v)
    if p["post_gamma"] is not None:
        v, err = norm64(v, err, layer, p["post_gamma"], p["post_beta"], d)
    for gate in (p["gate_rows"], p["gate"]):
        if gate is not None:
            v, err = v * gate.double(), err * gate.double().abs() + F32 * (v * gate.double()).abs()
    y = v + res_scale * p["x"].double()
    # res_scale is passed as a float.
    err = err + 3 * F32 * (v.abs() + abs(res_scale) * p["x"].double().abs())
    z, z_err = norm64(y, err, layer, p["pre_gamma"], p["pre_beta"], d)
    return y, err, z, z_err


def norm_inputs(M, d, layer, post, gate, block, seed):
    g = gen(seed)
    x = randn(g, M, d) * 3 + 0.7
    x[:, d // 2] *= 20
    return dict(
        x=x.bfloat16(), block=(randn(g, M, d) * 0.4 - 2.0).bfloat16() if block else None,
        post_gamma=1 + 0.3 * randn(g, d) if post else None,
        post_beta=0.3 * randn(g, d) if post and layer else None,
        gate=randn(g, d) if gate in ("vector", "both") else None,
        gate_rows=randn(g, M, d).bfloat16() if gate in ("rows", "both") else None,
        pre_gamma=1 + 0.3 * randn(g, d), pre_beta=0.3 * randn(g, d) if layer else None)


def block_norm(p, M, d, kind, res_scale, y=None, z=None, zq=None, scale=None, lds=None, eps=EPS):
    """lds: row strides by name where they are not d (zq: the padded width)."""
    torch = torch_cuda()
    ld = {**dict(x=d, block=d, gate_rows=d, y=d, z=d, zq=-(-d // 128) * 128), **(lds or {})}
    S.surge_op_block_norm(M, d, kind, p["x"], ld["x"], p["block"], ld["block"], p["post_gamma"],
                          p["post_beta"], p["gate"], p["gate_rows"], ld["gate_rows"], res_scale,
                          p["pre_gamma"] if z is not None or zq is not None else None,
                          p["pre_beta"] if z is not None or zq is not None else None, eps, y,
                          ld["y"], z, ld["z"], zq, ld["zq"], scale, torch.cuda.current_stream())


def check_i8(zq, scale, z, z_err, d):
    """int8 rows: within half a step of z, which the kernel knows to z_err, and
    a scale that takes the row's largest value to 127."""
    amax = z.abs().max(1, keepdim=True).values
    off = z_err.max(1, keepdim=True).values + 4 * F32 * amax
    s = scale.double()[:, None]
    assert ((s * 127 - amax).abs() <= off).all()
    assert (zq[:, :d].abs().max(1).values == 127).all()
    within(zq[:, :d].double() * s, z, 0.5 * s * (1 + 512 * F32) + 2 * off)
    assert (zq[:, d:] == 0).all()


NORM_SHAPES = [(1, 8), (3, 40), (5, 128), (130, 384), (9, 632), (33, 768), (64, 1024), (7, 1032),
               (5, 2048), (6, 2056), (3, 4096), (4, 6904), (2, 8192), (20_001, 256)]


@pytest.mark.parametrize("M,d", NORM_SHAPES)
@pytest.mark.parametrize("kind", [S.NORM_LAYER, S.NORM_RMS])
@pytest.mark.parametrize("post,gate,block", [(True, "none", True), (True, "both", True),
                                             (False, "rows", True), (True, "vector", True),
                                             (False, "none", False)])
def test_block_norm(M, d, kind, post, gate, block):
    torch = torch_cuda()
    layer = kind == S.NORM_LAYER
    p = norm_inputs(M, d, layer, post, gate, block, M + d + kind)
    cols = -(-d // 128) * 128
    y = torch.full((M + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    z = torch.full((M + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    zq = torch.full((M + 1, cols), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((M + 1,), -1.0, device="cuda")
    block_norm(p, M, d, kind, 0.7, y, z, zq, scale)
    ry, ey, rz, ez = norm_reference(p, layer, 0.7, d)
    within(y[:M], ry, BF16 * ry.abs() + 1.01 * ey, "y")
    within(z[:M], rz, BF16 * rz.abs() + 1.01 * ez, "z")
    check_i8(zq[:M], scale[:M], rz, ez, d)
    assert (y[M] == 7).all() and (z[M] == 7).all() and (zq[M] == 99).all() and scale[M] == -1.0


@pytest.mark.parametrize("outputs", [("y",), ("z",), ("zq",), ("y", "zq")])
def test_block_norm_of_some_outputs(outputs):
    """Each set of outputs has the bits of the call that makes all."""
    torch = torch_cuda()
    M, d = 77, 384
    p = norm_inputs(M, d, True, True, "both", True, 3)

    def buffers():
        return dict(y=torch.zeros(M, d, dtype=torch.bfloat16, device="cuda"),
                    z=torch.zeros(M, d, dtype=torch.bfloat16, device="cuda"),
                    zq=torch.zeros(M, d, dtype=torch.int8, device="cuda"),
                    scale=torch.zeros(M, device="cuda"))

    full, some = buffers(), buffers()
    block_norm(p, M, d, S.NORM_LAYER, 1.0, **full)
    block_norm(p, M, d, S.NORM_LAYER, 1.0,
               **{k: v for k, v in some.items() if k in outputs or (k == "scale" and "zq" in outputs)})
    for k in outputs:
        assert torch.equal(some[k], full[k]), k


@pytest.mark.parametrize("d", [384, 1024, 4104])
@pytest.mark.parametrize("y_over,z_over", [("x", "block"), ("block", "x"), ("gate_rows", "x"), ("x", None)])
def test_block_norm_in_place(d, y_over, z_over):
    torch = torch_cuda()
    M = 300
    p = norm_inputs(M, d, True, True, "rows", True, d)
    y, z = (torch.empty(M, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    block_norm(p, M, d, S.NORM_LAYER, 1.0, y, z)
    p2 = {k: v.clone() if v is not None else None for k, v in p.items()}
    y2, z2 = p2[y_over], p2[z_over] if z_over else torch.empty_like(z)
    block_norm(p2, M, d, S.NORM_LAYER, 1.0, y2, z2)
    assert torch.equal(y, y2) and torch.equal(z, z2)


def test_block_norm_strides():
    torch = torch_cuda()
    M, d = 50, 632
    p = norm_inputs(M, d, True, True, "rows", True, 8)
    wide, lds = dict(p), {}
    for k, extra in (("x", 8), ("block", 40), ("gate_rows", 16)):
        wide[k], _ = strided(p[k], extra)
        lds[k] = d + extra
    outs = {}
    for k, extra, t in (("y", 24, torch.bfloat16), ("z", 8, torch.bfloat16)):
        outs[k] = torch.full((M, d + extra), 7.0, dtype=t, device="cuda")
        lds[k] = d + extra
    outs["zq"] = torch.full((M, 640 + 16), 99, dtype=torch.int8, device="cuda")
    lds["zq"] = 656
    scale = torch.empty(M, device="cuda")
    block_norm(wide, M, d, S.NORM_LAYER, 1.0, outs["y"], outs["z"], outs["zq"], scale, lds)
    ry, ey, rz, ez = norm_reference(p, True, 1.0, d)
    within(outs["y"][:, :d], ry, BF16 * ry.abs() + 1.01 * ey)
    within(outs["z"][:, :d], rz, BF16 * rz.abs() + 1.01 * ez)
    check_i8(outs["zq"][:, :640], scale, rz, ez, d)
    assert (outs["y"][:, d:] == 7).all() and (outs["z"][:, d:] == 7).all() and (outs["zq"][:, 640:] == 99).all()


def test_block_norm_strides_past_32_bits():
    torch = torch_cuda()
    M, d, ld = 1100, 128, 1 << 22
    p = norm_inputs(M, d, True, True, "none", True, 4)
    x = torch.empty(M, ld, dtype=torch.bfloat16, device="cuda")
    x[:, :d] = p["x"]
    z = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    block_norm({**p, "x": x}, M, d, S.NORM_LAYER, 1.0, x, z, lds=dict(x=ld, y=ld))
    ry, ey, rz, ez = norm_reference(p, True, 1.0, d)
    within(x[:, :d], ry, BF16 * ry.abs() + 1.01 * ey)
    within(z, rz, BF16 * rz.abs() + 1.01 * ez)


def test_block_norm_of_rows_that_are_not_finite():
    """A NaN or an infinity stays in its row."""
    torch = torch_cuda()
    M, d = 9, 256
    p = norm_inputs(M, d, False, True, "none", True, 5)
    clean = {k: v.clone() if v is not None else None for k, v in p.items()}
    p["x"][2, 3], p["block"][5, 200] = math.nan, math.inf
    out = []
    for q in (p, clean):
        y = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
        zq = torch.empty(M, d, dtype=torch.int8, device="cuda")
        scale = torch.empty(M, device="cuda")
        block_norm(q, M, d, S.NORM_RMS, 1.0, y, None, zq, scale)
        out.append((y, zq, scale))
    keep = [i for i in range(M) if i not in (2, 5)]
    for a, b in zip(*out):
        assert torch.equal(a[keep], b[keep])
    assert out[0][2][[2, 5]].isnan().all() and (out[0][1][[2, 5]] == 0).all()


# ---------------------------------------------------------------------------
# Cross attention
# ---------------------------------------------------------------------------

def cu_of(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def cross_inputs(q_lengths, kv_lengths, heads, kv_heads, dh, seed, mask=None):
    """mask: share of the states that are left out; their rows of K and V hold
    infinities and NaN."""
    torch = torch_cuda()
    g = gen(seed)
    tq, tk = int(sum(q_lengths)), int(sum(kv_lengths))
    kv = randn(g, tk, 2 * kv_heads * dh).bfloat16()
    p = dict(cu_q=cu_of(q_lengths), cu_kv=cu_of(kv_lengths), heads=heads, kv_heads=kv_heads, dh=dh,
             q=randn(g, tq, heads * dh).bfloat16(), kv=kv, mask=None, scale=1 / math.sqrt(dh))
    if mask is not None:
        on = torch.rand(tk, generator=g, device="cuda") >= mask
        if len(kv_lengths) > 2:  # a text with no state left, one with its first and one with its last
            for i, keep in ((0, None), (1, 0), (2, -1)):
                a, b = int(p["cu_kv"][i]), int(p["cu_kv"][i + 1])
                on[a:b] = False
                if keep is not None and b > a:
                    on[a if keep == 0 else b - 1] = True
        kv[~on] = math.nan
        kv[~on, ::3] = math.inf
        kv[~on, 1::3] = -math.inf
        p["mask"] = on.to(torch.uint8) * 255
    return p


def cross_call(p, out, plan=None, workspace=None, stream=None):
    torch = torch_cuda()
    d, w = p["heads"] * p["dh"], p["kv_heads"] * p["dh"]
    plan = plan or S.CrossPlan(p["cu_q"], p["cu_kv"], p["heads"], p["kv_heads"], p["dh"])
    if workspace is None and plan.workspace_bytes:
        workspace = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
    S.surge_op_cross_attention(plan, p["q"], p["q"].stride(0), p["kv"], 2 * w, p["kv"][:, w:], 2 * w,
                               p["mask"], p["scale"], workspace, out, out.stride(0),
                               stream or torch.cuda.current_stream())
    return plan, workspace


def cross_reference(p):
    """Output and tolerance.  A probability is off by its rounding to bf16 and
    by its score's fp32 error (dh + 2 roundings of the sum of magnitudes, as a
    relative error, plus 8 roundings around the exponential); the sums add a
    rounding per 32-key step and part."""
    torch = torch_cuda()
    heads, kv_heads, dh = p["heads"], p["kv_heads"], p["dh"]
    group, w = heads // kv_heads, kv_heads * dh
    ref = torch.zeros(p["q"].shape, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(ref)
    for i in range(len(p["cu_q"]) - 1):
        a, b = int(p["cu_q"][i]), int(p["cu_q"][i + 1])
        c, d = int(p["cu_kv"][i]), int(p["cu_kv"][i + 1])
        keys = torch.arange(c, d, device="cuda")
        if p["mask"] is not None:
            keys = keys[p["mask"][c:d] != 0]
        if b == a or not len(keys):
            continue
        k = p["kv"][keys, :w].double().view(-1, kv_heads, dh).permute(1, 2, 0).contiguous()
        v = p["kv"][keys, w:].double().view(-1, kv_heads, dh).permute(1, 0, 2).contiguous()
        q = p["q"][a:b].double().view(b - a, kv_heads, group, dh).permute(1, 0, 2, 3) \
            .reshape(kv_heads, -1, dh)
        prob = torch.softmax(torch.bmm(q, k) * p["scale"], 2)
        size = torch.bmm(q.abs(), k.abs()).amax(2, keepdim=True) * p["scale"]
        o, o_abs = torch.bmm(prob, v), torch.bmm(prob, v.abs())
        rel = BF16 + 2 * (dh + 2) * F32 * size + (16 + 2 * (len(keys) // 32 + 1)) * F32
        t = BF16 * o.abs() + 1.01 * rel * o_abs
        for x, to in ((o, ref), (t, tol)):
            to[a:b] = x.view(kv_heads, b - a, group, dh).permute(1, 0, 2, 3).reshape(b - a, -1)
    return ref, tol


Q_MIX = [5, 3, 2, 1, 31, 0, 32, 33, 1, 64, 65, 7, 127, 200, 1, 0, 129, 16]
KV_MIX = [40, 33, 70, 1, 31, 32, 33, 0, 64, 65, 127, 128, 129, 2, 500, 3, 257, 1000]


@pytest.mark.parametrize("heads,kv_heads,dh", [(12, 12, 32), (4, 4, 64), (12, 12, 64), (2, 2, 128),
                                               (8, 2, 64), (6, 1, 32), (8, 1, 128), (9, 3, 64),
                                               (32, 8, 128)])
@pytest.mark.parametrize("mask", [None, 0.3, 0.97])
def test_cross_attention(heads, kv_heads, dh, mask):
    torch = torch_cuda()
    p = cross_inputs(Q_MIX, KV_MIX, heads, kv_heads, dh, heads + dh, mask)
    out = torch.full((p["q"].shape[0] + 3, heads * dh + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    ref, tol = cross_reference(p)
    n = p["q"].shape[0]
    within(out[:n, :heads * dh], ref, tol)
    assert (out[n:] == 7).all() and (out[:n, heads * dh:] == 7).all()
    empty = slice(int(p["cu_q"][5]), int(p["cu_q"][6]))
    assert (out[empty, :heads * dh] == 0).all()
    if mask is not None:
        assert (out[:5, :heads * dh] == 0).all()  # the text with no state left


# One query or a few, keys split over units; ends inside a block, parts of one key.
LONG = [(1, 5000, 4, 4, 64), (1, 20_011, 32, 8, 128), (3, 8193, 2, 2, 32), (40, 3001, 2, 1, 64),
        (1, 70_001, 1, 1, 128), (200, 2049, 2, 2, 128), (150, 4097, 8, 2, 64), (1, 257, 1, 1, 64)]


@pytest.mark.parametrize("q,kv,heads,kv_heads,dh", LONG)
@pytest.mark.parametrize("mask", [None, 0.5])
def test_cross_attention_over_long_texts(q, kv, heads, kv_heads, dh, mask):
    torch = torch_cuda()
    p = cross_inputs([q], [kv], heads, kv_heads, dh, q + kv, mask)
    if mask is not None:  # whole parts without a key, the first among them
        p["mask"][:kv // 3] = 0
    out = torch.full((q, heads * dh), math.nan, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    ref, tol = cross_reference(p)
    within(out, ref, tol)


# The chip full of units of 128 rows: their blocks are of 32 keys at d_head 128.
@pytest.mark.parametrize("seqs,q,kv,heads,kv_heads,dh", [(96, 128, 300, 8, 8, 128), (48, 60, 333, 32, 8, 128),
                                                         (300, 97, 290, 8, 8, 128), (300, 70, 260, 8, 8, 64)])
@pytest.mark.parametrize("mask", [None, 0.4])
def test_cross_attention_on_a_full_chip(seqs, q, kv, heads, kv_heads, dh, mask):
    torch = torch_cuda()
    q_lengths = [q - i % 7 for i in range(seqs)]
    kv_lengths = [0 if i == 5 else kv - (i * 37) % (kv // 2) for i in range(seqs)]
    p = cross_inputs(q_lengths, kv_lengths, heads, kv_heads, dh, seqs + kv, mask)
    out = torch.full((sum(q_lengths) + 1, heads * dh), math.nan, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    ref, tol = cross_reference(p)
    within(out[:-1], ref, tol)
    assert out[-1].isnan().all()


def test_cross_attention_long_and_short_texts_together():
    torch = torch_cuda()
    kv = [3, 9000, 0, 17, 40_000, 1, 64, 2500]
    q = [1, 1, 1, 5, 2, 1, 130, 33]
    p = cross_inputs(q, kv, 4, 2, 64, 1)
    out = torch.full((sum(q), 256), math.nan, dtype=torch.bfloat16, device="cuda")
    plan, _ = cross_call(p, out)
    assert plan.n_parts > 0
    ref, tol = cross_reference(p)
    within(out, ref, tol)
    again = torch.empty_like(out)
    cross_call(p, again)
    assert torch.equal(out, again)  # no order of arrival in the result


def test_cross_attention_masked_out_or_without_states():
    torch = torch_cuda()
    for kv in ([0, 0], [3000, 40]):
        p = cross_inputs([1, 70], kv, 4, 2, 64, 2, 0.1)
        p["mask"][:] = 0
        p["kv"][:] = math.nan
        out = torch.full((71, 256), math.nan, dtype=torch.bfloat16, device="cuda")
        cross_call(p, out)
        assert (out == 0).all()


def test_cross_attention_large_scores():
    """Scores of thousands: the running maximum keeps the exponentials finite."""
    torch = torch_cuda()
    p = cross_inputs([40, 1], [300, 4000], 2, 2, 64, 3)
    p["q"] *= 100
    p["kv"][:, :128] = p["kv"][:, :128] * 10
    # Exact ties and a lone winner: the winner's own row of V.
    out = torch.empty(41, 128, dtype=torch.bfloat16, device="cuda")
    cross_call(p, out)
    assert torch.isfinite(out).all()
    p["kv"][:, :128] = 0  # every score 0: the mean of V
    cross_call(p, out)
    ref, tol = cross_reference(p)
    within(out, ref, tol)


def test_cross_attention_rows_past_32_bits():
    """K and V rows whose offsets pass 2^32 elements, as slices of a long cache."""
    torch = torch_cuda()
    kv, ld = 1100, 1 << 22
    p = cross_inputs([1, 40], [100, 1000], 2, 2, 64, 12)
    big = torch.empty(kv, ld, dtype=torch.bfloat16, device="cuda")
    big[:, :256] = p["kv"]
    out = torch.empty(41, 128, dtype=torch.bfloat16, device="cuda")
    plan = S.CrossPlan(p["cu_q"], p["cu_kv"], 2, 2, 64)
    ws = torch.empty(max(plan.workspace_bytes, 16), dtype=torch.uint8, device="cuda")
    S.surge_op_cross_attention(plan, p["q"], 128, big, ld, big[:, 128:], ld, None, p["scale"], ws, out,
                               128, torch.cuda.current_stream())
    ref, tol = cross_reference(p)
    within(out, ref, tol)


def test_cross_attention_refusals_with_a_plan():
    torch = torch_cuda()
    p = cross_inputs([1], [9000], 2, 2, 64, 4)
    plan = S.CrossPlan(p["cu_q"], p["cu_kv"], 2, 2, 64)
    assert plan.workspace_bytes > 0
    out = torch.full((1, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    good = dict(plan=plan, d_q=p["q"], ld_q=128, d_k=p["kv"], ld_k=256, d_v=p["kv"][:, 128:], ld_v=256,
                key_mask=None, scale=0.125, workspace=ws, d_out=out, ld_out=128)
    for change in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                   dict(scale=3e38), dict(d_out=p["kv"], ld_out=256),
                   dict(workspace=None), dict(workspace=ws[16:]), dict(d_q=None), dict(d_k=None),
                   dict(d_v=None), dict(d_out=None), dict(ld_q=120), dict(ld_k=132), dict(ld_v=64),
                   dict(ld_out=1 << 23), dict(d_out=p["q"]), dict(d_q=p["q"].data_ptr() + 2)):
        with pytest.raises(S.SurgeError) as e:
            S.surge_op_cross_attention(**{**good, **change})
        assert e.value.status in (S.SURGE_ERR_INVALID_ARGUMENT, S.SURGE_ERR_CAPACITY)
    torch.cuda.synchronize()
    assert (out == 7).all()
    plan.close()
    with pytest.raises(S.SurgeError):
        S.surge_op_cross_attention(**good)


def test_cross_attention_on_two_streams():
    """One plan, two streams, a workspace each."""
    torch = torch_cuda()
    p = cross_inputs([1, 2], [9000, 12_000], 8, 2, 128, 5)
    other = {**p, "q": -p["q"]}
    plan = S.CrossPlan(p["cu_q"], p["cu_kv"], 8, 2, 128)
    want = []
    for x in (p, other):
        o = torch.empty(3, 1024, dtype=torch.bfloat16, device="cuda")
        cross_call(x, o, plan)
        want.append(o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.empty_like(o) for o in want]
    spaces = [torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, s, w in zip((p, other), got, streams, spaces):
            cross_call(x, o, plan, w, s)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---------------------------------------------------------------------------
# The operators together: one block of a reader
# ---------------------------------------------------------------------------

class Reader:
    """n = Norm(x) in int8; Q = n Wq, K|V = states Wkv; A = attention; y = r x
    + gate Norm(A Wo); n' = Norm(y) in bf16."""

    def __init__(self, q_lengths, kv_lengths, d, heads, seed):
        torch = torch_cuda()
        g = gen(seed)
        self.d, self.heads, self.dh = d, heads, d // heads
        self.x = randn(g, int(sum(q_lengths)), d).bfloat16()
        self.states = randn(g, int(sum(kv_lengths)), d).bfloat16()
        self.w, self.ws, self.bias = {}, {}, {}
        for name, n in (("q", d), ("kv", 2 * d), ("o", d)):
            q, s = quantized32(randn(g, n, d) / math.sqrt(d))
            self.w[name], self.ws[name] = q.cuda(), s.contiguous().cuda()
            self.bias[name] = 0.1 * randn(g, n)
        self.gamma = [1 + 0.1 * randn(g, d) for _ in range(3)]
        self.gate = 0.5 * randn(g, d)
        self.cu_q, self.cu_kv = cu_of(q_lengths), cu_of(kv_lengths)
        self.plan = S.CrossPlan(self.cu_q, self.cu_kv, heads, heads, self.dh)

        def empty(rows, cols, t=torch.bfloat16):
            return torch.empty(rows, cols, dtype=t, device="cuda")

        m, n = self.x.shape[0], self.states.shape[0]
        self.n8, self.ns = empty(m, d, torch.int8), torch.empty(m, device="cuda")
        self.s8, self.ss = empty(n, d, torch.int8), torch.empty(n, device="cuda")
        self.a8, self.as_ = empty(m, d, torch.int8), torch.empty(m, device="cuda")
        self.q, self.kv, self.a, self.o = empty(m, d), empty(n, 2 * d), empty(m, d), empty(m, d)
        self.y, self.z = empty(m, d), empty(m, d)
        self.ws_mem = empty(1, max(self.plan.workspace_bytes, 16), torch.uint8)

    def run(self, stream):
        d, m, n = self.d, self.x.shape[0], self.states.shape[0]
        norm = lambda **k: S.surge_op_block_norm(stream=stream, M=m, d=d, kind=S.NORM_RMS, **{**dict(  # noqa: E731
            d_x=self.x, ld_x=d, d_block=None, ld_block=0, post_gamma=None, post_beta=None, gate=None,
            gate_rows=None, ld_gate=0, res_scale=1.0, pre_beta=None, eps=EPS, d_y=None, ld_y=0,
            d_z=None, ld_z=0, d_zq=None, ld_zq=0, zq_scale=None), **k})
        norm(pre_gamma=self.gamma[0], d_zq=self.n8, ld_zq=d, zq_scale=self.ns)
        S.surge_op_quantize_rows(n, d, self.states, d, self.s8, d, self.ss, stream)
        for rows, x8, xs, name, y in ((m, self.n8, self.ns, "q", self.q), (n, self.s8, self.ss, "kv", self.kv)):
            S.surge_op_linear_i8(rows, y.shape[1], d, x8, d, xs, self.w[name], self.ws[name],
                                 self.bias[name], None, 0, 0, y, y.shape[1], stream)
        S.surge_op_cross_attention(self.plan, self.q, d, self.kv, 2 * d, self.kv[:, d:], 2 * d, None,
                                   1 / math.sqrt(self.dh), self.ws_mem, self.a, d, stream)
        S.surge_op_quantize_rows(m, d, self.a, d, self.a8, d, self.as_, stream)
        S.surge_op_linear_i8(m, d, d, self.a8, d, self.as_, self.w["o"], self.ws["o"], self.bias["o"],
                             None, 0, 0, self.o, d, stream)
        norm(d_block=self.o, ld_block=d, post_gamma=self.gamma[1], gate=self.gate,
             pre_gamma=self.gamma[2], d_y=self.y, ld_y=d, d_z=self.z, ld_z=d)

    def reference(self):
        """In 64 bits, quantized where the block quantizes and nowhere rounded
        to bf16 between."""
        torch = torch_cuda()

        def rms(v, gamma):
            return v / (v.pow(2).mean(1, keepdim=True) + EPS).sqrt() * gamma.double()

        def linear(v, name):
            a = v.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100)
            v = torch.round(v / a * 127) * a / 127
            w = self.w[name].double() * self.ws[name].double()[:, None]
            return v @ w.t().contiguous() + self.bias[name].double()

        x, d = self.x.double(), self.d
        q, kv = linear(rms(x, self.gamma[0]), "q"), linear(self.states.double(), "kv")
        a = torch.zeros_like(x)
        for i in range(len(self.cu_q) - 1):
            r, c = (slice(int(cu[i]), int(cu[i + 1])) for cu in (self.cu_q, self.cu_kv))
            if c.stop == c.start:
                continue
            h = lambda t: t.reshape(-1, self.heads, self.dh).permute(1, 0, 2).contiguous()  # noqa: E731
            s = torch.bmm(h(q[r]), h(kv[c, :d]).transpose(1, 2).contiguous()) / math.sqrt(self.dh)
            a[r] = torch.bmm(torch.softmax(s, 2), h(kv[c, d:])).permute(1, 0, 2).reshape(-1, d)
        y = x + self.gate.double() * rms(linear(a, "o"), self.gamma[1])
        return y, rms(y, self.gamma[2])

    def check(self):
        # Five stages round to bf16 (2^-9 of a value in the mean square) and a
        # rounding can move an int8 value by its step (at most 1/127 of the
        # row's largest, about 1/35 of its mean square): relative errors that
        # add up to well under 2^-5 over the rows.
        for got, ref in zip((self.y, self.z), self.reference()):
            assert ((got.double() - ref).norm() / ref.norm()) < 2.0 ** -6
            assert (got.double() - ref).abs().max() < 0.1 * ref.abs().max()


READERS = [([32] * 9, [48, 3, 200, 0, 17, 64, 65, 130, 9], 384, 12),
           ([1] * 64, list(range(8, 200, 3)), 1024, 16), ([70, 1], [5000, 20_000], 256, 2)]


@pytest.mark.parametrize("q,kv,d,heads", READERS)
def test_reader_block(q, kv, d, heads):
    torch = torch_cuda()
    r = Reader(q, kv, d, heads, d)
    r.run(torch.cuda.current_stream())
    r.check()


def test_reader_block_captured_and_replayed():
    """Two readers in a graph each, replayed with new inputs, eager work and
    synchronisations between: every replay has the eager call's bits."""
    torch = torch_cuda()
    readers = [Reader(*READERS[1], 11), Reader(*READERS[2], 12)]
    stream = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    for r in readers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            r.run(torch.cuda.current_stream())
        graphs.append(g)
    g = gen(1)
    for step in range(4):
        for r, graph in zip(readers, graphs):
            r.x.copy_(randn(g, *r.x.shape))
            r.run(torch.cuda.current_stream())
            torch.cuda.synchronize()
            want = (r.y.clone(), r.z.clone())
            r.y.zero_()
            r.z.zero_()
            graph.replay()
            if step % 2:
                torch.cuda.synchronize()
            assert torch.equal(r.y, want[0]) and torch.equal(r.z, want[1])
    # Both at the same time, on a stream each.
    for r, graph in zip(readers, graphs):
        r.run(torch.cuda.current_stream())
    torch.cuda.synchronize()
    want = [r.z.clone() for r in readers]
    streams = [torch.cuda.Stream() for _ in readers]
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for r, w in zip(readers, want):
        assert torch.equal(r.z, w)
