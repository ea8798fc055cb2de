"""Refusals of the reader's operators, all on the host: the pointers below are
addresses that nothing may touch, so every call has to end in its checks."""
import ctypes

import numpy as np
import pytest

from paper_2605_01060_amd import surge as S

A = 1 << 20  # 16-byte aligned addresses
X, Y, Z, Q, R = (A + (i << 12) for i in range(1, 6))
NAN, INF = float("nan"), float("inf")


def refused(fn, args, **change):
    with pytest.raises(S.SurgeError) as e:
        fn(**{**args, **change})
    assert e.value.status in (S.SURGE_ERR_INVALID_ARGUMENT, S.SURGE_ERR_CAPACITY), e.value
    return e.value


QUANT = dict(M=3, K=200, d_x=X, ld_x=200, d_q=Q, ld_q=256, d_scale=A)


@pytest.mark.parametrize("change", [
    dict(M=-1), dict(M=1 << 31), dict(K=0), dict(K=12), dict(K=16392, ld_x=16392, ld_q=16512),
    dict(d_x=0), dict(d_q=0), dict(d_scale=0), dict(d_x=A + 8), dict(d_q=A + 8), dict(ld_x=192),
    dict(ld_x=204), dict(ld_q=208), dict(ld_q=264), dict(ld_x=(1 << 22) + 8), dict(d_q=X),
])
def test_quantize_rows_refuses(change):
    refused(S.surge_op_quantize_rows, QUANT, **change)


LINEAR = dict(M=3, N=24, K=128, d_x=X, ld_x=128, d_x_scale=A, d_w=A, d_w_scale=A, d_bias=A, d_res=R,
              ld_res=24, epilogue=2, d_y=Y, ld_y=24)


@pytest.mark.parametrize("change", [
    dict(M=-1), dict(M=1 << 31), dict(N=0), dict(N=12), dict(N=(1 << 20) + 8), dict(K=0),
    dict(K=64), dict(K=192, ld_x=192), dict(K=65664, ld_x=65664), dict(epilogue=3),
    dict(epilogue=-1), dict(d_x=0), dict(d_x_scale=0), dict(d_w=0), dict(d_w_scale=0),
    dict(d_bias=0), dict(d_res=0), dict(d_y=0), dict(d_x=A + 4), dict(d_w=A + 8),
    dict(d_w_scale=A + 4), dict(d_bias=A + 8), dict(d_res=A + 2), dict(d_y=A + 8), dict(ld_x=112),
    dict(ld_x=136), dict(ld_y=16), dict(ld_y=28), dict(ld_res=16), dict(ld_x=1 << 23),
    dict(d_y=X), dict(d_y=A), dict(d_y=R, ld_y=32),
])
def test_linear_i8_refuses(change):
    refused(S.surge_op_linear_i8, LINEAR, **change)


NORM = dict(M=3, d=200, kind=S.NORM_LAYER, d_x=X, ld_x=200, d_block=R, ld_block=200, post_gamma=A,
            post_beta=A, gate=A, gate_rows=A, ld_gate=200, res_scale=1.0, pre_gamma=A, pre_beta=A,
            eps=1e-5, d_y=Y, ld_y=200, d_z=Z, ld_z=200, d_zq=Q, ld_zq=256, zq_scale=A)


@pytest.mark.parametrize("change", [
    dict(M=-1), dict(M=1 << 31), dict(d=0), dict(d=4), dict(d=8200, ld_x=8200), dict(kind=2),
    dict(kind=-1), dict(res_scale=NAN), dict(res_scale=INF), dict(eps=-1e-6), dict(eps=NAN),
    dict(eps=2.0), dict(d_block=0),
    dict(d_block=0, gate=0, gate_rows=0), dict(d_block=0, post_gamma=0, post_beta=0, gate_rows=0),
    dict(d_block=0, post_gamma=0, post_beta=0, gate=0), dict(d_y=0, d_z=0, d_zq=0),
    dict(post_gamma=0), dict(kind=S.NORM_RMS, pre_beta=0), dict(kind=S.NORM_RMS, post_beta=0),
    dict(d_z=0, d_zq=0), dict(pre_gamma=0, pre_beta=0), dict(d_x=0), dict(zq_scale=0),
    dict(d_x=A + 8), dict(d_block=A + 8), dict(gate_rows=A + 8), dict(gate=A + 4),
    dict(post_gamma=A + 4), dict(post_beta=A + 4), dict(pre_gamma=A + 4), dict(pre_beta=A + 4),
    dict(d_y=A + 8), dict(d_z=A + 8), dict(d_zq=A + 8), dict(ld_x=192), dict(ld_block=196),
    dict(ld_gate=100), dict(ld_y=192), dict(ld_z=204), dict(ld_zq=208),
    dict(d_z=Y), dict(d_zq=Y), dict(d_zq=Z), dict(d_zq=X), dict(d_zq=A), dict(d_y=X, ld_y=208),
    dict(d_z=R, ld_z=208), dict(d_y=A, ld_gate=208),
])
def test_block_norm_refuses(change):
    refused(S.surge_op_block_norm, NORM, **change)


def plan(**change):
    return {**dict(cu_q=np.array([0, 2, 2]), cu_kv=np.array([0, 0, 5]), n_heads=4, n_kv_heads=2,
                   d_head=64), **change}


@pytest.mark.parametrize("change", [
    dict(cu_q=np.array([0]), cu_kv=np.array([0])), dict(cu_q=np.array([1, 2, 2])),
    dict(cu_q=np.array([0, 2, 1])), dict(cu_kv=np.array([0, 5, 4])), dict(cu_kv=np.array([0, 0, 1 << 31])),
    dict(cu_q=np.array([0, 0, 1 << 31])), dict(cu_q=np.array([0, 0, 1 << 30])), dict(d_head=48),
    dict(d_head=256), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=3), dict(n_heads=2048),
    dict(n_kv_heads=-2),
])
def test_cross_plan_refuses(change):
    refused(S.surge_cross_plan_create, plan(**change))


def test_cross_plan_of_two_lengths():
    with pytest.raises(ValueError):
        S.CrossPlan(np.array([0, 1]), np.array([0, 1, 2]), 2, 2, 64)


def test_cross_attention_needs_a_plan():
    lib = S.lib()
    st = lib.surge_op_cross_attention(None, A, 64, A, 64, A, 64, None, 1.0, None, 0, A, 64, None)
    assert st == S.SURGE_ERR_INVALID_ARGUMENT
    assert lib.surge_cross_plan_info(None, None, None, None) == S.SURGE_ERR_INVALID_ARGUMENT
    assert lib.surge_cross_plan_create(1, None, None, 1, 1, 64, None) == S.SURGE_ERR_INVALID_ARGUMENT
    h = ctypes.c_void_p(7)
    cu = np.array([0, 1], np.int64)
    assert lib.surge_cross_plan_create(1, cu.ctypes.data, None, 1, 1, 64,
                                       ctypes.byref(h)) == S.SURGE_ERR_INVALID_ARGUMENT
    assert not h.value  # no handle of a plan that was not made
    lib.surge_cross_plan_destroy(None)


def test_no_rows_is_a_call_that_does_nothing():
    S.surge_op_quantize_rows(0, 128, 0, 0, 0, 0, 0)
    S.surge_op_linear_i8(0, 8, 128, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    S.surge_op_block_norm(**{**NORM, "M": 0})


def test_linear_i8_tile_of_refused_shapes():
    for shape in ((0, 8, 128), (1, 4, 128), (1, 8, 64), (1 << 31, 8, 128), (1, 8, 131072)):
        assert S.surge_op_linear_i8_tile(*shape) == (0, 0)
    assert S.surge_op_linear_i8_tile(1, 8, 128, 0) == (0, 0)
