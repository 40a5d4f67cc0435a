"""Refusals of the row operators (vt_linear, vt_linear_gated, vt_norm_rows, vt_rotate_heads,
vt_paged_append_heads), none of which reaches the GPU, and the projections' workspace size."""
import ctypes
import math

import pytest

from paper_2607_07046_amd import voltron as vt
from tests.test_paged_host import BOTH as POOL
from tests.test_paged_host import io as paged_io
from tests.test_paged_host import kv

P, Q, R = 0x10000, 0x20000, 0x30000  # aligned addresses that nothing reads
NAN, INF = math.nan, math.inf


def refused(status, call, *args):
    with pytest.raises(vt.VoltronError) as e:
        call(*args)
    assert e.value.status == status and e.value.detail
    return e.value.detail


def lin(**change):
    f = dict(type=vt.VT_T_F16, n_rows=3, n_in=20, n_out=10, x=P, ld_x=24, w=Q, ld_w=24, y=R, ld_y=16)
    f.update(change)
    return vt.vt_linear_io(**f)


def linear(io, ws=P, ws_bytes=1 << 30):
    vt.vt_linear(io, ws, ws_bytes, None)


def gated(io, ws=P, ws_bytes=1 << 30):
    vt.vt_linear_gated(io, ws, ws_bytes, None)


UP = dict(w_up=Q, ld_up=24)
LINEAR = [
    (vt.VT_ERR_ARG, dict(type=vt.VT_T_F8E4M3)), (vt.VT_ERR_ARG, dict(type=-1)), (vt.VT_ERR_ARG, dict(act=5)),
    (vt.VT_ERR_ARG, dict(act=-1)), (vt.VT_ERR_ARG, dict(n_rows=0)), (vt.VT_ERR_ARG, dict(n_rows=-1)),
    (vt.VT_ERR_ARG, dict(n_in=0)), (vt.VT_ERR_ARG, dict(n_out=0)),
    (vt.VT_ERR_UNSUPPORTED, dict(n_rows=(1 << 20) + 1)), (vt.VT_ERR_ARG, dict(x=None)), (vt.VT_ERR_ARG, dict(w=None)),
    (vt.VT_ERR_ARG, dict(y=None)), (vt.VT_ERR_ALIGN, dict(x=P + 8)), (vt.VT_ERR_ALIGN, dict(w=P + 2)),
    (vt.VT_ERR_ALIGN, dict(y=R + 4)), (vt.VT_ERR_ALIGN, dict(ld_x=28)), (vt.VT_ERR_ALIGN, dict(ld_w=28)),
    (vt.VT_ERR_ALIGN, dict(ld_y=12)), (vt.VT_ERR_ARG, dict(ld_x=16)), (vt.VT_ERR_ARG, dict(ld_w=-24)),
    (vt.VT_ERR_ARG, dict(ld_y=8)), (vt.VT_ERR_UNSUPPORTED, dict(ld_x=(1 << 22) + 8)),
    (vt.VT_ERR_UNSUPPORTED, dict(ld_w=(1 << 22) + 8)), (vt.VT_ERR_UNSUPPORTED, dict(ld_y=(1 << 32) + 8)),
    (vt.VT_ERR_ALIGN, dict(bias=P + 2)), (vt.VT_ERR_ALIGN, dict(residual=Q + 8, ld_res=16)),
    (vt.VT_ERR_ALIGN, dict(residual=Q, ld_res=12)), (vt.VT_ERR_ARG, dict(residual=Q, ld_res=8)),
    (vt.VT_ERR_ARG, dict(residual=Q)), (vt.VT_ERR_ARG, dict(residual=R, ld_res=24)), (vt.VT_ERR_ARG, dict(y=P)),
    (vt.VT_ERR_UNSUPPORTED, dict(n_rows=1 << 20, n_out=1 << 30, ld_y=1 << 30)),
]


@pytest.mark.parametrize("status,change", LINEAR)
def test_linear_refusals(status, change):
    refused(status, linear, lin(**change))
    refused(status, gated, lin(**UP, **change))


def test_linear_refusals_of_one_kind():
    refused(vt.VT_ERR_ARG, linear, lin(**UP))
    refused(vt.VT_ERR_ARG, linear, lin(bias_up=P))
    for status, change in ((vt.VT_ERR_ARG, {}), (vt.VT_ERR_ALIGN, dict(w_up=Q + 8, ld_up=24)),
                           (vt.VT_ERR_ALIGN, dict(w_up=Q, ld_up=25)), (vt.VT_ERR_ARG, dict(w_up=Q, ld_up=16)),
                           (vt.VT_ERR_UNSUPPORTED, dict(w_up=Q, ld_up=(1 << 22) + 8)),
                           (vt.VT_ERR_ALIGN, dict(bias_up=P + 4, **UP))):
        refused(status, gated, lin(**change))


def test_linear_workspace():
    size = vt.vt_linear_workspace_size(lin())
    assert size == (64 << 20) + 16384
    assert vt.vt_linear_workspace_size(lin(n_rows=1 << 20, n_in=16384, n_out=100000, w_up=Q)) == size
    for call, io in ((linear, lin()), (gated, lin(**UP))):
        refused(vt.VT_ERR_WORKSPACE, call, io, None, size)
        refused(vt.VT_ERR_WORKSPACE, call, io, P, size - 1)
        refused(vt.VT_ERR_ALIGN, call, io, P + 8, size)
    refused(vt.VT_ERR_ARG, vt.vt_linear_workspace_size, lin(n_in=0))
    lib = vt.load_library()
    assert lib.vt_linear_workspace_size(ctypes.byref(lin()), None) == vt.VT_ERR_ARG
    assert lib.vt_linear_workspace_size(None, ctypes.byref(ctypes.c_size_t())) == vt.VT_ERR_ARG
    assert lib.vt_linear(None, P, size, None) == vt.VT_ERR_ARG
    assert lib.vt_linear_gated(None, P, size, None) == vt.VT_ERR_ARG


def norm(**change):
    f = dict(type=vt.VT_T_F16, n_rows=3, hidden=20, eps=1e-5, x=P, ld_x=24, gain=Q, y=R, ld_y=24)
    f.update(change)
    return vt.vt_norm_io(**f)


@pytest.mark.parametrize("status,change", [
    (vt.VT_ERR_ARG, dict(type=vt.VT_T_F8E4M3)), (vt.VT_ERR_ARG, dict(n_rows=0)), (vt.VT_ERR_ARG, dict(hidden=0)),
    (vt.VT_ERR_UNSUPPORTED, dict(n_rows=(1 << 20) + 1)), (vt.VT_ERR_UNSUPPORTED, dict(hidden=16385, ld_x=16400)),
    (vt.VT_ERR_ARG, dict(eps=-1e-5)), (vt.VT_ERR_ARG, dict(eps=NAN)), (vt.VT_ERR_ARG, dict(eps=INF)),
    (vt.VT_ERR_ARG, dict(x=None)), (vt.VT_ERR_ARG, dict(gain=None)), (vt.VT_ERR_ARG, dict(y=None)),
    (vt.VT_ERR_ALIGN, dict(x=P + 2)), (vt.VT_ERR_ALIGN, dict(gain=Q + 8)), (vt.VT_ERR_ALIGN, dict(y=R + 8)),
    (vt.VT_ERR_ALIGN, dict(partial=Q + 8, ld_partial=24)), (vt.VT_ERR_ALIGN, dict(peer=Q, ld_peer=20)),
    (vt.VT_ERR_ALIGN, dict(h=Q + 8, ld_h=24)), (vt.VT_ERR_ARG, dict(ld_x=16)), (vt.VT_ERR_ARG, dict(ld_y=16)),
    (vt.VT_ERR_ARG, dict(partial=Q)), (vt.VT_ERR_ARG, dict(peer=Q, ld_peer=16)), (vt.VT_ERR_ARG, dict(h=Q, ld_h=16)),
    (vt.VT_ERR_ARG, dict(ld_x=(1 << 32) + 8)), (vt.VT_ERR_ARG, dict(h=R, ld_h=24)),
    (vt.VT_ERR_ARG, dict(y=P, ld_y=32)), (vt.VT_ERR_ARG, dict(h=P, ld_h=32)),
    (vt.VT_ERR_ARG, dict(partial=Q + 64, ld_partial=24, h=Q + 64, ld_h=32))])
def test_norm_refusals(status, change):
    refused(status, vt.vt_norm_rows, norm(**change))


def test_null_descriptors():
    lib = vt.load_library()
    assert lib.vt_norm_rows(None, None) == vt.VT_ERR_ARG
    assert lib.vt_rotate_heads(None, None, None, None) == vt.VT_ERR_ARG
    assert lib.vt_paged_append_heads(None, ctypes.byref(paged_io()), None, None, None) == vt.VT_ERR_ARG
    assert lib.vt_paged_append_heads(ctypes.byref(kv()), None, None, None, None) == vt.VT_ERR_ARG


def heads(**change):
    f = dict(type=vt.VT_T_F16, n_tok=3, head_dim=64, pos=P, n_q_heads=4, q=P, ld_q=256, q_out=Q, ld_qo=256, n_k_heads=2,
             k=P, ld_k=128, k_out=Q, ld_ko=128)
    f.update(change)
    return vt.vt_heads_io(**f)


@pytest.mark.parametrize("status,change", [
    (vt.VT_ERR_ARG, dict(type=vt.VT_T_F8E4M3)), (vt.VT_ERR_UNSUPPORTED, dict(head_dim=96)),
    (vt.VT_ERR_ARG, dict(n_tok=0)), (vt.VT_ERR_UNSUPPORTED, dict(n_tok=(1 << 20) + 1)),
    (vt.VT_ERR_ARG, dict(n_q_heads=-1)), (vt.VT_ERR_ARG, dict(n_k_heads=-2)), (vt.VT_ERR_ARG, dict(n_q_heads=0, n_k_heads=0)),
    (vt.VT_ERR_UNSUPPORTED, dict(n_q_heads=1025)), (vt.VT_ERR_UNSUPPORTED, dict(n_k_heads=1025)),
    (vt.VT_ERR_ALIGN, dict(pos=P + 2)), (vt.VT_ERR_ARG, dict(pos=None, pos0=-1)),
    (vt.VT_ERR_ARG, dict(pos=None, pos0=2 ** 31 - 2)),
    (vt.VT_ERR_ARG, dict(q=None)), (vt.VT_ERR_ARG, dict(q_out=None)), (vt.VT_ERR_ARG, dict(k=None)),
    (vt.VT_ERR_ARG, dict(k_out=None)), (vt.VT_ERR_ALIGN, dict(q=P + 8)), (vt.VT_ERR_ALIGN, dict(k_out=Q + 2)),
    (vt.VT_ERR_ALIGN, dict(ld_q=260)), (vt.VT_ERR_ARG, dict(ld_qo=248)), (vt.VT_ERR_ARG, dict(ld_k=120)),
    (vt.VT_ERR_ARG, dict(ld_ko=(1 << 32) + 8)), (vt.VT_ERR_ARG, dict(q_out=P, ld_qo=264)),
    (vt.VT_ERR_ARG, dict(k_out=P, ld_ko=136))])
def test_rotate_refusals(status, change):
    refused(status, vt.vt_rotate_heads, heads(**change))


ROPE = [dict(dims=3), dict(dims=66), dict(dims=-2), dict(flags=2), dict(base=-1.0), dict(base=NAN), dict(base=INF),
        dict(factor=0.5), dict(factor=-2.0), dict(factor=NAN), dict(factor=INF), dict(low=-1.0, high=2.0, context=4),
        dict(low=1.0, context=4), dict(low=2.0, high=2.0, context=4), dict(low=4.0, high=2.0, context=4),
        dict(low=1.0, high=4.0), dict(low=1.0, high=4.0, context=-5), dict(low=NAN, high=2.0, context=4),
        dict(high=INF, context=4), dict(amplitude=-1.0), dict(amplitude=NAN), dict(amplitude=INF)]


@pytest.mark.parametrize("change", ROPE)
def test_rope_refusals(change):
    f = dict(base=10000.0)
    f.update(change)
    rope = vt.vt_rope(**f)
    refused(vt.VT_ERR_ARG, vt.vt_rotate_heads, heads(), None, rope)
    refused(vt.VT_ERR_ARG, vt.vt_paged_append_heads, kv(), paged_io(), None, rope)


@pytest.mark.parametrize("status,change", [
    (vt.VT_ERR_ALIGN, dict(q_gain=P + 8)), (vt.VT_ERR_ALIGN, dict(k_gain=P + 2)), (vt.VT_ERR_ARG, dict(eps=-1.0)),
    (vt.VT_ERR_ARG, dict(eps=NAN)), (vt.VT_ERR_ARG, dict(eps=INF))])
def test_head_norm_refusals(status, change):
    n = vt.vt_head_norm(**change)
    refused(status, vt.vt_rotate_heads, heads(), n)
    refused(status, vt.vt_paged_append_heads, kv(), paged_io(), n)


@pytest.mark.parametrize("status,k,i", POOL)
def test_append_heads_refuses_what_append_does(status, k, i):
    refused(status, vt.vt_paged_append_heads, kv(**k), paged_io(**i))


@pytest.mark.parametrize("status,i", [
    (vt.VT_ERR_ARG, dict(k=None)), (vt.VT_ERR_ARG, dict(v=None)), (vt.VT_ERR_ALIGN, dict(k=P + 2)),
    (vt.VT_ERR_ALIGN, dict(ld_v=129)), (vt.VT_ERR_ARG, dict(ld_k=120)), (vt.VT_ERR_ALIGN, dict(q=P + 8)),
    (vt.VT_ERR_ARG, dict(q=P, q_rot=P, ld_qr=264))])
def test_append_heads_refusals(status, i):
    refused(status, vt.vt_paged_append_heads, kv(), paged_io(**i))
