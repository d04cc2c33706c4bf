"""Refusals of the gated layer and of the calls on activations kept in 8 bits: found on the host, before anything is launched (no GPU
needed), each with its own status; size queries."""
import ctypes

import pytest
import torch

from paper_2405_16325_amd import binding as sl

P = ctypes.c_void_p(4096)          # aligned, never dereferenced: every call here is refused on the host
ODD = ctypes.c_void_p(4096 + 8)
ODD16 = ctypes.c_void_p(4096 + 16)
NULL, SHAPE, ALIGN, VALUE = sl.SLOPE_ERR_NULL, sl.SLOPE_ERR_SHAPE, sl.SLOPE_ERR_ALIGN, sl.SLOPE_ERR_VALUE


def call(name, args, **changed):
    args = dict(args)
    assert set(changed) <= set(args)
    args.update(changed)
    return getattr(sl.lib(), name)(*args.values())


FWD = dict(x=P, b=4, vals=P, meta=P, d_ff=64, d_in=128, act=0, l=P, r_=P, r=32, h=P, gu=P, q=P, scale=P, ws=P, ws_bytes=1 << 40, stream=None)
BWD = dict(dh=P, gu=P, q=P, scale=P, b=4, d_ff=64, act=0, dgu=P, h=P, stream=None)
KEEP = dict(x=P, rows=4, d=64, q=P, scale=P, stream=None)
BACK = dict(q=P, scale=P, rows=4, d=64, x=P, stream=None)
WGRAD = dict(dy=P, q=P, scale=P, b=700, meta=P, d_out=4160, d_in=2112, dw=P, ws=P, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("changed,status", [
    (dict(x=None), NULL), (dict(vals=None), NULL), (dict(meta=None), NULL), (dict(h=None), NULL), (dict(q=None), NULL),
    (dict(scale=None), NULL), (dict(l=None), NULL), (dict(r_=None), NULL), (dict(ws=None), NULL),
    (dict(b=0), SHAPE), (dict(b=1 << 31), SHAPE), (dict(d_ff=0), SHAPE), (dict(d_ff=-8), SHAPE), (dict(d_ff=12), SHAPE),
    (dict(d_ff=(1 << 22) + 8), SHAPE), (dict(d_ff=(1 << 62) + 64), SHAPE), (dict(d_in=4), SHAPE), (dict(d_in=1 << 31), SHAPE), (dict(r=-32), SHAPE),
    (dict(r=33), sl.SLOPE_ERR_UNSUPPORTED), (dict(r=544), sl.SLOPE_ERR_UNSUPPORTED), (dict(act=3), VALUE), (dict(act=-1), VALUE),
    (dict(x=ODD), ALIGN), (dict(h=ODD), ALIGN), (dict(gu=ODD), ALIGN), (dict(q=ODD), ALIGN), (dict(scale=ODD), ALIGN),
    (dict(ws=ODD16), ALIGN), (dict(ws_bytes=0), sl.SLOPE_ERR_WORKSPACE)])
def test_forward_refusals(changed, status):
    assert call("slope_gated_fwd", FWD, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(dh=None), NULL), (dict(dgu=None), NULL), (dict(gu=None, q=None), NULL), (dict(gu=None, scale=None), NULL), (dict(b=0), SHAPE),
    (dict(d_ff=12), SHAPE), (dict(d_ff=(1 << 22) + 8), SHAPE), (dict(b=(1 << 31) - 1, d_ff=1 << 22), SHAPE), (dict(act=7), VALUE), (dict(dh=ODD), ALIGN), (dict(gu=ODD), ALIGN),
    (dict(gu=None, q=ODD), ALIGN), (dict(h=ODD), ALIGN), (dict(dgu=ODD), ALIGN)])
def test_gradient_refusals(changed, status):
    assert call("slope_gated_bwd", BWD, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(rows=0), SHAPE), (dict(rows=1 << 31), SHAPE),
    (dict(d=12), SHAPE), (dict(d=1 << 31), SHAPE), (dict(x=ODD), ALIGN), (dict(q=ODD), ALIGN), (dict(scale=ODD), ALIGN)])
def test_checkpoint_refusals(changed, status):
    assert call("slope_checkpoint_q8", KEEP, **changed) == status
    assert call("slope_restore_q8", BACK, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(dy=None), NULL), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(meta=None), NULL), (dict(dw=None), NULL),
    (dict(ws=None), NULL), (dict(b=0), SHAPE), (dict(d_out=12), SHAPE), (dict(d_in=0), SHAPE), (dict(dy=ODD), ALIGN),
    (dict(scale=ODD), ALIGN), (dict(ws=ODD16), ALIGN), (dict(ws_bytes=0), sl.SLOPE_ERR_WORKSPACE)])
def test_weight_gradient_refusals(changed, status):
    assert call("slope_wgrad_masked_q8", WGRAD, **changed) == status


def test_size_queries():
    lib = sl.lib()
    assert lib.slope_checkpoint_scale_bytes(3, 64) == 6 and lib.slope_checkpoint_scale_bytes(3, 72) == 9
    assert lib.slope_checkpoint_scale_bytes(0, 64) == 0 and lib.slope_checkpoint_scale_bytes(3, 12) == 0
    for b, d_in, d_out in ((1, 64, 64), (700, 2112, 4160), (16384, 9216, 36864)):
        assert lib.slope_wgrad_masked_q8_workspace_bytes(b, d_in, d_out) == lib.slope_workspace_bytes(sl.SLOPE_CALL_WGRAD_MASKED_Q8, b, d_in, d_out, 0)
        assert lib.slope_wgrad_masked_q8_workspace_bytes(b, d_in, d_out) >= (2 * b * d_in if d_in > 64 else 0)
    for b, d_in, d_out in ((1, 64, 64), (300, 2048, 2048), (1000, 1000, 1000)):          # nothing to allocate where X is restored on its way
        assert lib.slope_wgrad_masked_q8_workspace_bytes(b, d_in, d_out) == 0
    for b, d_in, d_ff, r in ((1, 768, 2048, 0), (777, 5120, 13648, 64), (64, 9216, 24576, 128)):
        need = lib.slope_gated_fwd_workspace_bytes(b, d_in, d_ff, r, 8)
        assert need == lib.slope_workspace_bytes(sl.SLOPE_CALL_GATED_FWD, b, d_in, d_ff, r) and need >= 2 * b * r
        assert need == lib.slope_gated_fwd_workspace_bytes(b, d_in, d_ff, r, 16) >= lib.slope_gated_fwd_workspace_bytes(b, d_in, d_ff, r, 0)
        for kept, none in ((8, {}), (0, dict(gu=None, q=None, scale=None))):
            short = lib.slope_gated_fwd_workspace_bytes(b, d_in, d_ff, 64, kept) - 1
            assert call("slope_gated_fwd", FWD, b=b, d_in=d_in, d_ff=d_ff, r=64, ws_bytes=short, **none) == sl.SLOPE_ERR_WORKSPACE
    assert lib.slope_gated_fwd_workspace_bytes(1, 768, 2048, 0, 0) == 0                  # nothing to allocate for the smallest calls
    assert lib.slope_gated_fwd_workspace_bytes(0, 64, 64, 0, 0) == 0 and lib.slope_gated_fwd_workspace_bytes(4, 64, 12, 0, 0) == 0


def test_the_binding_refuses_what_is_not_a_device_matrix():
    x = torch.zeros(4, 64, dtype=sl.BF16)
    for f in (lambda: sl.slope_checkpoint_q8(x), lambda: sl.slope_checkpoint_q8(x[0]), lambda: sl.slope_restore_q8(x, x),
              lambda: sl.slope_gated_bwd(x, gu=x), lambda: sl.slope_gated_bwd(x), lambda: sl.slope_gated_bwd(x, gu=x, q8=x),
              lambda: sl.slope_gated_fwd(x, x, x), lambda: sl.slope_wgrad_masked_q8(x, x, x, x)):
        with pytest.raises(ValueError):
            f()
