"""Refusals of the norm, 8-bit product and optimizer calls: argument errors are found on the host, before anything is launched
(no GPU needed), each with its own status; size queries; the table of a set of tensors."""
import ctypes
import struct

import pytest
import torch

from paper_2405_16325_amd import binding as sl

P = ctypes.c_void_p(4096)          # aligned, never dereferenced: every call here is refused on the host
ODD = ctypes.c_void_p(4096 + 8)
ODD4 = ctypes.c_void_p(4096 + 2)
INF, NAN = float("inf"), float("nan")


def call(name, args, **changed):
    args = dict(args)
    assert set(changed) <= set(args)
    args.update(changed)
    return getattr(sl.lib(), name)(*args.values())


FWD = dict(x=P, res=P, w=P, b=4, d=64, eps=1e-5, h=P, y=P, rstd=P, q=P, scale=P, stream=None)
BWD = dict(dy=P, h=P, w=P, rstd=P, dh=P, b=4, d=64, dx=P, dw=P, ws=P, ws_bytes=1 << 30, stream=None)
QUANT = dict(vals=P, d_out=8, d_in=64, q=P, scale=P, stream=None)
Q8 = dict(q=P, xs=P, b=4, wq=P, meta=P, ws=P, d_out=64, d_in=64, add=P, y=P, scratch=P, scratch_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("changed,status", [
    (dict(x=None), sl.SLOPE_ERR_NULL), (dict(w=None), sl.SLOPE_ERR_NULL), (dict(y=None, q=None, scale=None), sl.SLOPE_ERR_NULL),
    (dict(h=None), sl.SLOPE_ERR_NULL), (dict(res=None), sl.SLOPE_ERR_NULL), (dict(q=None), sl.SLOPE_ERR_NULL),
    (dict(scale=None), sl.SLOPE_ERR_NULL), (dict(b=0), sl.SLOPE_ERR_SHAPE), (dict(b=-1), sl.SLOPE_ERR_SHAPE),
    (dict(b=1 << 31), sl.SLOPE_ERR_SHAPE), (dict(d=0), sl.SLOPE_ERR_SHAPE), (dict(d=12), sl.SLOPE_ERR_SHAPE),
    (dict(d=1 << 24), sl.SLOPE_ERR_SHAPE), (dict(x=ODD), sl.SLOPE_ERR_ALIGN), (dict(res=ODD), sl.SLOPE_ERR_ALIGN),
    (dict(q=ODD), sl.SLOPE_ERR_ALIGN), (dict(scale=ODD), sl.SLOPE_ERR_ALIGN), (dict(rstd=ODD), sl.SLOPE_ERR_ALIGN),
    (dict(eps=0.0), sl.SLOPE_ERR_VALUE), (dict(eps=-1.0), sl.SLOPE_ERR_VALUE), (dict(eps=NAN), sl.SLOPE_ERR_VALUE),
    (dict(eps=INF), sl.SLOPE_ERR_VALUE), (dict(eps=1e-60), sl.SLOPE_ERR_VALUE)])
def test_norm_refusals(changed, status):
    assert call("slope_rmsnorm_fwd", FWD, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(dy=None), sl.SLOPE_ERR_NULL), (dict(rstd=None), sl.SLOPE_ERR_NULL), (dict(dw=None), sl.SLOPE_ERR_NULL),
    (dict(ws=None), sl.SLOPE_ERR_NULL), (dict(b=0), sl.SLOPE_ERR_SHAPE), (dict(d=20), sl.SLOPE_ERR_SHAPE),
    (dict(dh=ODD), sl.SLOPE_ERR_ALIGN), (dict(ws=ctypes.c_void_p(4096 + 16)), sl.SLOPE_ERR_ALIGN),
    (dict(ws_bytes=0), sl.SLOPE_ERR_WORKSPACE)])
def test_norm_gradient_refusals(changed, status):
    assert call("slope_rmsnorm_bwd", BWD, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(vals=None), sl.SLOPE_ERR_NULL), (dict(scale=None), sl.SLOPE_ERR_NULL), (dict(d_out=0), sl.SLOPE_ERR_SHAPE),
    (dict(d_in=12), sl.SLOPE_ERR_SHAPE), (dict(q=ODD), sl.SLOPE_ERR_ALIGN)])
def test_quantize_refusals(changed, status):
    assert call("slope_quantize_packed", QUANT, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(q=None), sl.SLOPE_ERR_NULL), (dict(xs=None), sl.SLOPE_ERR_NULL), (dict(meta=None), sl.SLOPE_ERR_NULL),
    (dict(ws=None), sl.SLOPE_ERR_NULL), (dict(y=None), sl.SLOPE_ERR_NULL), (dict(b=0), sl.SLOPE_ERR_SHAPE),
    (dict(d_out=12), sl.SLOPE_ERR_SHAPE), (dict(d_in=4), sl.SLOPE_ERR_SHAPE), (dict(d_in=1 << 31), sl.SLOPE_ERR_SHAPE),
    (dict(wq=ODD), sl.SLOPE_ERR_ALIGN), (dict(add=ODD), sl.SLOPE_ERR_ALIGN), (dict(y=ODD), sl.SLOPE_ERR_ALIGN),
    (dict(scratch=ctypes.c_void_p(4096 + 128)), sl.SLOPE_ERR_ALIGN)])
def test_product_refusals(changed, status):
    assert call("slope_spmm_fwd_q8", Q8, **changed) == status


def test_size_queries():
    lib = sl.lib()
    assert lib.slope_rmsnorm_bwd_workspace_bytes(4, 64) >= 64 * 4 and lib.slope_rmsnorm_bwd_workspace_bytes(4, 64) % 256 == 0
    assert lib.slope_rmsnorm_bwd_workspace_bytes(0, 64) == 0 and lib.slope_rmsnorm_bwd_workspace_bytes(4, 12) == 0
    assert lib.slope_workspace_bytes(sl.SLOPE_CALL_RMSNORM_BWD, 100, 768, 0, 0) == lib.slope_rmsnorm_bwd_workspace_bytes(100, 768)
    for b, d_in, d_out in ((1, 9216, 36864), (64, 36864, 9216), (777, 5120, 20480)):
        assert lib.slope_workspace_bytes(sl.SLOPE_CALL_SPMM_FWD_Q8, b, d_in, d_out, 0) == lib.slope_spmm_fwd_q8_workspace_bytes(b, d_in, d_out)
    assert lib.slope_spmm_fwd_q8_workspace_bytes(0, 64, 64) == 0
    assert b"scalar" in lib.slope_status_string(sl.SLOPE_ERR_VALUE)


def tensor(**changed):
    t = sl.AdamWTensor(4096, 8192, 12288, 16384, 20480, 24576, 28672, 1000, 0.1, 16)
    for k, v in changed.items():
        setattr(t, k, v)
    return t


def table_of(*tensors, bits=32, room=None):
    array = (sl.AdamWTensor * len(tensors))(*tensors)
    need = sl.lib().slope_adamw_table_bytes(array, len(tensors))
    host = torch.zeros(max(need, 64) if room is None else room, dtype=torch.uint8)
    return sl.lib().slope_adamw_table(array, len(tensors), bits, host.data_ptr(), host.numel()), host, need


@pytest.mark.parametrize("changed,bits,status", [
    (dict(param=None, master=None), 32, sl.SLOPE_ERR_NULL), (dict(grad=None), 32, sl.SLOPE_ERR_NULL), (dict(m=None), 32, sl.SLOPE_ERR_NULL),
    (dict(v=None), 8, sl.SLOPE_ERR_NULL), (dict(m_scale=None), 8, sl.SLOPE_ERR_NULL), (dict(v_scale=None), 8, sl.SLOPE_ERR_NULL),
    (dict(n=-1), 32, sl.SLOPE_ERR_SHAPE), (dict(n=1 << 41), 32, sl.SLOPE_ERR_SHAPE), (dict(grad=4104), 32, sl.SLOPE_ERR_ALIGN),
    (dict(m=4104), 32, sl.SLOPE_ERR_ALIGN), (dict(v_scale=4098), 8, sl.SLOPE_ERR_ALIGN), (dict(grad_bits=8), 32, sl.SLOPE_ERR_UNSUPPORTED),
    (dict(weight_decay=NAN), 32, sl.SLOPE_ERR_VALUE), (dict(weight_decay=INF), 8, sl.SLOPE_ERR_VALUE)])
def test_table_refusals(changed, bits, status):
    good, host, _ = table_of(tensor(), tensor(n=5), bits=bits)
    assert good == sl.SLOPE_OK
    assert table_of(tensor(), tensor(**changed), bits=bits, room=4096)[0] == status


def test_tables():
    assert table_of(tensor(), bits=16)[0] == sl.SLOPE_ERR_UNSUPPORTED
    assert table_of(tensor(n=10 ** 6), room=64)[0] == sl.SLOPE_ERR_WORKSPACE
    assert sl.lib().slope_adamw_table_bytes(None, 3) == 0 and sl.lib().slope_adamw_table(None, 1, 32, 4096, 64) == sl.SLOPE_ERR_NULL
    # optional pointers, and nothing asked of a tensor without elements
    assert table_of(tensor(param=None), tensor(master=None, m_scale=None, v_scale=None), sl.AdamWTensor())[0] == sl.SLOPE_OK
    # every chunk of every tensor is listed once, and the tensors as they were given
    sizes = [4096, 0, 1, 4097, 12288]
    status, host, need = table_of(*(tensor(n=n) for n in sizes))
    assert status == sl.SLOPE_OK
    raw = host.numpy().tobytes()
    step = ctypes.sizeof(sl.AdamWTensor)
    listed = [struct.unpack_from("<ii", raw, at) for at in range(64 + len(sizes) * step, need, 8)]
    assert listed == [(i, k) for i, n in enumerate(sizes) for k in range((n + 4095) // 4096)]
    assert [sl.AdamWTensor.from_buffer_copy(raw, 64 + i * step).n for i in range(len(sizes))] == sizes


NORM = dict(table=None, device=P, inv=1.0, most=1.0, control=P, ws=P, ws_bytes=1 << 20, stream=None)
STEP = dict(table=None, device=P, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, scale=1.0, step=1, control=None, stream=None)


def test_step_and_norm_refusals():
    _, host, _ = table_of(tensor())
    good = host.data_ptr()
    for name, args in (("slope_grad_norm", NORM), ("slope_adamw_step", STEP)):
        assert call(name, args) == sl.SLOPE_ERR_NULL                                  # no table
        assert call(name, args, table=good, device=None) == sl.SLOPE_ERR_NULL
        assert call(name, args, table=good, device=ODD) == sl.SLOPE_ERR_ALIGN
        assert call(name, args, table=good, control=ODD) == sl.SLOPE_ERR_ALIGN
        blank = torch.zeros(64, dtype=torch.uint8)
        assert call(name, args, table=blank.data_ptr()) == sl.SLOPE_ERR_UNSUPPORTED   # not a table
    for changed, status in ((dict(control=None), sl.SLOPE_ERR_NULL), (dict(ws=None), sl.SLOPE_ERR_NULL),
                            (dict(ws=ctypes.c_void_p(4096 + 16)), sl.SLOPE_ERR_ALIGN), (dict(inv=0.0), sl.SLOPE_ERR_VALUE),
                            (dict(inv=INF), sl.SLOPE_ERR_VALUE), (dict(most=0.0), sl.SLOPE_ERR_VALUE), (dict(most=NAN), sl.SLOPE_ERR_VALUE),
                            (dict(ws_bytes=0), sl.SLOPE_ERR_WORKSPACE)):
        assert call("slope_grad_norm", NORM, table=good, **changed) == status, changed
    for changed in (dict(lr=-1.0), dict(lr=INF), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=NAN), dict(eps=0.0), dict(eps=INF),
                    dict(step=0), dict(step=(1 << 24) + 1), dict(scale=INF), dict(scale=NAN)):
        assert call("slope_adamw_step", STEP, table=good, **changed) == sl.SLOPE_ERR_VALUE, changed


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        sl.slope_rmsnorm_fwd(x, x[0], 1e-5)
    with pytest.raises(ValueError, match="matrix"):
        sl.slope_rmsnorm_fwd(x[0], x[0], 1e-5)
    with pytest.raises(ValueError, match="device"):
        sl.slope_rmsnorm_bwd(x, x, x[0], x[:, 0].float())
    with pytest.raises(ValueError, match="device"):
        sl.slope_quantize_packed(x)
    q = x.to(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="device"):
        sl.slope_spmm_fwd_q8(q, x[:, 0].float(), q, q.view(torch.uint8)[:, :16], x[:, 0].float())
    g = torch.zeros(8)
    with pytest.raises(ValueError, match="entry"):
        sl.slope_adamw_plan([x], [g, g], [g], [g])
    with pytest.raises(ValueError, match="entry"):
        sl.slope_adamw_plan([], [], [], [])
    with pytest.raises(ValueError, match="both missing"):
        sl.slope_adamw_plan(None, [g], [g], [g])
    with pytest.raises(ValueError, match="grads"):
        sl.slope_adamw_plan([g], [g.half()], [g], [g])
    with pytest.raises(ValueError, match="device"):
        sl.slope_adamw_plan(None, [g], [g], [g], masters=[g])


@pytest.mark.parametrize("eps", [1e-39, 1e-44, 2.0 ** -126 - 2.0 ** -149, 2.0 ** 125 * (1 + 2.0 ** -23), 3e38])
def test_an_optimizer_eps_whose_reciprocal_fp32_does_not_hold(eps):
    """Below the smallest normal number the step's reciprocal is infinite, and an element without a gradient became 0 x infinity;
    past 2^126 it is subnormal and would be taken for zero."""
    _, host, _ = table_of(tensor())
    assert call("slope_adamw_step", STEP, table=host.data_ptr(), eps=eps) == sl.SLOPE_ERR_VALUE


@pytest.mark.parametrize("scale", [3.5e38, -3.5e38, 1e300])
def test_a_gradient_scale_that_is_infinite_in_fp32(scale):
    _, host, _ = table_of(tensor())
    assert call("slope_adamw_step", STEP, table=host.data_ptr(), scale=scale) == sl.SLOPE_ERR_VALUE
