"""Argument checks of the residual norm, on the CPU: the C entry points refuse
before anything is enqueued, and the binding before the library is called."""

import ctypes

import pytest
import torch

from paper_1709_02755_amd import lm, sru

OK, E_NULL, E_SHAPE, E_FLAG, E_WS, E_HIP, E_ALIGN = range(7)
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10002)  # bf16 aligned only


def forward(**kw):
    a = dict(M=4, d=8, dtype=1, res=0, gate=0, eps=1e-6, x=FAKE, ldx=8, y=FAKE, ldy=8, z=FAKE,
             ldz=8, w_post=FAKE, scale=FAKE, w_pre=FAKE, x_out=FAKE, ldxo=8, o=FAKE, ldo=8,
             rstd=FAKE)
    a.update(kw)
    return sru.lib().sru_residual_norm_forward(*a.values(), None)


def backward(**kw):
    a = dict(M=4, d=8, dtype=1, res=0, gate=0, x=FAKE, ldx=8, y=FAKE, ldy=8, z=FAKE, ldz=8,
             w_post=FAKE, scale=FAKE, w_pre=FAKE, rstd=FAKE, dx_out=FAKE, lddxo=8, do=FAKE, lddo=8,
             dx=FAKE, lddx=8, dy=FAKE, lddy=8, dz=FAKE, lddz=8, dw_post=FAKE, dscale=FAKE,
             dw_pre=FAKE, ws=None, n=0)
    a.update(kw)
    return sru.lib().sru_residual_norm_backward(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), E_FLAG), (dict(dtype=0, res=1), E_FLAG), (dict(res=2), E_FLAG),
    (dict(gate=2), E_FLAG), (dict(gate=-1), E_FLAG), (dict(M=0), E_SHAPE), (dict(d=0), E_SHAPE),
    (dict(d=16385), E_SHAPE), (dict(x=None), E_NULL), (dict(ldx=7), E_SHAPE),
    (dict(ldy=7), E_SHAPE), (dict(ldz=1 << 40), E_SHAPE), (dict(x=HALF), E_ALIGN),
    (dict(y=ODD), E_ALIGN), (dict(rstd=None), E_NULL), (dict(scale=HALF), E_ALIGN)])
def test_both_calls_check_their_inputs(kw, want):
    assert forward(**kw) == want
    assert backward(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(eps=0.0), E_SHAPE), (dict(eps=float("nan")), E_SHAPE), (dict(eps=float("inf")), E_SHAPE),
    (dict(x_out=None), E_NULL), (dict(o=None), E_NULL), (dict(w_pre=None), E_NULL),
    (dict(y=None), E_NULL), (dict(y=None, z=None, w_post=None, scale=None), E_NULL),
    (dict(y=None, z=None, w_post=None, scale=None, x_out=None, w_pre=None, o=None), E_NULL),
    (dict(ldo=7), E_SHAPE), (dict(o=ODD), E_ALIGN), (dict(x_out=HALF), E_ALIGN)])
def test_forward_refusals(kw, want):
    assert forward(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dx=None), E_NULL), (dict(dy=None), E_NULL), (dict(dz=None), E_NULL),
    (dict(z=None), E_NULL), (dict(dw_post=None), E_NULL), (dict(w_post=None), E_NULL),
    (dict(scale=None), E_NULL), (dict(dw_pre=None), E_NULL), (dict(lddx=7), E_SHAPE),
    (dict(lddo=7), E_SHAPE), (dict(dz=ODD), E_ALIGN), (dict(dw_pre=HALF), E_ALIGN),
    ({}, E_WS), (dict(ws=FAKE, n=16), E_WS), (dict(ws=HALF, n=1 << 20), E_ALIGN)])
def test_backward_refusals(kw, want):
    assert backward(**kw) == want


def test_workspace_query():
    q = sru.lib().sru_residual_norm_backward_workspace_bytes
    assert q(4, 8) % 256 == 0 and q(4, 8) >= 3 * 8 * 4
    assert q(0, 8) == 0 and q(4, 16385) == 0 and q(-1, 8) == 0
    assert q(1 << 30, 8192) < 64 << 20  # does not grow with the rows


class Stub:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 512

        def call(*a):
            self.calls.append((name, a))
            return 0
        return call


@pytest.fixture
def stub(monkeypatch):
    s = Stub()
    monkeypatch.setattr(sru, "_lib", s)
    monkeypatch.setattr(sru, "_on_gpu", lambda t: True)
    monkeypatch.setattr(sru, "_stream", lambda: None)
    return s


B16 = torch.bfloat16


def test_binding(stub):
    M, d = 3, 8
    x, y, w = torch.zeros((M, d)), torch.zeros((M, d), dtype=B16), torch.zeros(d)
    p = dict(w_post=w, z=y, scale=w, w_pre=w)
    fw = lm.residual_norm_forward(x, y, **p)
    assert fw["x_out"].dtype == torch.float32 and fw["o"].dtype == B16
    assert fw["rstd"].shape == (M, 2)
    g = lm.residual_norm_backward(x, y, fw["rstd"], x, y, **p)
    assert [g[n].dtype for n in ("dx", "dy", "dz", "dw_pre")] == [torch.float32, B16, B16,
                                                                 torch.float32]
    assert lm.residual_norm_forward(x, w_pre=w)["x_out"] is None
    assert lm.residual_norm_forward(x, y)["o"] is None
    # pitches: slices of one projection, leading dimensions, a single row
    wide = torch.zeros((M, 3 * d), dtype=B16)
    lm.residual_norm_forward(x, wide[:, d:2 * d], z=wide[:, :d], w_pre=w)
    a = stub.calls[-1][1]
    assert (a[7], a[9], a[11]) == (d, 3 * d, 3 * d)
    x3, wide3 = torch.zeros((2, 3, d)), torch.zeros((2, 3, 3 * d), dtype=B16)
    lm.residual_norm_forward(x3, wide3[..., d:2 * d])
    assert stub.calls[-1][1][9] == 3 * d and stub.calls[-1][1][0] == 6
    reached = len(stub.calls)
    bad = [
        lambda: lm.residual_norm_forward(x.double(), y),
        lambda: lm.residual_norm_forward(x, y[:, :4]),
        lambda: lm.residual_norm_forward(y, x),                       # bf16 beside fp32
        lambda: lm.residual_norm_forward(x, y, z=x),
        lambda: lm.residual_norm_forward(x, y, w_post=w[:4]),
        lambda: lm.residual_norm_forward(x, y, scale=w.to(B16)),
        lambda: lm.residual_norm_forward(x),                          # nothing to do
        lambda: lm.residual_norm_forward(x, z=y, w_pre=w),            # a gate of nothing
        lambda: lm.residual_norm_forward(x, torch.zeros((d, M), dtype=B16).t()),
        lambda: lm.residual_norm_forward(x, y[:1].expand(M, d)),
        lambda: lm.residual_norm_forward(x3, torch.zeros((2, 4, d), dtype=B16)[:, :3]),
        lambda: lm.residual_norm_forward(x, y, out=dict(x_out=y)),
        lambda: lm.residual_norm_forward(x, y, w_pre=w, out=dict(o=x)),
        lambda: lm.residual_norm_forward(x, y, out=dict(rstd=w)),
        lambda: lm.residual_norm_backward(x, y, w, x, y, **p),
        lambda: lm.residual_norm_backward(x, y, fw["rstd"], y, y, **p),
        lambda: lm.residual_norm_backward(x, y, fw["rstd"], x, x, **p),
        lambda: lm.residual_norm_backward(x, y, fw["rstd"], x, y, **p, out=dict(dy=x)),
        lambda: lm.residual_norm_backward(x, y, fw["rstd"], x, y, **p, ws=w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert len(stub.calls) == reached, i


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        lm.residual_norm_forward(torch.zeros((2, 8)), w_pre=torch.zeros(8))


@pytest.mark.parametrize("shape", [((1 << 32) + 5, 1), (1 << 31, 1), (1 << 16, 1 << 16, 2),
                                   (1, (1 << 32) + 5)])
def test_sizes_past_32_bits_are_refused(shape, stub):
    """By the binding: the library's sizes are ints.  (Tensors without memory.)"""
    x, w = torch.empty(shape, device="meta"), torch.empty(shape[-1], device="meta")
    with pytest.raises(ValueError, match="large"):
        lm.residual_norm_forward(x, x, w_pre=w)
    with pytest.raises(ValueError, match="large"):
        lm.residual_norm_backward(x, x, torch.empty((*shape[:-1], 2), device="meta"), x, x,
                                  w_pre=w)
    assert stub.calls == []


def test_first_norm_of_a_full_precision_residual(stub):
    """The norm of x alone, o in bfloat16 beside a float32 x, as the C call has it."""
    M, d = 3, 8
    x, y, w = torch.zeros((M, d)), torch.zeros((M, d), dtype=B16), torch.zeros(d)
    fw = lm.residual_norm_forward(x, w_pre=w, dtype=B16)
    assert fw["o"].dtype == B16 and fw["x_out"] is None
    assert stub.calls[-1][1][2:4] == (lm.DTYPE_BF16, lm.DTYPE_FP32)
    assert lm.residual_norm_forward(x, w_pre=w, dtype=B16, out=dict(o=y))["o"] is y
    assert lm.residual_norm_forward(y, w_pre=w, dtype=B16)["o"].dtype == B16
    assert lm.residual_norm_forward(x, y, w_pre=w, dtype=B16)["o"].dtype == B16
    assert lm.residual_norm_forward(x, w_pre=w)["o"].dtype == torch.float32
    g = lm.residual_norm_backward(x, None, fw["rstd"], x, y, w_pre=w)
    assert g["dx"].dtype == torch.float32
    assert stub.calls[-1][1][2:4] == (lm.DTYPE_BF16, lm.DTYPE_FP32)
    assert lm.residual_norm_backward(x, None, fw["rstd"], x, w_pre=w)["dx"].dtype == torch.float32
    reached = len(stub.calls)
    bad = [
        lambda: lm.residual_norm_forward(y, w_pre=w, dtype=torch.float32),
        lambda: lm.residual_norm_forward(x, w_pre=w, dtype=torch.half),
        lambda: lm.residual_norm_forward(x, y, w_pre=w, dtype=torch.float32),
        lambda: lm.residual_norm_forward(x, w_pre=w, dtype=B16, out=dict(o=x)),
        lambda: lm.residual_norm_backward(y, None, fw["rstd"], y, x, w_pre=w),
        lambda: lm.residual_norm_backward(x, None, fw["rstd"], y, y, w_pre=w),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert len(stub.calls) == reached, i
