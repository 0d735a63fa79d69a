"""Argument checks of the gated linear recurrence, on the CPU: the C entry points
refuse before anything is enqueued, and the binding before the library is
called."""

import ctypes

import pytest
import torch

from paper_1709_02755_amd import lm, sru

OK, E_NULL, E_SHAPE, E_FLAG, E_WS, E_HIP, E_ALIGN = range(7)
FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10002)
B16 = torch.bfloat16
L, B, D = 1000, 2, 8


def forward(**kw):
    a = dict(L=L, B=B, d=D, dtype=1)
    for n in ("x", "r", "i"):
        a.update({n: FAKE, n + "_t": B * D, n + "_b": D})
    a.update(lam=FAKE, c=8.0, h0=None, mask=None, reset=None, H=FAKE, H_t=B * D, H_b=D,
             h_last=None, states=None, ws=FAKE, n=1 << 20)
    a.update(kw)
    return sru.lib().sru_lru_forward(*a.values(), None)


def backward(**kw):
    a = dict(L=L, B=B, d=D, dtype=1)
    for n in ("x", "r", "i"):
        a.update({n: FAKE, n + "_t": B * D, n + "_b": D})
    a.update(lam=FAKE, c=8.0, states=FAKE, dH=FAKE, dH_t=B * D, dH_b=D, dh_last=None, mask=None,
             reset=None)
    for n in ("dx", "dr", "di"):
        a.update({n: FAKE, n + "_t": B * D, n + "_b": D})
    a.update(dlam=FAKE, dh0=None, ws=FAKE, n=1 << 20)
    a.update(kw)
    return sru.lib().sru_lru_backward(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), E_FLAG), (dict(L=0), E_SHAPE), (dict(B=0), E_SHAPE), (dict(d=-1), E_SHAPE),
    (dict(L=1 << 20, B=1 << 12), E_SHAPE), (dict(L=1 << 30, B=1, d=1 << 20), E_SHAPE),
    (dict(c=-1.0), E_SHAPE), (dict(c=float("nan")), E_SHAPE), (dict(c=float("inf")), E_SHAPE),
    (dict(x=None), E_NULL), (dict(r=None), E_NULL), (dict(i=None), E_NULL), (dict(lam=None), E_NULL),
    (dict(x_t=-1), E_SHAPE), (dict(i_b=1 << 41), E_SHAPE), (dict(r=ODD), E_ALIGN),
    (dict(lam=HALF), E_ALIGN), (dict(ws=None), E_WS), (dict(n=64), E_WS), (dict(ws=HALF), E_ALIGN)])
def test_both_calls_check_their_inputs(kw, want):
    assert forward(**kw) == want
    assert backward(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(H=None), E_NULL), (dict(H_t=D), E_SHAPE), (dict(H_b=0), E_SHAPE), (dict(H_b=D - 1), E_SHAPE),
    (dict(H_t=B * D - 1), E_SHAPE), (dict(H_t=D, H_b=(L - 1) * D), E_SHAPE), (dict(H=ODD), E_ALIGN),
    (dict(h_last=HALF), E_ALIGN), (dict(states=HALF), E_ALIGN), (dict(h0=HALF), E_ALIGN)])
def test_forward_refusals(kw, want):
    assert forward(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(states=None), E_NULL), (dict(dH=None), E_NULL), (dict(dx=None), E_NULL),
    (dict(dr=None), E_NULL), (dict(di=None), E_NULL), (dict(dlam=None), E_NULL),
    (dict(dr_t=0), E_SHAPE), (dict(di_b=3), E_SHAPE), (dict(dx=ODD), E_ALIGN),
    (dict(dh_last=HALF), E_ALIGN), (dict(dlam=HALF), E_ALIGN)])
def test_backward_refusals(kw, want):
    assert backward(**kw) == want


def test_workspace_queries():
    f, b = sru.lib().sru_lru_forward_workspace_bytes, sru.lib().sru_lru_backward_workspace_bytes
    assert f(1, 4, 64) == 0 and f(64, 4, 64) == 0        # one workgroup's steps
    assert f(1000, 4, 64) > 0 and f(1000, 4, 64) % 256 == 0
    assert b(1, 4, 64) >= 4 * 4 * 64                     # sums for lam
    assert f(0, 4, 64) == 0 and b(10, 0, 64) == 0


def test_sizes_that_fit_a_launch():
    """What is refused by its size is what no launch takes, not a long sequence of
    many channels."""
    f, b = sru.lib().sru_lru_forward_workspace_bytes, sru.lib().sru_lru_backward_workspace_bytes
    assert b(100000, 64, 2048) == 4 * 64 * 2048 and f(100000, 64, 2048) == 0
    assert b(1, 1 << 23, 1) == 0        # 2^23 workgroups


@pytest.mark.parametrize("L,B,d", [(1, 1, 2 ** 31 - 1), (8, 1, 2 ** 31 - 63), (1, 1, 2 ** 31 - 65),
                                   (1, 3, 2 ** 29), (1, 2 ** 22, 64)])
def test_widths_past_every_launch(L, B, d):
    """Refused before a launch, also where a width rounded up to whole waves is
    no int any more."""
    f, b = sru.lib().sru_lru_forward_workspace_bytes, sru.lib().sru_lru_backward_workspace_bytes
    assert f(L, B, d) == 0 and b(L, B, d) == 0
    size = dict(L=L, B=B, d=d)
    for n in ("x", "r", "i", "H", "dH", "dx", "dr", "di"):
        size.update({n + "_t": B * d, n + "_b": d})
    for call, names in ((forward, "xriH"), (backward, ("x", "r", "i", "dH", "dx", "dr", "di"))):
        kw = {k: v for k, v in size.items() if k in "LBd" or k[:-2] in names}
        assert call(**kw) == E_SHAPE


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


def test_binding(stub):
    L, B, d = 9, 2, 4
    x, lam = torch.zeros((L, B, d), dtype=B16), torch.zeros(d)
    h0, m = torch.zeros((B, d)), torch.zeros((L, B), dtype=torch.uint8)
    fw = lm.lru_forward(x, x, x, lam, h0, mask=m, reset=m)
    assert fw["H"].dtype == B16 and fw["states"].shape == (2, B, d)
    g = lm.lru_backward(x, x, x, lam, fw["states"], x, h0, mask=m)
    assert g["dx"].shape == x.shape and g["dlam"].shape == (d,) and g["dh0"].shape == (B, d)
    # distances: slices of a projection, [B, L, d] memory
    U = torch.zeros((L, B, 3, d), dtype=B16)
    xs, rs, bs = U[:, :, 0], U[:, :, 1], torch.zeros((B, L, d), dtype=B16).transpose(0, 1)
    lm.lru_forward(xs, rs, bs, lam)
    a = stub.calls[-1][1]
    assert a[5:7] == (B * 3 * d, 3 * d) and a[8:10] == (B * 3 * d, 3 * d) and a[11:13] == (d, L * d)
    h = torch.zeros((B, d))
    y = lm.lru_step(U[0, :, 0], U[0, :, 1], U[0, :, 2], lam, h)
    a = stub.calls[-1][1]
    assert y.shape == (B, d) and a[0:3] == (1, B, d) and a[6] == 3 * d
    assert a[15] == a[21] == h.data_ptr()     # the state, in place
    reached = len(stub.calls)
    st = fw["states"]
    bad = [
        lambda: lm.lru_forward(x[0], x, x, lam),
        lambda: lm.lru_forward(x.half(), x, x, lam),
        lambda: lm.lru_forward(x, x.float(), x, lam),
        lambda: lm.lru_forward(x, x, x[:, :1], lam),
        lambda: lm.lru_forward(x, x, None, lam),
        lambda: lm.lru_forward(x.transpose(1, 2), x, x, lam),
        lambda: lm.lru_forward(x, x, torch.zeros((L, d, B), dtype=B16).transpose(1, 2), lam),
        lambda: lm.lru_forward(x, x, x, lam.to(B16)),
        lambda: lm.lru_forward(x, x, x, lam, h0[:1]),
        lambda: lm.lru_forward(x, x, x, lam, mask=m.float()),
        lambda: lm.lru_forward(x, x, x, lam, reset=m[:3]),
        lambda: lm.lru_forward(x, x, x, lam, out=dict(H=x.float())),
        lambda: lm.lru_forward(x, x, x, lam, out=dict(states=st[:1])),
        lambda: lm.lru_forward(x, x, x, lam, ws=lam),
        lambda: lm.lru_backward(x, x, x, lam, st[:1], x),
        lambda: lm.lru_backward(x, x, x, lam, st, x.float()),
        lambda: lm.lru_backward(x, x, x, lam, st, x, h0[0]),
        lambda: lm.lru_backward(x, x, x, lam, st, x, out=dict(dr=x[:4])),
        lambda: lm.lru_step(x, x[0], x[0], lam, h),
        lambda: lm.lru_step(x[0], x[0].float(), x[0], lam, h),
        lambda: lm.lru_step(x[0], x[0], x[0].t(), lam, h),
        lambda: lm.lru_step(x[0], x[0], x[0], lam, h.to(B16)),
        lambda: lm.lru_step(x[0], x[0], x[0], lam, None),
        lambda: lm.lru_step(x[0], x[0], x[0], lam, h, out=h),
        lambda: lm.lru_step(x[0], x[0], x[0], lam, h, mask=m),
        lambda: lm.lru_step(x[0], x[0], x[0], lam, h, reset=m[0].bool()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert len(stub.calls) == reached, i


def test_host_tensors_are_refused():
    x = torch.zeros((2, 1, 8))
    with pytest.raises(ValueError, match="GPU"):
        lm.lru_forward(x, x, x, torch.zeros(8))


@pytest.mark.parametrize("shape", [((1 << 32) + 5, 1, 1), (1, (1 << 32) + 5, 1),
                                   (1, 1, (1 << 32) + 5), (1 << 31, 1, 1)])
def test_sizes_past_32_bits_are_refused(shape, stub):
    """By the binding: the library's sizes are ints.  (Tensors without memory.)"""
    L, B, d = shape
    x, lam = torch.empty(shape, device="meta"), torch.empty(d, device="meta")
    states = torch.empty((-(-L // 8), B, d), device="meta")
    with pytest.raises(ValueError, match="large"):
        lm.lru_forward(x, x, x, lam)
    with pytest.raises(ValueError, match="large"):
        lm.lru_backward(x, x, x, lam, states, x)
    if L == 1:
        with pytest.raises(ValueError, match="large"):
            lm.lru_step(x[0], x[0], x[0], lam, torch.empty((B, d), device="meta"))
    assert stub.calls == []
