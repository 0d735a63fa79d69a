"""Argument checks of the vocabulary row calls, on the CPU: the C entry points
refuse before anything is enqueued, and the binding before the library is
called (a stub library records what is reached)."""

import ctypes

import pytest
import torch

from paper_1709_02755_amd import lm, sru

OK, E_NULL, E_SHAPE, E_FLAG, E_WS, E_HIP, E_ALIGN = range(7)
FAKE = ctypes.c_void_p(0x10000)     # never dereferenced
ODD = ctypes.c_void_p(0x10001)
HALF = ctypes.c_void_p(0x10004)     # 4-byte aligned
NAN, INF = float("nan"), float("inf")


def logprobs(**kw):
    a = dict(z=FAKE, ld=100, dtype=0, tok=FAKE, N=600, V=100, top=0, T=1.0, lp=FAKE, ent=FAKE,
             stats=FAKE, ids=None, tl=None, ws=None, n=0)
    a.update(kw)
    return sru.lib().sru_token_logprobs(a["z"], a["ld"], a["dtype"], a["tok"], a["N"], a["V"],
                                        a["top"], a["T"], a["lp"], a["ent"], a["stats"], a["ids"],
                                        a["tl"], a["ws"], a["n"], None)


def logprobs_backward(**kw):
    a = dict(z=FAKE, ld=100, dtype=0, tok=FAKE, stats=FAKE, ent=FAKE, dlp=FAKE, dent=None,
             ids=None, dtop=None, N=600, V=100, top=0, T=1.0, dz=FAKE, ldd=100)
    a.update(kw)
    return sru.lib().sru_token_logprobs_backward(*a.values(), None)


def distill(name, **kw):
    a = dict(z=FAKE, ld=100, dtype=0, ids=FAKE, t=FAKE, tdtype=0, stats=FAKE, dloss=FAKE, N=600,
             V=100, K=4, T=1.0, loss=FAKE, dz=FAKE, ldd=100, ws=None, n=0)
    a.update(kw)
    front = [a[k] for k in ("z", "ld", "dtype", "ids", "t", "tdtype")]
    size = [a[k] for k in ("N", "V", "K", "T")]
    ws = [a["ws"], a["n"], None]
    lib = sru.lib()
    if name == "forward":
        return lib.sru_distill_forward(*front, *size, a["loss"], a["stats"], *ws)
    if name == "backward":
        return lib.sru_distill_backward(*front, a["stats"], a["dloss"], *size, a["dz"], a["ldd"],
                                        None)
    return lib.sru_distill_forward_backward(*front, a["dloss"], *size, a["loss"], a["stats"],
                                            a["dz"], a["ldd"], *ws)


ROWS = [(dict(dtype=2), E_FLAG), (dict(N=0), E_SHAPE), (dict(V=0), E_SHAPE), (dict(N=-1), E_SHAPE),
        (dict(ld=99), E_SHAPE), (dict(V=1 << 30, ld=1 << 30), E_SHAPE),
        (dict(ld=1 << 40), E_SHAPE), (dict(T=0.0), E_SHAPE), (dict(T=-1.0), E_SHAPE),
        (dict(T=NAN), E_SHAPE), (dict(T=INF), E_SHAPE), (dict(T=1e-45), E_SHAPE),
        (dict(z=None), E_NULL), (dict(z=ctypes.c_void_p(0x10002)), E_ALIGN),
        (dict(z=ODD, dtype=1), E_ALIGN)]


@pytest.mark.parametrize("kw,want", ROWS)
def test_rows_are_checked_by_every_call(kw, want):
    assert logprobs(**kw) == want
    assert logprobs_backward(**kw) == want
    for name in ("forward", "backward", "forward_backward"):
        assert distill(name, **kw) == want


@pytest.mark.parametrize("T", [4e-39, 3.5e-39, 3e-39])
def test_temperatures_whose_exponents_are_no_numbers(T):
    """1 / T is finite here and log2(e) / T, which the kernels use, is not."""
    test_rows_are_checked_by_every_call(dict(T=T), E_SHAPE)


@pytest.mark.parametrize("kw,want", [
    (dict(top=65), E_SHAPE), (dict(top=-1), E_SHAPE), (dict(top=8, V=7, ld=7), E_SHAPE),
    (dict(tok=None), E_NULL), (dict(lp=None), E_NULL), (dict(ent=None), E_NULL),
    (dict(stats=None), E_NULL), (dict(top=1), E_NULL), (dict(top=1, ids=FAKE), E_NULL),
    (dict(tok=HALF), E_ALIGN), (dict(lp=ODD), E_ALIGN), (dict(top=1, ids=HALF, tl=FAKE), E_ALIGN),
    (dict(N=1, V=100000, ld=100000), E_WS), (dict(N=1, V=100000, ld=100000, ws=FAKE, n=16), E_WS),
    (dict(N=1, V=100000, ld=100000, ws=HALF, n=1 << 20), E_ALIGN)])
def test_logprobs_refusals(kw, want):
    assert logprobs(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(ldd=99), E_SHAPE), (dict(dz=None), E_NULL), (dict(dz=ODD), E_ALIGN),
    (dict(tok=None), E_NULL), (dict(stats=None), E_NULL), (dict(dent=FAKE, ent=None), E_NULL),
    (dict(dtop=FAKE), E_SHAPE), (dict(dtop=FAKE, top=3), E_NULL),
    (dict(dtop=FAKE, top=3, ids=HALF), E_ALIGN), (dict(dlp=ODD), E_ALIGN)])
def test_logprobs_backward_refusals(kw, want):
    assert logprobs_backward(**kw) == want


@pytest.mark.parametrize("name", ["forward", "backward", "forward_backward"])
@pytest.mark.parametrize("kw,want", [
    (dict(tdtype=2), E_FLAG), (dict(K=0), E_SHAPE), (dict(K=1025), E_SHAPE),
    (dict(ids=None), E_NULL), (dict(t=None), E_NULL), (dict(ids=HALF), E_ALIGN),
    (dict(t=ODD), E_ALIGN), (dict(stats=None), E_NULL), (dict(stats=ODD), E_ALIGN)])
def test_distill_refusals(name, kw, want):
    assert distill(name, **kw) == want


def test_distill_outputs_and_workspace():
    assert distill("forward", loss=None) == E_NULL
    assert distill("backward", dloss=None) == E_NULL
    assert distill("backward", ldd=9) == E_SHAPE
    assert distill("forward_backward", dz=None) == E_NULL
    few = dict(N=2, V=100000, ld=100000, ldd=100000)
    for name in ("forward", "forward_backward"):
        assert distill(name, **few) == E_WS
        assert distill(name, ws=HALF, n=1 << 20, **few) == E_ALIGN


def test_workspace_queries():
    lib = sru.lib()
    assert lib.sru_token_logprobs_workspace_bytes(1, 100000, 0, 20) % 256 == 0
    assert lib.sru_token_logprobs_workspace_bytes(1, 100000, 0, 20) > 0
    assert lib.sru_token_logprobs_workspace_bytes(4096, 100000, 1, 20) == 0  # a row each
    assert lib.sru_token_logprobs_workspace_bytes(1, 100000, 5, 20) == 0
    assert lib.sru_token_logprobs_workspace_bytes(0, 100000, 0, 0) == 0
    assert lib.sru_distill_workspace_bytes(1, 100000, 0) > 0
    assert lib.sru_distill_workspace_bytes(1, 10, 0) == 0


def test_rows_of_every_count():
    """Counts of rows up to the largest int have a cut (the sums of sizes are
    looked at in the sanitized build)."""
    lib, most = sru.lib(), 2 ** 31 - 1
    for N in (most, most - 510, most - 512):
        for V in (1, 65536, 2 ** 30):
            assert lib.sru_token_logprobs_workspace_bytes(N, V, 1, 20) == 0  # a row each
            assert lib.sru_distill_workspace_bytes(N, V, 0) == 0


class Stub:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 512

        def call(*a):
            self.calls.append(name)
            return 0
        return call


@pytest.fixture
def stub(monkeypatch):
    s = Stub()
    monkeypatch.setattr(sru, "_lib", s)
    monkeypatch.setattr(sru, "_on_gpu", lambda t: True)
    monkeypatch.setattr(sru, "_stream", lambda: None)
    return s


N, V, K = 3, 10, 4


def test_binding_checks_every_tensor(stub):
    z, tok, f = torch.zeros((N, V)), torch.zeros(N, dtype=torch.int64), torch.zeros(N)
    fw = lm.token_logprobs(z, tok, top=2)
    assert stub.calls == ["sru_token_logprobs"]
    assert fw["top_ids"].shape == (N, 2) and fw["stats"].shape == (N, 2)
    ids, t = torch.zeros((N, K), dtype=torch.int64), torch.zeros((N, K))
    stats = torch.zeros((N, 2))
    dtop = torch.zeros((N, 2))
    assert lm.token_logprobs_backward(z, tok, fw, f, f, dtop).shape == (N, V)
    assert lm.distill_forward_backward(z, ids, t, f)["dlogits"].shape == (N, V)
    reached = len(stub.calls)
    bad = [
        lambda: lm.token_logprobs(z.double(), tok),
        lambda: lm.token_logprobs(z[0], tok),
        lambda: lm.token_logprobs(None, tok),
        lambda: lm.token_logprobs(torch.zeros((V, N)).t(), tok),
        lambda: lm.token_logprobs(z[:1].expand(N, V), tok),
        lambda: lm.token_logprobs(z, tok[:2]),
        lambda: lm.token_logprobs(z, tok.int()),
        lambda: lm.token_logprobs(z, tok, temperature=0.0),
        lambda: lm.token_logprobs(z, tok, temperature=float("inf")),
        lambda: lm.token_logprobs(z, tok, out=dict(logprob=torch.zeros(N + 1))),
        lambda: lm.token_logprobs(z, tok, ws=torch.zeros(512)),
        lambda: lm.token_logprobs_backward(z, tok, fw, f[:1]),
        lambda: lm.token_logprobs_backward(z, tok, dict(fw, stats=stats[:1]), f),
        lambda: lm.token_logprobs_backward(z, tok, fw, f, None, torch.zeros((N, 3))),
        lambda: lm.token_logprobs_backward(z, tok, dict(fw, top_ids=None), f, None, dtop),
        lambda: lm.token_logprobs_backward(z, tok, fw, f, dlogits=z.bfloat16()),
        lambda: lm.token_logprobs_backward(z, tok, fw, f, dlogits=torch.zeros((N, V + 1))),
        lambda: lm.distill_forward(z, ids[:, :3], t),
        lambda: lm.distill_forward(z, ids, t.half()),
        lambda: lm.distill_forward(z, ids, torch.zeros((K, N)).t()),
        lambda: lm.distill_backward(z, ids, t, stats[:2], f),
        lambda: lm.distill_backward(z, ids, t, stats, None),
        lambda: lm.distill_forward_backward(z, ids, t, f.double()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert len(stub.calls) == reached, i


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        lm.token_logprobs(torch.zeros((N, V)), torch.zeros(N, dtype=torch.int64))


@pytest.mark.parametrize("top", [-1, 65, 1 << 32, 1 << 40])
def test_alternatives_out_of_range(top, stub):
    """Refused before anything of their size is allocated."""
    with pytest.raises(ValueError, match="top"):
        lm.token_logprobs(torch.zeros((N, V)), torch.zeros(N, dtype=torch.int64), top=top)
    assert stub.calls == []


BIG = (1 << 32) + 5  # cut to 32 bits it is 5


def test_sizes_past_32_bits_are_refused(stub):
    """By the binding: the library's sizes are ints.  (Tensors without memory.)"""
    def z(n, v):
        return torch.empty((n, v), device="meta")

    def i64(*shape):
        return torch.empty(shape, dtype=torch.int64, device="meta")

    for n, v in ((BIG, 1), (1, BIG), (1 << 31, 1)):
        f = torch.empty(n, device="meta")
        fw = dict(stats=z(n, 2), entropy=f, top_ids=None)
        for call in (lambda: lm.token_logprobs(z(n, v), i64(n)),
                     lambda: lm.token_logprobs_backward(z(n, v), i64(n), fw, f),
                     lambda: lm.distill_forward(z(n, v), i64(n, 2), z(n, 2)),
                     lambda: lm.distill_backward(z(n, v), i64(n, 2), z(n, 2), fw["stats"], f),
                     lambda: lm.distill_forward_backward(z(n, v), i64(n, 2), z(n, 2), f)):
            with pytest.raises(ValueError, match="large"):
                call()
    with pytest.raises(ValueError, match="large"):
        lm.distill_forward(z(3, 10), i64(3, BIG), z(3, BIG))
    assert stub.calls == []
