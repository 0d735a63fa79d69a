"""Vocabulary rows on the GPU against a plain 64-bit implementation: log
probabilities, entropy and top alternatives, distillation, their gradients.

Tolerances.  fp32 results: x = (z - max) / T carries two roundings, so a term
e^x is off by 2^-23 |x| + 2^-23 relative, |x| <= 60 where it counts (below, e^x
adds less than 2^-80); a sum over a row adds (V / 512 + 16) 2^-24.  With V <=
70,001 that is below 2e-5 of a term of weight 1; log probabilities and
entropies are then within 2e-5 + 1e-6 |value|, gradients within 2e-5 of the
largest weight in the row.  bf16 gradients add half a step of bf16: 8 significant
bits, so up to 2^-8 of the value."""

import math

import pytest
import torch

from paper_1709_02755_amd import lm, sru

pytestmark = pytest.mark.gpu

INF = math.inf
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: -3.3895313892515355e38}


def rows(N, V, dtype, seed, ties=False, pitch=None, offset=0):
    """Random logits on the GPU, in memory of the given pitch and offset."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((N, V), generator=g, dtype=torch.float64) * 3
    if ties:
        z = torch.round(z * 2) / 2  # many equal values, and zeros of both signs
    z = z.to(dtype)
    pitch = V if pitch is None else pitch
    buf = torch.full((N * pitch + offset + 16,), float("nan"), dtype=dtype)
    view = buf.cuda()[offset:offset + N * pitch].view(N, pitch)[:, :V]
    view.copy_(z)
    return view


def plain(z, tokens, top, T):
    """logprob, entropy, top_ids, top_logprobs, log p and p in 64 bits on the CPU."""
    z = z.detach().cpu().double()
    N, V = z.shape
    m = z.max(1, keepdim=True)[0]
    empty = m == -INF
    x = torch.where(empty, -INF, (z - torch.where(empty, 0.0, m)) / T)
    S = torch.exp(x).sum(1, keepdim=True)
    lp = torch.where(empty, -INF, x - torch.log(S))
    p = torch.where(empty, 0.0, torch.exp(x) / S)
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    bad = torch.isnan(z).any(1) | (z == INF).any(1)
    lp[bad], p[bad], ent[bad] = math.nan, math.nan, math.nan
    tok = tokens.cpu()
    ok = (tok >= 0) & (tok < V)
    logprob = torch.where(ok, lp.gather(1, tok.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    ids, tl = [], []
    for n in range(N):
        row = z[n].tolist()
        order = sorted((j for j in range(V) if row[j] == row[j]), key=lambda j: (-row[j], j))[:top]
        ids.append(order + [-1] * (top - len(order)))
        tl.append([float(lp[n, j]) for j in order] + [-INF] * (top - len(order)))
    return (logprob, ent, torch.tensor(ids, dtype=torch.int64).reshape(N, top),
            torch.tensor(tl, dtype=torch.float64).reshape(N, top), lp, p)


def close(name, got, ref, scale=None, bf16=False):
    # results are fp32: a log probability beyond its range is infinite
    got, ref = got.detach().cpu().double(), ref.float().double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), name
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), name
    ok = torch.isfinite(ref)
    tol = 2e-5 * (1.0 if scale is None else scale.expand_as(ref)[ok]) + 1e-6 * ref[ok].abs()
    if bf16:
        tol = tol + 2.0 ** -8 * ref[ok].abs()
    err = (got[ok] - ref[ok]).abs()
    assert bool((err <= tol).all()), (name, float((err - tol).max()))


def run_logprobs(z, tokens, top, T, **kw):
    fw = lm.token_logprobs(z, tokens, top=top, temperature=T, **kw)
    torch.cuda.synchronize()
    return fw


def check_logprobs(z, tokens, top, T):
    fw = run_logprobs(z, tokens, top, T)
    lp, ent, ids, tl, _, _ = plain(z, tokens, top, T)
    close("logprob", fw["logprob"], lp)
    close("entropy", fw["entropy"], ent)
    if top:
        assert torch.equal(fw["top_ids"].cpu(), ids)
        close("top_logprobs", fw["top_logprobs"], tl)
    else:
        assert fw["top_ids"] is None
    return fw


def grad_plain(z, tokens, ids, lp, p, ent, dlp, dent, dtop, T):
    N, V = z.shape
    tok = tokens.cpu()
    up = torch.zeros((N, V), dtype=torch.float64)
    for n in range(N):
        if dlp is not None and 0 <= tok[n] < V:
            up[n, tok[n]] += float(dlp[n])
        if dtop is not None:
            for k in range(dtop.shape[1]):
                if ids[n, k] >= 0:
                    up[n, ids[n, k]] += float(dtop[n, k])
    dz = up - p * up.sum(1, keepdim=True)
    if dent is not None:
        dz = dz - dent.cpu().double()[:, None] * torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
    empty = (z.detach().cpu().double() == -INF).all(1)
    dz[empty] = 0.0
    return dz / T


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 8), (3, 9), (2, 64), (4, 65), (3, 1000), (2, 4095), (3, 4097),
          (1, 30011), (2, 70001), (700, 257), (600, 5003)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", SHAPES)
def test_logprobs_and_gradient(N, V, dtype):
    g = torch.Generator().manual_seed(N * 100003 + V)
    tokens = torch.randint(-1, V + 1, (N,), generator=g).cuda()  # some outside the vocabulary
    top = min(V, 20) if N < 100 else min(V, 3)
    T = (1.0, 0.7, 2.0)[V % 3]
    z = rows(N, V, dtype, V, ties=V % 2 == 0)
    fw = check_logprobs(z, tokens, top, T)
    _, ent, ids, _, lp, p = plain(z, tokens, top, T)
    dlp, dent = torch.randn(N, generator=g), torch.randn(N, generator=g) * 0.1
    dtop = torch.randn((N, top), generator=g)
    for use in ((dlp, None, None), (dlp, dent, dtop), (None, dent, None), (None, None, dtop)):
        up = [None if t is None else t.cuda() for t in use]
        got = lm.token_logprobs_backward(z, tokens, fw, *up, temperature=T)
        ref = grad_plain(z, tokens, ids, lp, p, ent, *use, T)
        weight = sum(t.double().abs().reshape(N, -1).sum(1) for t in use if t is not None)
        close("dlogits", got, ref, (weight / T * (1 + ent.abs()))[:, None], dtype == torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(2, 64), (3, 5003), (2, 70001)])
def test_most_alternatives_and_their_gradient(N, V, dtype):
    T, top = 1.2, lm.MAX_TOP
    g = torch.Generator().manual_seed(V)
    tokens = torch.randint(0, V, (N,), generator=g).cuda()
    z = rows(N, V, dtype, V + 1)
    fw = check_logprobs(z, tokens, top, T)
    _, ent, ids, _, lp, p = plain(z, tokens, top, T)
    tokens[0] = ids[0, 5]  # one of the alternatives
    dlp, dtop = torch.randn(N, generator=g), torch.randn((N, top), generator=g)
    got = lm.token_logprobs_backward(z, tokens, fw, dlp.cuda(), None, dtop.cuda(), temperature=T)
    ref = grad_plain(z, tokens, ids, lp, p, ent, dlp, None, dtop, T)
    weight = dlp.double().abs() + dtop.double().abs().sum(1)
    close("dlogits", got, ref, (weight / T)[:, None], dtype == torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pitch,offset", [(1003, 1), (1003, 5), (1008, 3), (1001, 0)])
def test_strided_rows(pitch, offset, dtype):
    """Rows whose starts differ in alignment, read and written in place and
    into memory of another alignment; nothing between the rows is touched."""
    N, V, T = 6, 1001, 0.9
    z = rows(N, V, dtype, 5, pitch=pitch, offset=offset)
    tokens = torch.tensor([0, 1000, 7, -1, 500, 993]).cuda()
    fw = check_logprobs(z, tokens, 7, T)
    _, ent, ids, _, lp, p = plain(z, tokens, 7, T)
    dlp, dtop = torch.linspace(-1, 1, N), torch.linspace(-1, 1, N * 7).reshape(N, 7)
    ref = grad_plain(z, tokens, ids, lp, p, ent, dlp, None, dtop, T)
    scale = ((dlp.abs() + dtop.abs().sum(1)) / T)[:, None].double()
    fresh = lm.token_logprobs_backward(z, tokens, fw, dlp.cuda(), None, dtop.cuda(), temperature=T)
    close("dlogits", fresh, ref, scale, dtype == torch.bfloat16)
    shifted = rows(N, V, dtype, 6, pitch=pitch + 1, offset=offset + 1)
    lm.token_logprobs_backward(z, tokens, fw, dlp.cuda(), None, dtop.cuda(), temperature=T,
                               dlogits=shifted)
    assert torch.equal(shifted, fresh)
    lm.token_logprobs_backward(z, tokens, fw, dlp.cuda(), None, dtop.cuda(), temperature=T,
                               dlogits=z)
    assert torch.equal(z, fresh)
    gap = z.as_strided((N - 1, pitch - V), (pitch, 1), z.storage_offset() + V)
    assert bool(torch.isnan(gap).all())


def special_rows(V, dtype):
    """Rows that go wrong: nothing possible, one token possible, the type's
    lowest value everywhere and in places, NaN, +inf, no padding, huge values."""
    z = torch.randn((9, V), generator=torch.Generator().manual_seed(3))
    z[0] = -INF
    z[1] = -INF
    z[1, V // 2] = 1.5
    z[2] = LOWEST[dtype]
    z[3, V // 3:] = LOWEST[dtype]
    z[4, V - 1] = math.nan
    z[5, 0] = INF
    z[6, ::2] = -INF
    z[7] = 1e30 * z[7]
    return z.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,T", [(33, 0.5), (5000, 1.0), (70000, 0.3)])
def test_special_rows(V, T, dtype):
    z = special_rows(V, dtype)
    N = z.shape[0]
    tokens = torch.full((N,), V // 2).cuda()
    top = 6
    fw = check_logprobs(z, tokens, top, T)
    _, ent, ids, _, lp, p = plain(z, tokens, top, T)
    dlp, dent = torch.ones(N), torch.full((N,), 0.5)
    got = lm.token_logprobs_backward(z, tokens, fw, dlp.cuda(), dent.cuda(), temperature=T).cpu()
    ref = grad_plain(z, tokens, ids, lp, p, ent, dlp, dent, None, T)
    fine = torch.tensor([0, 1, 2, 3, 6, 7, 8])
    scale = ((1 + ent.abs()) / T)[:, None]
    close("dlogits", got[fine], ref[fine], scale[fine], dtype == torch.bfloat16)
    assert bool((got[0] == 0).all())  # nothing possible: nothing to learn
    assert bool(torch.isnan(got[4]).any()) and bool(torch.isnan(got[5]).any())


@pytest.mark.parametrize("order", ["up", "down", "equal"])
@pytest.mark.parametrize("top", [1, 5, 64])
def test_top_of_ordered_rows(order, top):
    """Every value better than all before it, every one worse, all alike."""
    V = 20001
    z = torch.arange(V, dtype=torch.float32) / 1000
    z = {"up": z, "down": z.flip(0), "equal": torch.zeros(V)}[order]
    z = torch.stack([z, z]).cuda()
    fw = check_logprobs(z, torch.tensor([0, 1]).cuda(), top, 1.0)
    want = list(range(V))[::-1][:top] if order == "up" else list(range(top))
    assert fw["top_ids"][0].tolist() == want


def teacher(N, V, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] if K <= V else
                       torch.randint(0, V, (K,), generator=g) for _ in range(N)])
    t = torch.randn((N, K), generator=g) * 2
    return ids, t.to(dtype)


def distill_plain(z, ids, t, dloss, T):
    z, t = z.detach().cpu().double(), t.cpu().double()
    N, V = z.shape
    _, _, _, _, lp, q = plain(z, torch.zeros(N, dtype=torch.int64), 0, T)
    loss, dz = torch.zeros(N, dtype=torch.float64), torch.zeros_like(z)
    for n in range(N):
        kept = [k for k in range(ids.shape[1]) if 0 <= ids[n, k] < V and t[n, k] != -INF]
        if not kept:
            continue
        p = torch.softmax(t[n, kept] / T, 0)
        for pk, k in zip(p.tolist(), kept):
            if pk > 0:
                loss[n] += pk * (math.log(pk) - float(lp[n, ids[n, k]]))
        if bool((z[n] == -INF).all()):
            continue
        dz[n] = q[n]
        for pk, k in zip(p.tolist(), kept):
            dz[n, ids[n, k]] -= pk
        dz[n] *= float(dloss[n]) / T
    return loss, dz


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (2, 7, 3), (3, 64, 64), (4, 65, 9), (2, 4097, 128),
                                   (3, 300, 1024), (1, 70001, 17), (700, 257, 5), (600, 5003, 40)])
def test_distill(N, V, K, dtype):
    T = (1.0, 2.0, 0.8)[K % 3]
    z = rows(N, V, dtype, V + K)
    tt = torch.float32 if N % 2 else dtype
    ids, t = teacher(N, V, K, tt, K)
    ids[0, K // 2:] = -1          # cut
    if N > 1:
        t[1, 0] = -INF            # no probability
        ids[1, K - 1] = V         # outside the vocabulary
        ids[-1] = ids[-1, 0]      # one id K times
    dloss = torch.linspace(-1, 2, N) if N > 1 else torch.tensor([0.7])
    loss, dz = distill_plain(z, ids, t, dloss, T)
    args = z, ids.cuda(), t.cuda()
    fw = lm.distill_forward(*args, temperature=T)
    close("loss", fw["loss"], loss)
    got = lm.distill_backward(*args, fw["stats"], dloss.cuda(), temperature=T)
    scale = (dloss.abs() / T)[:, None].double()
    close("dlogits", got, dz, scale, dtype == torch.bfloat16)
    both = lm.distill_forward_backward(*args, dloss.cuda(), temperature=T)
    for n in ("loss", "stats"):
        assert torch.equal(both[n], fw[n]), n
    assert torch.equal(both["dlogits"], got)
    # in place, over strided rows
    zs = rows(N, V, dtype, V + K, pitch=V + 3, offset=2)
    lm.distill_forward_backward(zs, *args[1:], dloss.cuda(), temperature=T, dlogits=zs)
    close("in place", zs, dz, scale, dtype == torch.bfloat16)


def test_distill_special_rows():
    V, T = 3000, 0.5
    z = special_rows(V, torch.float32)
    N = z.shape[0]
    ids, t = teacher(N, V, 8, torch.float32, 9)
    ids[1, 0] = V // 2
    ids[8] = -1
    dloss = torch.ones(N)
    loss, dz = distill_plain(z, ids, t, dloss, T)
    both = lm.distill_forward_backward(z, ids.cuda(), t.cuda(), dloss.cuda(), temperature=T)
    got, gl = both["dlogits"].cpu(), both["loss"].cpu().double()
    assert gl[0] == INF and gl[1] == INF and gl[8] == 0
    assert math.isnan(gl[4]) and math.isnan(gl[5])
    fine = torch.tensor([2, 7, 8])
    # row 7: logits of 1e30, a difference of two of them rounds at 1e30 2^-24 / T
    assert bool(torch.isfinite(gl[fine]).all())
    close("loss", gl[torch.tensor([2, 8])], loss[torch.tensor([2, 8])])
    keep = torch.tensor([0, 1, 2, 3, 6, 7, 8])
    close("dlogits", got[keep], dz[keep], torch.full((7, 1), 1 / T, dtype=torch.float64))
    assert bool((got[0] == 0).all()) and bool((got[8] == 0).all())
    # a teacher with a NaN logit
    t[2, 3] = math.nan
    assert math.isnan(float(lm.distill_forward(z, ids.cuda(), t.cuda())["loss"][2]))


def test_gradients_against_differences():
    """Central differences of the 64-bit functions along random directions."""
    N, V, K, T, eps = 4, 37, 5, 0.8, 1e-5
    g = torch.Generator().manual_seed(11)
    z = torch.randn((N, V), generator=g)
    tokens = torch.tensor([3, 36, 0, 7])
    ids, t = teacher(N, V, K, torch.float32, 12)
    dlp, dent = torch.randn(N, generator=g), torch.randn(N, generator=g)
    dtop = torch.randn((N, K), generator=g)
    fw = lm.token_logprobs(z.cuda(), tokens.cuda(), top=K, temperature=T)
    got = lm.token_logprobs_backward(z.cuda(), tokens.cuda(), fw, dlp.cuda(), dent.cuda(),
                                     dtop.cuda(), temperature=T).cpu().double()
    both = lm.distill_forward_backward(z.cuda(), ids.cuda(), t.cuda(), dlp.cuda(), temperature=T)

    def f(zz):
        lp, ent, _, tl, _, _ = plain(zz, tokens, K, T)
        return float((dlp * lp).sum() + (dent * ent).sum() + (dtop * tl).sum())

    def h(zz):
        return float((dlp * distill_plain(zz, ids, t, dlp, T)[0]).sum())

    for _ in range(4):
        d = torch.randn((N, V), generator=g, dtype=torch.float64)
        for fn, grad in ((f, got), (h, both["dlogits"].cpu().double())):
            slope = (fn(z.double() + eps * d) - fn(z.double() - eps * d)) / (2 * eps)
            assert abs(slope - float((grad * d).sum())) <= 1e-4 * (1 + abs(slope))


def test_same_bits_on_another_stream_and_in_a_graph():
    """Two calls, one on a side stream, and replays of a captured call (with
    other work between them) give the same bits."""
    N, V, K, T = 3, 50001, 12, 1.3
    z = rows(N, V, torch.bfloat16, 8)
    tokens = torch.tensor([5, -1, 50000]).cuda()
    ids, t = (a.cuda() for a in teacher(N, V, K, torch.float32, 2))
    dl = torch.tensor([0.5, -1.0, 2.0]).cuda()

    def step(zz):
        fw = lm.token_logprobs(zz, tokens, top=20, temperature=T)
        g = lm.token_logprobs_backward(zz, tokens, fw, dl, dl, temperature=T)
        b = lm.distill_forward_backward(zz, ids, t, dl, temperature=T)
        return [fw["logprob"], fw["entropy"], fw["top_ids"], fw["top_logprobs"], g, b["loss"],
                b["dlogits"]]

    want = [v.clone() for v in step(z)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step(z)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(z)
    for _ in range(3):
        step(rows(N, V, torch.bfloat16, 9))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held))


def test_rows_past_32_bits():
    """Rows that start past 2^31 elements and past 2^32 bytes."""
    V, pitch = 1000, 1 << 28
    buf = torch.zeros((9 * pitch + 1000,), dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((10, V), (pitch, 1))
    z.copy_(rows(10, V, torch.bfloat16, 4))
    tokens = torch.arange(10).cuda()
    fw = check_logprobs(z, tokens, 3, 1.0)
    dlp = torch.ones(10).cuda()
    ref = lm.token_logprobs_backward(z.contiguous(), tokens, fw, dlp)
    lm.token_logprobs_backward(z, tokens, fw, dlp, dlogits=z)
    assert torch.equal(z, ref)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 64])
def test_more_rows_than_a_launch_has_workgroups(V, dtype):
    """Rows that a workgroup comes to after its first: the bits of the same rows in
    a call of their own."""
    N, K, T, last = (1 << 20) + 37, 3, 0.8, 50
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn((N, V), generator=g, device="cuda").to(dtype)
    tokens = torch.randint(-1, V, (N,), generator=g, device="cuda")
    ids = torch.randint(-1, V, (N, K), generator=g, device="cuda")
    t = torch.randn((N, K), generator=g, device="cuda")
    dl = torch.randn(N, generator=g, device="cuda")
    dtop = torch.randn((N, K), generator=g, device="cuda")

    def step(z, tokens, ids, t, dl, dtop):
        fw = lm.token_logprobs(z, tokens, top=K, temperature=T)
        plain_fw = lm.token_logprobs(z, tokens, temperature=T)
        b = lm.distill_forward_backward(z, ids, t, dl, temperature=T)
        two = lm.distill_forward(z, ids, t, temperature=T)
        return [fw["logprob"], fw["entropy"], fw["top_ids"], fw["top_logprobs"],
                plain_fw["logprob"],
                lm.token_logprobs_backward(z, tokens, fw, dl, dl, dtop, temperature=T),
                b["loss"], b["dlogits"], two["loss"],
                lm.distill_backward(z, ids, t, two["stats"], dl, temperature=T)]

    args = z, tokens, ids, t, dl, dtop
    whole = step(*args)
    part = step(*(a[N - last:].contiguous() for a in args))
    for a, b in zip(whole, part):
        assert torch.equal(a[N - last:], b)


def test_refusals():
    z = torch.zeros((2, 8), device="cuda")
    tok = torch.zeros(2, dtype=torch.int64, device="cuda")
    ids, t = torch.zeros((2, 3), dtype=torch.int64, device="cuda"), torch.zeros((2, 3), device="cuda")
    for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=-1.0)):
        with pytest.raises(ValueError):
            lm.token_logprobs(z, tok, **bad)
    with pytest.raises(ValueError):
        lm.token_logprobs(z.half(), tok)
    with pytest.raises(ValueError):
        lm.token_logprobs(z, tok.int())
    with pytest.raises(ValueError):
        lm.token_logprobs(z.t(), tok)
    with pytest.raises(ValueError):
        lm.token_logprobs(z[:1].expand(2, 8), tok)
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.token_logprobs(z, tok, top=9)
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.token_logprobs(z[:0], tok[:0])
    with pytest.raises(ValueError):
        lm.distill_forward(z, ids[:, :2], t)
    with pytest.raises(ValueError):
        lm.distill_backward(z, ids, t, torch.zeros((2,), device="cuda"), torch.zeros(2, device="cuda"))
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.distill_forward(z, ids.new_zeros((2, 1025)), t.new_zeros((2, 1025)))
