"""The residual norm on the GPU against a plain 64-bit implementation (its
gradients by automatic differentiation), at widths on both sides of every way a
row is held, row by row and strided, with every part left out.

Tolerances: a row's sums carry (d / 64 + 16) 2^-24 relative at most, 2^-16 at d =
16384; each value then about ten roundings of 2^-24 and a gate within 2^-21.  So
fp32 results are within 4e-5 of the magnitude of what they are made of (a norm's
gradient is a difference: of its two terms, not of what is left), bf16 ones add
half a step, 2^-8 of the value."""

import math

import pytest
import torch

from paper_1709_02755_amd import lm, sru

pytestmark = pytest.mark.gpu

F32, B16 = torch.float32, torch.bfloat16
EPS = 1e-5
TYPES = [(F32, F32), (B16, F32), (B16, B16)]


def inputs(M, d, act, res, seed, drop=()):
    g = torch.Generator().manual_seed(seed)

    def r(*shape):
        return torch.randn(shape, generator=g)

    t = dict(x=(2 * r(M, d)).to(res), y=r(M, d).to(act), z=(2 * r(M, d)).to(act),
             w_post=1 + 0.3 * r(d), scale=0.5 + 0.2 * r(d), w_pre=1 + 0.3 * r(d),
             dx_out=r(M, d).to(res), do=r(M, d).to(act))
    for n in drop:
        t[n] = None
    return t


def plain(t, gate, eps=EPS):
    """(x_out, o) and the gradients, in 64 bits on the CPU."""
    v = {n: None if a is None else a.detach().cpu().double().requires_grad_(True)
         for n, a in t.items()}

    def norm(a, w):
        return a / torch.sqrt(a.square().mean(-1, keepdim=True) + eps) * w

    x_out, o = v["x"], None
    if v["y"] is not None:
        u = v["y"] if v["w_post"] is None else norm(v["y"], v["w_post"])
        if v["z"] is not None:
            s = 1 / (1 + torch.exp(-v["z"]))
            u = u * (v["z"] * s if gate == lm.GATE_SILU else s)
        x_out = v["x"] + (u if v["scale"] is None else v["scale"] * u)
    if v["w_pre"] is not None:
        o = norm(x_out, v["w_pre"])
    total = 0.0
    if t["dx_out"] is not None:
        total = total + (x_out * v["dx_out"].detach()).sum()
    if o is not None and t["do"] is not None:
        total = total + (o * v["do"].detach()).sum()
    if torch.is_tensor(total):
        total.backward()
    grads = {n: None if v[n] is None else (torch.zeros_like(v[n]) if v[n].grad is None
                                           else v[n].grad)
             for n in ("x", "y", "z", "w_post", "scale", "w_pre")}
    return x_out.detach(), None if o is None else o.detach(), grads


def magnitudes(t, gate, eps=EPS):
    """Of what each result is made of: sums of absolute values, a row's largest
    one where a row's sum enters."""
    v = {n: None if a is None else a.detach().cpu().double() for n, a in t.items()}

    def top(a):
        return a.abs().amax(-1, keepdim=True)

    def rstd(a):
        return 1 / torch.sqrt(a.square().mean(-1, keepdim=True) + eps)

    one = torch.ones_like(v["x"])
    x_out, u, yh, g, slope = v["x"], None, None, one, one
    if v["y"] is not None:
        yh = v["y"] if v["w_post"] is None else v["y"] * rstd(v["y"])
        n = yh if v["w_post"] is None else yh * v["w_post"]
        if v["z"] is not None:
            s = 1 / (1 + torch.exp(-v["z"]))
            g = v["z"] * s if gate == lm.GATE_SILU else s
            slope = (s + g.abs() * (1 - s)) if gate == lm.GATE_SILU else s
        u = n * g
        x_out = v["x"] + (u if v["scale"] is None else v["scale"] * u)
    mag = {"x_out": top(v["x"]) + (0 if u is None else top(x_out - v["x"]))}
    dx = 0 * mag["x_out"] + 1e-30
    if v["dx_out"] is not None:
        dx = dx + top(v["dx_out"])
    if v["w_pre"] is not None:
        xh = x_out * rstd(x_out)
        mag["o"] = top(xh * v["w_pre"]) + mag["x_out"] * top(rstd(x_out) * v["w_pre"])
        mag["w_pre"] = one.sum(0) * 1e-30
        if v["do"] is not None:
            w = v["do"] * v["w_pre"]
            dx = dx + rstd(x_out) * (top(w) + top(xh) * (w * xh).abs().mean(-1, keepdim=True))
            xs = xh.abs() + mag["x_out"] * rstd(x_out)
            mag["w_pre"] = (v["do"].abs() * xs).sum(0)
    mag["x"] = dx
    if u is not None:
        sc = 1.0 if v["scale"] is None else v["scale"].abs()
        mag["scale"] = (dx * u.abs()).sum(0)
        du = dx * sc * one
        mag["z"] = top(du * n * slope)
        dn = du * g.abs()
        mag["w_post"] = (dn * yh.abs()).sum(0)
        mag["y"] = top(dn)
        if v["w_post"] is not None:
            w = dn * v["w_post"].abs()
            mag["y"] = rstd(v["y"]) * (top(w) + top(yh) * (w * yh.abs()).mean(-1, keepdim=True))
    return mag


def close(name, got, ref, scale):
    got = got.detach()
    bf16 = got.dtype == B16
    got = got.cpu().double()
    assert got.shape == ref.shape, name
    tol = 4e-5 * scale + (2.0 ** -8 * ref.abs() if bf16 else 0.0)
    err = (got - ref).abs()
    assert bool((err <= tol).all()), (name, float((err - tol).max()))


def dev(t):
    return {n: None if a is None else a.cuda() for n, a in t.items()}


def run(t, gate, **out):
    p = dict(w_post=t["w_post"], z=t["z"], scale=t["scale"], w_pre=t["w_pre"], gate=gate, eps=EPS)
    fw = lm.residual_norm_forward(t["x"], t["y"], **p)
    g = lm.residual_norm_backward(t["x"], t["y"], fw["rstd"], t["dx_out"], t["do"], **p, **out)
    torch.cuda.synchronize()
    return fw, g


def check(t, gate):
    x_out, o, ref = plain(t, gate)
    mag = magnitudes(t, gate)
    fw, g = run(dev(t), gate)
    if t["y"] is not None:
        close("x_out", fw["x_out"], x_out, mag["x_out"])
    else:
        assert fw["x_out"] is None
    if t["w_pre"] is not None:
        close("o", fw["o"], o, mag["o"])
    else:
        assert fw["o"] is None
    for n, r in ref.items():
        if r is None:
            assert g["d" + n] is None
        else:
            close("d" + n, g["d" + n], r, mag[n])
    return fw, g


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("M,d", [(1, 1), (3, 7), (5, 64), (9, 300), (4, 512), (7, 513), (6, 1000),
                                 (13, 1024), (3, 1025), (5, 2048), (3, 2056), (2, 4096), (3, 4100),
                                 (2, 8191), (3, 8192), (2, 8200), (2, 16384), (1, 16383)])
def test_values_and_gradients(M, d, act, res):
    check(inputs(M, d, act, res, d + M), lm.GATE_SILU if M % 2 else lm.GATE_SIGMOID)


PARTS = [("z",), ("w_post",), ("scale",), ("w_pre", "do"), ("z", "w_post"), ("do",), ("dx_out",),
         ("dx_out", "do"), ("y", "z", "w_post", "scale"), ("z", "w_post", "scale", "w_pre", "do"),
         ("y", "z", "w_post", "scale", "dx_out")]


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("drop", PARTS)
def test_parts_left_out(drop, act, res):
    if "y" in drop and act != res:
        act = res  # without a block's output there is one type
    for d in (40, 1500):
        check(inputs(6, d, act, res, 2, drop), lm.GATE_SILU)


@pytest.mark.parametrize("M,d", [(5, 40), (3, 1024), (4, 1277), (2, 6001)])
def test_norm_alone_beside_a_full_precision_residual(M, d):
    """What a bfloat16 model's first block reads of a float32 residual."""
    t = inputs(M, d, B16, F32, d, ("y", "z", "w_post", "scale"))
    _, o, ref = plain(t, lm.GATE_SILU)
    mag = magnitudes(t, lm.GATE_SILU)
    v = dev(t)
    fw = lm.residual_norm_forward(v["x"], w_pre=v["w_pre"], eps=EPS, dtype=B16)
    g = lm.residual_norm_backward(v["x"], None, fw["rstd"], v["dx_out"], v["do"], w_pre=v["w_pre"],
                                  eps=EPS)
    torch.cuda.synchronize()
    assert fw["o"].dtype == B16 and g["dx"].dtype == F32
    close("o", fw["o"], o, mag["o"])
    close("dx", g["dx"], ref["x"], mag["x"])
    close("dw_pre", g["dw_pre"], ref["w_pre"], mag["w_pre"])


@pytest.mark.parametrize("d", [64, 1024])
def test_many_rows(d):
    """More rows than the gradient's workgroups take at a time."""
    t = inputs(5000, d, B16, F32, 5)
    x_out, o, ref = plain(t, lm.GATE_SILU)
    fw, g = run(dev(t), lm.GATE_SILU)
    mag = magnitudes(t, lm.GATE_SILU)
    close("o", fw["o"], o, mag["o"])
    for n in ref:
        close(n, g["d" + n], ref[n], mag[n])


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("d,pitch,offset", [(256, 768, 256), (256, 771, 5), (33, 70, 1)])
def test_strided_rows_and_own_memory(d, pitch, offset, act, res):
    """Slices of a projection in, slices of its gradient out; x_out over x and
    dx over dx_out.  The same bits as contiguous rows where both are read in 16
    bytes, and nothing beside the rows is touched."""
    M = 11
    t = inputs(M, d, act, res, 7)
    mag = magnitudes(t, lm.GATE_SILU)
    t = dev(t)
    p = dict(w_post=t["w_post"], scale=t["scale"], w_pre=t["w_pre"], eps=EPS)
    fw, g = run(t, lm.GATE_SILU)

    def slice_of(a):
        buf = torch.full((M * pitch + offset,), 7.0, dtype=a.dtype, device="cuda")
        s = buf[offset:].view(M, pitch)[:, :d]
        s.copy_(a)
        return s, buf

    (y, _), (z, _), (xs, _) = slice_of(t["y"]), slice_of(t["z"]), slice_of(t["x"])
    f2 = lm.residual_norm_forward(xs, y, z=z, **p)
    for n in ("x_out", "o"):
        close(n, f2[n], fw[n].cpu().double(), mag[n])
    (dy, bufy), (dz, _) = slice_of(t["y"]), slice_of(t["z"])
    (do, _), (dxo, _) = slice_of(t["do"]), slice_of(t["dx_out"])
    g2 = lm.residual_norm_backward(xs, y, f2["rstd"], dxo, do, z=z, **p,
                                   out=dict(dy=dy, dz=dz, dx=dxo))
    assert g2["dy"] is dy and g2["dx"] is dxo
    for n in ("x", "y", "z", "w_post", "scale", "w_pre"):
        close(n, g2["d" + n], g["d" + n].cpu().double(), mag[n])
    rest = bufy[offset:].view(M, pitch)[:, d:]
    assert bool((rest == 7.0).all()) and bool((bufy[:offset] == 7.0).all())
    f3 = lm.residual_norm_forward(xs, y, z=z, **p, out=dict(x_out=xs))
    assert f3["x_out"] is xs and torch.equal(xs, f2["x_out"])
    assert torch.equal(f3["o"], f2["o"])


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("d,pitch,offset", [(33, 39, 3), (1001, 1003, 1), (4099, 4100, 2),
                                            (8191, 8193, 7)])
def test_nothing_beside_ragged_rows(d, pitch, offset, act, res):
    """Outputs whose rows end inside 16 bytes and start between them: what lies
    between the rows, before and after them stays."""
    M = 6
    t = inputs(M, d, act, res, 8)
    mag = magnitudes(t, lm.GATE_SILU)
    t = dev(t)
    p = dict(w_post=t["w_post"], scale=t["scale"], w_pre=t["w_pre"], eps=EPS)
    fw, g = run(t, lm.GATE_SILU)
    bufs = {}

    def out_of(n, dtype):
        buf = torch.full((M * pitch + offset + 8,), 7.0, dtype=dtype, device="cuda")
        bufs[n] = buf
        return buf[offset:offset + M * pitch].view(M, pitch)[:, :d]

    f2 = lm.residual_norm_forward(t["x"], t["y"], z=t["z"], **p,
                                  out=dict(x_out=out_of("x_out", res), o=out_of("o", act)))
    g2 = lm.residual_norm_backward(t["x"], t["y"], f2["rstd"], t["dx_out"], t["do"], z=t["z"], **p,
                                   out=dict(dx=out_of("dx", res), dy=out_of("dy", act),
                                            dz=out_of("dz", act)))
    for n in ("x_out", "o"):
        close(n, f2[n], fw[n].cpu().double(), mag[n])
    for n in ("x", "y", "z", "w_post", "scale", "w_pre"):
        close(n, g2["d" + n], g["d" + n].cpu().double(), mag[n])
    for n, buf in bufs.items():
        rest = buf[offset:offset + M * pitch].view(M, pitch)[:, d:]
        assert bool((rest == 7.0).all()), n
        assert bool((buf[:offset] == 7.0).all()) and bool((buf[-8:] == 7.0).all()), n


def test_leading_dimensions():
    t = dev(inputs(12, 40, B16, B16, 9))
    fw, g = run(t, lm.GATE_SILU)
    t3 = {n: a.view(4, 3, 40) if a.dim() == 2 else a for n, a in t.items()}
    f3, g3 = run(t3, lm.GATE_SILU)
    assert f3["o"].shape == (4, 3, 40) and f3["rstd"].shape == (4, 3, 2)
    assert torch.equal(f3["o"].view(12, 40), fw["o"])
    assert torch.equal(g3["dy"].view(12, 40), g["dy"]) and torch.equal(g3["dw_pre"], g["dw_pre"])
    with pytest.raises(ValueError, match="equal distances"):
        wide = torch.zeros((4, 4, 40), dtype=B16, device="cuda")[:, :3]
        lm.residual_norm_forward(wide, t3["y"], w_pre=t["w_pre"])


def test_rows_of_zeros_and_of_no_number():
    """A row of zeros has finite results; NaN and infinity stay in their row."""
    t = inputs(6, 96, F32, F32, 4)
    t["x"][0] = 0
    t["y"][0] = 0
    t["y"][2, 5] = math.nan
    t["x"][3, 1] = math.inf
    t["z"][4, :] = -200.0  # the gate is closed
    fw, g = run(dev(t), lm.GATE_SILU)
    assert bool((fw["o"][0] == 0).all()) and bool(torch.isfinite(g["dy"][0]).all())
    for n in (fw["x_out"], fw["o"], g["dx"], g["dy"]):
        assert bool(torch.isnan(n[2]).any()) and bool(torch.isfinite(n[[0, 1, 4, 5]]).all())
    assert torch.equal(fw["x_out"][4], dev(t)["x"][4])
    assert not bool(torch.isfinite(fw["o"][3]).all())


def test_gradient_against_differences():
    t = inputs(3, 20, F32, F32, 6)
    _, g = run(dev(t), lm.GATE_SILU)

    def f(v):
        x_out, o, _ = plain(v, lm.GATE_SILU)
        return float((x_out * t["dx_out"].double()).sum() + (o * t["do"].double()).sum())

    gen = torch.Generator().manual_seed(1)
    for n in ("x", "y", "z", "w_post", "scale", "w_pre"):
        d = torch.randn(t[n].shape, generator=gen, dtype=torch.float64)
        e = 1e-5
        up = f({**t, n: t[n].double() + e * d})
        down = f({**t, n: t[n].double() - e * d})
        slope = (up - down) / (2 * e)
        assert abs(slope - float((g["d" + n].cpu().double() * d).sum())) <= 1e-4 * (1 + abs(slope))


def test_same_bits_on_another_stream_and_in_a_graph():
    t = dev(inputs(700, 1024, B16, F32, 8))

    def step(v):
        fw, g = run_nosync(v)
        return [fw["x_out"], fw["o"]] + [g[n] for n in sorted(g)]

    def run_nosync(v):
        p = dict(w_post=v["w_post"], z=v["z"], scale=v["scale"], w_pre=v["w_pre"], eps=EPS)
        fw = lm.residual_norm_forward(v["x"], v["y"], **p)
        return fw, lm.residual_norm_backward(v["x"], v["y"], fw["rstd"], v["dx_out"], v["do"], **p)

    want = [a.clone() for a in step(t)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step(t)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(t)
    other = dev(inputs(700, 1024, B16, F32, 9))
    for _ in range(3):
        step(other)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held))


def test_rows_past_32_bits():
    """Rows that start past 2^31 elements."""
    d, pitch = 520, 1 << 28
    buf = torch.zeros((9 * pitch + d,), dtype=B16, device="cuda")
    t = dev(inputs(10, d, B16, B16, 3))
    fw, g = run(t, lm.GATE_SILU)
    y = buf.as_strided((10, d), (pitch, 1))
    y.copy_(t["y"])
    f2, g2 = run({**t, "y": y}, lm.GATE_SILU, out=dict(dy=y))
    assert torch.equal(f2["o"], fw["o"]) and torch.equal(y, g["dy"])


@pytest.mark.parametrize("d", [1032, 1033])
def test_more_rows_than_a_launch_has_workgroups(d):
    """Rows that a workgroup comes to after its first: the bits of the same rows in
    a call of their own."""
    M, last = (1 << 20) + 9, 20
    y = torch.randn((M, d), device="cuda").to(B16)
    w = torch.linspace(0.5, 1.5, d, device="cuda")
    p = dict(w_post=w, scale=w, w_pre=w, eps=EPS)
    whole = lm.residual_norm_forward(y, y, z=y, **p)
    end = y[M - last:].clone()
    part = lm.residual_norm_forward(end, end, z=end, **p)
    for n in ("x_out", "o", "rstd"):
        assert torch.equal(whole[n][M - last:], part[n]), n


def test_refusals():
    t = dev(inputs(4, 32, B16, F32, 1))
    p = dict(w_pre=t["w_pre"])
    bad = [dict(x=t["x"].half()), dict(y=t["y"].float(), x=t["x"].bfloat16()),
           dict(y=t["y"][:, :16]), dict(y=t["y"][:2]), dict(z=t["z"].float()),
           dict(w_pre=t["w_pre"].bfloat16()), dict(scale=t["scale"][:3]),
           dict(y=None, scale=t["scale"]), dict(y=None, w_pre=None),
           dict(x=t["x"].t().contiguous().t())]
    for kw in bad:
        a = dict(x=t["x"], y=t["y"], **p)
        a.update(kw)
        with pytest.raises(ValueError):
            lm.residual_norm_forward(**a)
    with pytest.raises(sru.SruError, match="FLAG"):
        lm.residual_norm_forward(t["x"], t["y"], gate=2, **p)
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.residual_norm_forward(t["x"], t["y"], eps=0.0, **p)
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.residual_norm_forward(torch.zeros((1, 16385), device="cuda"),
                                 torch.zeros((1, 16385), device="cuda"))
    with pytest.raises(sru.SruError, match="SHAPE"):
        lm.residual_norm_forward(t["x"][:0], t["y"][:0], **p)
