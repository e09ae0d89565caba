"""The fused norms between a block's linears and their gradients, against the definition in 64 bits.

Tolerances, u = 2^-24.  A sum over a row is a tree of at most 40 additions deep (8 in a chunk, 5 chunks, 5 shuffles, 16 warps, with room), so a
mean is off by at most 40 u mean|v| and a mean square by 42 u of itself; the factor 1 / sqrt adds three roundings and halves the mean square's.  With
d = f (40 u mean|v|) the normalised value is off by at most d + 26 u |n|, and the few roundings of weight, modulation and shift by 6 u of their terms.
"""
import math

import numpy as np
import pytest

from test_gpu_fp8 import _rotation

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def _stats(v, kind):
    c = v - v.mean(1, keepdim=True) if kind == "layer" else v
    return c, 1.0 / (c.square().mean(1, keepdim=True) + EPS).sqrt()


def _norm(v, kind):
    c, f = _stats(v, kind)
    return c * f


def _norm_tol(v, kind):
    c, f = _stats(v, kind)
    return f * 40 * U * v.abs().mean(1, keepdim=True) + 26 * U * (c * f).abs()


def _rounded(tol, ref, dtype):
    import torch
    return tol + torch.finfo(dtype).eps / 2 * (ref.abs() + tol)


def _case(M, D, norm="layer", post="none", stream="bf16", rps=None, gate=True, mod=True, weight=False, alpha=1.0, seed=0, offset=0.0, branch=True):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    rps = rps or M
    S = -(-M // rps)
    dtype = torch.float32 if stream == "fp32" else torch.bfloat16
    wide = (2 * r(M, D + 16) + offset).to(dtype)
    c = {"x": wide[:, :D], "b": (r(M, D + 8) * torch.exp(r(M, 1))).bfloat16()[:, :D] if branch else None}
    m = (0.5 * r(S, 3 * D + 8)).bfloat16()
    c["gate"] = m[:, 2 * D:3 * D] if gate and branch else None
    c["shift"], c["scale"] = (m[:, :D], m[:, D:2 * D]) if mod else (None, None)
    c["weight"] = (1 + 0.2 * r(D)).bfloat16() if weight else None
    c["post_weight"] = (1 + 0.2 * r(D)).bfloat16() if weight and branch else None
    c["kw"] = dict(norm=norm, post=post, rps=rps, alpha=alpha)
    return c


def _given(c):
    from paper_2503_06564_b200 import trdq
    kinds = {"none": trdq.NORM_NONE, "layer": trdq.NORM_LAYER, "rms": trdq.NORM_RMS}
    kw = c["kw"]
    return dict(gate=c["gate"], shift=c["shift"], scale=c["scale"], weight=c["weight"], post_weight=c["post_weight"], norm=kinds[kw["norm"]],
                post_norm=kinds[kw["post"]], rows_per_sample=kw["rps"], eps=EPS, res_scale=kw["alpha"])


def _wide(p, c):
    """A parameter of samples, one row per row; in double."""
    return None if p is None else p.double().repeat_interleave(c["kw"]["rps"], 0)[: c["x"].shape[0]]


def _residual(c):
    """(r, tolerance before its rounding) in double."""
    kw = c["kw"]
    xa = kw["alpha"] * c["x"].double()
    if c["b"] is None:
        return xa, U * xa.abs()
    u, tol = c["b"].double(), 0.0
    if kw["post"] != "none":
        u, tol = _norm(u, kw["post"]), _norm_tol(u, kw["post"])
    factor = 1.0
    if c["post_weight"] is not None:
        factor = factor * c["post_weight"].double()
    if c["gate"] is not None:
        factor = factor * _wide(c["gate"], c)
    u = u * factor
    return xa + u, (tol * abs(factor) if kw["post"] != "none" else 0.0) + 4 * U * (u.abs() + xa.abs())


def _hidden(c, r):
    """(h, tolerance before its rounding) from the stored r."""
    kw = c["kw"]
    r = r.double()
    n, tol = _norm(r, kw["norm"]), _norm_tol(r, kw["norm"])
    factor = 1.0
    if c["weight"] is not None:
        factor = factor * c["weight"].double()
    if c["scale"] is not None:
        factor = factor * (1 + _wide(c["scale"], c))
    h = n * factor
    tol = tol * abs(factor) + 6 * U * h.abs()
    if c["shift"] is not None:
        h = h + _wide(c["shift"], c)
        tol = tol + U * (h.abs() + _wide(c["shift"], c).abs())
    return h, tol


def _within(got, ref, tol):
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), f"{(err / tol).max().item():.3f} of the tolerance at {int((err / tol).argmax())}"


SHAPES = [(1, 8), (1, 4096), (2, 128), (3, 136), (9, 1152), (33, 1280), (17, 1288), (64, 2560), (5, 2568), (12, 5120), (7, 5128), (11, 8192), (300, 64)]
KINDS = [dict(), dict(norm="rms", post="rms", gate=False, mod=False, weight=True), dict(norm="rms", post="layer", weight=True, alpha=0.5),
         dict(post="rms", gate=False, weight=True, mod=True), dict(branch=False), dict(branch=False, norm="rms", mod=False, weight=True, alpha=-2.0),
         dict(gate=False, mod=False)]


@pytest.mark.parametrize("M, D", SHAPES)
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_forward(M, D, stream):
    import torch
    from paper_2503_06564_b200 import trdq
    for i, kind in enumerate(KINDS):
        for rps in {1, max(1, M // 3), M}:
            c = _case(M, D, stream=stream, rps=rps, seed=M * D + i, offset=3.0 * (i % 2), **kind)
            store = torch.full((M + 1, D + 24), 5.0, dtype=c["x"].dtype, device="cuda")
            hout = torch.full((M + 1, D + 8), 5.0, dtype=torch.bfloat16, device="cuda")
            r, h = trdq.trdq_gated_norm(c["x"], c["b"], resid=store[:M, :D], out=hout[:M, :D], **_given(c))
            ref, tol = _residual(c)
            _within(r, ref, _rounded(tol, ref, r.dtype))
            ref, tol = _hidden(c, r)
            _within(h, ref, _rounded(tol, ref, h.dtype))
            assert bool((store[M] == 5).all()) and bool((store[:, D:] == 5).all()) and bool((hout[M] == 5).all()) and bool((hout[:, D:] == 5).all())
            # the residual sum in place of x
            x = c["x"].clone()
            r2, h2 = trdq.trdq_gated_norm(x, c["b"], resid=x, **_given(c))
            assert r2.data_ptr() == x.data_ptr() and torch.equal(r2, r) and torch.equal(h2, h)


@pytest.mark.parametrize("M, D", [(1, 128), (1, 4096), (9, 1152), (33, 1280), (17, 2560), (7, 5120), (11, 8192), (300, 256)])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("rotated", [False, True])
def test_forward_codes(M, D, stream, rotated):
    import torch
    from paper_2503_06564_b200 import trdq
    rot, signs, smooth = _rotation(np.random.default_rng(D), D)
    for i, kind in enumerate(KINDS[:3]):
        c = _case(M, D, stream=stream, rps=max(1, M // 2), seed=M + D + i, **kind)
        r, h = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))
        r2, codes, scales = trdq.trdq_gated_norm_fp8(rot if rotated else None, 800, c["x"], c["b"], **_given(c))
        assert torch.equal(r, r2)
        v, tol = _hidden(c, r)
        v, tol = v.view(M, -1, 128), tol.view(M, -1, 128)
        if rotated:
            vec = torch.from_numpy(signs[1].astype(np.float64) * smooth[1] * 2.0 ** -3.5).cuda().view(1, -1, 128)
            n = torch.arange(128, device="cuda")
            H = 1.0 - 2.0 * (sum(((n[:, None] & n[None, :]) >> k) & 1 for k in range(7)) & 1).double()
            v, tol = v * vec, tol * vec.abs()
            # seven stages of additions and the rounded vector, over the block's absolute sum
            tol = (tol.sum(2, keepdim=True) + 10 * U * v.abs().sum(2, keepdim=True)).expand_as(v)
            v = v @ H
        top, ttol = v.abs().amax(2), tol.amax(2)
        s = scales.t().double()
        assert bool(((s - top / 448).abs() <= ttol / 448 + 2 * U * s).all())
        value = codes.float().double().view(M, -1, 128) * s[:, :, None]
        # half a step of the code: 2^-4 of the value (eps / 2), at least half of the spacing 2^-9 of the smallest codes; 4 u for the factor
        half = torch.maximum(v.abs() * 2.0 ** -4, s[:, :, None] * 2.0 ** -10) * (1 + 2.0 ** -4)
        _within(value, v, half + tol + ttol[:, :, None] + 4 * U * v.abs())
        # and against the codes of a fp32 evaluation almost all are the same: a wrong rounding would differ everywhere
        exact = (v / (top / 448).clamp_min(1e-300)[:, :, None])
        _, e = torch.frexp(exact)
        step = torch.exp2((e - 4).clamp_min(-9).double())
        nearest = (torch.round(exact / step) * step).clamp(-448, 448)
        assert (nearest != codes.float().double().view(M, -1, 128)).double().mean().item() <= 1e-3


def test_r_need_not_be_stored():
    import ctypes as C
    import torch
    from paper_2503_06564_b200 import trdq
    c = _case(5, 256, rps=2)
    r, h = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))
    g = _given(c)
    op = trdq._gated_norm_op("", c["x"], c["b"], g["gate"], g["shift"], g["scale"], None, None, g["norm"], g["post_norm"], 2, EPS, 1.0)
    out = torch.empty_like(h)
    assert trdq.lib().trdq_gated_norm(C.byref(op), None, 0, out.data_ptr(), 256, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, h)


def test_rows_that_are_not_finite_stay_by_themselves():
    import torch
    from paper_2503_06564_b200 import trdq
    c = _case(6, 1152, rps=3)
    clean = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))
    x, b = c["x"].clone(), c["b"].clone()
    x[1, 5], b[3, 7], x[4, 0] = float("nan"), float("inf"), -float("inf")
    r, h = trdq.trdq_gated_norm(x, b, **_given(c))
    for row in (0, 2, 5):
        assert torch.equal(r[row], clean[0][row]) and torch.equal(h[row], clean[1][row])
    for row in (1, 3, 4):
        assert bool(h[row].isnan().all())
    z = torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    assert bool((trdq.trdq_gated_norm(z, z)[1] == 0).all())   # eps keeps a constant row finite


# -------------------------------------------------------------------------------------------------------- gradients
def _reference_gradients(c, r, dh, dr):
    """Differentiates the definition in double; the stored r stands where the sum stood."""
    import torch
    kw = c["kw"]
    leaf = {k: c[k].double().requires_grad_() for k in ("b", "gate", "shift", "scale", "weight", "post_weight") if c[k] is not None}
    x = torch.zeros(r.shape, dtype=torch.float64, device="cuda", requires_grad=True)
    rows = torch.arange(r.shape[0], device="cuda") // kw["rps"]
    s = kw["alpha"] * x
    if "b" in leaf:
        u = leaf["b"] if kw["post"] == "none" else _norm(leaf["b"], kw["post"])
        u = u * leaf["post_weight"] if "post_weight" in leaf else u
        s = s + (u * leaf["gate"][rows] if "gate" in leaf else u)
    s = s + (r.double() - s).detach()
    h = _norm(s, kw["norm"])
    h = h * leaf["weight"] if "weight" in leaf else h
    h = h * (1 + leaf["scale"][rows]) + leaf["shift"][rows] if "scale" in leaf else h
    loss = (h * dh.double()).sum()
    if dr is not None:
        loss = loss + (s * dr.double()).sum()
    names = {"dx": x, "db": leaf.get("b"), **{"d" + k: leaf[k] for k in leaf if k != "b"}}
    names = {k: v for k, v in names.items() if v is not None}
    return dict(zip(names, torch.autograd.grad(loss, list(names.values()))))


def _gradient_tolerances(c, r, dh, dr):
    """Before their rounding.  The terms of each formula with absolute values; a term carries the relative error of the statistics and of
    one more row sum (2 x 40 u), of n itself (its d above, relative to the row's spread) and a handful of roundings: 128 u with the
    mean |v| of the row over its spread on top."""
    import torch
    kw = c["kw"]
    r64, dh = r.double(), dh.double().abs()
    cr, f = _stats(r64, kw["norm"])
    n = (cr * f).abs()
    dn_n = f * 40 * U * r64.abs().mean(1, keepdim=True) + 26 * U * n       # error of n
    gain = torch.ones_like(n)
    if c["scale"] is not None:
        gain = gain * (1 + _wide(c["scale"], c)).abs()
    if c["weight"] is not None:
        gain = gain * c["weight"].double().abs()
    dn = dh * gain
    ms = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    term = f * (dn + n * ms(dn * n) + ms(dn))
    dR = term + (dr.double().abs() if dr is not None else 0.0)
    e = 128 * U * dR + f * (dn_n * ms(dn * n) + n * ms(dn * dn_n))
    tol = {"dx": abs(kw["alpha"]) * e}
    rows = torch.arange(r.shape[0], device="cuda") // kw["rps"]
    S, deep = int(rows[-1]) + 1, (min(kw["rps"], 2 ** 20) + 64) * U

    def per_sample(v):
        return torch.zeros((S, v.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, rows, v)

    w = 1.0 if c["weight"] is None else c["weight"].double().abs()
    if c["scale"] is not None:
        tol["dshift"] = deep * per_sample(dh)
        tol["dscale"] = w * per_sample(deep * dh * n + dh * dn_n)
    total = (r.shape[0] + 64) * U
    if c["weight"] is not None:
        g = 1.0 if c["scale"] is None else (1 + _wide(c["scale"], c)).abs()
        tol["dweight"] = (g * (total * dh * n + dh * dn_n)).sum(0)
    if c["b"] is not None:
        b64 = c["b"].double()
        m, dm = b64.abs(), 0.0 * b64
        fb = torch.ones_like(f)
        if kw["post"] != "none":
            cb, fb = _stats(b64, kw["post"])
            m, dm = (cb * fb).abs(), _norm_tol(b64, kw["post"])
        p = 1.0 if c["post_weight"] is None else c["post_weight"].double().abs()
        g = torch.ones_like(n) if c["gate"] is None else _wide(c["gate"], c).abs()
        if c["gate"] is not None:
            tol["dgate"] = p * per_sample(deep * dR * m + e * m + dR * dm)
        if c["post_weight"] is not None:
            tol["dpost_weight"] = (g * (total * dR * m + e * m + dR * dm)).sum(0)
        du, de = dR * g * p, e * g * p
        if kw["post"] != "none":
            de = fb * (de + m * ms(de * m) + ms(de) + m * ms(du * dm) + dm * ms(du * m)) + 128 * U * fb * (du + m * ms(du * m) + ms(du))
            du = fb * (du + m * ms(du * m) + ms(du))
        tol["db"] = de + 4 * U * du
    return tol


BACKWARD_SHAPES = [(1, 8), (2, 128), (1, 4096), (3, 136), (40, 1152), (19, 4096), (7, 4104), (10, 8192), (700, 264), (2100, 64)]


@pytest.mark.parametrize("M, D", BACKWARD_SHAPES)
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_gradients(M, D, stream):
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(M + D)
    for i, kind in enumerate(KINDS):
        for rps in {1, max(1, M // 3), M}:
            c = _case(M, D, stream=stream, rps=rps, seed=M * D + i, offset=2.0 * (i % 2), **kind)
            r = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))[0]
            dh = torch.randn((M, D + 8), generator=gen, device="cuda").bfloat16()[:, :D]
            dr = None if i == 2 else torch.randn((M, D + 16), generator=gen, device="cuda").to(r.dtype)[:, :D]
            got = trdq.trdq_gated_norm_backward(r, c["b"], dh, dr, **_given(c))
            want, tol = _reference_gradients(c, r, dh, dr), _gradient_tolerances(c, r, dh, dr)
            assert {k for k, v in got.items() if v is not None} == set(want) == set(tol)
            for k, ref in want.items():
                assert got[k].shape == ref.shape
                _within(got[k], ref, _rounded(tol[k], ref, got[k].dtype) + 1e-300)
            again = trdq.trdq_gated_norm_backward(r, c["b"], dh, dr, **_given(c))
            assert all(torch.equal(v, again[k]) for k, v in got.items() if v is not None)
            if dr is not None:   # the gradient of r turned into that of x where it is
                d = dr.clone()
                assert torch.equal(trdq.trdq_gated_norm_backward(r, c["b"], dh, d, dX=d, **_given(c))["dx"], got["dx"]) and torch.equal(d, got["dx"])


def test_gradients_against_differences():
    """Central differences of the kernels' own forward pass, along its gradient for every input.  The loss sum(h dh) + sum(r dr) has N = 64 x 512 terms;
    h is rounded to bf16 (standard deviation 2^-9 / sqrt(3) of its value), so a difference carries a noise of about sqrt(2 N) 2^-9 0.58 = 0.3, and three of them
    over the step 2 x 0.05 is 9; the step's cubic remainder is of the order 0.05^2 of the derivative, whose size is about sqrt(N) = 180 per unit.  That
    holds for steps of 0.05 of what a norm divides by: the rows of b have spreads from 0.1 to 10, so a row of x or b steps by 0.05 of its own spread."""
    import torch
    from paper_2503_06564_b200 import trdq
    c = _case(64, 512, norm="layer", post="rms", stream="fp32", rps=16, weight=True, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(9)
    dh, dr = torch.randn((64, 512), generator=gen, device="cuda").bfloat16(), torch.randn((64, 512), generator=gen, device="cuda")
    r, _ = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))
    g = trdq.trdq_gated_norm_backward(r, c["b"], dh, dr, **_given(c))

    def loss(c):
        r, h = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))
        return ((h.double() * dh.double()).sum() + (r.double() * dr.double()).sum()).item()

    for name, grad in (("x", "dx"), ("b", "db"), ("gate", "dgate"), ("shift", "dshift"), ("scale", "dscale"), ("weight", "dweight"), ("post_weight", "dpost_weight")):
        # the directional derivative along the gradient is large against the noise; steps on the grid of the input's type
        direction = g[grad].double()
        if name in ("x", "b"):
            direction = direction / direction.square().mean(1, keepdim=True).sqrt() * c[name].double().square().mean(1, keepdim=True).sqrt()
        else:
            direction = direction / direction.square().mean().sqrt()
        up, down = dict(c), dict(c)
        step = 0.05
        up[name] = (c[name].double() + step * direction).to(c[name].dtype)
        down[name] = (c[name].double() - step * direction).to(c[name].dtype)
        moved = up[name].double() - down[name].double()
        want = (g[grad].double() * moved).sum().item()
        assert abs(loss(up) - loss(down) - want) <= 0.05 * abs(want) + 1.0, name


def test_gradients_that_are_not_wanted():
    import torch
    from paper_2503_06564_b200 import trdq
    c = _case(20, 256, rps=10, gate=False, mod=False)
    dh = torch.randn((20, 256), device="cuda").bfloat16()
    g = trdq.trdq_gated_norm_backward(c["x"], c["b"], dh, **_given(c))
    assert {k for k, v in g.items() if v is not None} == {"dx", "db"}
    none = _case(0, 64, weight=True, rps=4)
    g = trdq.trdq_gated_norm_backward(none["x"], none["b"], torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), **_given(none))
    assert bool((g["dweight"] == 0).all()) and g["dgate"].shape == (0, 64) and g["dx"].shape == (0, 64)


def test_refusals():
    import torch
    from paper_2503_06564_b200 import trdq
    c = _case(6, 128, rps=3)
    given = _given(c)
    rot = _rotation(np.random.default_rng(0), 256)[0]
    for call, status in ((lambda: trdq.trdq_gated_norm(c["x"], c["b"], **(given | dict(rows_per_sample=2))), 2),      # three samples, two rows of parameters
                         (lambda: trdq.trdq_gated_norm(c["x"], c["b"], **(given | dict(rows_per_sample=0))), 2),
                         (lambda: trdq.trdq_gated_norm(c["x"], None, **given), 1), (lambda: trdq.trdq_gated_norm(c["x"], c["b"], **(given | dict(norm=0))), 2),
                         (lambda: trdq.trdq_gated_norm(c["x"][:, :100], c["b"][:, :100]), 2), (lambda: trdq.trdq_gated_norm(c["x"], c["b"][:5]), 2),
                         (lambda: trdq.trdq_gated_norm(c["x"][:, 4:124], c["b"][:, :120]), 3), (lambda: trdq.trdq_gated_norm_fp8(rot, 0, c["x"], c["b"]), 10),
                         (lambda: trdq.trdq_gated_norm(c["x"].cpu(), c["b"]), 10),
                         (lambda: trdq.trdq_gated_norm_backward(c["x"], c["b"], c["b"][:3], **given), 2),
                         (lambda: trdq.trdq_gated_norm_backward(c["x"], c["b"], c["b"], workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), **given), 8)):
        with pytest.raises(trdq.TrdqError) as e:
            call()
        assert e.value.status == status
    for call in (lambda: trdq.trdq_gated_norm(c["x"].half(), c["b"]), lambda: trdq.trdq_gated_norm(c["x"], c["b"].float()),
                 lambda: trdq.trdq_gated_norm(c["x"], c["b"], gate=c["gate"].float(), rows_per_sample=3),
                 lambda: trdq.trdq_gated_norm(c["x"], c["b"], resid=c["x"].float())):
        with pytest.raises(AssertionError):
            call()
    assert math.isfinite(trdq.trdq_gated_norm(c["x"], c["b"], **given)[1].float().sum().item())


@pytest.mark.parametrize("M, D, rps", [(5000, 64, 1), (5000, 64, 3), (5000, 64, 4), (5000, 64, 9), (5000, 64, 2500), (2000, 1152, 12), (2000, 1152, 16), (1999, 1152, 667),
                                       (700, 2560, 100)])
def test_gradients_of_samples_that_end_anywhere(M, D, rps):
    """Each CTA takes a run of rows whatever their samples: samples shorter and longer than a run, that begin where a run begins or inside it."""
    from paper_2503_06564_b200 import trdq
    import torch
    gen = torch.Generator(device="cuda").manual_seed(M + rps)
    c = _case(M, D, rps=rps, weight=True, seed=rps)
    r = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))[0]
    # eighths of small integers: their sums are exact in fp32, so dshift shows whether each row is in one sum, and in the right one
    dh = (torch.randint(-3, 4, (M, D), generator=gen, device="cuda") / 8).bfloat16()
    got = trdq.trdq_gated_norm_backward(r, c["b"], dh, None, **_given(c))
    assert torch.equal(got["dshift"].double(), torch.stack([d.double().sum(0) for d in dh.split(rps)]))
    want, tol = _reference_gradients(c, r, dh, None), _gradient_tolerances(c, r, dh, None)
    for k, ref in want.items():
        _within(got[k], ref, _rounded(tol[k], ref, got[k].dtype) + 1e-300)
    again = trdq.trdq_gated_norm_backward(r, c["b"], dh, None, **_given(c))
    assert all(torch.equal(v, again[k]) for k, v in got.items() if v is not None)


@pytest.mark.parametrize("M, D, rps", [(400, 4104, 7), (333, 8192, 100), (500, 5120, 500)])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("post", ["none", "layer"])
def test_gradients_of_wide_rows(M, D, rps, stream, post):
    """Two chunks a thread, several rows and samples a run."""
    from paper_2503_06564_b200 import trdq
    import torch
    gen = torch.Generator(device="cuda").manual_seed(M + D)
    c = _case(M, D, rps=rps, stream=stream, post=post, weight=True, seed=D, alpha=0.5)
    r = trdq.trdq_gated_norm(c["x"], c["b"], **_given(c))[0]
    dh, dr = torch.randn((M, D), generator=gen, device="cuda").bfloat16(), torch.randn((M, D + 16), generator=gen, device="cuda").to(r.dtype)[:, :D]
    got = trdq.trdq_gated_norm_backward(r, c["b"], dh, dr, **_given(c))
    want, tol = _reference_gradients(c, r, dh, dr), _gradient_tolerances(c, r, dh, dr)
    for k, ref in want.items():
        _within(got[k], ref, _rounded(tol[k], ref, got[k].dtype) + 1e-300)
    again = trdq.trdq_gated_norm_backward(r, c["b"], dh, dr, **_given(c))
    assert all(torch.equal(v, again[k]) for k, v in got.items() if v is not None)


@pytest.mark.parametrize("M, D, rps", [(3000, 1152, 1), (3001, 1152, 13), (2999, 640, 700), (900, 5120, 11)])
@pytest.mark.parametrize("rotated", [False, True])
def test_many_rows_as_few(M, D, rps, rotated):
    """Runs of several rows a CTA, samples that change inside them: the bits of the same rows a sample at a time."""
    from paper_2503_06564_b200 import trdq
    import torch
    c = _case(M, D, rps=rps, post="rms", weight=True, seed=M + D)
    given = _given(c)
    rot = None
    if rotated:
        rng = np.random.default_rng(3)
        rot = trdq.Rotation(D, [0, 1000], (rng.integers(0, 2, (1, D)) * 2 - 1).astype(np.int8), rng.uniform(0.5, 2.0, (1, D)).astype(np.float32))
    whole = trdq.trdq_gated_norm(c["x"], c["b"], **given) + trdq.trdq_gated_norm_fp8(rot, 5, c["x"], c["b"], **given)
    for s in sorted({0, 1, (M // rps) // 2, (M - 1) // rps}):
        rows, one = slice(s * rps, min(M, s * rps + rps)), dict(given)
        one["rows_per_sample"] = rps
        for name in ("gate", "shift", "scale"):
            one[name] = given[name][s:s + 1]
        part = trdq.trdq_gated_norm(c["x"][rows], c["b"][rows], **one) + trdq.trdq_gated_norm_fp8(rot, 5, c["x"][rows], c["b"][rows], **one)
        for w, p in zip(whole, part):
            w = w[rows] if w.shape[0] == M else w[:, rows]
            assert torch.equal(w.contiguous().view(torch.uint8), p.contiguous().view(torch.uint8))
