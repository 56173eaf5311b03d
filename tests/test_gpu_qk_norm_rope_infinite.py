"""Norm and rotation of rows with elements that are not finite, element by element against the formula: what it does not bring into a
result does not reach it.  (Squares of an infinity make the inverse length 0, and 0 times infinity is no number: that is the formula.)"""
import math

import pytest

pytestmark = pytest.mark.gpu

INF = math.inf


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def formula(x, w, table, norm, pairs, scale):
    """One row [d] at a position's table row [rot], in 64 bits, each feature from the terms that are its own."""
    import torch
    d, rot = x.numel(), 0 if table is None else table.numel()
    r = 1.0 if norm == 0 else ((x * x).sum() / (d if norm == 1 else 1) + 1e-6).rsqrt()
    n = (r * x) * w
    y = n.clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        c, s = table[i], table[rot // 2 + i]
        y[a], y[b] = n[a] * c - n[b] * s, n[b] * c + n[a] * s
    return scale * y


def gradient(x, g, w, table, norm, pairs, scale):
    import torch
    d, rot = x.numel(), 0 if table is None else table.numel()
    u = g.clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
        c, s = table[i], table[rot // 2 + i]
        u[a], u[b] = g[a] * c + g[b] * s, g[b] * c - g[a] * s
    z = scale * u * w
    if norm == 0:
        return z
    r = ((x * x).sum() / (d if norm == 1 else 1) + 1e-6).rsqrt()
    n = r * x
    return r * (z - n * ((n * z).sum() / (d if norm == 1 else 1)))


def same(got, want, bf16, what):
    """Equal kinds of numbers in every place, finite ones to 2^-18 of the row's largest (2^-8 of themselves more in bf16)."""
    import torch
    got = got.double().cpu()
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(want)), (what, kind.__name__, kind(got).nonzero().flatten().tolist(), kind(want).nonzero().flatten().tolist())
    fin = torch.isfinite(want)
    if fin.any():
        tol = 2.0 ** -18 * want[fin].abs().max() + (2.0 ** -8 * want[fin].abs() if bf16 else 0) + 1e-30
        assert ((got[fin] - want[fin]).abs() <= tol).all(), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [0, 16, 32, 64])
@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("value", [INF, -INF, math.nan])
def test_where_a_number_that_is_not_finite_arrives(dtype, rot, pairs, norm, value):
    """Rows of x, and of the result's gradient, with one such element in turn at rotated and unrotated features; the others of order 1."""
    import torch
    gen = torch.Generator().manual_seed(rot + norm)
    dt, d = torch.bfloat16 if dtype == "bf16" else torch.float32, 64
    places = [0, 1, 6, 15, 16, 17, 30, 31, 32, 33, 47, 62, 63]
    T = len(places) + 1
    x, g = (torch.randn(T, d, generator=gen).to(dt) for _ in range(2))
    w, scale = torch.rand(d, generator=gen) + 0.5, 0.125
    angle = 0.1 + torch.arange(T, dtype=torch.float64)[:, None] * 0.3 ** torch.arange(rot // 2, dtype=torch.float64)
    table = torch.cat((angle.cos(), angle.sin()), 1).float() if rot else None
    sick_x, sick_g = x.clone(), g.clone()
    for t, p in enumerate(places):
        sick_x[t, p] = value
        sick_g[t, p] = value
    how = dict(cos_sin=None if table is None else table.cuda(), q_weight=w.cuda(), norm=norm, eps=1e-6, rotation=pairs, q_scale=scale)
    out = lsm().lsm_qk_norm_rope(sick_x.cuda().view(1, 1, T, d), None, **how)[0][0, 0]
    back = lambda x_, g_: lsm().lsm_qk_norm_rope_bwd(x_.cuda().view(1, 1, T, d), None, g_.cuda().view(1, 1, T, d), None, **how)["dq"][0, 0]
    dx_of_x, dx_of_g = back(sick_x, g), back(x, sick_g)
    torch.cuda.synchronize()
    wd, bf = w.double(), dtype == "bf16"
    for t in range(T):
        row = None if table is None else table[t].double()
        what = (t, places[t] if t < len(places) else None)
        same(out[t], formula(sick_x[t].double(), wd, row, norm, pairs, scale), bf, ("y",) + what)
        same(dx_of_x[t], gradient(sick_x[t].double(), g[t].double(), wd, row, norm, pairs, scale), bf, ("dx of x",) + what)
        if norm == 0:  # with a norm every element of the gradient reaches all of dx
            same(dx_of_g[t], gradient(x[t].double(), sick_g[t].double(), wd, row, norm, pairs, scale), bf, ("dx of dy",) + what)
