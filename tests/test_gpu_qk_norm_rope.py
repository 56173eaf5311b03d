"""Norm and rotation of queries and keys (lsm_qk_norm_rope, lsm_qk_norm_rope_bwd) against the formulas in 64 bits.

Tolerances.  A row's sum of d squares, its inverse root, two coefficients and a sum of two products are fewer than 16
roundings of 2^-24 in a chain, so an output is within 2^-20 of (|x c| + |x' s|) r, and a stored bf16 within half a unit in
its last place (2^-8 of its size) of that.  In the backward pass z and (n . z) take as many again: 2^-19 of
r (|z| + |n| sum |n z|).  A weight's gradient is a sum over rows: a lane adds at most a few tens of terms in a row, then come
trees: 64 * 2^-24 of the sum of the terms' sizes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-6


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def table(n_pos, rot):
    import torch
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 1000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat((a.cos(), a.sin()), 1).float()


def rotate(x, cs, pairs, back=False):
    """x [B,H,T,d], cs [B,T,rot] or None, all in 64 bits."""
    import torch
    if cs is None:
        return x
    rot = cs.shape[-1]
    c, s = cs[:, None, :, :rot // 2], cs[:, None, :, rot // 2:]
    s = -s if back else s
    y = x.clone()
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def inverse_length(x, norm):
    import torch
    if norm == 0:
        return torch.ones_like(x[..., :1])
    q = (x * x).sum(-1, keepdim=True)
    return ((q / x.shape[-1] if norm == 1 else q) + EPS).rsqrt()


def reference(x, w, cs, norm, pairs, scale, g=None):
    """y and its error scale; with g also dx, its error scale, dw and the sum of its terms' sizes (64 bits, [B,H,T,d])."""
    import torch
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w
    r = inverse_length(x, norm)
    n = r * x
    out = scale * rotate(n * w, cs, pairs)
    size = abs(scale) * rotate((n * w).abs(), None if cs is None else cs.abs(), pairs).abs() + abs(scale) * 2 * (n * w).abs().amax(-1, keepdim=True)
    if g is None:
        return out, size
    u = scale * rotate(g, cs, pairs, back=True)
    z = u * w
    d = 1 if norm == 2 else x.shape[-1]
    along = (n * z).sum(-1, keepdim=True) / d * (norm != 0)
    dx = r * (z - n * along)
    zmax = 2 * abs(scale) * g.abs().amax(-1, keepdim=True) * w.abs().max()
    dx_size = r * (zmax + n.abs() * (n.abs() * zmax).sum(-1, keepdim=True) / d * (norm != 0))
    return out, size, dx, dx_size, (u * n).sum((0, 1, 2)), (2 * abs(scale) * g.abs().amax(-1, keepdim=True) * n.abs()).sum((0, 1, 2))


def near(got, ref, size, rel, bf16, what):
    import torch
    got = got.double().cpu()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= rel * size + (2.0 ** -8 * ref.abs() if bf16 else 0) + 1e-40)
    assert not bad.any(), (what, int(bad.sum()), float((got - ref).abs()[bad].max()))


def put(x, layout, dt, fused=False):
    """[B,H,T,d] in 64 bits -> the device tensor in `layout`; fused: a slice of a wider tensor, not dense over its axes."""
    import torch
    x = x if layout == 0 else x.transpose(1, 2)
    x = x.to(dt)
    if not fused:
        return x.contiguous().cuda()
    wide = torch.full(x.shape[:2] + (x.shape[2] + 3, x.shape[3] + 16), float("nan"), dtype=dt, device="cuda")
    view = wide[:, :, 1:1 + x.shape[2], 16:]
    view.copy_(x)
    return view


def back(x, layout):
    return x if layout == 0 else x.transpose(1, 2)


def case(B, T, Hq, Hk, d, dtype, norm, pairs, rot, weights=True, layout=0, out_layout=0, fused=False, cached=True, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda *s: torch.randn(*s, generator=gen).to(dt).double()
    q, gq = rnd(B, Hq, T, d), rnd(B, Hq, T, d)
    k, gk = (rnd(B, Hk, T, d), rnd(B, Hk, T, d)) if Hk else (None, None)
    wq = (1 + 0.3 * torch.randn(d, generator=gen)) if weights else None
    wk = (1 + 0.3 * torch.randn(d, generator=gen)) if weights and Hk else None
    n_pos = T + 50
    cs = table(n_pos, rot) if rot else None
    pos = torch.randint(0, n_pos, (B, T), generator=gen, dtype=torch.int32) if cached and rot else None
    at = torch.arange(T).expand(B, T) if pos is None else pos.long()
    rows = None if cs is None else cs.double()[at]
    scale = d ** -0.5
    how = dict(cos_sin=None if cs is None else cs.cuda(), positions=None if pos is None else pos.cuda(),
               q_weight=None if wq is None else wq.cuda(), k_weight=None if wk is None else wk.cuda(), norm=norm, eps=EPS,
               rotation=int(pairs), q_scale=scale, k_scale=1.5, layout=layout, out_layout=out_layout)
    dq, dk = put(q, layout, dt, fused), None if k is None else put(k, layout, dt, fused)
    o = lsm().lsm_qk_norm_rope(dq, dk, **how)
    r = lsm().lsm_qk_norm_rope_bwd(dq, dk, put(gq, out_layout, dt, fused), None if k is None else put(gk, out_layout, dt, fused), **how)
    torch.cuda.synchronize()
    bf = dtype == "bf16"
    for n, x, w, g, sc, got, dx, dw in (("q", q, wq, gq, scale, o[0], r["dq"], r["d_q_weight"]),
                                        ("k", k, wk, gk, 1.5, o[1], r["dk"], r["d_k_weight"])):
        if x is None:
            assert got is None and dx is None and dw is None
            continue
        sc = float(np.float32(sc))
        ref = reference(x, None if w is None else w.double(), rows, norm, pairs, sc, g)
        near(back(got, out_layout), ref[0], ref[1], 2.0 ** -20, bf, n + "_out")
        near(back(dx, layout), ref[2], ref[3], 2.0 ** -19, bf, "d" + n)
        if w is None:
            assert dw is None
        else:
            near(dw, ref[4], ref[5], 64 * 2.0 ** -24, False, "d_%s_weight" % n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("pairs", [False, True])
def test_values_and_gradients(dtype, d, norm, pairs):
    for i, (B, T, Hq, Hk) in enumerate([(1, 1, 1, 1), (2, 5, 3, 1), (1, 37, 6, 2)]):
        for rot in (0, 16, 48, d):
            case(B, T, Hq, Hk, d, dtype, norm, pairs, rot, weights=i != 1, seed=i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,out_layout", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("fused", [False, True])
def test_orders_and_strides(dtype, layout, out_layout, fused):
    case(3, 9, 4, 2, 128, dtype, 1, False, 128, layout=layout, out_layout=out_layout, fused=fused)
    case(2, 6, 5, 5, 64, dtype, 2, True, 32, layout=layout, out_layout=out_layout, fused=fused, cached=False)


@pytest.mark.parametrize("dtype,T,H", [("bf16", 1, 70), ("bf16", 300, 33), ("f32", 129, 9), ("bf16", 4099, 2)])
def test_many_heads_and_many_tokens(dtype, T, H):
    """Head ranges of one and of several heads, tokens that do not fill the last group, more items than workgroups."""
    case(1, T, H, 1, 128, dtype, 1, False, 64)
    case(2, T, 3, 0, 64, dtype, 1, True, 64, cached=False)


def test_one_token_of_three_axes():
    import torch
    pkg = lsm()
    q, k = (torch.randn(5, h, 128, device="cuda").to(torch.bfloat16) for h in (4, 2))
    cs, pos = table(100, 128).cuda(), torch.tensor([0, 99, 3, 7, 50], dtype=torch.int32, device="cuda")
    w = torch.rand(128, device="cuda")
    a = pkg.lsm_qk_norm_rope(q, k, cs, pos, w, w)
    b = pkg.lsm_qk_norm_rope(q[:, :, None], k[:, :, None], cs, pos[:, None].contiguous(), w, w)
    assert a[0].shape == q.shape and a[1].shape == k.shape
    assert torch.equal(a[0], b[0][:, :, 0]) and torch.equal(a[1], b[1][:, :, 0])


def test_results_into_slices_of_given_tensors():
    import torch
    pkg = lsm()
    fused = torch.randn(2, 11, 9, 64, device="cuda").to(torch.bfloat16)
    q, k = fused[:, :, :4], fused[:, :, 4:6]
    cs = table(11, 64).cuda()
    plain = pkg.lsm_qk_norm_rope(q, k, cs, layout=1, out_layout=0)
    wide = torch.zeros(2, 8, 11, 64, device="cuda", dtype=torch.bfloat16)
    got = pkg.lsm_qk_norm_rope(q, k, cs, layout=1, out_layout=0, q_out=wide[:, 1:5], k_out=wide[:, 5:7])
    assert got[0].data_ptr() == wide[:, 1:5].data_ptr()
    assert torch.equal(wide[:, 1:5], plain[0]) and torch.equal(wide[:, 5:7], plain[1])
    assert not wide[:, 0].any() and not wide[:, 7].any()
    grads = pkg.lsm_qk_norm_rope_bwd(q, k, plain[0], plain[1], cs, layout=1, out_layout=0)
    d_fused = torch.zeros_like(fused)
    pkg.lsm_qk_norm_rope_bwd(q, k, plain[0], plain[1], cs, layout=1, out_layout=0, dq=d_fused[:, :, :4], dk=d_fused[:, :, 4:6])
    assert torch.equal(d_fused[:, :, :4], grads["dq"]) and torch.equal(d_fused[:, :, 4:6], grads["dk"])
    assert not d_fused[:, :, 6:].any()


def test_repeated_inputs_and_results_in_place():
    import torch
    pkg = lsm()
    cs, w = table(11, 64).cuda(), torch.linspace(0.5, 1.5, 64, device="cuda")
    one = torch.randn(1, 1, 11, 64, device="cuda")
    q, g = one.expand(3, 4, 11, 64), torch.randn(3, 4, 1, 64, device="cuda").expand(3, 4, 11, 64)
    got, ref = pkg.lsm_qk_norm_rope(q, q, cs, None, w), pkg.lsm_qk_norm_rope(q.contiguous(), q.contiguous(), cs, None, w)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    got, plain = pkg.lsm_qk_norm_rope_bwd(q, q, g, g, cs, None, w), pkg.lsm_qk_norm_rope_bwd(q.contiguous(), q.contiguous(), g.contiguous(),
                                                                                          g.contiguous(), cs, None, w)
    for n in ("dq", "dk", "d_q_weight"):
        assert torch.equal(got[n], plain[n]), n
    for bad in (torch.zeros(1, 4, 11, 64, device="cuda").expand(3, 4, 11, 64), torch.zeros(3, 1, 11, 64, device="cuda").expand(3, 4, 11, 64)):
        with pytest.raises(pkg.LsmError):
            pkg.lsm_qk_norm_rope(q, q, cs, None, w, q_out=bad)
        with pytest.raises(pkg.LsmError):
            pkg.lsm_qk_norm_rope_bwd(q, q, g, g, cs, None, w, dk=bad)
    mine = q.contiguous()
    other = mine.clone()
    out = pkg.lsm_qk_norm_rope(mine, other, cs, None, w, q_out=mine, k_out=other)
    assert out[0] is mine and torch.equal(mine, ref[0]) and torch.equal(other, ref[1])


@pytest.mark.parametrize("pairs", [0, 1])
def test_gradient_is_the_slope_of_the_forward_formula(pairs):
    """Central differences of the forward formula in 64 bits against the kernel's gradients in fp32."""
    import torch
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(1, 2, 3, 64, generator=gen)
    g, w, cs = torch.randn(1, 2, 3, 64, generator=gen), torch.rand(64, generator=gen) + 0.5, table(3, 32)
    for norm in (0, 1, 2):
        r = lsm().lsm_qk_norm_rope_bwd(x.cuda(), None, g.cuda(), None, cs.cuda(), q_weight=w.cuda(), norm=norm, eps=EPS,
                                       rotation=pairs, q_scale=0.125)

        def loss(x_, w_):
            return (reference(x_, w_, cs.double()[None], norm, bool(pairs), 0.125)[0] * g.double()).sum()
        h = 1e-5
        for what, base, got in (("x", x.double(), r["dq"]), ("w", w.double(), r["d_q_weight"])):
            slope = torch.zeros_like(base)
            for i in range(base.numel()):
                e = torch.zeros(base.numel(), dtype=torch.float64)
                e[i] = h
                e = e.view(base.shape)
                up, down = ((loss(base + e, w.double()), loss(base - e, w.double())) if what == "x" else
                            (loss(x.double(), base + e), loss(x.double(), base - e)))
                slope.view(-1)[i] = (up - down) / (2 * h)
            # differences: h^2 times third derivatives of order 1; the kernel: 2^-19 of sums of a few terms of order 1
            assert (got.double().cpu() - slope).abs().max() <= 2e-5, (norm, what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_outside_the_table_and_rows_that_are_not_finite(dtype):
    import torch
    pkg = lsm()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.randn(1, 3, 8, 128, device="cuda").to(dt)
    cs = table(20, 64).cuda()
    pos = torch.arange(8, dtype=torch.int32, device="cuda")[None].contiguous()
    good = pkg.lsm_qk_norm_rope(q, q, cs, pos)
    dgood = pkg.lsm_qk_norm_rope_bwd(q, q, q, q, cs, pos)
    bad_pos = pos.clone()
    bad_pos[0, 2], bad_pos[0, 5], bad_pos[0, 6] = -1, 20, 2 ** 31 - 1
    for got, ref in ((pkg.lsm_qk_norm_rope(q, q, cs, bad_pos), good),
                     ([pkg.lsm_qk_norm_rope_bwd(q, q, q, q, cs, bad_pos)[n] for n in ("dq", "dk")], (dgood["dq"], dgood["dk"]))):
        for a, b in zip(got, ref):
            for t in range(8):
                assert torch.isnan(a[:, :, t]).all() if t in (2, 5, 6) else torch.equal(a[:, :, t], b[:, :, t]), t
    sick = q.clone()
    sick[0, 1, 3, 7], sick[0, 2, 4, 100], sick[0, 0, 7, 70] = float("nan"), float("inf"), -float("inf")
    got, dgot = pkg.lsm_qk_norm_rope(sick, None, cs, pos)[0], pkg.lsm_qk_norm_rope_bwd(sick, None, q, None, cs, pos)["dq"]
    for h in range(3):
        for t in range(8):
            if (h, t) in ((1, 3), (2, 4), (0, 7)):
                assert not torch.isfinite(got[0, h, t]).all() and not torch.isfinite(dgot[0, h, t]).all()
            else:
                assert torch.equal(got[0, h, t], good[0][0, h, t]) and torch.equal(dgot[0, h, t], dgood["dq"][0, h, t])
    zero = torch.zeros(1, 1, 3, 128, device="cuda", dtype=dt)
    for norm in (1, 2):
        assert not pkg.lsm_qk_norm_rope(zero, None, cs, norm=norm)[0].any()
        d = pkg.lsm_qk_norm_rope_bwd(zero, None, q[:, :1, :3], None, cs, norm=norm)["dq"]
        assert torch.isfinite(d).all() and d.any()


def test_offsets_beyond_32_bits():
    import torch
    pkg = lsm()
    far = 2 ** 31 + 64
    wide = torch.empty(far + 4 * 64, device="cuda", dtype=torch.bfloat16)
    q = wide.as_strided((1, 2, 4, 64), (0, far, 64, 1))
    q.copy_(torch.randn(1, 2, 4, 64, device="cuda"))
    near_by, cs = q.contiguous(), table(4, 64).cuda()
    out = torch.empty_like(wide).as_strided((1, 2, 4, 64), (0, far, 64, 1))
    pkg.lsm_qk_norm_rope(q, None, cs, q_out=out)
    assert torch.equal(out, pkg.lsm_qk_norm_rope(near_by, None, cs)[0])
    pkg.lsm_qk_norm_rope_bwd(q, None, q, None, cs, dq=out)
    assert torch.equal(out, pkg.lsm_qk_norm_rope_bwd(near_by, None, near_by, None, cs)["dq"])


def test_another_stream_and_replays_of_a_graph():
    import torch
    pkg = lsm()
    q = torch.randn(2, 4, 33, 128, device="cuda").to(torch.bfloat16)
    cs, w = table(33, 128).cuda(), torch.rand(128, device="cuda")
    run = lambda **kw: (pkg.lsm_qk_norm_rope(q, q, cs, q_weight=w, k_weight=w, **kw),
                        pkg.lsm_qk_norm_rope_bwd(q, q, q, q, cs, q_weight=w, k_weight=w, **kw))
    flat = lambda r: list(r[0]) + [r[1][n] for n in ("dq", "dk", "d_q_weight", "d_k_weight")]
    eager = [t.clone() for t in flat(run())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = flat(run(stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = flat(run())
    for _ in range(3):
        for t in outs:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        (q.float() * 2).sum().item()


def test_refusals():
    import torch
    pkg = lsm()
    q = torch.zeros(2, 4, 8, 128, device="cuda", dtype=torch.bfloat16)
    cs = table(8, 128).cuda()
    for bad in (dict(q=q.half()), dict(q=q.cpu()), dict(q=q.transpose(2, 3)), dict(k=q.float()), dict(k=q[:, :, :4]),
                dict(q_weight=torch.ones(64, device="cuda")), dict(q_weight=torch.ones(128, device="cuda", dtype=torch.bfloat16)),
                dict(cos_sin=cs.double()), dict(positions=torch.zeros(2, 8, device="cuda")),
                dict(positions=torch.zeros(8, device="cuda", dtype=torch.int32)), dict(k=None, k_weight=torch.ones(128, device="cuda")),
                dict(q_out=torch.empty(2, 4, 7, 128, device="cuda", dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            pkg.lsm_qk_norm_rope(**{**dict(q=q, k=q, cos_sin=cs), **bad})
    for bad in (dict(cos_sin=table(7, 128).cuda()),              # T beyond the table
                dict(cos_sin=table(8, 24).cuda()),               # not a multiple of 16
                dict(cos_sin=table(8, 144).cuda()),              # wider than the head
                dict(eps=0.0), dict(norm=3), dict(rotation=2),
                dict(q=torch.zeros(2, 4, 8, 96, device="cuda"), k=None),
                dict(q=torch.zeros(2, 4, 8, 132, device="cuda")[..., :128], k=None, norm=7),
                dict(q=torch.zeros(2, 4, 8, 130, device="cuda")[..., :128], k=None)):
        with pytest.raises(pkg.LsmError):
            pkg.lsm_qk_norm_rope(**{**dict(q=q, k=q, cos_sin=cs), **bad})
    with pytest.raises(ValueError):
        pkg.lsm_qk_norm_rope_bwd(q, q, q, q[:, :2])
