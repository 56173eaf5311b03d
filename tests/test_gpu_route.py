"""Routing (lsm_moe_route, its gradient) and the plan (lsm_moe_plan) against plain forms in 64 bits and sorting.

Tolerance.  A weight is a quotient of exponentials of fp32 differences of at most some tens: the difference's rounding moves an
exponential by 2^-24 of its exponent's size (32 at most where it counts: 2^-19), exponential, sum of up to 256 and quotient by a few
2^-24.  Weights are held to 2^-19 of themselves; a gradient w (d - along), whose `along` is a sum of up to 16 terms, to 2^-19 of |w| times the
largest |d|, and stored as bf16 to half a step (2^-8) more."""
import pytest

pytestmark = pytest.mark.gpu
INF = float("inf")


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def make(n, E, dtype="f32", seed=0, bars=0.0, padding=0.0, values=None):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = 2 * torch.randn(n, E, generator=gen)
    if values:  # few different ones: many ties
        x = torch.randint(0, values, (n, E), generator=gen).float() - values // 2
    x[:, torch.rand(E, generator=gen) < bars] = -INF
    x[torch.rand(n, generator=gen) < padding] = -INF
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def plain(x, k, renormalise, d=None):
    """weights, chosen and d_logits for finite logits and -inf."""
    import torch
    x = x.double().cpu().requires_grad_()
    value, chosen = torch.sort(x.detach(), dim=-1, descending=True, stable=True)
    value, chosen = value[:, :k], chosen[:, :k]
    there = value > -INF
    some = torch.where(there[:, :1], x, torch.zeros_like(x))
    w = torch.softmax(some, -1).gather(1, chosen)
    if renormalise:
        w = torch.softmax(some.gather(1, chosen), -1)
    w = torch.where(there, w, torch.zeros_like(w))
    if d is None:
        return w.detach(), chosen.masked_fill(~there, -1), None
    g, = torch.autograd.grad(w, x, torch.where(there, d.double().cpu(), 0.0))
    return w.detach(), chosen.masked_fill(~there, -1), g


def check(x, k, renormalise=True, seed=5):
    import torch
    n, E = x.shape
    d = torch.randn(n, k, generator=torch.Generator().manual_seed(seed)).cuda()
    w, c = lsm().lsm_moe_route(x, k, renormalise=renormalise)
    g = lsm().lsm_moe_route_bwd(x, c, d, renormalise=renormalise)
    assert w.dtype == torch.float32 and c.dtype == torch.int32 and g.dtype == x.dtype
    w_, c_, g_ = plain(x, k, renormalise, d)
    assert torch.equal(c.cpu().long(), c_)
    assert ((w.cpu().double() - w_).abs() <= 2.0 ** -19 * w_).all()
    p = torch.zeros(n, E, dtype=torch.float64).scatter_add_(1, c_.clamp(min=0), w_)
    if not renormalise:
        p = torch.softmax(torch.where(c_[:, :1] >= 0, x.double().cpu(), 0.0), -1) * (c_[:, :1] >= 0)
    tol = 2.0 ** -19 * p * d.abs().max(-1, keepdim=True).values.cpu() + (2.0 ** -8 * g_.abs() + 2.0 ** -133 if x.dtype == torch.bfloat16 else 0)
    assert ((g.cpu().double() - g_).abs() <= tol).all()
    return w, c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,k", [(1, 1, 1), (1, 64, 8), (3, 7, 7), (4, 64, 16), (33, 60, 4), (257, 65, 3), (100, 128, 6), (50, 129, 16),
                                   (31, 256, 8), (70, 16, 16), (5000, 64, 8)])
def test_values_and_gradients(dtype, n, E, k):
    check(make(n, E, dtype, seed=n + E), k, True)
    check(make(n, E, dtype, seed=n + E + 1), k, False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_the_lowest_index(dtype):
    for values in (1, 2, 5):
        check(make(200, 130, dtype, seed=values, values=values), 8)
    x = make(4, 64, dtype)
    x[:] = 0.0
    x[:, ::2] = -0.0  # equal to 0
    _, c = check(x, 5)
    assert (c.cpu() == __import__("torch").arange(5)).all()


@pytest.mark.parametrize("renormalise", [True, False])
def test_masks_that_leave_few_or_none(renormalise):
    import torch
    x = make(300, 40, "f32", seed=2, bars=0.5, padding=0.2)
    check(x, 8, renormalise)
    x[:, 3:] = -INF  # three experts left, eight wanted
    w, c = check(x, 8, renormalise)
    assert (c[:, 3:] == -1).all() and (w[:, 3:] == 0).all()
    x[:] = -INF
    w, c = check(x, 8, renormalise)
    assert (c == -1).all() and (w == 0).all()
    low = torch.finfo(torch.float32).min  # the type's lowest value is a number, not a mask
    x[:] = low
    w, c = check(x, 8, True)
    assert (c.cpu() == torch.arange(8)).all() and (w == 0.125).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_that_are_not_finite(dtype):
    import torch
    x = make(6, 20, dtype, seed=3)
    want = x.clone()
    x[0, 4] = float("nan")
    want[0, 4] = -INF
    x[1, 7] = INF
    want[1, 7] = torch.finfo(x.dtype).max
    x[2] = float("nan")
    want[2] = -INF
    for renormalise in (True, False):
        a, b = lsm().lsm_moe_route(x, 4, renormalise), lsm().lsm_moe_route(want, 4, renormalise)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.isfinite(a[0]).all()
        d = torch.randn(6, 4, device="cuda")
        assert torch.equal(lsm().lsm_moe_route_bwd(x, a[1], d, renormalise), lsm().lsm_moe_route_bwd(want, b[1], d, renormalise))
    assert a[1][1, 0] == 7 and a[0][1, 0] == 1.0 and (a[1][2] == -1).all()


def test_gradient_against_differences():
    import torch
    x = make(5, 12, "f32", seed=8)
    d = torch.randn(5, 3, generator=torch.Generator().manual_seed(1)).cuda()
    for renormalise in (True, False):
        _, c = lsm().lsm_moe_route(x, 3, renormalise)
        g = lsm().lsm_moe_route_bwd(x, c, d, renormalise)
        step = 2.0 ** -6
        for t, e in ((0, int(c[0, 0])), (1, int(c[1, 2])), (2, 5), (4, 0)):
            up, down = x.clone(), x.clone()
            up[t, e] += step
            down[t, e] -= step
            a, b = (lsm().lsm_moe_route(y, 3, renormalise) for y in (up, down))
            if not (torch.equal(a[1], c) and torch.equal(b[1], c)):
                continue
            # central difference: third derivatives (below 4 of the weights) times step^2 / 6, and 2^-22 of the weights over the step
            want = float(((a[0] - b[0]) * d).sum()) / (2 * step)
            assert abs(float(g[t, e]) - want) <= (4 * step * step / 6 + 2.0 ** -22 * 3 / step) * 3 * float(d.abs().max())


def test_a_gradient_for_experts_of_ones_own():
    """Experts in another order, one that stands twice, and places without one."""
    import torch
    x = make(2, 10, "f32", seed=4)
    c = torch.tensor([[3, 7, 3, -1], [9, 0, 12, 5]], dtype=torch.int32, device="cuda")
    d = torch.randn(2, 4, generator=torch.Generator().manual_seed(2)).cuda()
    d[0, 3] = float("nan")  # not used
    d[1, 2] = float("nan")
    for renormalise in (True, False):
        g = lsm().lsm_moe_route_bwd(x, c, d, renormalise).double().cpu()
        for t, (S, dw) in enumerate((((3, 7), (d[0, 0] + d[0, 2], d[0, 1])), ((9, 0, 5), (d[1, 0], d[1, 1], d[1, 3])))):
            z = x[t].double().cpu().requires_grad_()
            w = torch.softmax(z[list(S)], 0) if renormalise else torch.softmax(z, 0)[list(S)]
            want, = torch.autograd.grad(w, z, torch.stack(dw).double().cpu())
            assert ((g[t] - want).abs() <= 2.0 ** -18 * float(torch.stack(dw).abs().max())).all()


# ---- the plan ------------------------------------------------------------------------------------------------------

def check_plan(c, E):
    import torch
    offsets, order, place = lsm().lsm_moe_plan(c, E)
    flat = c.cpu().long().view(-1)
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    want = torch.sort(key, stable=True).indices
    counts = torch.bincount(key, minlength=E + 1)[:E]
    total = int(counts.sum())
    assert torch.equal(offsets.cpu().long(), torch.cat((torch.zeros(1, dtype=torch.long), counts.cumsum(0))))
    assert torch.equal(order.cpu().long()[:total], want[:total]) and (order.cpu()[total:] == -1).all()
    at = torch.full_like(flat, -1)
    at[want[:total]] = torch.arange(total)
    assert torch.equal(place.cpu().long().view(-1), at) and place.shape == c.shape


@pytest.mark.parametrize("n,k,E", [(1, 1, 1), (1, 8, 64), (5, 3, 256), (63, 1, 2), (64, 2, 64), (1023, 8, 64), (1024, 8, 17), (1025, 8, 64),
                                   (4099, 2, 129), (20000, 8, 64), (70001, 5, 256), (300000, 1, 3)])
def test_plan(n, k, E):
    """Below, at and above the pairs that one workgroup sorts (8192)."""
    import torch
    gen = torch.Generator().manual_seed(n + E)
    c = torch.randint(0, E, (n, k), generator=gen, dtype=torch.int32)
    check_plan(c.cuda(), E)
    c[torch.rand(n, k, generator=gen) < 0.3] = -1
    c[torch.rand(n, k, generator=gen) < 0.05] = E
    c[0, 0] = 2 ** 31 - 1
    check_plan(c.cuda(), E)


def test_plan_of_one_expert_and_of_none():
    import torch
    check_plan(torch.full((3000, 4), 5, dtype=torch.int32, device="cuda"), 9)
    check_plan(torch.full((3000, 4), -1, dtype=torch.int32, device="cuda"), 9)


def test_captured_and_replayed():
    """Route, plan and gradient in a graph whose logits change between replays."""
    import torch
    x = make(3000, 64, "f32", seed=1)
    d = torch.randn(3000, 4, device="cuda")

    def run():
        w, c = lsm().lsm_moe_route(x, 4)
        return (w, c) + lsm().lsm_moe_plan(c, 64) + (lsm().lsm_moe_route_bwd(x, c, d),)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for seed in (2, 3, 4):
        x.copy_(make(3000, 64, "f32", seed=seed))
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_on_another_stream():
    import torch
    x = make(2000, 64, "f32", seed=6)
    want = lsm().lsm_moe_route(x, 8)
    plan = lsm().lsm_moe_plan(want[1], 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = lsm().lsm_moe_route(x, 8, stream=side)
    again = lsm().lsm_moe_plan(got[1], 64, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + again, want + plan))
