"""The experts of many tokens (lsm_moe_experts, lsm_moe_experts_bwd) against the formulas in 64 bits.

Tolerances.  A product's sum over K fp32 products of random sign is within 2^-24 * 2 sqrt(K) of their root-mean-square sum; with K up to
some thousand and two or three products behind one another that is below 2^-16 of a row's root mean square; ten times that (seven
standard deviations and more) is asked of fp32 results, and 2^-22 of the value for what follows the last sum.  The row is that of the
operand that the last product takes: a hidden gradient da_f, the sum of products that need not be small where it is, is off by so much
of the root mean square of da over f, and moves d_w_gate_up[f, d] by that times x_d.  With one pair an expert (3 tokens, 64 experts) that is
|x_d| rms_f(da) 2^-16 against |x_d| |da_f|, whatever |da_f|: the results' root mean square along f belongs into the tolerance
beside that along d.  With bf16 elements one operand of the last product has been
rounded: the activations (y), their gradients (dx, d_w_gate_up), the weighted activations (d_w_down).  Each rounding is off by at
most 2^-8 of the value, independently: the standard deviation of a result's error is at most 2^-8 / sqrt(3) times the root of the sum of
the squared products, which is formed in 64 bits too; seven of those are asked (some million results), and half a step, 2^-8, of the stored value.
Routing weights' gradients are fp32 sums of unrounded numbers."""
import math

import pytest

pytestmark = pytest.mark.gpu


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def make(n, D, F, E, k, dtype, seed=0, dropped=0.0, residual=True, skew=0.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda std, *s: (std * torch.randn(*s, generator=gen)).to(dt).cuda()
    out = torch.randn(n, E, generator=gen) + skew * torch.randn(E, generator=gen)
    value, chosen = out.sort(-1, descending=True)
    weights, chosen = torch.softmax(value[:, :k], -1), chosen[:, :k].int()
    gone = torch.rand(n, k, generator=gen) < dropped
    return dict(x=rnd(1, n, D), weights=weights.masked_fill(gone, 0.0).cuda(), chosen=chosen.masked_fill(gone, -1).cuda(),
                w_gate_up=rnd(D ** -0.5, E, 2 * F, D), w_down=rnd(F ** -0.5, E, D, F), residual=rnd(1, n, D) if residual else None,
                d_y=rnd(1, n, D))


def reference(a):
    """Results in 64 bits, and for each the root of the sum of the squares that a rounded operand's error is spread over."""
    import torch
    x, p, dy = a["x"].double(), a["weights"].double(), a["d_y"].double()
    E, D, F = a["w_down"].shape
    zero = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)
    y = zero(x) if a["residual"] is None else a["residual"].double().clone()
    r = dict(y=y, dx=zero(x), d_weights=zero(p), d_w_gate_up=zero(a["w_gate_up"]), d_w_down=zero(a["w_down"]))
    s = {k: zero(v) for k, v in r.items()}
    for e in range(E):
        rows, slot = (a["chosen"] == e).nonzero(as_tuple=True)
        if rows.numel() == 0:
            continue
        W1, W2, xe, g, pe = a["w_gate_up"][e].double(), a["w_down"][e].double(), x[rows], dy[rows], p[rows, slot][:, None]
        gate, up = (xe @ W1.t().contiguous()).split(F, -1)
        sig = torch.sigmoid(gate)
        h = gate * sig * up
        t = g @ W2
        da = torch.cat((pe * t * up * (sig + gate * sig * (1 - sig)), pe * t * gate * sig), -1)
        r["y"].index_add_(0, rows, pe * (h @ W2.t().contiguous()))
        s["y"].index_add_(0, rows, pe.square() * (h.square() @ W2.square().t().contiguous()))
        r["dx"].index_add_(0, rows, da @ W1)
        s["dx"].index_add_(0, rows, da.square() @ W1.square())
        r["d_weights"][rows, slot] = (t * h).sum(-1)
        s["d_weights"][rows, slot] = (t * h).square().sum(-1)
        r["d_w_gate_up"][e] = da.t().contiguous() @ xe
        s["d_w_gate_up"][e] = da.square().t().contiguous() @ xe.square()
        r["d_w_down"][e] = g.t().contiguous() @ (pe * h)
        s["d_w_down"][e] = g.square().t().contiguous() @ (pe * h).square()
    return r, {k: v.sqrt() for k, v in s.items()}


def compare(name, got, want, spread, bf16):
    import torch
    assert got.shape == want.shape, name
    scale = torch.maximum(spread, spread.square().mean(-1, keepdim=True).sqrt())
    if name == "d_w_gate_up":
        scale = torch.maximum(scale, spread.square().mean(-2, keepdim=True).sqrt())
    fp32 = 10 * 2.0 ** -16 * scale + 2.0 ** -22 * want.abs()
    tol = fp32 + (7 * 2.0 ** -8 / math.sqrt(3) * spread + 2.0 ** -8 * want.abs() if bf16 else 0)
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (name, int(bad.sum()), float((err / tol.clamp(min=1e-300)).max()))


def run(a, **kw):
    plan = lsm().lsm_moe_plan(a["chosen"], a["w_down"].shape[0])
    what = a["x"], a["weights"], plan, a["w_gate_up"], a["w_down"]
    return dict(lsm().lsm_moe_experts_bwd(*what, a["d_y"], **kw), y=lsm().lsm_moe_experts(*what, residual=a["residual"]))


def check(a):
    import torch
    got = run(a)
    torch.cuda.synchronize()
    want, spread = reference(a)
    for name, w in want.items():
        assert got[name].dtype == (torch.float32 if name == "d_weights" else a["x"].dtype)
        compare(name, got[name], w, spread[name], got[name].dtype == torch.bfloat16)
    return got


# n, D, F, E, k: one token; fewer pairs than experts; rows per expert around each tile's (32, 64, 128, 256); widths beside tiles'
SIZES = [(1, 8, 8, 1, 1), (1, 64, 72, 8, 2), (3, 264, 136, 64, 4), (31, 128, 128, 1, 1), (33, 136, 40, 1, 1), (64, 256, 264, 2, 1),
         (65, 72, 520, 1, 1), (100, 512, 64, 5, 5), (200, 320, 200, 3, 2), (257, 264, 392, 2, 2), (700, 128, 136, 4, 2), (1100, 200, 136, 2, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,F,E,k", SIZES)
def test_values_and_gradients(dtype, n, D, F, E, k):
    check(make(n, D, F, E, k, dtype, seed=n + D, residual=n % 2 == 0))


# sizes with which each of the seven tiles is the one chosen for each of the products, in either type
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,F,E,k", [(18, 264, 208, 64, 3), (2090, 136, 96, 64, 2), (11292, 40, 72, 8, 2), (7222, 40, 256, 33, 1),
                                       (15443, 192, 40, 8, 2), (2647, 728, 48, 5, 2), (12, 168, 1048, 33, 2), (12665, 72, 80, 33, 3),
                                       (154, 888, 40, 64, 1), (18941, 136, 40, 8, 2), (1200, 1032, 520, 4, 2), (6000, 264, 392, 3, 1)])
def test_every_tile(dtype, n, D, F, E, k):
    check(make(n, D, F, E, k, dtype, seed=n + F, skew=0.5, dropped=0.1))


# The largest tiles in more number than there are compute units, so that workgroups go on to a second and a third: 298 or 550 tiles of rows, one to
# four of columns; products of 2, 3, 4, 5, 9 and 13 steps (a step is 32 numbers), of which those below five are filled up.
@pytest.mark.parametrize("full,D,F", [(45, 128, 72), (45, 136, 72), (24, 264, 64), (24, 392, 264)])
def test_tiles_that_follow_one_another(full, D, F):
    """Every expert has `full` whole tiles of 256 rows and a last one of 1, 64, 65, 128, 129 or no rows: waves with rows behind the last, and columns
    behind the widths, store nothing between two tiles."""
    import torch
    last = [1, 64, 65, 128, 129, 0, 0, 129, 128, 65, 64, 1]
    experts = torch.cat([torch.full((256 * full + r,), e, dtype=torch.int32) for e, r in enumerate(last)] + [torch.full((37,), -1, dtype=torch.int32)])
    n = experts.numel()
    a = make(n, D, F, 12, 1, "bf16", seed=D + F)
    gen = torch.Generator().manual_seed(full)
    a["chosen"] = experts[torch.randperm(n, generator=gen)][:, None].cuda()
    a["weights"] = (0.25 + torch.rand(n, 1, generator=gen)).cuda()
    check(a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_longer_list_than_is_held_at_a_time(dtype):
    """Weight gradients over 5000 pairs of an expert: the list of rows (2048 at a time) is filled again and again."""
    check(make(5000, 64, 72, 1, 1, dtype, seed=5))
    check(make(3000, 72, 64, 3, 2, dtype, seed=6, skew=2.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_pairs_and_experts_without_tokens(dtype):
    import torch
    a = make(150, 128, 72, 40, 3, dtype, seed=7, dropped=0.4, skew=3.0)
    a["chosen"][a["chosen"] == 11] = -1
    a["chosen"][:4] = -1  # tokens that go nowhere
    a["x"][0] = float("nan")
    a["d_y"][1] = float("inf")  # of tokens that no expert sees: not read
    a["residual"][0] = 1.0
    want = {k: v.clone() if v is not None else None for k, v in a.items()}
    want["x"][0] = 0
    want["d_y"][1] = 0
    got = run(a)
    r, s = reference(want)
    for name in r:
        compare(name, got[name], r[name], s[name], got[name].dtype == torch.bfloat16)
    assert (got["d_w_gate_up"][11] == 0).all() and (got["d_w_down"][11] == 0).all()
    assert (got["dx"][:4] == 0).all() and (got["d_weights"][a["chosen"] < 0] == 0).all()
    a["chosen"][:] = -1  # no pair at all
    got = run(a)
    assert torch.equal(got["y"], a["residual"]) and all((got[n] == 0).all() for n in r if n != "y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_stays_with_its_token_and_expert(dtype):
    import torch
    a = make(90, 128, 72, 4, 1, dtype, seed=9)
    clean = run(a)
    a["x"][17, 5] = float("nan")
    e = int(a["chosen"][17, 0])
    a["w_down"][(e + 1) % 4, 3, 2] = float("inf")  # feature 3 of every token of that expert
    got = run(a)
    other = torch.arange(90, device="cuda") != 17
    inf_tokens = (a["chosen"][:, 0] == (e + 1) % 4)
    assert torch.isnan(got["y"][17]).all() and torch.isnan(got["dx"][17]).all()
    assert torch.equal(got["y"][other & ~inf_tokens], clean["y"][other & ~inf_tokens])
    assert torch.equal(got["dx"][other & ~inf_tokens], clean["dx"][other & ~inf_tokens])
    keep = torch.arange(128, device="cuda") != 3
    assert torch.equal(got["y"][inf_tokens][:, keep], clean["y"][inf_tokens][:, keep]) and not torch.isfinite(got["y"][inf_tokens][:, 3]).any()
    for name in ("d_w_gate_up", "d_w_down"):
        for q in range(4):
            if q not in (e, (e + 1) % 4):
                assert torch.equal(got[name][q], clean[name][q])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_small_numbers(dtype):
    """Pairs' rows far beyond fp16's range: the same result times a power of two."""
    import torch
    a = make(130, 128, 72, 3, 2, dtype, seed=10, residual=False)
    base = run(a)
    for scale in (2.0 ** 60, 2.0 ** -60):
        b = dict(a, w_down=a["w_down"] * scale)
        assert torch.equal(run(b)["y"], base["y"] * scale)
        b = dict(a, d_y=a["d_y"] * scale)
        got = run(b)
        for name in ("dx", "d_weights", "d_w_gate_up", "d_w_down"):
            assert torch.equal(got[name], base[name] * scale), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,E,k", [(70, 256, 16), (300, 129, 6), (9, 255, 3), (500, 253, 1)])
def test_many_experts(dtype, n, E, k):
    check(make(n, 64, 40, E, k, dtype, seed=E, skew=1.0, dropped=0.05))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_the_workspace_held_does_not_matter(dtype):
    """Workspaces of NaN (all bits set), widths that are neither whole tiles nor whole lines of the caches."""
    import torch
    for n, D, F in ((9, 72, 104), (37, 72, 104), (300, 136, 40), (2100, 264, 72)):
        a = make(n, D, F, 5, 2, dtype, seed=n, dropped=0.2)
        want = run(a)
        plan = lsm().lsm_moe_plan(a["chosen"], 5)
        what = a["x"], a["weights"], plan, a["w_gate_up"], a["w_down"]
        ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda")
        y = lsm().lsm_moe_experts(*what, residual=a["residual"], workspace=ws)
        ws.fill_(255)
        got = dict(lsm().lsm_moe_experts_bwd(*what, a["d_y"], workspace=ws), y=y)
        for name in want:
            assert torch.equal(got[name], want[name]), (name, n)


def test_rows_almost_four_gigabytes_apart():
    """Offsets that need all of 32 bits: the last rows of x and d_y begin just below 2^32 bytes."""
    import torch
    a = make(16, 72, 40, 3, 2, "bf16", seed=21)
    want = run(a)
    stride = (1 << 27) - 256
    far = torch.empty(16 * stride, dtype=torch.bfloat16, device="cuda")
    for name in ("x", "d_y"):
        b = dict(a)
        b[name] = far.as_strided((16, 72), (stride, 1))
        b[name].copy_(a[name])
        got = run(b)
        assert all(torch.equal(got[q], want[q]) for q in want), name


def test_an_expert_of_almost_four_gigabytes():
    """65528 x 16376: all zeros but the last eight features and columns, which are an expert of 8 x 8."""
    import torch
    D, F = 65528, 16376
    small = make(5, 8, 8, 1, 1, "bf16", seed=22, residual=False)
    big = dict(small, x=torch.zeros(5, D, dtype=torch.bfloat16, device="cuda"), d_y=torch.zeros(5, D, dtype=torch.bfloat16, device="cuda"),
               w_gate_up=torch.zeros(1, 2 * F, D, dtype=torch.bfloat16, device="cuda"), w_down=torch.zeros(1, D, F, dtype=torch.bfloat16, device="cuda"))
    big["x"][:, -8:], big["d_y"][:, -8:] = small["x"], small["d_y"]
    big["w_gate_up"][0, F - 8:F, -8:], big["w_gate_up"][0, -8:, -8:] = small["w_gate_up"][0, :8], small["w_gate_up"][0, 8:]
    big["w_down"][0, -8:, -8:] = small["w_down"][0]
    got = run(big)
    want, spread = reference(small)
    cut = dict(y=got["y"][:, -8:], dx=got["dx"][:, -8:], d_weights=got["d_weights"], d_w_down=got["d_w_down"][:, -8:, -8:],
               d_w_gate_up=torch.cat((got["d_w_gate_up"][:, F - 8:F, -8:], got["d_w_gate_up"][:, -8:, -8:]), 1))
    for name in want:
        compare(name, cut[name], want[name], spread[name], name != "d_weights")
    for name in ("y", "dx"):
        assert (got[name][:, :-8] == 0).all()
    assert int((got["d_w_gate_up"] != 0).sum()) <= 2 * 64 and int((got["d_w_down"] != 0).sum()) <= 64


def test_rows_further_apart():
    """x and d_y as columns of wider tensors, with numbers that are not finite between the rows."""
    import torch
    a = make(70, 128, 72, 4, 2, "bf16", seed=11)
    want = run(a)
    wide = torch.full((70, 200), float("nan"), dtype=torch.bfloat16, device="cuda")
    b = dict(a, x=wide.clone()[:, 16:144], d_y=wide.clone()[:, 64:192])
    b["x"].copy_(a["x"])
    b["d_y"].copy_(a["d_y"])
    got = run(b)
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_gradients_against_differences():
    import torch
    a = make(12, 16, 24, 3, 2, "f32", seed=12)
    got = run(a)
    plan = lsm().lsm_moe_plan(a["chosen"], 3)
    gen = torch.Generator().manual_seed(3)
    for name, grad in (("x", "dx"), ("weights", "d_weights"), ("w_gate_up", "d_w_gate_up"), ("w_down", "d_w_down")):
        way = torch.randn(a[name].shape, generator=gen).cuda()
        step = 2.0 ** -8
        value = []
        for s in (step, -step):
            b = dict(a)
            b[name] = a[name] + s * way
            y = lsm().lsm_moe_experts(b["x"], b["weights"], plan, b["w_gate_up"], b["w_down"], residual=a["residual"])
            value.append(float((y.double() * a["d_y"].double()).sum()))
        want = (value[0] - value[1]) / (2 * step)
        # third derivatives along the way (cubed lengths of it, some tens) times step^2 / 6, and the rounding of 192 results over the step
        size = float(got[grad].double().norm() * way.double().norm())
        assert abs(float((got[grad].double() * way.double()).sum()) - want) <= 2e-3 * size, name


@pytest.mark.parametrize("n,D,F,E,k", [(1, 256, 136, 4, 1), (1, 1032, 520, 16, 4), (5, 264, 2056, 8, 2), (16, 72, 264, 1, 1), (16, 520, 136, 40, 16)])
def test_few_tokens_are_rounded_once(n, D, F, E, k):
    """Up to 16 tokens only the result is rounded to bf16 (half a step, 2^-8 of it); a pair's row to half precision before that: with a
    power of two for a stretch of it, so 2^-11 of each number, or 2^-25 of the stretch's largest; and what is left of a number that is rounded in two
    halves is 2^-16 of it, spread over the sum as the spread of its products is.  fp32 sums as everywhere in this file."""
    import torch
    a = make(n, D, F, E, k, "bf16", seed=n + D, residual=False)
    got = run(a)
    want, spread = reference(a)
    for name in ("y", "dx"):
        parts = 2.0 ** -11 * 7 * spread[name].square().mean(-1, keepdim=True).sqrt().clamp(min=0)
        scale = torch.maximum(spread[name], spread[name].square().mean(-1, keepdim=True).sqrt())
        tol = 2.0 ** -8 * want[name].abs() + parts * k ** 0.5 + (10 * 2.0 ** -16 + 7 * 2.0 ** -16) * scale
        err = (got[name].double() - want[name]).abs()
        assert (err <= tol).all(), (name, float((err / tol.clamp(min=1e-300)).max()))


def half_step(want):
    """Of bf16, at each value: numbers of 2^e to 2^(e + 1) are 2^(e - 7) apart."""
    import torch
    return torch.ldexp(torch.ones_like(want), torch.frexp(want)[1] - 9)


@pytest.mark.parametrize("n,D,F,E,k", [(16, 1032, 264, 4, 1), (16, 520, 136, 40, 16), (5, 2056, 520, 8, 2), (1, 2056, 1032, 16, 4)])
def test_nothing_but_the_result_of_few_tokens_is_rounded(n, D, F, E, k):
    """Up to 16 tokens: half a step of the result at its own size, and beside that what a remainder's own rounding leaves of activations and their
    gradients, 2^-17 of each at most (2^-8 of a remainder that is 2^-9 of them), independently: 7 / sqrt(3) 2^-17 of the products' root sum of squares,
    and seven standard deviations of 2^-24 * 2 sqrt(2056) for the fp32 sums of two products behind one another, below 7 * 2^-17 of their root mean square."""
    import torch
    a = make(n, D, F, E, k, "bf16", seed=n + F, residual=False)
    got = run(a)
    want, spread = reference(a)
    for name in ("y", "dx"):
        scale = torch.maximum(spread[name], spread[name].square().mean(-1, keepdim=True).sqrt())
        tol = half_step(want[name]) + (7 / math.sqrt(3) + 7) * 2.0 ** -17 * scale
        bad = ~((got[name].double() - want[name]).abs() <= tol)
        assert not bad.any(), (name, int(bad.sum()))


@pytest.mark.parametrize("n,E,k", [(5, 4, 2), (70, 3, 1), (300, 2, 2), (9000, 12, 4)])
def test_a_pairs_row_is_whole_until_it_is_added(n, E, k):
    """Activations that bf16 holds: the gate is 64, whose sigmoid is 1, the factor a whole number up to 96.  What is rounded is then the result alone: half a
    step of it at its own size, and 2^-18 of the products' sum of sizes, for no more than 64 fp32 roundings of 2^-24 behind one another."""
    import torch
    D, F = 264, 40
    gen = torch.Generator().manual_seed(n)
    a = make(n, D, F, E, k, "bf16", seed=n, residual=False)
    a["x"][:, 0] = 1
    a["x"][:, 1:7] = torch.tensor([-2.0, -1.0, 1.0, 2.0])[torch.randint(0, 4, (n, 6), generator=gen)].to(a["x"])
    a["w_gate_up"].zero_()
    a["w_gate_up"][:, :F, 0] = 64
    a["w_gate_up"][:, F:, 1:7] = torch.randint(-8, 9, (E, F, 6), generator=gen).to(a["x"])
    plan = lsm().lsm_moe_plan(a["chosen"], E)
    got = lsm().lsm_moe_experts(a["x"], a["weights"], plan, a["w_gate_up"], a["w_down"])
    want, size = torch.zeros(n, D, dtype=torch.float64, device="cuda"), torch.zeros(n, D, dtype=torch.float64, device="cuda")
    for j in range(k):
        e = a["chosen"][:, j].long()
        h = 64 * (a["x"][:, 1:7].double()[:, None] * a["w_gate_up"].double()[e, F:, 1:7]).sum(-1)
        for f in range(F):
            one = a["weights"][:, j, None].double() * h[:, f, None] * a["w_down"].double()[e, :, f]
            want += one
            size += one.abs()
    bad = ~((got.double() - want).abs() <= half_step(want) + 2.0 ** -18 * size)
    assert not bad.any(), int(bad.sum())


def test_frozen_experts():
    import torch
    a = make(40, 64, 40, 3, 2, "bf16", seed=13)
    want = run(a)
    got = run(a, weight_grads=False)
    assert got["d_w_gate_up"] is None and got["d_w_down"] is None
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["d_weights"], want["d_weights"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_bits_twice_and_two_calls_at_once(dtype):
    import torch
    a, b = make(400, 136, 72, 5, 2, dtype, seed=14), make(300, 136, 72, 5, 2, dtype, seed=15)
    want_a, want_b = run(a), run(b)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        got_a = run(a)
    with torch.cuda.stream(t):
        got_b = run(b)
    torch.cuda.synchronize()
    assert all(torch.equal(got_a[n], want_a[n]) and torch.equal(got_b[n], want_b[n]) for n in want_a)


def test_captured_and_replayed():
    """Forward and backward in a graph with a plan that changes from replay to replay, eager work between them."""
    import torch
    a = make(500, 128, 72, 6, 2, "bf16", seed=16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(a)
    for seed in (17, 18, 19):
        for n, v in make(500, 128, 72, 6, 2, "bf16", seed=seed, dropped=0.2 * (seed - 17)).items():
            a[n].copy_(v)
        want = {n: v.clone() for n, v in run(a).items()}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in want)


def test_a_given_workspace_and_result():
    import torch
    a = make(77, 64, 40, 3, 2, "bf16", seed=20)
    want = run(a)["y"]
    plan = lsm().lsm_moe_plan(a["chosen"], 3)
    y, ws = torch.empty_like(a["x"]), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    got = lsm().lsm_moe_experts(a["x"], a["weights"], plan, a["w_gate_up"], a["w_down"], residual=a["residual"], y=y, workspace=ws)
    assert got is y and torch.equal(y, want)
    with pytest.raises(lsm().LsmError):
        lsm().lsm_moe_experts(a["x"], a["weights"], plan, a["w_gate_up"], a["w_down"], workspace=ws[:1024])


def test_the_same_as_the_decode_step():
    """With lsm_moe_route, the layer that lsm_moe_step is for few tokens."""
    import torch
    gen = torch.Generator().manual_seed(21)
    x, router = torch.randn(60, 128, generator=gen).cuda(), (torch.randn(12, 128, generator=gen) / 6).cuda()
    a = make(60, 128, 72, 12, 3, "f32", seed=22)
    want = lsm().lsm_moe_step(x, router, a["w_gate_up"], a["w_down"], 3, residual=a["residual"])
    w, c = lsm().lsm_moe_route(x @ router.t(), 3)
    got = lsm().lsm_moe_experts(x, w, lsm().lsm_moe_plan(c, 12), a["w_gate_up"], a["w_down"], residual=a["residual"])
    # both within 10 * 2^-16 of the 64-bit result's root mean square
    assert float((got - want).abs().max()) <= 20 * 2.0 ** -16 * float(want.square().mean().sqrt())
