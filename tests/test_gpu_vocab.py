"""The losses over a vocabulary (lsm_linear_cross_entropy, lsm_linear_distill and their gradients) against the definitions in 64 bits.

Tolerances.  A logit is an fp32 sum of D products: within 2^-24 * 2 sqrt(D) of the products' root-mean-square sum, which is below
8 here, and 2^-22 of itself: under 2^-16 with seven standard deviations for D up to 1000.  lse and loss move by no more than the logits (their derivatives by
the logits sum to 1, the loss's to 2 in size) and by a few 2^-23 of their own size: 2^-15 + 2^-21 |value|.  A gradient of a logit
moves by p times 2^-15 and, with bf16 elements, by half a step, 2^-8, when it is rounded on its way into the next product; independent roundings
give a result whose error's standard deviation is 2^-8 / sqrt(3) times the root of the sum of the squared products, formed in 64 bits too.
Seven of them are asked and half a step of the stored value; of fp32 elements 2^-15 times the sum of p times the weights' size, and ten times
2^-24 * 2 sqrt(K) of the squared products' root for the sum itself."""
import math

import pytest

pytestmark = pytest.mark.gpu
INF = float("inf")


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def make(n, D, V, K, dtype, seed=0, left_out=0.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    a = dict(x=torch.randn(n, D, generator=gen).to(dt).cuda(), w=(2 * D ** -0.5 * torch.randn(V, D, generator=gen)).to(dt).cuda(),
             d_loss=(0.5 + torch.rand(n, generator=gen)).cuda(), teacher=None)
    if K:
        a["index"] = torch.randint(0, V, (n, K), generator=gen, dtype=torch.int32).cuda()
        a["teacher"] = (3 * torch.randn(n, K, generator=gen)).cuda()
        a["index"][(torch.rand(n, generator=gen) < left_out).cuda()] = -1
    else:
        a["index"] = torch.randint(0, V, (n,), generator=gen, dtype=torch.int32).cuda()
        a["index"][(torch.rand(n, generator=gen) < left_out).cuda()] = -100
    return a


def reference(a, tau=1.0):
    import torch
    n, V = a["x"].shape[0], a["w"].shape[0]
    if a["teacher"] is None:
        index = a["index"].long()[:, None]
        there = (index >= 0) & (index < V)
        share = there.double()
    else:
        index = a["index"].long()
        logit = torch.nan_to_num(a["teacher"].double(), nan=-INF, posinf=torch.finfo(torch.float32).max, neginf=-INF)
        there = (index >= 0) & (index < V) & (logit > -INF)
        top = torch.where(there, logit, -INF).max(1, keepdim=True).values.clamp(min=-1e39)
        share = torch.where(there, torch.exp((logit - top) / tau), 0.0)
        share = share / share.sum(1, keepdim=True).clamp(min=1e-300)
    counts = there.any(1)
    x = torch.where(counts[:, None], a["x"].double(), 0.0)
    w = a["w"].double()
    z = x @ w.t().contiguous() / tau
    lse = torch.logsumexp(z, 1)
    at = torch.where(there, index, 0)
    loss = (torch.special.xlogy(share, share) + share * (lse[:, None] - z.gather(1, at))).sum(1)
    p = torch.exp(z - lse[:, None])
    weight = torch.where(counts, a["d_loss"].double(), 0.0)[:, None] / tau
    g = weight * p.scatter_add(1, at, -share)
    r = dict(loss=torch.where(counts, loss, 0.0), lse=torch.where(counts, lse, 0.0), dx=g @ w, dw=g.t().contiguous() @ x)
    spread = dict(dx=(g.square() @ w.square()).sqrt(), dw=(g.square().t().contiguous() @ x.square()).sqrt())
    moved = dict(dx=(weight * p) @ w.abs(), dw=(weight * p).t().contiguous() @ x.abs())
    return r, spread, moved, dict(dx=V, dw=n)


def run(a, tau=1.0, **kw):
    what = [a["x"], a["w"], a["index"]] + ([] if a["teacher"] is None else [a["teacher"]])
    fwd, bwd = ((lsm().lsm_linear_cross_entropy, lsm().lsm_linear_cross_entropy_bwd) if a["teacher"] is None else
                (lsm().lsm_linear_distill, lsm().lsm_linear_distill_bwd))
    loss, lse = fwd(*what, temperature=tau)
    return dict(bwd(*what, lse, a["d_loss"], temperature=tau, **kw), loss=loss, lse=lse)


def check(a, tau=1.0):
    import torch
    got = run(a, tau)
    torch.cuda.synchronize()
    want, spread, moved, K = reference(a, tau)
    for name in ("loss", "lse"):
        assert got[name].dtype == torch.float32
        err = (got[name].double() - want[name]).abs()
        bad = ~(err <= (2.0 ** -15) / min(tau, 1.0) + 2.0 ** -21 * want[name].abs())
        assert not bad.any(), (name, float(err.max()))
    for name in ("dx", "dw"):
        assert got[name].dtype == a["x"].dtype
        tol = 2.0 ** -15 / min(tau, 1.0) * moved[name] + (10 * 2.0 ** -23 * math.sqrt(K[name]) + 2.0 ** -20) * spread[name]
        if a["x"].dtype == torch.bfloat16:
            tol = tol + 7 * 2.0 ** -8 / math.sqrt(3) * spread[name] + 2.0 ** -8 * want[name].abs()
        err = (got[name].double() - want[name]).abs()
        bad = ~(err <= tol + 1e-30)
        assert not bad.any(), (name, int(bad.sum()), float((err / (tol + 1e-30)).max()))
    return got


# n, D, V: one token; rows around each tile's (32, 64, 128, 256); vocabularies beside 64, 128 and 256, odd and smaller than a tile
SIZES = [(1, 8, 1), (1, 64, 50), (3, 72, 1001), (32, 128, 257), (33, 264, 130), (64, 136, 513), (70, 128, 2047), (129, 520, 300),
         (257, 64, 1025), (300, 200, 777), (600, 72, 2049)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,V", SIZES)
def test_cross_entropy(dtype, n, D, V):
    check(make(n, D, V, 0, dtype, seed=n + V, left_out=0.3 if n > 3 else 0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,V,K", [(1, 8, 1, 1), (1, 64, 50, 3), (3, 72, 1001, 20), (33, 264, 300, 64), (70, 128, 2047, 65), (129, 520, 3001, 100),
                                     (257, 64, 1025, 1), (300, 72, 777, 256), (600, 64, 2049, 8)])
def test_distillation(dtype, n, D, V, K):
    """With replacement: entries of the same token among them."""
    check(make(n, D, V, K, dtype, seed=n + V, left_out=0.2 if n > 3 else 0.0), tau=2.0 if n % 2 else 1.0)


# sizes with which each of the seven tiles is the one chosen for each of the products, in either type
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 70])
@pytest.mark.parametrize("n,D,V", [(1, 24, 18658), (790, 24, 1331), (8195, 24, 452), (37, 24, 64137), (8173, 24, 1028), (2, 136, 54471), (1, 24, 2580),
                                   (213, 24, 541), (82, 24, 2750), (1, 152, 2729), (18331, 464, 51), (1000, 520, 5003), (2500, 264, 3001)])
def test_every_tile(dtype, K, n, D, V):
    check(make(n, D, V, K, dtype, seed=n + V, left_out=0.1 if n > 3 else 0.0))


# The largest tiles in more number than there are compute units, so that workgroups go on to a second and a third: `rows` of the tokens count, a
# last tile of 1, 64, 129 or all of its 256 rows; products of 1, 5 and 9 steps (a step is 32 numbers), of which those below five are filled up.
@pytest.mark.parametrize("n,D,V,rows", [(3000, 24, 9001, 2561), (3000, 24, 9001, 2816), (4001, 136, 9001, 3969), (6000, 264, 5001, 5184)])
def test_tiles_that_follow_one_another(n, D, V, rows):
    import torch
    a = make(n, D, V, 0, "bf16", seed=rows)
    a["index"][torch.randperm(n, generator=torch.Generator().manual_seed(V))[rows:].cuda()] = -100
    check(a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,K,where", [(70, 2047, 70, (490, 540)), (33, 1024, 256, (0, 1024)), (300, 513, 5, (508, 513)), (5, 70001, 66, (511, 514)),
                                         (64, 4096, 64, (4032, 4096))])
def test_entries_close_together(dtype, n, V, K, where):
    """A teacher's tokens within a few columns, on both sides of a border, most of them several times, at the vocabulary's ends; some rows
    with entries that do not count between them."""
    import torch
    a = make(n, 72, V, K, dtype, seed=n + K)
    a["index"] = (where[0] + a["index"] % (where[1] - where[0])).int()
    a["index"][::3, ::2] = torch.tensor([-1, V], dtype=torch.int32).cuda()[torch.arange((K + 1) // 2).cuda() % 2]
    a["teacher"][1::4, 1::3] = -INF
    check(a)


@pytest.mark.parametrize("K", [0, 9])
@pytest.mark.parametrize("n,D,V", [(1, 64, 777), (1, 1032, 50), (3, 264, 20001), (16, 136, 3001), (16, 2056, 700)])
def test_few_tokens_are_rounded_once(n, D, V, K):
    """Up to 16 tokens only dx and dw are rounded to bf16 (half a step, 2^-8); what is left of a number in two halves is 2^-16 of it.  fp32 as in
    check()."""
    import torch
    a = make(n, D, V, K, "bf16", seed=n + V)
    got = run(a)
    want, spread, moved, length = reference(a)
    for name in ("dx", "dw"):
        tol = 2.0 ** -15 * moved[name] + (10 * 2.0 ** -23 * math.sqrt(length[name]) + 2.0 ** -20 + 7 * 2.0 ** -16) * spread[name]
        err = (got[name].double() - want[name]).abs()
        tol = tol + 2.0 ** -8 * want[name].abs() + 1e-30
        assert (err <= tol).all(), (name, float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_temperatures(dtype):
    for tau in (0.5, 3.0):
        check(make(40, 64, 500, 0, dtype, seed=1), tau)
        check(make(40, 64, 500, 7, dtype, seed=2), tau)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_vocabulary_in_pieces(dtype):
    """More tokens than one piece of the gradient holds: 33000 x 8192 of bf16 (half of fp32) are above it; a few rows count."""
    import torch
    a = make(33000, 16, 9001, 0, dtype, seed=3)
    a["index"][torch.arange(33000, device="cuda") % 97 != 5] = -100
    p = lsm().train._vocab_params(33000, 16, 9001, 0, 1 if dtype == "bf16" else 0, 1.0, 0, 16)
    assert p[2] < 33000 * 9001 * a["x"].element_size()
    got = run(a)
    keep = (a["index"] >= 0).nonzero().squeeze(1)
    b = dict(a, x=a["x"][keep].contiguous(), index=a["index"][keep].contiguous(), d_loss=a["d_loss"][keep].contiguous())
    want, spread, moved, K = reference(b)
    for name, full in (("loss", got["loss"][keep]), ("lse", got["lse"][keep]), ("dx", got["dx"][keep]), ("dw", got["dw"])):
        bf16 = full.dtype == torch.bfloat16
        if name in moved:
            tol = 2.0 ** -15 * moved[name] + (10 * 2.0 ** -23 * math.sqrt(K[name]) + 2.0 ** -20) * spread[name]
            tol = tol + (7 * 2.0 ** -8 / math.sqrt(3) * spread[name] + 2.0 ** -8 * want[name].abs() if bf16 else 0)
        else:
            tol = 2.0 ** -15 + 2.0 ** -21 * want[name].abs()
        assert ((full.double() - want[name]).abs() <= tol + 1e-30).all(), name
    gone = a["index"] < 0
    assert (got["dx"][gone] == 0).all() and (got["loss"][gone] == 0).all() and (got["lse"][gone] == 0).all()


@pytest.mark.parametrize("n,D,V,pieces", [(3, 1024, 50257, 1), (64, 1024, 20001, 1), (700, 1032, 33000, 1), (8191, 1032, 20001, 2)])
def test_what_fits_into_one_piece_is_one(n, D, V, pieces):
    """Launches of the logits' gradient: 8191 x 16384 of bf16 is what a piece holds."""
    import torch
    a = make(n, D, V, 0, "bf16", seed=n)
    loss, lse = lsm().lsm_linear_cross_entropy(a["x"], a["w"], a["index"])
    lsm().lsm_profile_start()
    lsm().lsm_linear_cross_entropy_bwd(a["x"], a["w"], a["index"], lse, a["d_loss"])
    torch.cuda.synchronize()
    names = [name for name, _ in lsm().lsm_profile_stop()]
    assert names.count("vocab_grad") == names.count("vocab_dw") == names.count("vocab_dx") == pieces


def test_whole_pieces_that_end_with_full_rounds():
    """8191 tokens of which most count, three pieces: 51 columns of tiles, of the 64 that fit, twice, and what is left; dx's sums go from piece to piece."""
    check(make(8191, 1032, 40001, 0, "bf16", seed=41, left_out=0.3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,D,V,left_out", [(2100, 72, 20001, 0.9), (1500, 264, 9001, 0.7), (8000, 24, 5001, 0.997), (700, 520, 6000, 0.5), (3000, 72, 3001, 1.0)])
def test_few_tokens_of_many_count(dtype, n, D, V, left_out):
    """dx's sums are then in more shares of the vocabulary than with all tokens; with none there is nothing to do."""
    check(make(n, D, V, 0, dtype, seed=n, left_out=left_out))


@pytest.mark.parametrize("K", [0, 5])
def test_tokens_left_out_are_not_read(K):
    import torch
    a = make(100, 64, 300, K, "bf16", seed=4)
    out = torch.arange(100, device="cuda") % 3 == 1
    a["index"][out] = -100 if K else 300
    a["x"][out] = float("nan")
    a["d_loss"][out] = INF
    if K:
        a["teacher"][out] = float("nan")
    got = check(dict(a, x=torch.where(out[:, None], torch.zeros_like(a["x"]), a["x"])))
    here = run(a)
    assert all(torch.equal(here[n], got[n]) for n in got)
    assert (here["dx"][out] == 0).all() and (here["loss"][out] == 0).all() and (here["lse"][out] == 0).all()
    a["index"][:] = -1  # none is left
    got = run(a)
    assert all((got[n] == 0).all() for n in got)


def test_entries_that_do_not_count():
    """Of a teacher's entries: an index beyond either end, -inf, NaN; +inf takes all; every entry the same token."""
    import torch
    a = make(8, 64, 200, 6, "f32", seed=5)
    a["index"][0, 2], a["index"][1, 0], a["index"][2, 5] = -1, 200, 2 ** 31 - 1
    a["teacher"][3, 1] = -INF
    a["teacher"][4, 4] = float("nan")
    a["teacher"][5, 3] = INF
    a["index"][6] = 77
    a["teacher"][7] = -INF  # left out
    got = check(a, 1.5)
    assert got["loss"][7] == 0 and (got["dx"][7] == 0).all()


def test_one_entry_is_a_target():
    import torch
    a = make(50, 64, 300, 1, "f32", seed=6)
    b = dict(a, index=a["index"][:, 0].contiguous(), teacher=None)
    got, want = run(a), run(b)
    assert all(torch.equal(got[n], want[n]) for n in ("lse", "loss"))
    for n in ("dx", "dw"):  # the target's share is subtracted before or after the token's weight
        assert float((got[n] - want[n]).abs().max()) <= 2.0 ** -21 * float(want[n].abs().max())


def test_what_is_not_finite():
    import torch
    a = make(70, 64, 300, 0, "f32", seed=7)
    clean = run(a)
    a["x"][9, 3] = float("nan")
    got = run(a)
    other = torch.arange(70, device="cuda") != 9
    for n in ("loss", "lse", "dx"):
        assert torch.equal(got[n][other], clean[n][other]) and torch.isnan(got[n][9]).all()
    a = make(70, 64, 300, 0, "f32", seed=7)
    a["w"][250] = 0
    a["w"][250, 0] = -INF  # a token that is impossible where the feature is positive, and certain where it is negative
    a["x"][:, 0] = a["x"][:, 0].abs() + 0.1
    a["index"][a["index"] == 250] = 3
    loss, lse = lsm().lsm_linear_cross_entropy(a["x"], a["w"], a["index"])
    keep = torch.arange(300, device="cuda") != 250
    z = (a["x"].double() @ a["w"][keep].double().t().contiguous())
    assert ((lse.double() - torch.logsumexp(z, 1)).abs() <= 2.0 ** -15).all() and torch.isfinite(loss).all()


def test_large_logits():
    """Logits of some hundreds: the maximum is taken out before the exponentials.  Held to 2^-24 * 16 of the largest logit's size, by
    which its rounding moves every difference."""
    import torch
    a = make(40, 64, 500, 0, "f32", seed=8)
    a["w"] *= 60
    got = run(a)
    want, _, _, _ = reference(a)
    tol = 2.0 ** -20 * 60 * 8 * 3
    assert ((got["loss"].double() - want["loss"]).abs() <= tol).all() and torch.isfinite(got["dx"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 7])
def test_what_the_workspace_held_does_not_matter(dtype, K):
    """Workspaces of NaN (all bits set), vocabularies that end inside a tile, tokens left out."""
    import torch
    for n, D, V in ((5, 72, 1001), (300, 136, 777), (2100, 72, 3001)):
        a = make(n, D, V, K, dtype, seed=n, left_out=0.3)
        want = run(a)
        ws = torch.full((1 << 27,), 255, dtype=torch.uint8, device="cuda")
        fwd, bwd, what = ((lsm().lsm_linear_cross_entropy, lsm().lsm_linear_cross_entropy_bwd, ()) if K == 0 else
                          (lsm().lsm_linear_distill, lsm().lsm_linear_distill_bwd, (a["teacher"],)))
        loss, lse = fwd(a["x"], a["w"], a["index"], *what, workspace=ws)
        ws.fill_(255)
        got = dict(bwd(a["x"], a["w"], a["index"], *what, lse, a["d_loss"], workspace=ws), loss=loss, lse=lse)
        for name in want:
            assert torch.equal(got[name], want[name]), (name, n)


@pytest.mark.parametrize("K", [0, 7])
def test_rows_almost_four_gigabytes_apart(K):
    """Offsets that need all of 32 bits: the last row of x begins just below 2^32 bytes."""
    import torch
    a = make(16, 72, 300, K, "bf16", seed=31)
    want = run(a)
    stride = (1 << 27) - 256
    far = torch.empty(16 * stride, dtype=torch.bfloat16, device="cuda")
    b = dict(a, x=far.as_strided((16, 72), (stride, 1)))
    b["x"].copy_(a["x"])
    got = run(b)
    assert all(torch.equal(got[q], want[q]) for q in want)


def test_a_vocabulary_of_more_than_four_gigabytes():
    """2^24 - 3 columns of 136: rows of w and its gradient behind 2^32 bytes, targets at both ends."""
    import torch
    V, D = (1 << 24) - 3, 136
    gen = torch.Generator("cuda").manual_seed(32)
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    w[-4:] = torch.randn(4, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(3, D, generator=gen, device="cuda", dtype=torch.bfloat16) / 8
    target = torch.tensor([V - 1, 0, V - 3], dtype=torch.int32, device="cuda")
    loss, lse = lsm().lsm_linear_cross_entropy(x, w, target)
    got = lsm().lsm_linear_cross_entropy_bwd(x, w, target, lse, torch.ones(3, device="cuda"))
    z = x.double() @ w[-4:].double().t().contiguous()                      # all other logits are 0
    want = torch.log(torch.exp(z).sum(1) + (V - 4))
    at = torch.stack((z[0, 3], torch.zeros_like(z[0, 0]), z[2, 1]))
    # lse is about 16.6: fp32 sums of 2^24 terms, a few tens at a time, then of parts: within 64 x 2^-24 of the sum, and 2^-23 of 17
    assert ((lse.double() - want).abs() <= 64 * 2.0 ** -24 + 17 * 2.0 ** -23).all() and ((loss.double() - (want - at)).abs() <= 2.0 ** -15).all()
    g = torch.zeros(3, 4, dtype=torch.float64, device="cuda")
    g += torch.exp(z - want[:, None])
    g[0, 3] -= 1
    g[2, 1] -= 1
    dw = g.t().contiguous() @ x.double()
    size = g.abs().t().contiguous() @ x.double().abs()                     # roundings of g and of the result, 2^-8 each, and 2^-18 of p
    assert ((got["dw"][-4:].double() - dw).abs() <= 2.1 * 2.0 ** -8 * size).all()
    row0 = (torch.exp(-want)[:, None] - torch.tensor([[0.0], [1.0], [0.0]], device="cuda").double()) * x.double()
    assert ((got["dw"][0].double() - row0.sum(0)).abs() <= 2.1 * 2.0 ** -8 * row0.abs().sum(0)).all()
    dx = g @ w[-4:].double()
    assert ((got["dx"].double() - dx).abs() <= 2.1 * 2.0 ** -8 * (g.abs() @ w[-4:].double().abs())).all()


def test_rows_further_apart_and_no_weight_gradient():
    import torch
    a = make(70, 64, 300, 0, "bf16", seed=9)
    want = run(a)
    wide = torch.full((70, 104), float("nan"), dtype=torch.bfloat16, device="cuda")
    b = dict(a, x=wide[:, 24:88])
    b["x"].copy_(a["x"])
    got = run(b)
    assert all(torch.equal(got[n], want[n]) for n in want)
    got = run(a, weight_grad=False)
    assert got["dw"] is None and torch.equal(got["dx"], want["dx"])


@pytest.mark.parametrize("K", [0, 4])
def test_gradients_against_differences(K):
    import torch
    a = make(10, 24, 60, K, "f32", seed=10)
    got = run(a, 1.3)
    gen = torch.Generator().manual_seed(4)
    for name, grad in (("x", "dx"), ("w", "dw")):
        way = torch.randn(a[name].shape, generator=gen).cuda()
        step, value = 2.0 ** -8, []
        for s in (step, -step):
            value.append(float((run({**a, name: a[name] + s * way}, 1.3)["loss"].double() * a["d_loss"].double()).sum()))
        size = float(got[grad].double().norm() * way.double().norm())
        # third derivatives along the way times step^2 / 6, the rounding of ten losses over the step
        assert abs(float((got[grad].double() * way.double()).sum()) - (value[0] - value[1]) / (2 * step)) <= 2e-3 * size, name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 9])
def test_the_same_bits_twice_and_two_calls_at_once(dtype, K):
    import torch
    a, b = make(300, 64, 1000, K, dtype, seed=11), make(200, 64, 900, K, dtype, seed=12)
    want_a, want_b = run(a), run(b)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s):
        got_a = run(a)
    with torch.cuda.stream(t):
        got_b = run(b)
    torch.cuda.synchronize()
    assert all(torch.equal(got_a[n], want_a[n]) and torch.equal(got_b[n], want_b[n]) for n in want_a)


@pytest.mark.parametrize("K", [0, 6])
def test_captured_and_replayed(K):
    """Forward and backward in a graph; targets and how many count change from replay to replay, eager work between them."""
    import torch
    a = make(400, 64, 900, K, "bf16", seed=13)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(a)
    for seed in (14, 15, 16):
        for n, v in make(400, 64, 900, K, "bf16", seed=seed, left_out=0.3 * (seed - 14)).items():
            if v is not None:
                a[n].copy_(v)
        want = {n: v.clone() for n, v in run(a).items()}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in want)
