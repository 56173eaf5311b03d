"""Beam selection where some scores are huge or infinite: the first step, masks of large negative numbers, masked ends of a row.

Every candidate is held to its own size.  A score c + ((x - m) - log s) is four roundings of 2^-24 of numbers no larger than
|c| + |x - m| + log V, and log s, whose sum's terms and trees are off by 2^-20 at most: so a candidate of score y is within
e = 2^-20 (1 + |y| + |c| + log V), an infinite y or c counting as 0.  Of two candidates the one returned may be worse than the one left
out by the two e, no more; in one beam, where scores fall with the logits, not at all.  The check itself is tried on wrong results."""
import math

import pytest
import torch

INF = math.inf


def definition(x, scores, finished, eos):
    """[B, K, V] scores in 64 bits; x: finite or -inf."""
    m = x.amax(-1, keepdim=True)
    s = scores[..., None] + ((x - m) - torch.exp(x - m).sum(-1, keepdim=True).log())
    s = torch.where(torch.isnan(s), -INF, s)
    if finished is not None:
        alone = torch.full_like(s, -INF)
        alone[..., eos] = scores
        s = torch.where(finished[..., None], alone, s)
    return s


def verify(x, scores, finished, eos, got, parent, token, ended):
    """x [B, K, V], scores [B, K] in 64 bits, the rest as returned: raises AssertionError unless it is the n best, best first."""
    B, K, V = x.shape
    n = got.shape[1]
    true = definition(x, scores, finished, eos)
    finite = lambda a: torch.where(torch.isfinite(a), a, 0.0)
    size = (2.0 ** -20 * (1 + finite(true).abs() + finite(scores).abs()[..., None] + math.log(V))).view(B, K * V)
    flat = true.view(B, K * V)
    assert ((0 <= parent) & (parent < K)).all() and ((0 <= token) & (token < V)).all()
    at = parent.long() * V + token.long()
    assert (at.sort(1).values.diff(dim=1) > 0).all(), "a candidate twice"
    got, t, e = got.double(), flat.gather(1, at), size.gather(1, at)
    none = torch.isneginf(t)
    assert (torch.isneginf(got) == none).all(), "the wrong ones are at -inf"
    assert (none | ((got - t).abs() <= e)).all(), "a score is off"
    assert (none.int().diff(dim=1) >= 0).all() and (none[:, 1:] | (got.diff(dim=1) <= 0)).all(), "not best first"
    assert ((got[:, 1:] != got[:, :-1]) | (at.diff(dim=1) > 0)).all(), "equal scores out of order"
    out = torch.ones_like(flat, dtype=torch.bool).scatter_(1, at, False)
    rest = torch.where(out, flat - size, -INF).amax(1)
    some = none.any(1)
    assert torch.isneginf(rest[some]).all(), "a finite candidate was left out"
    assert (rest <= t[:, -1] + e[:, -1])[~some].all(), "a better candidate was left out"
    for b in some.nonzero().flatten().tolist():
        low = at[b][none[b]]
        assert torch.equal(low, torch.isneginf(flat[b]).nonzero().flatten()[:low.numel()]), "candidates at -inf do not come by index"
    # In a beam: whoever comes before a returned one and has no smaller logit is returned too.
    live = ~none if finished is None else ~none & ~finished.gather(1, parent.long())
    index = torch.arange(V, device=x.device)
    beams = torch.arange(B, device=x.device)
    for i in range(n):
        k, tk = parent[:, i].long(), token[:, i].long()
        row = x[beams, k]
        ahead = out.view(B, K, V)[beams, k] & (index < tk[:, None]) & (row >= row.gather(1, tk[:, None]))
        assert not (ahead.any(1) & live[:, i]).any(), "a better logit of the same beam was left out"
    if eos is not None:
        was = finished.gather(1, parent.long()) if finished is not None else False
        assert (ended.bool() == (was | (token == eos))).all()


def ideal(x, scores, n, finished, eos):
    """The definition's own result."""
    B, K, V = x.shape
    s, at = definition(x, scores, finished, eos).view(B, K * V).sort(dim=1, descending=True, stable=True)
    parent, token = at[:, :n] // V, at[:, :n] % V
    ended = None if eos is None else (finished.gather(1, parent) if finished is not None else False) | (token == eos)
    return s[:, :n], parent, token, ended


def masks(dtype_min):
    return {"first step": None, "-1e9": -1e9, "lowest": dtype_min, "-inf": -INF, "-30": -30.0}


def host_case(kind):
    gen = torch.Generator().manual_seed(7)
    B, K, V = 2, 4, 601
    x, scores = 3 * torch.randn(B, K, V, generator=gen).double(), -8 * torch.rand(B, K, generator=gen).double()
    low = masks(torch.finfo(torch.float32).min)[kind]
    if low is None:
        scores[:, 1:] = -INF
    else:
        x[:, :, V // 3:] = low
    return x, scores


@pytest.mark.parametrize("kind", list(masks(0)))
def test_the_check_accepts_the_definition_and_refuses_what_is_wrong(kind):
    x, scores = host_case(kind)
    B, K, V = x.shape
    n = 6
    good = ideal(x, scores, n + 1, None, None)
    verify(x, scores, None, None, *[a[:, :n] if a is not None else None for a in good])
    low, worst = (a[:, :n] for a in definition(x, scores, None, None).view(B, K * V).sort(dim=1, stable=True))
    without = lambda i: [torch.cat((a[:, :i], a[:, i + 1:]), 1) for a in good[:3]] + [None]
    wrong = {
        "the best one left out": without(0),
        "one in the middle left out": without(2),
        "scores off": [good[0][:, :n] + 1e-3, good[1][:, :n], good[2][:, :n], None],
        "the worst": [low, worst // V, worst % V, None],
        "the worst, scores off by 1000": [low - 1000, worst // V, worst % V, None],
        "two exchanged": [a[:, [1, 0] + list(range(2, n))] for a in good[:3]] + [None],
    }
    for what, result in wrong.items():
        with pytest.raises(AssertionError):
            verify(x, scores, None, None, *result)
            pytest.fail("accepted: " + what, pytrace=False)


def test_the_check_knows_ties_and_finished_beams():
    x, scores = torch.zeros(1, 2, 9).double(), torch.zeros(1, 2).double()
    verify(x, scores, None, None, *ideal(x, scores, 4, None, None))
    s, parent, token, _ = ideal(x, scores, 4, None, None)
    with pytest.raises(AssertionError):
        verify(x, scores, None, None, s, parent, token + 1, None)         # the first one of equal ones left out
    done = torch.tensor([[True, False]])
    verify(x, scores, done, 3, *ideal(x, scores, 4, done, 3))
    s, parent, token, ended = ideal(x, scores, 4, done, 3)
    with pytest.raises(AssertionError):
        verify(x, scores, done, 3, s, parent, token, ~ended)
    none = torch.full((1, 2), -INF).double()
    s, parent, token, _ = ideal(x, none, 4, None, None)
    verify(x, none, None, None, s, parent, token, None)
    with pytest.raises(AssertionError):
        verify(x, none, None, None, s, parent, token + 1, None)


def check(logits, scores, n=None, finished=None, eos=None):
    import paper_2503_05447_amd as lsm
    verify(logits.double(), scores.double(), finished, eos, *lsm.lsm_beam_select(logits, scores, n, finished, eos))


def device_case(B, K, V, dtype, seed, pad=1):
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    return (3 * torch.randn(B, K, V + pad, generator=gen)).to(dt).cuda()[:, :, :V], (-8 * torch.rand(B, K, generator=gen)).cuda()


SHAPES = [(1, 4, 32000, 4), (3, 5, 5003, 10), (2, 1, 70001, 32), (64, 8, 25001, 8), (32, 32, 8201, 32)]  # the last two: several tiles a slice


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,V,n", SHAPES)
def test_random_logits_and_the_first_step(dtype, B, K, V, n):
    logits, scores = device_case(B, K, V, dtype, seed=V)
    check(logits, scores, n)
    scores[:, 1:] = -INF
    check(logits, scores, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["-1e9", "lowest", "-inf", "-30"])
@pytest.mark.parametrize("B,K,V,n", SHAPES)
def test_masked_parts_of_a_row(dtype, kind, B, K, V, n):
    """The end, the beginning, and all but a few places of a row masked; with the first step's scores; with finished beams."""
    logits, scores = device_case(B, K, V, dtype, seed=V + 1)
    low = masks(torch.finfo(logits.dtype).min)[kind]
    token = torch.arange(V, device="cuda")
    first = scores.clone()
    first[:, 1:] = -INF
    done = torch.rand(B, K, generator=torch.Generator().manual_seed(V)).cuda() < 0.3
    for out in (token >= V // 3, token < V - V // 5, (token % 4999 != 17) & (token != V - 1)):
        masked = logits.masked_fill(out, low)
        check(masked, scores, n)
        check(masked, first, n)
        check(masked, scores, n, done, V - 2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_best_candidate_wherever_it_stands(dtype):
    """One high logit a beam at the edges of pieces, tiles and slices, above logits that rise or fall along the row."""
    for B, K, V in ((2, 3, 20005), (64, 8, 25001)):
        logits, scores = device_case(B, K, V, dtype, seed=5)
        ramp = torch.linspace(-4, 4, V, device="cuda").to(logits.dtype)
        for base in (logits, logits + ramp, logits - ramp):
            for at in (0, 1, 4095, 4096, 8191, 8192, 16383, 16384, V - 2, V - 1):
                x = base.clone()
                x[:, :, at] = 20
                check(x, scores, K)
