"""One step of a beam search (lsm_beam_select) and the states that follow it (lsm_state_reorder).

The selection is checked in two ways.  Exactly, on logits from a grid on which fp32 arithmetic rounds nothing that decides (all
logits of a row equal, or one-hot: m and the log-normaliser are then known numbers) and on masks: parents and tokens must be
the ones the definition's order gives, ties included.  And on random logits against scores in 64 bits: the scores returned are
within the rounding of the formula of the true ones of the candidates returned, they are the best ones up to that rounding,
and equal or neighbouring scores stand in the order of their candidates.

Tolerance of a score c + ((x - m) - log s): four roundings of 2^-24 of numbers no larger than |c| + |x - m| + log V, and log s:
a sum of positive terms, each with 2^-22 for its exponential and its share of the sum's roundings (slices of a few tens of
additions and trees): 2^-20 together."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

INF = math.inf


def lsm():
    import paper_2503_05447_amd as pkg
    return pkg


def true_scores(logits, scores, finished, eos, largest):
    """[B, K V] in 64 bits."""
    x = logits.double().cpu().numpy()
    x = np.minimum(np.where(np.isnan(x), -INF, x), largest)
    m = x.max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        lp = (x - m) - np.log(np.exp(x - m).sum(-1, keepdims=True))
        s = scores.double().cpu().numpy()[..., None] + lp
    s = np.where(np.isnan(s), -INF, s)
    if finished is not None:
        alone = np.full_like(s, -INF)
        alone[..., eos] = scores.double().cpu().numpy()
        s = np.where(finished.cpu().numpy()[..., None], alone, s)
    return s.reshape(s.shape[0], -1)


def select(logits, scores, n_out=None, finished=None, eos=None):
    import torch
    out = lsm().lsm_beam_select(logits, scores, n_out, finished, eos)
    torch.cuda.synchronize()
    return out


def check(logits, scores, n_out=None, finished=None, eos=None):
    import torch
    B, K, V = logits.shape
    n = n_out or K
    got, parent, token, ended = (t if t is None else t.cpu().numpy() for t in select(logits, scores, n_out, finished, eos))
    largest = torch.finfo(logits.dtype).max
    true = true_scores(logits, scores, finished, eos, largest)
    x = logits.float().cpu().numpy()
    size = 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(true), true, 0)) + np.abs(scores.double().cpu().numpy()).clip(max=1e30).max() + math.log(V))
    for b in range(B):
        index = parent[b].astype(np.int64) * V + token[b]
        assert (0 <= parent[b]).all() and (parent[b] < K).all() and (0 <= token[b]).all() and (token[b] < V).all()
        assert len(set(index.tolist())) == n, "a candidate twice"
        t = true[b][index]
        assert (np.isneginf(got[b]) == np.isneginf(t)).all()
        fin = np.isfinite(t)
        assert (np.abs(got[b][fin] - t[fin]) <= size[b][index][fin]).all(), np.abs(got[b][fin] - t[fin]).max()
        assert (np.diff(got[b][fin]) <= 0).all() and (np.diff(fin.astype(int)) <= 0).all()
        for i in range(n - 1):
            if got[b][i] == got[b][i + 1]:
                assert index[i] < index[i + 1], "equal scores out of order"
        # equal logits of a beam have one score: whoever is in, those before it are too
        for i in np.nonzero(fin)[0]:
            k, tk = parent[b][i], token[b][i]
            if finished is None or not finished[b, k]:
                same = np.nonzero(x[b, k, :tk] == x[b, k, tk])[0]
                assert set((k * V + same).tolist()) <= set(index.tolist()), "an equal logit before it was left out"
        # nothing left out is better than the last one by more than the rounding
        rest = true[b].copy()
        rest[index] = -INF
        tol = 2 * size[b].max()
        if fin.all():
            assert rest.max() <= t[-1] + tol
        else:
            assert np.isneginf(rest).all()
            low = index[~fin]
            others = np.setdiff1d(np.nonzero(np.isneginf(true[b]))[0], low)
            assert (np.diff(low) > 0).all() and (len(others) == 0 or low.max() < others.min())
        if eos is not None:
            was = finished.cpu().numpy()[b][parent[b]] if finished is not None else np.zeros(n, bool)
            assert (ended[b] == (was | (token[b] == eos))).all()
    return got, parent, token, ended


def random_case(B, K, V, dtype, pad=0, seed=0, spread=3.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    wide = (spread * torch.randn(B, K, V + pad, generator=gen)).to(dt).cuda()
    scores = -8 * torch.rand(B, K, generator=gen)
    return wide[:, :, :V], scores.cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,V,n,pad", [(1, 1, 1, 1, 0), (1, 1, 7, 5, 0), (2, 3, 5, 15, 0), (1, 4, 1000, 4, 0), (3, 2, 4097, 4, 1),
                                         (2, 5, 16385, 10, 3), (1, 32, 999, 32, 0), (1, 1, 70001, 32, 5), (7, 4, 33333, 8, 0)])
def test_random_logits(dtype, B, K, V, n, pad):
    logits, scores = random_case(B, K, V, dtype, pad, seed=V)
    check(logits, scores, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_slices(dtype):
    """Enough beams for the longer slices of the first kernel, several of them a row, and rows that begin inside a piece."""
    logits, scores = random_case(16, 32, 20003, dtype, 1, seed=3)
    check(logits, scores, 32)
    logits, scores = random_case(64, 8, 17001, dtype, 0, seed=4)
    check(logits, scores, 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_logits_finished_beams_and_the_first_step(dtype):
    import torch
    logits, scores = random_case(4, 4, 5003, dtype, 2, seed=9)
    few = logits.clone()
    keep = torch.zeros(5003, dtype=torch.bool, device="cuda")
    keep[[3, 17, 4999]] = True
    for low in (-INF, torch.finfo(logits.dtype).min, -1e9, -30.0):
        check(few.masked_fill(~keep, low), scores, 8)
    first = scores.clone()
    first[:, 1:] = -INF
    check(logits, first, 4)
    check(logits.masked_fill(~keep, -INF), first, 8)       # three candidates, the others at -inf by their index
    done = torch.tensor([[1, 0, 0, 0], [0, 0, 0, 0], [1, 1, 1, 1], [0, 1, 0, 1]], dtype=torch.bool, device="cuda")
    check(logits, scores, 8, done, 77)
    check(logits, scores, 8, None, 77)
    check(logits, first, 8, done, 0)
    check(torch.full_like(logits, -INF), scores, 6)
    check(torch.full_like(logits, -INF), scores, 6, done, 5002)
    none = torch.full_like(scores, -INF)
    check(logits, none, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_that_are_not_numbers(dtype):
    import torch
    logits, scores = random_case(3, 2, 9001, dtype, 0, seed=10)
    logits[0, 0, 100], logits[0, 1, ::3], logits[1, 1] = float("nan"), float("nan"), float("nan")
    logits[2, 0, 7], logits[2, 0, 8999] = INF, INF
    got, parent, token, _ = check(logits, scores, 6)
    assert (parent[1] == 0).all()
    both = [t for p, t in zip(parent[2], token[2]) if p == 0][:2]
    assert set(both) <= {7, 8999}
    scores[0, 0] = float("nan")
    got, parent, token, _ = select(logits, scores, 4)
    assert (parent[0] == 1).all()


def ordered_pick(true, n):
    return np.lexsort((np.arange(true.size), -true))[:n]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [33, 4096, 20001])
@pytest.mark.parametrize("value", [0.0, -0.0, 1.0, -3.0, -1e9, "lowest"])
def test_equal_logits_go_by_index(dtype, V, value):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.finfo(dt).min if value == "lowest" else value
    logits = torch.full((2, 3, V), x, dtype=dt, device="cuda")
    scores = torch.tensor([[-1.0, -1.0, -1.0], [-2.0, -1.0, -1.0]], device="cuda")
    for n in (1, 5, 32):
        _, parent, token, _ = select(logits, scores, n)
        assert (parent.cpu().numpy() == [[0], [1]]).all() and (token.cpu().numpy() == np.arange(n)).all()
    # steps of a whole number between blocks of equal logits: the blocks by value, inside them by index
    logits = logits * 0 + 1.0
    logits[:, :, V // 2:] += 2.0
    logits[:, 1, V - 3:] += 1.0
    for n in (4, 17, 32):
        got, parent, token, _ = (t if t is None else t.cpu().numpy() for t in select(logits, scores, n))
        for b in range(2):
            true = true_scores(logits, scores, None, None, 3e38)[b]
            want = ordered_pick(np.round(true, 4), n)   # true differences are 0 or far larger
            rounded = {}
            index = parent[b].astype(np.int64) * V + token[b]
            # beams of one score can differ in the last bit of their normalisers: compare inside each beam
            for k in range(3):
                mine, ref = index[parent[b] == k], [i for i in want if i // V == k]
                assert list(mine[:len(ref)]) == ref[:len(mine)], (n, b, k)


def test_close_logits_whose_scores_round_to_one_number():
    """A score far from 0 swallows differences of small logits: what is dropped from a slice by its logit may be due by index."""
    import torch
    V = 40000
    base = torch.arange(V, device="cuda", dtype=torch.float32) * 2.0 ** -40 + 1.0   # all the same in fp32 but for the last bits
    for scores in ([[-4096.0]], [[0.0]]):
        s = torch.tensor(scores, device="cuda")
        logits = base.view(1, 1, V).clone()
        logits[0, 0] += torch.arange(V, device="cuda") % 7 * 2.0 ** -22
        got, parent, token, _ = select(logits, s, 20)
        x = logits[0, 0].cpu().numpy()
        m = x.max()
        # the formula in fp32 with the normaliser that the result implies
        lse = np.float32(math.log(np.exp(x.astype(np.float64) - m).sum()))
        y = (np.float32(s.item()) + ((x - m) - lse)).astype(np.float32)
        assert list(token[0].cpu().numpy()) == list(np.lexsort((np.arange(V), -y))[:20])
    logits = torch.zeros(1, 4, V, device="cuda")
    logits[0, 2] += torch.arange(V, device="cuda") * 1e-9
    s = torch.tensor([[-3e6, -3e6, -1e6, -3e6]], device="cuda")
    _, parent, token, _ = select(logits, s, 32)
    assert (parent == 2).all() and (token[0].cpu().numpy() == np.arange(32)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rising_logits(dtype):
    """Neighbours are the largest: more of them above one bound than a workgroup's list holds."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (torch.arange(65536, device="cuda") // 16 * 0.0078125).to(dt).view(1, 1, -1)
    for y in (x, x.flip(-1).contiguous()):
        check(y, torch.zeros(1, 1, device="cuda"), 32)
    big = torch.zeros(1, 1, 65536, device="cuda", dtype=dt)
    lanes = torch.arange(65536, device="cuda") // 8 % 64 < 33      # whole lanes of large and different values
    big[0, 0, lanes] = (100 + torch.rand(int(lanes.sum()), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 50).to(dt)
    check(big, torch.zeros(1, 1, device="cuda"), 32)
    check(big.expand(600, 1, -1).contiguous()[:, :, :16383], torch.zeros(600, 1, device="cuda"), 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices_of_several_tiles(dtype):
    """Enough beams for a workgroup to take several tiles of a row: what a later tile holds against the first one's bound."""
    import torch
    B, K, V = 64, 8, 40001
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    low = torch.finfo(dt).min
    at = torch.arange(V, device="cuda")
    logits, scores = random_case(B, K, V, dtype, 1, seed=12)
    scores = torch.where(torch.arange(K, device="cuda") == 5, scores + 30, scores).contiguous()   # one beam has nearly all
    for n in (8, 32):
        check(logits, scores, n)
        late = logits.clone()
        late[:, :, :V // 3] = -INF                                   # nothing in the first tiles
        check(late, scores, n)
        late[:, :, V // 3:] = low                                    # ... and the lowest number in all the others
        late[:, 5, V - 2] = 0
        check(late, scores, n)
        late[:, :, 100], late[:, :, 200] = 1, low
        check(late, scores, n)
        ties = logits * 0 + (at // 5003 % 3).to(dt)                  # blocks of equal ones, the largest in the third and sixth
        check(ties, scores, n)
        ties = logits * 0 - 3
        ties[:, :, 30000:] = 2                                       # more than a list holds, in later tiles only
        ties[:, :, 39990:] = 2.5
        check(ties, scores, n)
        check((at * 2.0 ** -9).to(dt).expand(B, K, V).contiguous(), scores, n)
    check(torch.where(torch.rand(B, K, V, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) < 1e-3, logits, -INF), scores, 32)


def test_offsets_beyond_32_bits():
    import torch
    V, stride = 1000, 2 ** 30 + 8
    wide = torch.empty(2 * stride + V, device="cuda", dtype=torch.bfloat16)
    logits = wide.as_strided((1, 3, V), (3 * stride, stride, 1))
    logits.copy_(3 * torch.randn(1, 3, V, device="cuda"))
    scores = torch.tensor([[-5.0, -4.0, -3.0]], device="cuda")
    a, b = select(logits, scores, 6), select(logits.contiguous(), scores, 6)
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


@pytest.mark.parametrize("K", [1, 2, 4, 5, 8, 11, 16, 32])
def test_states_follow_their_beams(K):
    import torch
    B = 3
    gen = torch.Generator(device="cuda").manual_seed(K)
    parent = torch.randint(0, K, (B, K), generator=gen, device="cuda", dtype=torch.int32)
    parent[0] = torch.arange(K, device="cuda").flip(0)             # a permutation
    states = [torch.randn(B * K, 2, 64, 64, generator=gen, device="cuda"), torch.randn(B, K, 3, 5, generator=gen, device="cuda"),
              torch.randint(0, 9, (B * K, 77), generator=gen, device="cuda", dtype=torch.int32),
              torch.randn(B * K, 4, 128, generator=gen, device="cuda").to(torch.bfloat16),
              torch.arange(B * K, device="cuda", dtype=torch.int32)]
    rows = (torch.arange(B, device="cuda")[:, None] * K + parent).view(-1)
    want = [s.reshape(B * K, -1)[rows].view(s.shape) for s in states]
    lsm().lsm_state_reorder(states, parent)
    assert all(torch.equal(a, b) for a, b in zip(states, want))
    many = [torch.randn(B * K, 8, generator=gen, device="cuda") for _ in range(70)]     # more than one launch takes
    want = [s[rows] for s in many]
    lsm().lsm_state_reorder(many, parent)
    assert all(torch.equal(a, b) for a, b in zip(many, want))
    one, kept = torch.randn(B * K, 6, device="cuda"), torch.arange(K, device="cuda", dtype=torch.int32).expand(B, K).contiguous()
    before = one.clone()
    lsm().lsm_state_reorder(one, kept)
    assert torch.equal(one, before)
    kept[1, K - 1] = K
    if K > 1:
        kept[2, 0] = -1
    lsm().lsm_state_reorder(one, kept)
    bad = [2 * K - 1] + ([2 * K] if K > 1 else [])
    assert all(torch.isnan(one[i]).all() if i in bad else torch.equal(one[i], before[i]) for i in range(B * K))


def test_rows_beyond_32_bits():
    import torch
    n = 2 ** 29 + 4                      # 2 GiB and a bit a row
    s = torch.zeros(4, n, device="cuda")
    s[:, -1] = torch.arange(4.0, device="cuda")
    s[:, 0] = 10 + torch.arange(4.0, device="cuda")
    lsm().lsm_state_reorder(s, torch.tensor([[3, 0, 2, 2]], dtype=torch.int32, device="cuda"))
    assert s[:, -1].tolist() == [3, 0, 2, 2] and s[:, 0].tolist() == [13, 10, 12, 12]


def test_another_stream_and_replays_of_a_graph():
    import torch
    pkg = lsm()
    logits, scores = random_case(5, 4, 30001, "bf16", 0, seed=2)
    done = torch.rand(5, 4, device="cuda") < 0.3
    start = torch.randn(20, 2, 64, 64, device="cuda")
    state = start.clone()

    def step(**kw):
        r = pkg.lsm_beam_select(logits, scores, 4, done, 3, **kw)
        pkg.lsm_state_reorder(state, r[1], **kw)
        return list(r)
    eager = [t.clone() for t in step()]
    moved = state.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    state.copy_(start)
    torch.cuda.synchronize()
    got = step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager)) and torch.equal(state, moved)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        state.copy_(start)
        for t in outs:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)) and torch.equal(state, moved)
        (logits.float() * 2).sum().item()


def test_refusals():
    import torch
    pkg = lsm()
    logits, scores = random_case(2, 4, 100, "f32")
    done = torch.zeros(2, 4, dtype=torch.bool, device="cuda")
    for bad in (dict(logits=logits.half()), dict(logits=logits.cpu()), dict(logits=logits[0]), dict(logits=logits.transpose(1, 2)),
                dict(logits=torch.zeros(2, 6, 100, device="cuda")[:, :4]), dict(scores=scores[:, :3]), dict(scores=scores.double()),
                dict(finished=done), dict(finished=done.int(), eos=3)):
        with pytest.raises(ValueError):
            pkg.lsm_beam_select(**{**dict(logits=logits, scores=scores), **bad})
    for bad in (dict(n_out=0), dict(n_out=33), dict(n_out=-1), dict(eos=100), dict(logits=logits[:1, :1, :3].contiguous(), scores=scores[:1, :1].contiguous(), n_out=4),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(pkg.LsmError):
            pkg.lsm_beam_select(**{**dict(logits=logits, scores=scores), **bad})
    with pytest.raises(pkg.LsmError):
        pkg.lsm_beam_select(torch.zeros(1, 33, 50, device="cuda"), torch.zeros(1, 33, device="cuda"))
    parent = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    s = torch.zeros(8, 6, device="cuda")
    for bad in (s[:7], s.cpu(), s[:, :3], torch.zeros(8, 0, device="cuda")):
        with pytest.raises(ValueError):
            pkg.lsm_state_reorder(bad, parent)
    with pytest.raises(ValueError):
        pkg.lsm_state_reorder(s, parent.long())
    with pytest.raises(ValueError):
        pkg.lsm_state_reorder(s, parent.view(-1))
    with pytest.raises(pkg.LsmError):
        pkg.lsm_state_reorder(torch.zeros(8, 3, device="cuda", dtype=torch.bfloat16), parent)


def test_nothing_is_moved_when_one_of_many_states_is_refused():
    import torch
    pkg = lsm()
    parent = torch.tensor([[1, 1, 0, 3]], dtype=torch.int32, device="cuda")
    start = torch.arange(4 * 4, dtype=torch.float32, device="cuda").view(4, 4)
    shifted = torch.zeros(4 * 4 + 1, device="cuda")[1:].view(4, 4)
    for bad in (torch.zeros(4, 3, device="cuda", dtype=torch.bfloat16), shifted):
        states = [start.clone() for _ in range(70)]
        with pytest.raises(pkg.LsmError):
            pkg.lsm_state_reorder(states + [bad], parent)
        assert all(torch.equal(s, start) for s in states)
    with pytest.raises(ValueError):
        pkg.lsm_state_reorder(torch.zeros((), device="cuda"), parent)
