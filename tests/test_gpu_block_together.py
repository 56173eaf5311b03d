"""The operators as a model uses them: the beam search of examples/beam_decode.py against the same search written out plainly in
64 bits, and the gradient of norm, rotation and token mixer chained."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("beam_decode", os.path.join(ROOT, "examples", "beam_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(m, tokens):
    """Log-probabilities of every next token of one sequence, token by token, in 64 bits on the CPU."""
    import torch
    d_ = lambda t: t.double().cpu()
    H, d, k = m["heads"], m["d"], m["top_k"]
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    cos, sin = d_(m["cos_sin"]).chunk(2, 1)
    x = d_(m["embed"])[tokens]
    T = len(tokens)
    for w in m["layers"]:
        y = norm(x)
        q, kk, v = (y @ d_(w["qkv"]).t()).view(T, 3, H, d).unbind(1)
        turn = lambda z: torch.cat((z[..., :d // 2] * cos[:T, None] - z[..., d // 2:] * sin[:T, None],
                                    z[..., d // 2:] * cos[:T, None] + z[..., :d // 2] * sin[:T, None]), -1)
        q, kk = turn(norm(q)) * d ** -0.5, turn(norm(kk)) * d ** -0.5
        a = torch.sigmoid(y @ d_(w["decay"]).t() + 4)
        state, o = torch.zeros(H, d, d, dtype=torch.float64), []
        for t in range(T):
            state = a[t][:, None, None] * state + kk[t][:, :, None] * v[t][:, None, :]
            o.append((q[t][:, None, :] @ state)[:, 0].reshape(-1))
        x = x + torch.stack(o) @ d_(w["out"]).t()
        y, res = norm(x), x
        p = torch.softmax(y @ d_(w["router"]).t(), -1)
        x = res.clone()
        for t in range(T):
            top = torch.topk(p[t], k).indices
            for e in top.tolist():
                gate, up = (d_(w["w_gate_up"][e]) @ y[t]).chunk(2)
                x[t] += p[t, e] / p[t, top].sum() * (d_(w["w_down"][e]) @ (gate * torch.sigmoid(gate) * up))
    return torch.log_softmax(norm(x) @ d_(m["head"]).t(), -1)


def plain_beams(m, prompt, beams, steps, eos):
    """[(tokens, score)] by the definition: all continuations of all beams, the best first, equal ones by beam and token."""
    live = [((), 0.0, False)]
    for _ in range(steps):
        cand = []
        for b, (toks, s, ended) in enumerate(live):
            if ended:
                cand.append((-s, b, eos, toks + (eos,), True))
                continue
            lp = plain_logits(m, prompt + list(toks))[-1]
            cand += [(-(s + lp[t].item()), b, t, toks + (t,), t == eos) for t in range(lp.numel())]
        live = [(toks, -s, e) for s, _, _, toks, e in sorted(cand)[:beams]]
    return [(toks, s) for toks, s, _ in live]


@pytest.mark.parametrize("eos", [3, 11])
def test_beam_search_of_a_small_model(eos):
    """fp32 throughout: every operator is within 1e-4 of its result, the residual stream's scale is 1, and the log-probabilities of
    five tokens are held to 2e-3; neighbouring candidates of these seeds are further apart than that, so the beams are the same."""
    import torch
    ex = example()
    m = ex.make_model(hidden=64, heads=2, d=64, layers=2, experts=8, top_k=2, width=40, vocab=19, positions=32, dtype=torch.float32, seed=4)
    prompts = torch.randint(0, 19, (2, 9), device="cuda", generator=torch.Generator("cuda").manual_seed(eos))
    history, scores = ex.beam_search(m, prompts, 3, 5, eos)
    torch.cuda.synchronize()
    for b in range(2):
        want = plain_beams(m, prompts[b].tolist(), 3, 5, eos)
        for k, (toks, s) in enumerate(want):
            assert abs(scores[b, k].item() - s) <= 2e-3, (b, k)
            assert history[b, k].tolist() == list(toks), (b, k)


def test_gradient_through_norm_rotation_and_mixer():
    """d loss / d (raw q, raw k, weights): lsm_chunk_bwd hands its gradients to lsm_qk_norm_rope_bwd.  fp32, 1e-4 of the root mean
    square as for the mixer alone."""
    import torch
    import paper_2503_05447_amd as lsm
    gen = torch.Generator().manual_seed(2)
    B, T, H, d = 1, 50, 2, 64
    raw = [torch.randn(B, T, H, d, generator=gen, dtype=torch.float32) for _ in range(4)]
    w = [torch.rand(d, generator=gen) + 0.5 for _ in range(2)]
    g = -torch.rand(B, T, H, generator=gen) * 0.1
    angle = torch.arange(T)[:, None] * 100.0 ** (-torch.arange(0, d, 2) / d)
    cs = torch.cat((angle.cos(), angle.sin()), 1).float()
    q, k, v, d_o = (t.cuda() for t in raw)
    wq, wk, gd, table = w[0].cuda(), w[1].cuda(), g.cuda(), cs.cuda()
    how = dict(cos_sin=table, q_weight=wq, k_weight=wk, norm=lsm.NORM_L2, layout=lsm.LAYOUT_BTHD)
    qn, kn = lsm.lsm_qk_norm_rope(q, k, **how)
    o, _ = lsm.lsm_chunk_fwd(qn, kn, v, gd, lsm.DECAY_SCALAR, layout=lsm.LAYOUT_BTHD)
    r = lsm.lsm_chunk_bwd(qn, kn, v, gd, lsm.DECAY_SCALAR, d_o, layout=lsm.LAYOUT_BTHD)
    dr = lsm.lsm_qk_norm_rope_bwd(q, k, r["dq"], r["dk"], **how)
    torch.cuda.synchronize()
    leaf = [t.double().requires_grad_() for t in raw[:2] + w]
    cos, sin = cs.double()[None, :, None].chunk(2, -1)

    def head(x, weight):
        n = x * torch.rsqrt(x.square().sum(-1, keepdim=True) + 1e-6) * weight
        a, b = n.chunk(2, -1)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    qd, kd, vd = head(leaf[0], leaf[2]), head(leaf[1], leaf[3]), raw[2].double()
    state, loss, out = torch.zeros(B, H, d, d, dtype=torch.float64), 0.0, []
    for t in range(T):
        state = g[:, t].double().exp()[..., None, None] * state + kd[:, t][..., :, None] * vd[:, t][..., None, :]
        out.append((qd[:, t][..., None, :] @ state)[..., 0, :])
    want_o = torch.stack(out, 1)
    grads = torch.autograd.grad((want_o * raw[3].double()).sum(), leaf)
    for got, want in zip([o, dr["dq"], dr["dk"], dr["d_q_weight"], dr["d_k_weight"]], [want_o.detach()] + list(grads)):
        assert (got.double().cpu() - want).abs().max() <= 1e-4 * want.square().mean().sqrt()
