"""The operators as a training step uses them: loss and gradients of examples/train_step.py against the same model written out
plainly in 64 bits with automatic differentiation, and the step captured into a graph.

Tolerance of the fp32 model: each operator is within 2^-13 of its results' root mean square (the mixer's own tests ask 1e-4 of the
largest), and two layers with their backward passes put some twenty of them behind one another: 20 x 2^-13 = 2.4e-3 of a gradient's
root mean square if all errors went the same way; 2e-3 is asked."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_loss(m, p, tokens, teacher):
    """The same loss in 64 bits on the CPU, token by token; p: the parameters there, in the order of parameters()."""
    import torch
    H, d, B, T = m["heads"], m["d"], *tokens.shape
    p = iter(p)
    embed, head = next(p), next(p)
    layers = [{n: next(p) for n in w} for w in m["layers"]]
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    cos, sin = m["cos_sin"].double().cpu()[:T, None].chunk(2, -1)
    turn = lambda z: torch.cat((z[..., :d // 2] * cos - z[..., d // 2:] * sin, z[..., d // 2:] * cos + z[..., :d // 2] * sin), -1)
    x = embed[tokens] * m["hidden"] ** 0.5
    for w in layers:
        y = norm(x)
        q, k, v = (y @ w["qkv"].t()).unflatten(-1, (3 * H, d)).split(H, 2)
        q, k = turn(norm(q) * w["q_weight"]) * d ** -0.5, turn(norm(k) * w["k_weight"]) * d ** -0.5
        a = torch.sigmoid(y @ w["decay"].t() + 4)
        state, o = torch.zeros(B, H, d, d, dtype=torch.float64), []
        for t in range(T):
            state = a[:, t, :, None, None] * state + k[:, t, :, :, None] * v[:, t, :, None, :]
            o.append((q[:, t, :, None, :] @ state)[:, :, 0])
        x = (x + torch.stack(o, 1).flatten(2) @ w["out"].t()).flatten(0, 1)
        y = norm(x)
        value, chosen = torch.topk(y @ w["router"].t(), m["top_k"])
        share, out = torch.softmax(value, -1), []
        for i in range(B * T):
            z = x[i]
            for j in range(m["top_k"]):
                e = chosen[i, j]
                gate, up = (w["w_gate_up"][e] @ y[i]).chunk(2)
                z = z + share[i, j] * (w["w_down"][e] @ (gate * torch.sigmoid(gate) * up))
            out.append(z)
        x = torch.stack(out).view(B, T, -1)
    logp = norm(x.flatten(0, 1)) @ head.t()
    if teacher is None:
        logp = torch.log_softmax(logp, -1).view(B, T, -1)[:, :-1]
        return -logp.gather(2, tokens[:, 1:, None]).mean()
    index, logits, tau = teacher
    share = torch.softmax(logits.double() / tau, -1)
    return (share * (share.log() - torch.log_softmax(logp / tau, -1).gather(1, index.long()))).sum(1).mean()


@pytest.mark.parametrize("distill", [False, True])
def test_loss_and_gradients(distill):
    import torch
    ex = example()
    m = ex.make_model(hidden=72, heads=2, d=64, layers=2, experts=6, top_k=2, width=40, vocab=301, positions=64, dtype=torch.float32, seed=3)
    gen = torch.Generator().manual_seed(4)
    tokens, teacher = torch.randint(0, 301, (2, 37), generator=gen), None
    if distill:
        teacher = (torch.randint(0, 301, (74, 5), generator=gen, dtype=torch.int32), torch.randn(74, 5, generator=gen), 2.0)
    on_gpu = None if teacher is None else (teacher[0].cuda(), teacher[1].cuda(), teacher[2])
    params = ex.parameters(m)
    loss = ex.loss_of(m, tokens.cuda(), on_gpu)
    got = torch.autograd.grad(loss, params)
    leaves = [p.detach().double().cpu().requires_grad_() for p in params]
    want_loss = plain_loss(m, leaves, tokens, teacher)
    want = torch.autograd.grad(want_loss, leaves)
    assert abs(loss.item() - want_loss.item()) <= 1e-4 * abs(want_loss.item())
    for p, g, w in zip(params, got, want):
        rms = w.square().mean().sqrt()
        err = (g.double().cpu() - w).square().mean().sqrt()
        assert err <= 2e-3 * rms, (tuple(p.shape), float(err / rms))


@pytest.mark.parametrize("distill", [False, True])
def test_a_step_in_bf16_runs(distill):
    import torch
    ex = example()
    m = ex.make_model(hidden=256, heads=2, d=128, layers=2, experts=8, top_k=2, width=264, vocab=1001, positions=512)
    tokens = torch.randint(0, 1001, (2, 300), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    teacher = None
    if distill:
        teacher = (torch.randint(0, 1001, (600, 8), device="cuda", dtype=torch.int32), torch.randn(600, 8, device="cuda"), 1.0)
    grads = torch.autograd.grad(ex.loss_of(m, tokens, teacher), ex.parameters(m))
    assert all(torch.isfinite(g).all() and g.float().abs().max() > 0 for g in grads)


def test_operators_of_a_step_captured_and_replayed():
    """Routing, plan, experts and loss with all their gradients as one graph, while tensors of an eager step live."""
    import torch
    import paper_2503_05447_amd as lsm
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(300, 64, generator=gen).cuda()
    logits = torch.randn(300, 6, generator=gen).cuda()
    w1, w2 = (torch.randn(6, 80, 64, generator=gen) / 8).cuda(), (torch.randn(6, 64, 40, generator=gen) / 6).cuda()
    head = (torch.randn(501, 64, generator=gen) / 8).cuda()
    target = torch.randint(-50, 501, (300,), generator=gen, dtype=torch.int32).cuda()
    d_loss = torch.full((300,), 1 / 300, device="cuda")

    def step():
        weights, chosen = lsm.lsm_moe_route(logits, 2)
        plan = lsm.lsm_moe_plan(chosen, 6)
        y = lsm.lsm_moe_experts(x, weights, plan, w1, w2, residual=x)
        loss, lse = lsm.lsm_linear_cross_entropy(y, head, target)
        g = lsm.lsm_linear_cross_entropy_bwd(y, head, target, lse, d_loss)
        e = lsm.lsm_moe_experts_bwd(x, weights, plan, w1, w2, g["dx"])
        return [loss, g["dw"], e["dx"], e["d_w_gate_up"], e["d_w_down"], lsm.lsm_moe_route_bwd(logits, chosen, e["d_weights"])]
    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        if i:
            logits.copy_(torch.randn(300, 6, generator=gen))
            x.copy_(torch.randn(300, 64, generator=gen))
            eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
