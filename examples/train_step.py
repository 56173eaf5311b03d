"""A training step of a small Linear-MoE model of random weights: how the operators of this library follow each other forward and
backward.

A layer: projection -> lsm_qk_norm_rope -> lsm_chunk_fwd -> projection, then lsm_moe_route -> lsm_moe_plan -> lsm_moe_experts; at the end
lsm_linear_cross_entropy, or with a teacher's best logits lsm_linear_distill.  Each operator's backward call is wrapped for torch's
automatic differentiation, once: a derivative of the gradients is refused.  Projections, norms of the residual stream and the optimizer are torch.

    python examples/train_step.py [--batch 4] [--tokens 2048] [--steps 10] [--teacher 32]
"""
import argparse
import functools
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_05447_amd as lsm  # noqa: E402


def once(backward):
    """The operators' gradients are constants to automatic differentiation: under create_graph what follows from them would silently be
    differentiated as if they were, whether or not the gradients that come in require one."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        if torch.is_grad_enabled():
            raise RuntimeError("the gradients of these operators cannot be differentiated again (create_graph)")
        return backward(ctx, *grads)
    return run


class NormRotation(torch.autograd.Function):
    """q, k [B,T,H,d] -> normalised, weighted and rotated."""
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos_sin, q_scale, k_scale):
        ctx.how = dict(cos_sin=cos_sin, q_scale=q_scale, k_scale=k_scale, layout=lsm.LAYOUT_BTHD)
        ctx.save_for_backward(q, k, q_weight, k_weight)
        return lsm.lsm_qk_norm_rope(q, k, q_weight=q_weight, k_weight=k_weight, **ctx.how)

    @staticmethod
    @once
    def backward(ctx, d_q, d_k):
        q, k, q_weight, k_weight = ctx.saved_tensors
        g = lsm.lsm_qk_norm_rope_bwd(q, k, d_q.contiguous(), d_k.contiguous(), q_weight=q_weight, k_weight=k_weight, **ctx.how)
        return g["dq"], g["dk"], g["d_q_weight"], g["d_k_weight"], None, None, None


class Mixer(torch.autograd.Function):
    """The token mixer with a scalar decay a token."""
    @staticmethod
    def forward(ctx, q, k, v, g):
        ctx.save_for_backward(q, k, v, g)
        return lsm.lsm_chunk_fwd(q, k, v, g, lsm.DECAY_SCALAR, layout=lsm.LAYOUT_BTHD)[0]

    @staticmethod
    @once
    def backward(ctx, d_o):
        r = lsm.lsm_chunk_bwd(*ctx.saved_tensors, lsm.DECAY_SCALAR, d_o.contiguous(), layout=lsm.LAYOUT_BTHD)
        return r["dq"], r["dk"], r["dv"], r["dg"]


class Experts(torch.autograd.Function):
    """residual + the chosen experts of the rows of x, from the router's outputs."""
    @staticmethod
    def forward(ctx, x, logits, w_gate_up, w_down, residual, top_k):
        weights, chosen = lsm.lsm_moe_route(logits, top_k)
        ctx.plan = lsm.lsm_moe_plan(chosen, w_down.shape[0])
        ctx.save_for_backward(x, logits, weights, chosen, w_gate_up, w_down)
        return lsm.lsm_moe_experts(x, weights, ctx.plan, w_gate_up, w_down, residual=residual)

    @staticmethod
    @once
    def backward(ctx, d_y):
        x, logits, weights, chosen, w_gate_up, w_down = ctx.saved_tensors
        g = lsm.lsm_moe_experts_bwd(x, weights, ctx.plan, w_gate_up, w_down, d_y.contiguous())
        return g["dx"], lsm.lsm_moe_route_bwd(logits, chosen, g["d_weights"]), g["d_w_gate_up"], g["d_w_down"], d_y, None


class CrossEntropy(torch.autograd.Function):
    """Loss of each row of x; the logits x w^T are never there."""
    @staticmethod
    def forward(ctx, x, w, target):
        loss, lse = lsm.lsm_linear_cross_entropy(x, w, target)
        ctx.save_for_backward(x, w, target, lse)
        return loss

    @staticmethod
    @once
    def backward(ctx, d_loss):
        x, w, target, lse = ctx.saved_tensors
        g = lsm.lsm_linear_cross_entropy_bwd(x, w, target, lse, d_loss.contiguous())
        return g["dx"], g["dw"], None


class Distill(torch.autograd.Function):
    """The same against a teacher's best logits."""
    @staticmethod
    def forward(ctx, x, w, index, teacher, temperature):
        loss, lse = lsm.lsm_linear_distill(x, w, index, teacher, temperature)
        ctx.temperature = temperature
        ctx.save_for_backward(x, w, index, teacher, lse)
        return loss

    @staticmethod
    @once
    def backward(ctx, d_loss):
        x, w, index, teacher, lse = ctx.saved_tensors
        g = lsm.lsm_linear_distill_bwd(x, w, index, teacher, lse, d_loss.contiguous(), ctx.temperature)
        return g["dx"], g["dw"], None, None, None


def make_model(hidden=1024, heads=8, d=128, layers=4, experts=64, top_k=8, width=1024, vocab=32000, positions=4096,
               dtype=torch.bfloat16, seed=0):
    """Parameters of a Linear-MoE model whose mixer has a scalar decay a token (the Mamba2 row), and the rotation's table."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def weight(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).to(dtype).requires_grad_()
    layer = lambda: dict(qkv=weight(3 * heads * d, hidden), decay=weight(heads, hidden), out=weight(hidden, heads * d),  # noqa: E731
                         q_weight=torch.ones(d, device="cuda", requires_grad=True), k_weight=torch.ones(d, device="cuda", requires_grad=True),
                         router=weight(experts, hidden), w_gate_up=weight(experts, 2 * width, hidden), w_down=weight(experts, hidden, width))
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return dict(hidden=hidden, heads=heads, d=d, top_k=top_k, vocab=vocab, layers=[layer() for _ in range(layers)],
                embed=weight(vocab, hidden), head=weight(vocab, hidden), cos_sin=torch.cat((angle.cos(), angle.sin()), 1).float())


def parameters(m):
    return [m["embed"], m["head"]] + [p for w in m["layers"] for p in w.values()]


def norm(x):
    xf = x.float()
    return (xf * torch.rsqrt(xf.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def hidden_states(m, tokens):
    """The last layer's normalised rows [B T, hidden] for tokens [B, T]."""
    B, T = tokens.shape
    H, d = m["heads"], m["d"]
    x = m["embed"][tokens] * m["hidden"] ** 0.5
    for w in m["layers"]:
        y = norm(x)
        qkv = (y @ w["qkv"].t()).unflatten(-1, (3 * H, d))
        q, k = NormRotation.apply(qkv[:, :, :H], qkv[:, :, H:2 * H], w["q_weight"], w["k_weight"], m["cos_sin"], d ** -0.5, d ** -0.5)
        decay = torch.nn.functional.logsigmoid((y @ w["decay"].t()).float() + 4)
        o = Mixer.apply(q, k, qkv[:, :, 2 * H:].contiguous(), decay.contiguous())
        x = x + o.flatten(2) @ w["out"].t()
        rows = x.flatten(0, 1)
        y = norm(rows)
        x = Experts.apply(y, y @ w["router"].t(), w["w_gate_up"], w["w_down"], rows, m["top_k"]).view(B, T, -1)
    return norm(x.flatten(0, 1))


def loss_of(m, tokens, teacher=None):
    """Mean loss of the next token; the last token of each sequence has none.  teacher: (index, logits, temperature) of [B T, K]
    tokens and their logits, to be learnt from instead."""
    x = hidden_states(m, tokens)
    if teacher is not None:
        return Distill.apply(x, m["head"], *teacher).mean()
    target = torch.full_like(tokens, -100, dtype=torch.int32)
    target[:, :-1] = tokens[:, 1:]
    return CrossEntropy.apply(x, m["head"], target.flatten()).sum() / (tokens.shape[0] * (tokens.shape[1] - 1))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--teacher", type=int, default=0, help="learn from so many logits of a teacher a token")
    a = ap.parse_args()
    m = make_model()
    gen = torch.Generator("cuda").manual_seed(1)
    tokens = torch.randint(0, m["vocab"], (a.batch, a.tokens), device="cuda", generator=gen)
    teacher = None
    if a.teacher:
        n = a.batch * a.tokens
        teacher = (torch.randint(0, m["vocab"], (n, a.teacher), device="cuda", generator=gen, dtype=torch.int32),
                   3 * torch.randn(n, a.teacher, device="cuda", generator=gen), 2.0)
    optimizer = torch.optim.AdamW(parameters(m), lr=1e-4)
    for i in range(a.steps + 2):
        if i == 2:
            torch.cuda.synchronize()
            t = time.perf_counter()
        optimizer.zero_grad()
        loss = loss_of(m, tokens, teacher)
        loss.backward()
        optimizer.step()
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    print("%d x %d tokens: %.2f ms a step, %.2f M tokens/s, loss %.4f" % (a.batch, a.tokens, t * 1e3, tokens.numel() / t / 1e6, loss.item()))


if __name__ == "__main__":
    main()
