"""Beam search with a small Linear-MoE model of random weights: how the operators of this library follow each other.

Prefill of a prompt: projection -> lsm_qk_norm_rope -> lsm_chunk_fwd -> lsm_moe_step (blocks of 128 tokens).
A decoded token: projection -> lsm_qk_norm_rope -> lsm_step -> lsm_moe_step, then lsm_beam_select over the vocabulary and
lsm_state_reorder of every layer's recurrent states.  Projections, norms of the residual stream and the output head are torch.

    python examples/beam_decode.py [--batch 4] [--beams 4] [--steps 32]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_05447_amd as lsm  # noqa: E402


def make_model(hidden=1024, heads=8, d=128, layers=4, experts=64, top_k=8, width=1024, vocab=32000, positions=4096,
               dtype=torch.bfloat16, seed=0):
    """Weights of a Linear-MoE model whose mixer has a scalar decay a token (the Mamba2 row), and the rotation's table."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def weight(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).to(dtype)
    layer = lambda: dict(qkv=weight(3 * heads * d, hidden), decay=weight(heads, hidden), out=weight(hidden, heads * d),  # noqa: E731
                         q_weight=torch.ones(d, device="cuda"), k_weight=torch.ones(d, device="cuda"),
                         router=weight(experts, hidden), w_gate_up=weight(experts, 2 * width, hidden),
                         w_down=weight(experts, hidden, width))
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return dict(hidden=hidden, heads=heads, d=d, top_k=top_k, vocab=vocab, dtype=dtype, layers=[layer() for _ in range(layers)],
                embed=weight(vocab, hidden) * hidden ** 0.5, head=weight(vocab, hidden),
                cos_sin=torch.cat((angle.cos(), angle.sin()), 1).float())


def norm(x):
    xf = x.float()
    return (xf * torch.rsqrt(xf.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def mixer_inputs(m, w, x, positions, layout):
    """q, k, v and the log-decay of [.., hidden] rows x; q and k straight from the fused projection's output."""
    H, d = m["heads"], m["d"]
    y = norm(x)
    qkv = (y @ w["qkv"].t()).unflatten(-1, (3 * H, d))
    # one token: [B, 3H, d] is [B, heads, d]; a prompt: [B, T, 3H, d]
    q, k = lsm.lsm_qk_norm_rope(qkv[..., :H, :], qkv[..., H:2 * H, :], m["cos_sin"], positions, w["q_weight"], w["k_weight"],
                                norm=lsm.NORM_RMS, q_scale=d ** -0.5, k_scale=d ** -0.5, layout=layout)
    decay = torch.nn.functional.logsigmoid((y @ w["decay"].t()).float() + 4)
    return q, k, qkv[..., 2 * H:, :].contiguous(), decay.contiguous()


def experts(m, w, x):
    """x + the experts' output for rows x [n, hidden], 128 at a time."""
    parts = [lsm.lsm_moe_step(norm(p), w["router"], w["w_gate_up"], w["w_down"], m["top_k"], residual=p) for p in x.split(128)]
    return parts[0] if len(parts) == 1 else torch.cat(parts)


def prefill(m, tokens):
    """Logits after the prompts [B, T] and the layers' states [B, H, d, d]."""
    B, T = tokens.shape
    x, states = m["embed"][tokens], []
    for w in m["layers"]:
        q, k, v, g = mixer_inputs(m, w, x, None, lsm.LAYOUT_BTHD)
        o, state = lsm.lsm_chunk_fwd(q, k, v, g, lsm.DECAY_SCALAR, layout=lsm.LAYOUT_BTHD)
        x = x + o.flatten(2) @ w["out"].t()
        x = experts(m, w, x.flatten(0, 1)).view(B, T, -1)
        states.append(state)
    return norm(x[:, -1]) @ m["head"].t(), states


def step(m, tokens, position, states):
    """Logits after one more token of each row; the states are updated in place."""
    x = m["embed"][tokens]
    positions = torch.full_like(tokens, position, dtype=torch.int32)
    for w, state in zip(m["layers"], states):
        q, k, v, g = mixer_inputs(m, w, x, positions, lsm.LAYOUT_BHTD)
        o = lsm.lsm_step(q, k, v, g, lsm.DECAY_SCALAR, state)
        x = experts(m, w, x + o.flatten(1) @ w["out"].t())
    return norm(x) @ m["head"].t()


def beam_search(m, prompts, beams, steps, eos):
    """Tokens [B, beams, steps] and log-probabilities [B, beams] of the best continuations, best first."""
    B, T = prompts.shape
    logits, states = prefill(m, prompts)
    states = [s.repeat_interleave(beams, 0) for s in states]      # every beam starts from its prompt's states
    logits = logits[:, None].expand(B, beams, -1).contiguous()
    scores = torch.full((B, beams), -float("inf"), device="cuda")  # at first one beam of each prompt counts
    scores[:, 0] = 0
    ended = torch.zeros(B, beams, dtype=torch.bool, device="cuda")
    history = torch.zeros(B, beams, steps, dtype=torch.int32, device="cuda")
    for i in range(steps):
        scores, parent, token, ended = lsm.lsm_beam_select(logits, scores, finished=ended, eos=eos)
        lsm.lsm_state_reorder(states + [history], parent)
        history[:, :, i] = token
        if i + 1 < steps:
            logits = step(m, token.view(-1).long(), T + i, states).view(B, beams, -1)
    return history, scores


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    m = make_model()
    prompts = torch.randint(0, m["vocab"], (a.batch, 200), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    beam_search(m, prompts, a.beams, 4, eos=2)
    torch.cuda.synchronize()
    t = time.perf_counter()
    history, scores = beam_search(m, prompts, a.beams, a.steps, eos=2)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print("best continuation of prompt 0 (log-probability %.3f): %s ..." % (scores[0, 0].item(), history[0, 0, :8].tolist()))
    print("%d prompts of %d tokens, %d beams, %d tokens: %.1f ms, %.2f ms a token" % (a.batch, prompts.shape[1], a.beams, a.steps,
                                                                                   t * 1e3, t * 1e3 / a.steps))


if __name__ == "__main__":
    main()
