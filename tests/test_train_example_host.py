"""The wrappers of examples/train_step.py for automatic differentiation, with plain stand-ins for the operators: no GPU is needed."""
import importlib.util
import os
import types

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def example(monkeypatch):
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    loss = lambda x, *rest: (x.square().sum(1), x.detach().sum(1))
    loss_bwd = lambda x, w, *rest: dict(dx=2 * x * rest[-1 if torch.is_tensor(rest[-1]) else -2][:, None], dw=torch.zeros_like(w))
    stand_ins = dict(
        LAYOUT_BTHD=0, DECAY_SCALAR=0, lsm_qk_norm_rope=lambda q, k, **kw: (q * q, k * k),
        lsm_qk_norm_rope_bwd=lambda q, k, dq, dk, q_weight, k_weight, **kw: dict(dq=2 * q * dq, dk=2 * k * dk, d_q_weight=q_weight * 0, d_k_weight=k_weight * 0),
        lsm_chunk_fwd=lambda q, k, v, g, *kind, **kw: (q * k * v,),
        lsm_chunk_bwd=lambda q, k, v, g, kind, d, **kw: dict(dq=d * k * v, dk=d * q * v, dv=d * q * k, dg=g * 0),
        lsm_moe_route=lambda logits, k: (logits[:, :k].detach(), torch.zeros(logits.shape[0], k, dtype=torch.int32)),
        lsm_moe_plan=lambda chosen, E: (), lsm_moe_experts=lambda x, w, plan, a, b, residual: residual + x * x,
        lsm_moe_experts_bwd=lambda x, w, plan, a, b, d: dict(dx=2 * x * d, d_weights=w, d_w_gate_up=a * 0, d_w_down=b * 0),
        lsm_moe_route_bwd=lambda logits, chosen, d: logits * 0,
        lsm_linear_cross_entropy=loss, lsm_linear_cross_entropy_bwd=loss_bwd, lsm_linear_distill=loss, lsm_linear_distill_bwd=loss_bwd)
    monkeypatch.setattr(m, "lsm", types.SimpleNamespace(**stand_ins))
    return m


def calls(m):
    gen = torch.Generator().manual_seed(1)
    t = lambda *s: torch.randn(*s, generator=gen).requires_grad_()
    whole = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return dict(NormRotation=lambda: m.NormRotation.apply(t(1, 3, 2, 4), t(1, 3, 2, 4), t(4), t(4), None, 1.0, 1.0)[0],
                Mixer=lambda: m.Mixer.apply(t(1, 3, 2, 4), t(1, 3, 2, 4), t(1, 3, 2, 4), t(1, 3, 2)),
                Experts=lambda: m.Experts.apply(t(5, 4), t(5, 3), t(3, 4, 4), t(3, 4, 2), t(5, 4), 2),
                CrossEntropy=lambda: m.CrossEntropy.apply(t(5, 4), t(7, 4), whole(5)),
                Distill=lambda: m.Distill.apply(t(5, 4), t(7, 4), whole(5, 2), torch.zeros(5, 2), 2.0))


@pytest.mark.parametrize("name", ["NormRotation", "Mixer", "Experts", "CrossEntropy", "Distill"])
def test_a_second_derivative_is_refused(example, name):
    """Where a loss is the result's sum the incoming gradient requires none, and torch's own products behind it would still be differentiated
    with the operator's gradient as a constant."""
    for loss in (torch.sum, lambda out: out.square().sum()):
        out = calls(example)[name]()
        leaf = out.grad_fn.next_functions[0][0].variable
        with pytest.raises(RuntimeError, match="cannot be differentiated again"):
            torch.autograd.grad(loss(out), leaf, create_graph=True)
        out = calls(example)[name]()
        leaf = out.grad_fn.next_functions[0][0].variable
        grad, = torch.autograd.grad(loss(out), leaf)
        assert grad.shape == leaf.shape and grad.abs().max() > 0


def test_every_wrapper_is_tried(example):
    there = {n for n, v in vars(example).items() if isinstance(v, type) and issubclass(v, torch.autograd.Function)}
    assert there == set(calls(example))
