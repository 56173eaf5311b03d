"""How the operators of include/lsm_block.h take their arguments, without a GPU: numbers enter a call by their value, never by the
object that holds them, and what must not overlap is refused before any HIP call."""
import ctypes

import pytest
import torch

import paper_2503_05447_amd as pkg
from paper_2503_05447_amd import block

SHAPE = -2


class OnDevice(torch.Tensor):
    """A CPU tensor that says it is on the device: marshalling alone is looked at, nothing is launched."""
    is_cuda = property(lambda self: True)


def tensor(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


class Recorder:
    """The library with its launching calls replaced: each leaves the parameter block that it was given."""
    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        if name in ("lsm_qk_norm_rope", "lsm_qk_norm_rope_bwd", "lsm_moe_step", "lsm_beam_select"):
            def call(p, *rest):
                got = type(p._obj)()
                ctypes.memmove(ctypes.byref(got), p, ctypes.sizeof(got))
                self.seen.append(got)
                return 0
            return call
        return getattr(pkg.library(), name)


@pytest.fixture
def seen(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(block, "library", lambda: lib)
    monkeypatch.setattr(block, "_stream_handle", lambda stream: None)
    return lib.seen


def qk_calls():
    q = tensor(1, 2, 8, 64)
    return (lambda **kw: block.lsm_qk_norm_rope(q, q, **kw), lambda **kw: block.lsm_qk_norm_rope_bwd(q, q, q, q, **kw))


@pytest.mark.parametrize("name", ["eps", "q_scale", "k_scale"])
def test_a_factor_that_changes_between_calls_is_read_again(seen, name):
    """A learnable temperature is a tensor that keeps its identity while an optimiser changes its value."""
    for call in qk_calls():
        for made in (torch.tensor, lambda x: torch.nn.Parameter(torch.tensor(x))):
            factor = made(0.5)
            call(**{name: factor})
            assert getattr(seen[-1], name) == 0.5
            with torch.no_grad():
                factor.mul_(2)
            call(**{name: factor})
            assert getattr(seen[-1], name) == 1.0
        call(**{name: 0.25})
        assert getattr(seen[-1], name) == 0.25


@pytest.mark.parametrize("name", ["norm", "rotation"])
def test_a_choice_that_changes_between_calls_is_read_again(seen, name):
    for call in qk_calls():
        choice = torch.tensor(1)
        call(**{name: choice})
        assert getattr(seen[-1], name) == 1
        choice.zero_()
        call(**{name: choice})
        assert getattr(seen[-1], name) == 0
        with pytest.raises(TypeError):
            call(**{name: 1.0})


def test_an_order_that_changes_between_calls_is_read_again(seen):
    for call in qk_calls():
        order = torch.tensor(block.LAYOUT_BHTD)
        call(layout=order)
        assert (seen[-1].H_q, seen[-1].T) == (2, 8)
        order.fill_(block.LAYOUT_BTHD)
        call(layout=order)
        assert (seen[-1].H_q, seen[-1].T) == (8, 2)


def test_numbers_of_experts_and_beams_that_change_between_calls_are_read_again(seen):
    x, router, gate_up, down = tensor(3, 16), tensor(8, 16), tensor(8, 16, 16), tensor(8, 16, 8)
    k = torch.tensor(2)
    block.lsm_moe_step(x, router, gate_up, down, k)
    assert seen[-1].top_k == 2
    k.fill_(4)
    block.lsm_moe_step(x, router, gate_up, down, k)
    assert seen[-1].top_k == 4
    n, eos = torch.tensor(2), torch.tensor(5)
    block.lsm_beam_select(tensor(1, 3, 50), tensor(1, 3), n, eos=eos)
    assert (seen[-1].n_out, seen[-1].eos) == (2, 5)
    n.fill_(3)
    eos.fill_(7)
    block.lsm_beam_select(tensor(1, 3, 50), tensor(1, 3), n, eos=eos)
    assert (seen[-1].n_out, seen[-1].eos) == (3, 7)
    for bad in (lambda: block.lsm_moe_step(x, router, gate_up, down, 2.0), lambda: block.lsm_beam_select(tensor(1, 3, 50), tensor(1, 3), 2.0),
                lambda: block.lsm_beam_select(tensor(1, 3, 50), tensor(1, 3), 2, eos=5.0)):
        with pytest.raises(TypeError):
            bad()
