"""Host-side checks of include/lsm_train.h and its binding that need no GPU: bad arguments are refused before any HIP call."""
import ctypes

import pytest
import torch

import paper_2503_05447_amd as pkg
from paper_2503_05447_amd import train

NULL, SHAPE, UNSUP, ALIGN, WS = -1, -2, -3, -4, -5
vp = ctypes.c_void_p


def route(size=None, **kw):
    c = dict(n=8, E=16, top_k=4, dtype=0, renormalise=1)
    c.update(kw)
    return train._RouteParams(ctypes.sizeof(train._RouteParams) if size is None else size, *c.values())


def experts(size=None, x_stride=None, dy_stride=None, **kw):
    c = dict(n=8, D=64, F=40, E=16, top_k=4, dtype=1, reserved=0)
    c.update(kw)
    return train._ExpertsParams(ctypes.sizeof(train._ExpertsParams) if size is None else size, *c.values(),
                                c["D"] if x_stride is None else x_stride, c["D"] if dy_stride is None else dy_stride)


def vocab(size=None, x_stride=None, **kw):
    c = dict(n=8, D=64, V=1000, K=0, dtype=1, temperature=1.0, reserved=0)
    c.update(kw)
    return train._VocabParams(ctypes.sizeof(train._VocabParams) if size is None else size, *c.values(), c["D"] if x_stride is None else x_stride)


def call(name, p, n, bytes_=1 << 50, **at):
    """lsm_<name> with n pointers 0x1000, 0x2000, .. and those of `at` (by place) instead."""
    ptr = [0x1000 * (i + 1) for i in range(n)]
    for k, v in at.items():
        ptr[int(k[1:])] = v
    f = getattr(pkg.library(), name)
    rest = [vp(a) for a in ptr] + ([ctypes.c_size_t(bytes_)] if len(f.argtypes) == n + 3 else []) + [vp(None)]
    return f(ctypes.byref(p) if p is not None else None, *rest)


CALLS = {"lsm_moe_route": (route, 3), "lsm_moe_route_bwd": (route, 4), "lsm_moe_plan": (route, 5), "lsm_moe_experts": (experts, 10),
         "lsm_moe_experts_bwd": (experts, 13), "lsm_vocab_loss": (vocab, 7), "lsm_vocab_loss_bwd": (vocab, 9)}
OPTIONAL = {"lsm_moe_experts": {7}, "lsm_moe_experts_bwd": set(), "lsm_vocab_loss": {3}, "lsm_vocab_loss_bwd": {3, 7}}


@pytest.mark.parametrize("name", CALLS)
def test_null_and_misaligned(name):
    make, n = CALLS[name]
    p = make(K=4) if make is vocab else make(n=5000) if name == "lsm_moe_plan" else make()
    assert call(name, None, n) == NULL
    has_ws = hasattr(pkg.library(), name + "_workspace_bytes")
    last = n - 1 if has_ws else n
    for i in range(last):
        got = call(name, p, n, **{"a%d" % i: None})
        if i not in OPTIONAL.get(name, set()) or (make is vocab and i == 3):
            assert got == NULL, i
        assert call(name, p, n, **{"a%d" % i: 0x1008}) == ALIGN, i
    if has_ws:
        assert call(name, p, n, **{"a%d" % last: None}) == WS
        assert call(name, p, n, **{"a%d" % last: 0x1004}) == ALIGN
        need = getattr(pkg.library(), name + "_workspace_bytes")(ctypes.byref(p))
        assert need > 0 and call(name, p, n, bytes_=need - 1) == WS
    assert call(name, make(size=8), n) == SHAPE


def test_route_refuses_bad_sizes():
    for name, n in (("lsm_moe_route", 3), ("lsm_moe_route_bwd", 4), ("lsm_moe_plan", 5)):
        for bad in (dict(n=0), dict(E=0), dict(top_k=0), dict(top_k=17, E=16), dict(n=(1 << 24) + 1, top_k=1), dict(n=1 << 23, top_k=3)):
            assert call(name, route(**bad), n) == SHAPE, (name, bad)
        for bad in (dict(E=257), dict(E=64, top_k=17)):
            assert call(name, route(**bad), n) == UNSUP, (name, bad)
        if name != "lsm_moe_plan":
            assert call(name, route(dtype=2), n) == UNSUP and call(name, route(renormalise=2), n) == UNSUP
    size = pkg.library().lsm_moe_plan_workspace_bytes
    assert size(ctypes.byref(route(n=2048, top_k=4))) == 0  # few pairs: none is needed
    assert size(ctypes.byref(route(n=0))) == 0 and size(ctypes.byref(route(n=1 << 20))) > 0


def test_experts_refuse_bad_sizes():
    for name, n in (("lsm_moe_experts", 10), ("lsm_moe_experts_bwd", 13)):
        for bad in (dict(n=0), dict(D=0), dict(F=0), dict(E=0), dict(top_k=0), dict(E=3), dict(n=1 << 23), dict(x_stride=56),
                    dict(x_stride=1 << 40), dict(n=1 << 20, top_k=1, D=2048), dict(D=65536, F=65536), dict(D=65536, F=8192, dtype=0)):
            assert call(name, experts(**bad), n) == SHAPE, (name, bad)
        for bad in (dict(dtype=2), dict(E=257), dict(top_k=17, E=64), dict(D=60), dict(F=36), dict(D=65544), dict(reserved=1)):
            assert call(name, experts(**bad), n) == UNSUP, (name, bad)
        assert call(name, experts(x_stride=68), n) == ALIGN
    assert call("lsm_moe_experts_bwd", experts(dy_stride=56), 13) == SHAPE
    assert call("lsm_moe_experts_bwd", experts(dy_stride=68), 13) == ALIGN
    p = experts()
    for i in (10, 11):  # both weights' gradients or neither
        assert call("lsm_moe_experts_bwd", p, 13, **{"a%d" % i: None}) == NULL
    for size in (pkg.library().lsm_moe_experts_workspace_bytes, pkg.library().lsm_moe_experts_bwd_workspace_bytes):
        assert size(ctypes.byref(experts(D=60))) == 0 and size(ctypes.byref(p)) > 0


def test_losses_refuse_bad_sizes():
    for name, n in (("lsm_vocab_loss", 7), ("lsm_vocab_loss_bwd", 9)):
        for bad in (dict(n=0), dict(D=0), dict(V=0), dict(K=-1), dict(n=(1 << 24) + 1), dict(V=(1 << 24) + 1), dict(temperature=0.0),
                    dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-39),
                    dict(x_stride=56), dict(n=1 << 24, K=17), dict(n=1 << 20, D=2048)):
            assert call(name, vocab(**bad), n) == SHAPE, (name, bad)
        for bad in (dict(dtype=2), dict(K=257), dict(D=60), dict(D=65544), dict(reserved=1)):
            assert call(name, vocab(**bad), n) == UNSUP, (name, bad)
        assert call(name, vocab(x_stride=68), n) == ALIGN
        assert call(name, vocab(K=0), n) == NULL               # a teacher without entries
        assert call(name, vocab(K=4), n, a3=None) == NULL      # entries without a teacher
    for size in (pkg.library().lsm_vocab_loss_workspace_bytes, pkg.library().lsm_vocab_loss_bwd_workspace_bytes):
        assert size(ctypes.byref(vocab(D=60))) == 0 and size(ctypes.byref(vocab(n=100000, V=131071))) > 0


def test_temperatures_whose_scale_is_not_finite_are_refused():
    """The kernels raise 2 to a power: 1 / (temperature log 2) is a number of fp32 from 2^-127.4 on."""
    for name, n in (("lsm_vocab_loss", 7), ("lsm_vocab_loss_bwd", 9)):
        for bad in (3.5e-39, 4.0e-39, 2.0 ** -128):
            assert call(name, vocab(temperature=bad), n, a3=None) == SHAPE, (name, bad)
    for size in (pkg.library().lsm_vocab_loss_workspace_bytes, pkg.library().lsm_vocab_loss_bwd_workspace_bytes):
        assert size(ctypes.byref(vocab(temperature=3.5e-39))) == 0
        for good in (2.0 ** -127, 2.0 ** -100, 1.0, 2.0 ** 126):
            assert size(ctypes.byref(vocab(temperature=good))) > 0


def test_products_that_no_launch_holds_are_refused():
    """2^32 threads are the most of a launch, 512 the most of a tile: 2^23 tiles or more are refused before anything runs."""
    many = experts(n=1 << 24, top_k=1, D=8, F=65536)             # 65536 x 512 tiles of the hidden layer
    assert call("lsm_moe_experts", many, 10) == SHAPE and call("lsm_moe_experts_bwd", many, 13) == SHAPE
    wide = experts(n=256, top_k=1, E=256, D=32768, F=32760, dtype=1)     # the weights' gradients alone
    assert call("lsm_moe_experts_bwd", wide, 13) == SHAPE
    assert call("lsm_vocab_loss", vocab(n=1 << 24, D=8, V=1 << 24, K=0, dtype=1), 7, a3=None) == SHAPE
    assert call("lsm_vocab_loss_bwd", vocab(n=1, D=65536, V=1 << 24, K=0, dtype=1), 9, a3=None) == SHAPE
    lib = pkg.library()
    for size, p in ((lib.lsm_moe_experts_workspace_bytes, many), (lib.lsm_moe_experts_bwd_workspace_bytes, wide)):
        assert size(ctypes.byref(p)) == 0
    large = experts(n=1 << 19, top_k=8, E=64, D=2048, F=1024, dtype=1)
    assert lib.lsm_moe_experts_workspace_bytes(ctypes.byref(large)) > 0 and lib.lsm_moe_experts_bwd_workspace_bytes(ctypes.byref(large)) > 0


def test_the_logits_are_never_kept():
    """What a backward call asks for is a piece of the vocabulary, whatever the vocabulary's size."""
    size = pkg.library().lsm_vocab_loss_bwd_workspace_bytes
    big = size(ctypes.byref(vocab(n=65536, D=1024, V=1 << 20)))
    assert big < 65536 * (1 << 20) * 2 / 16


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
        if name in CALLS:
            def take(p, *rest):
                got = type(p._obj)()
                ctypes.memmove(ctypes.byref(got), p, ctypes.sizeof(got))
                self.seen.append(got)
                return 0
            return take
        return getattr(pkg.library(), name)


@pytest.fixture
def seen(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(train, "library", lambda: r)
    monkeypatch.setattr(train, "_stream_handle", lambda stream: None)
    monkeypatch.setattr(train, "_current_device", lambda: -1)
    return r.seen


def plan(n, k, E):
    i = torch.int32
    return tensor(E + 1, dtype=i), tensor(n * k, dtype=i), tensor(n, k, dtype=i)


def test_binding_passes_sizes_and_strides(seen):
    wide = tensor(6, 80)
    pkg.lsm_moe_route(tensor(6, 9), 3, renormalise=False)
    assert (seen[-1].n, seen[-1].E, seen[-1].top_k, seen[-1].dtype, seen[-1].renormalise) == (6, 9, 3, 0, 0)
    pkg.lsm_moe_plan(tensor(6, 3, dtype=torch.int32), 9)
    assert (seen[-1].n, seen[-1].E, seen[-1].top_k) == (6, 9, 3)
    args = wide[:, :64], tensor(6, 3), plan(6, 3, 9), tensor(9, 80, 64), tensor(9, 64, 40)
    assert pkg.lsm_moe_experts(*args).shape == (6, 64)
    assert (seen[-1].n, seen[-1].D, seen[-1].F, seen[-1].E, seen[-1].top_k, seen[-1].x_stride) == (6, 64, 40, 9, 3, 80)
    got = pkg.lsm_moe_experts_bwd(*args, tensor(6, 96)[:, 16:80], weight_grads=False)
    assert (seen[-1].x_stride, seen[-1].dy_stride) == (80, 96) and got["d_w_down"] is None
    for temperature in (1.0, torch.tensor(2.0)):  # a number enters by its value
        pkg.lsm_linear_cross_entropy(wide[:, :64], tensor(50, 64), tensor(6, dtype=torch.int32), temperature=temperature)
        assert (seen[-1].n, seen[-1].D, seen[-1].V, seen[-1].K, seen[-1].x_stride) == (6, 64, 50, 0, 80)
        assert seen[-1].temperature == float(temperature)
    got = pkg.lsm_linear_distill_bwd(wide[:, :64], tensor(50, 64), tensor(6, 5, dtype=torch.int32), tensor(6, 5), tensor(6), tensor(6),
                                     weight_grad=False)
    assert seen[-1].K == 5 and got["dw"] is None and got["dx"].shape == (6, 64)


def test_binding_refuses(seen):
    i = torch.int32
    x, w, wgu, wd, p = tensor(6, 64), tensor(6, 3), tensor(9, 80, 64), tensor(9, 64, 40), plan(6, 3, 9)
    for bad in (lambda: pkg.lsm_moe_route(tensor(6, 9, dtype=torch.float16), 3), lambda: pkg.lsm_moe_route(tensor(9), 3),
                lambda: pkg.lsm_moe_route(tensor(6, 18)[:, ::2], 3), lambda: pkg.lsm_moe_route(torch.zeros(6, 9), 3),
                lambda: pkg.lsm_moe_route_bwd(tensor(6, 9), tensor(6, 3, dtype=i), tensor(6, 2)),
                lambda: pkg.lsm_moe_route_bwd(tensor(6, 9), tensor(6, 3), tensor(6, 3)),
                lambda: pkg.lsm_moe_plan(tensor(18, dtype=i), 9), lambda: pkg.lsm_moe_plan(tensor(6, 3, dtype=torch.int64), 9),
                lambda: pkg.lsm_moe_experts(x, w, plan(6, 3, 8), wgu, wd), lambda: pkg.lsm_moe_experts(x, w, plan(5, 3, 9), wgu, wd),
                lambda: pkg.lsm_moe_experts(x.t().contiguous().t(), w, p, wgu, wd), lambda: pkg.lsm_moe_experts(x, w, p, wgu, wd.to(torch.bfloat16)),
                lambda: pkg.lsm_moe_experts(x, w, p, wgu[:, :79], wd), lambda: pkg.lsm_moe_experts(x, w, p, wgu, wd, residual=tensor(5, 64)),
                lambda: pkg.lsm_moe_experts(x, w, p, wgu, wd, y=tensor(6, 128)[:, ::2]),
                lambda: pkg.lsm_moe_experts(x, w, p, wgu, wd, workspace=tensor(64, dtype=torch.uint8)[::2]),
                lambda: pkg.lsm_moe_experts_bwd(x, w, p, wgu, wd, None), lambda: pkg.lsm_moe_experts_bwd(x, w, p, wgu, wd, tensor(6, 72)),
                lambda: pkg.lsm_linear_cross_entropy(x, tensor(50, 72), tensor(6, dtype=i)),
                lambda: pkg.lsm_linear_cross_entropy(x, tensor(50, 64), tensor(6, dtype=torch.int64)),
                lambda: pkg.lsm_linear_cross_entropy_bwd(x, tensor(50, 64), tensor(6, dtype=i), tensor(5), tensor(6)),
                lambda: pkg.lsm_linear_distill(x, tensor(50, 64), tensor(6, 0, dtype=i), tensor(6, 0)),
                lambda: pkg.lsm_linear_distill(x, tensor(50, 64), tensor(6, 4, dtype=i), None),
                lambda: pkg.lsm_linear_distill(x, tensor(50, 64), tensor(6, 4, dtype=i), tensor(6, 5)),
                lambda: pkg.lsm_linear_distill_bwd(x, tensor(50, 64), tensor(6, dtype=i), tensor(6, 4), tensor(6), tensor(6))):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    assert not seen


def test_numbers_beyond_32_bits_are_refused(seen):
    """They would be taken for their lowest 32 bits."""
    with pytest.raises(ValueError):
        pkg.lsm_moe_route(tensor(6, 9), (1 << 32) + 3)
    with pytest.raises(ValueError):
        pkg.lsm_moe_plan(tensor(6, 3, dtype=torch.int32), (1 << 32) + 9)
    with pytest.raises(ValueError):
        train._vocab_params(6, 64, (1 << 32) + 50, 0, 0, 1.0, 0, 64)
    with pytest.raises(ValueError):
        train._experts_params((1 << 32) + 6, 64, 40, 9, 3, 0, 0, 64, 64)
    assert not seen


def test_another_device_is_refused(seen, monkeypatch):
    class Elsewhere(OnDevice):
        def get_device(self):
            return 1
    monkeypatch.setattr(train, "_current_device", lambda: 0)
    there = torch.zeros(6, 9).as_subclass(Elsewhere)
    with pytest.raises(ValueError, match="current device"):
        pkg.lsm_moe_route(there, 3)
    with pytest.raises(ValueError, match="need a contiguous tensor"):
        pkg.lsm_linear_cross_entropy(tensor(6, 64), torch.zeros(50, 64).as_subclass(Elsewhere), tensor(6, dtype=torch.int32))
    assert not seen
