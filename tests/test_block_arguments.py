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


def qk_status(entry, q_out, k_out, q_at=0x100000, q_out_at=0x200000, sizes=(3, 5, 4, 64), **strides):
    """Status of a call on B, T, H heads of d elements with the results' strides given."""
    B, T, H, d = sizes
    plain = (H * T * d, T * d, d)
    s = dict(q=plain, k=plain, q_out=plain, k_out=plain, dq=plain, dk=plain)
    s.update({"fwd": dict(q_out=q_out, k_out=k_out), "bwd": dict(dq=q_out, dk=k_out)}[entry])
    s.update(strides)
    p = block._QkParams(ctypes.sizeof(block._QkParams), B, T, H, H, d, 1, 1, 0, 0, 0, 1e-6, 1.0, 1.0, 0,
                        *[(ctypes.c_int64 * 3)(*x) for x in s.values()])
    at = [ctypes.c_void_p(x) for x in (q_at, 0x300000, None, None, None, None)]
    if entry == "fwd":
        return pkg.library().lsm_qk_norm_rope(ctypes.byref(p), *at, ctypes.c_void_p(q_out_at), ctypes.c_void_p(0x400001), None)
    return pkg.library().lsm_qk_norm_rope_bwd(ctypes.byref(p), *at, *[ctypes.c_void_p(x) for x in (0x500000, 0x600000, q_out_at, 0x400000)],
                                              None, None, ctypes.c_void_p(0x700000), 1, None)


def meet(sizes, strides):
    """Whether two rows of d elements share one, by going through all of them."""
    B, T, H, d = sizes
    at = sorted(b * strides[0] + h * strides[1] + t * strides[2] for b in range(B) for h in range(H) for t in range(T))
    return any(y - x < d for x, y in zip(at, at[1:]))


def test_results_whose_rows_share_elements_are_refused():
    """Against every row's place: a forward call that passes this check ends at the misaligned k_out, a backward call at its workspace."""
    import itertools
    import random
    rng = random.Random(0)
    passed = {"fwd": -4, "bwd": -5}
    seen = {True: 0, False: 0}
    for n in range(3000):
        sizes = (rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 4), 64)
        if n % 3 == 0:   # an order of the axes, perhaps with gaps, perhaps a little too near each other
            strides, step = [0, 0, 0], 64
            for axis in rng.sample(range(3), 3):
                step += 8 * rng.choice([0, 0, 0, 1, 5, -1])
                strides[axis] = step
                step *= (sizes[0], sizes[2], sizes[1])[axis]
        else:
            strides = [8 * rng.choice([-1, 1, 1, 1]) * rng.randint(0, 40) for _ in range(3)]
        want = meet(sizes, strides)
        seen[want] += 1
        plain = (sizes[2] * sizes[1] * 64, sizes[1] * 64, 64)
        for entry, which in itertools.product(("fwd", "bwd"), (0, 1)):
            outs = [plain, plain]
            outs[which] = strides
            if which == 1 and entry == "fwd":
                continue  # k_out stands for the call's end here
            assert qk_status(entry, *outs, sizes=sizes) == (SHAPE if want else passed[entry]), (entry, which, sizes, strides)
    assert min(seen.values()) > 500
    # long axes: heads beside each other in a token, heads that begin before the last one's end, more rows than fit
    for entry in ("fwd", "bwd"):
        assert qk_status(entry, (0, 64, 192), (0, 64000, 64), sizes=(1, 1000, 3, 64)) == passed[entry]
        assert qk_status(entry, (0, 64 * 999, 64), (0, 64000, 64), sizes=(1, 1000, 3, 64)) == SHAPE
        assert qk_status(entry, (64 * 3, 64 * 1001, 64 * 7), (700 * 51200, 51200, 64), sizes=(900, 800, 700, 64)) == SHAPE


def test_results_in_place_have_the_inputs_strides():
    """q_out = q with heads and tokens exchanged would overwrite rows that other waves have yet to read.  (A call that passes ends
    at the misaligned k_out.)"""
    bhtd, bthd, sizes = (4096, 512, 64), (4096, 64, 512), (2, 8, 8, 64)
    kw = dict(q_at=0x100000, sizes=sizes)
    assert qk_status("fwd", bhtd, bhtd, q_out_at=0x100000, q=bhtd, **kw) == -4
    assert qk_status("fwd", bthd, bhtd, q_out_at=0x100000, q=bthd, **kw) == -4
    assert qk_status("fwd", bthd, bhtd, q_out_at=0x100000, q=bhtd, **kw) == SHAPE
    assert qk_status("fwd", bhtd, bhtd, q_out_at=0x100000, q=bthd, **kw) == SHAPE
    assert qk_status("fwd", bhtd, bhtd, q_out_at=0x100000, q=(0, 512, 64), **kw) == SHAPE     # a repeated input is no place for results
    assert qk_status("fwd", bthd, bhtd, q_out_at=0x200000, q=bhtd, **kw) == -4                # two tensors: any order
    # the stride of an axis of one is never used
    assert qk_status("fwd", (8, 512, 64), bhtd, q_out_at=0x100000, q=(4096, 512, 64), q_at=0x100000, sizes=(1, 8, 8, 64)) == -4


def test_a_transposition_in_place_is_refused_through_the_binding(monkeypatch):
    monkeypatch.setattr(block, "_stream_handle", lambda stream: None)
    q = torch.zeros(1, 8, 8, 64).as_subclass(OnDevice)
    with pytest.raises(pkg.LsmError) as e:
        block.lsm_qk_norm_rope(q, None, layout=block.LAYOUT_BHTD, out_layout=block.LAYOUT_BTHD, q_out=q)
    assert e.value.status == SHAPE
    k = q.clone()
    with pytest.raises(pkg.LsmError) as e:
        block.lsm_qk_norm_rope(q.clone(), k, layout=block.LAYOUT_BTHD, out_layout=block.LAYOUT_BHTD, q_out=q, k_out=k)
    assert e.value.status == SHAPE


def beam_status(B, K, V, **kw):
    """Status of a selection whose last check, the alignment of a result, fails."""
    c = dict(n_out=1, dtype=1, eos=-1)
    c.update(kw)
    p = block._BeamParams(ctypes.sizeof(block._BeamParams), B, K, V, c["n_out"], c["dtype"], c["eos"], 0, V)
    at = [ctypes.c_void_p(x) for x in (0x1000, 0x2000, None, 0x3000, 0x4000, 0x5001, None, 0x6000)]
    return pkg.library().lsm_beam_select(ctypes.byref(p), *at, 1 << 62, None), pkg.library().lsm_beam_select_workspace_bytes(ctypes.byref(p))


def test_launches_of_more_threads_than_an_axis_takes_are_refused():
    """Fewer than 2^32 threads along an axis of a launch: 2^24 - 1 workgroups of 256, 2^23 - 1 of 512."""
    row = lambda T, d: ((T * d, T * d, d),) * 2
    at = dict(q_at=0x100000)
    most = ((1 << 24) - 1) * 16                               # tokens of 128 bf16 features, 16 to a workgroup
    for T, want in ((1 << 27, -4), (most, -4), (most + 1, SHAPE), (1 << 29, SHAPE), (1 << 30, SHAPE)):
        assert qk_status("fwd", *row(T, 128), sizes=(1, T, 1, 128), **at) == want, T
    assert qk_status("bwd", *row(1 << 30, 128), sizes=(1, 1 << 30, 1, 128), **at) == -5        # its workgroups take what there is in turn
    for B, K, V, want in (((1 << 23) - 1, 1, 1, -4), (1 << 23, 1, 1, SHAPE), ((1 << 19) - 1, 32, 1, -4), (1 << 19, 32, 1, SHAPE),
                          (1 << 18, 32, 1 << 14, -4), ((1 << 19) - 1, 32, 1 << 18, SHAPE)):
        status, need = beam_status(B, K, V)
        assert status == want and (need > 0) == (want != SHAPE), (B, K, V)


SHIM = """
/* HIP's launch replaced: the n-th one fails, all of them are counted. */
static int calls, fail_at, last;
int __hipPushCallConfiguration(void) { return 0; }
int __hipPopCallConfiguration(void) { return 0; }
int hipLaunchKernel(void) { return ++calls == fail_at ? (last = 9) : 0; }
int hipGetLastError(void) { int e = last; last = 0; return e; }
void shim_reset(int at) { calls = last = 0; fail_at = at; }
int shim_calls(void) { return calls; }
"""
AFTER_A_FAILED_LAUNCH = """
import ctypes, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2503_05447_amd import block
lib, vp, P = block.library(), ctypes.c_void_p, lambda *a: [ctypes.c_void_p(0x1000 * (i + 1)) for i in a]
beam = block._BeamParams(ctypes.sizeof(block._BeamParams), 1, 2, 100, 2, 0, -1, 0, 100)
moe = lambda n: block._MoeParams(ctypes.sizeof(block._MoeParams), n, 64, 32, 8, 2, 1, 1)
s = (ctypes.c_int64 * 3)(1024, 512, 64)
qk = block._QkParams(ctypes.sizeof(block._QkParams), 1, 8, 2, 2, 64, 1, 1, 0, 0, 0, 1e-6, 1.0, 1.0, 0, s, s, s, s, s, s)
calls = dict(
    beam=(2, lambda: lib.lsm_beam_select(ctypes.byref(beam), *P(0, 1), None, *P(2, 3, 4), None, *P(5), 1 << 40, None)),
    moe_2=(4, lambda: lib.lsm_moe_step(ctypes.byref(moe(2)), *P(0, 1, 2, 3, 4, 5, 6), 1 << 40, None)),
    moe_9=(5, lambda: lib.lsm_moe_step(ctypes.byref(moe(9)), *P(0, 1, 2, 3, 4, 5, 6), 1 << 40, None)),
    qk_bwd=(2, lambda: lib.lsm_qk_norm_rope_bwd(ctypes.byref(qk), *P(0, 1, 2, 3), None, None, *P(4, 5, 6, 7, 8, 9, 10), 1 << 40, None)))
for name, (launches, call) in calls.items():
    for at in range(launches + 1):
        shim.shim_reset(at)
        status = call()
        want = (0, launches) if at == 0 else (-6, at)
        assert (status, shim.shim_calls()) == want, (name, at, status, shim.shim_calls())
print("done")
"""


def test_nothing_is_launched_after_a_launch_that_failed(tmp_path):
    """What a kernel left out would have written is where the next ones find their addresses."""
    import os
    import shutil
    import subprocess
    import sys
    if shutil.which("gcc") is None:
        pytest.skip("no host compiler for the launch counter")
    (tmp_path / "shim.c").write_text(SHIM)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", tmp_path / "shim.so", tmp_path / "shim.c"], check=True)
    pkg.library()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-W", "ignore", "-c", AFTER_A_FAILED_LAUNCH, str(tmp_path / "shim.so"), root], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "done", r.stderr[-2000:]


def test_the_backward_workspace_of_invalid_strides_is_0():
    s = (4096, 512, 64)
    for bad in ("q", "k", "q_out", "k_out", "dq", "dk"):
        strides = {n: (4096, 512, 68) if n == bad else s for n in ("q", "k", "q_out", "k_out", "dq", "dk")}
        p = block._QkParams(ctypes.sizeof(block._QkParams), 2, 8, 8, 8, 64, 1, 1, 0, 0, 0, 1e-6, 1.0, 1.0, 0,
                            *[(ctypes.c_int64 * 3)(*x) for x in strides.values()])
        assert pkg.library().lsm_qk_norm_rope_bwd_workspace_bytes(ctypes.byref(p)) == 0, bad


def test_a_workspace_that_is_not_all_there_on_the_device_is_refused(seen):
    """Host memory, or one byte repeated: the kernels would write outside it."""
    q = tensor(1, 2, 8, 64)
    calls = (lambda ws: block.lsm_qk_norm_rope_bwd(q, q, q, q, workspace=ws),
             lambda ws: block.lsm_moe_step(tensor(3, 16), tensor(8, 16), tensor(8, 16, 16), tensor(8, 16, 8), 2, workspace=ws),
             lambda ws: block.lsm_beam_select(tensor(1, 3, 50), tensor(1, 3), workspace=ws))
    for call in calls:
        for bad in (torch.zeros(1 << 20, dtype=torch.uint8), tensor(1, dtype=torch.uint8).expand(1 << 20), tensor(1 << 20, 2, dtype=torch.uint8)[:, 0]):
            with pytest.raises(ValueError):
                call(bad)
        assert not seen
    for call in calls:
        call(tensor(1 << 20, dtype=torch.uint8))
    assert len(seen) == len(calls)


def reorder_status(at, size, parent=0x300000, B=2, K=4):
    """Status of a call whose last state is misaligned: one that passes what comes before it."""
    a, s = (ctypes.c_void_p * len(at))(*at), (ctypes.c_size_t * len(size))(*size)
    return pkg.library().lsm_state_reorder(a, s, len(at), ctypes.c_void_p(parent), B, K, None)


def test_states_that_share_memory_are_refused(monkeypatch):
    """Each is moved by its own workgroups: two that meet, or one that meets the parents, would be read while they change."""
    rows = 8
    assert reorder_status((0x10000, 0x10000), (64, 64)) == SHAPE
    assert reorder_status((0x20000, 0x10000, 0x10000 + rows * 64 - 16), (64, 64, 16)) == SHAPE
    assert reorder_status((0x10000, 0x10000 + rows * 64 - 32, 0x20000), (64, 64, 4)) == SHAPE
    assert reorder_status((0x300000 - rows * 64 + 16, 0x10000), (64, 64)) == SHAPE
    assert reorder_status((0x300000 + 16,), (4,)) == SHAPE
    # neighbours are not refused for it (but for a last row of 6 bytes)
    assert reorder_status((0x10000, 0x10000 + rows * 64, 0x300000 + rows * 4, 0x300000 - rows * 16, 0x50008), (64, 64, 16, 16, 8)) == -4
    # more than one launch takes
    monkeypatch.setattr(block, "_stream_handle", lambda stream: None)
    moved = []
    monkeypatch.setattr(block, "library", lambda: type("L", (), {"lsm_state_reorder": staticmethod(lambda *a: moved.append(a) or 0),
                                                                "lsm_status_string": staticmethod(pkg.library().lsm_status_string)}))
    states = [tensor(8, 4) for _ in range(70)]
    parent = tensor(2, 4, dtype=torch.int32)
    for extra in (states[3], states[3].view(-1)[:16].view(8, 2)):
        with pytest.raises(pkg.LsmError) as e:
            block.lsm_state_reorder(states + [extra], parent)
        assert e.value.status == SHAPE and not moved
    block.lsm_state_reorder(states, parent)
    assert len(moved) == 2
