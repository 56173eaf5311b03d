"""Host-side checks of include/lsm_block.h that need no GPU: bad arguments are refused before any HIP call."""
import ctypes

import paper_2503_05447_amd as pkg
from paper_2503_05447_amd import block

NULL, SHAPE, UNSUP, ALIGN, WS = -1, -2, -3, -4, -5
vp = ctypes.c_void_p


def qk_params(strides=None, size=None, reserved=0, **kw):
    c = dict(B=2, T=8, H_q=4, H_k=2, d=128, dtype=1, norm=1, rotation=0, rot_dim=128, n_pos=8, eps=1e-6, q_scale=1.0, k_scale=1.0)
    c.update(kw)
    s = {n: (4096, 1024, 128) for n in ("q", "k", "q_out", "k_out", "dq", "dk")}
    s.update(strides or {})
    return block._QkParams(ctypes.sizeof(block._QkParams) if size is None else size, *c.values(), reserved,
                           *[(ctypes.c_int64 * 3)(*v) for v in s.values()])


def qk(p, q=0x1000, k=0x2000, qw=0x3000, kw=0x4000, cs=0x5000, pos=0x6000, qo=0x7000, ko=0x8000):
    return pkg.library().lsm_qk_norm_rope(ctypes.byref(p), vp(q), vp(k), vp(qw), vp(kw), vp(cs), vp(pos), vp(qo), vp(ko), vp(None))


def qk_bwd(p, q=0x1000, k=0x2000, qw=0x3000, kw=0x4000, cs=0x5000, gq=0x6000, gk=0x7000, dq=0x8000, dk=0x9000, dqw=0xa000,
           dkw=0xb000, ws=0x10000, wsb=1 << 40):
    return pkg.library().lsm_qk_norm_rope_bwd(ctypes.byref(p), vp(q), vp(k), vp(qw), vp(kw), vp(cs), vp(None), vp(gq), vp(gk),
                                              vp(dq), vp(dk), vp(dqw), vp(dkw), vp(ws), wsb, vp(None))


def test_norm_and_rotation_refuse_bad_arguments():
    P = qk_params
    assert pkg.library().lsm_qk_norm_rope(None, *[vp(None)] * 9) == NULL
    for bad in (dict(B=0), dict(T=0), dict(H_q=0), dict(H_k=-1), dict(n_pos=-1), dict(n_pos=0), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(B=1 << 20, T=1 << 20), dict(H_q=1 << 21), dict(size=8)):
        assert qk(P(**bad)) == SHAPE, bad
        assert pkg.library().lsm_qk_norm_rope_bwd_workspace_bytes(ctypes.byref(P(**bad))) == 0
    for bad in (dict(d=96), dict(dtype=2), dict(norm=3), dict(norm=-1), dict(rotation=2), dict(rot_dim=24), dict(rot_dim=144),
                dict(reserved=1)):
        assert qk(P(**bad)) == UNSUP, bad
    for n in ("q", "k", "q_out", "k_out"):
        for i in range(3):
            s = [4096, 1024, 128]
            s[i] += 4
            assert qk(P(strides={n: s})) == ALIGN, (n, i)
    assert qk_bwd(P(strides={"dq": (4096, 1024, 130)})) == ALIGN
    assert qk(P(strides={"q": (4, 1024, 128)}, B=1), q=0x1008) == ALIGN     # an axis of one: its stride is free, the pointer is not
    for n in ("q", "qo", "cs", "ko", "k"):
        assert qk(P(), **{n: None}) == NULL, n
    for i in range(3):                                                         # rows that would be written more than once
        s = [4096, 1024, 128]
        s[i] = 0
        assert qk(P(strides={"q_out": s})) == SHAPE and qk(P(strides={"k_out": s})) == SHAPE
        assert qk_bwd(P(strides={"dq": s})) == SHAPE and qk_bwd(P(strides={"dk": s})) == SHAPE
        assert qk_bwd(P(strides={"q_out": s, "q": s}), wsb=16) == WS           # inputs may repeat
    assert qk(P(H_k=0)) == NULL and qk(P(H_k=0), k=None, ko=None) == NULL      # a k's weight without a k
    assert qk(P(rot_dim=0)) == NULL                                            # a table without a rotation
    assert qk(P(n_pos=7), pos=None) == SHAPE                                   # tokens beyond the table
    for n in ("q", "k", "qw", "kw", "cs", "pos", "qo", "ko"):
        assert qk(P(), **{n: 0x1004}) == ALIGN, n
    for n in ("gq", "gk", "dq", "dk"):
        assert qk_bwd(P(), **{n: None}) == NULL, n
    assert qk_bwd(P(), qw=None) == NULL and qk_bwd(P(), kw=None) == NULL       # a gradient without its weight
    assert qk_bwd(P(), ws=None) == WS and qk_bwd(P(), wsb=16) == WS
    for n in ("dqw", "dkw", "ws", "gk"):
        assert qk_bwd(P(), **{n: 0x1004}) == ALIGN, n


def beam_params(size=None, reserved=0, row_stride=None, **kw):
    c = dict(B=2, K=4, V=100, n_out=4, dtype=0, eos=-1)
    c.update(kw)
    return block._BeamParams(ctypes.sizeof(block._BeamParams) if size is None else size, *c.values(), reserved,
                             c["V"] if row_stride is None else row_stride)


def beam(p, x=0x1000, s=0x2000, f=None, o=0x3000, par=0x4000, tok=0x5000, of=None, ws=0x10000, wsb=1 << 40):
    return pkg.library().lsm_beam_select(ctypes.byref(p), vp(x), vp(s), vp(f), vp(o), vp(par), vp(tok), vp(of), vp(ws), wsb, vp(None))


def test_beam_selection_refuses_bad_arguments():
    P = beam_params
    need = pkg.library().lsm_beam_select_workspace_bytes
    assert pkg.library().lsm_beam_select(None, *[vp(None)] * 8, 0, vp(None)) == NULL
    for bad in (dict(B=0), dict(K=0), dict(V=0), dict(n_out=0), dict(row_stride=99), dict(K=1, V=3, n_out=4), dict(eos=100), dict(eos=-2),
                dict(K=32, V=(1 << 20) + 1), dict(size=4), dict(row_stride=1 << 41), dict(B=1 << 30)):
        assert beam(P(**bad)) == SHAPE, bad
        assert need(ctypes.byref(P(**bad))) == 0
    for bad in (dict(dtype=2), dict(K=33), dict(n_out=33), dict(reserved=1)):
        assert beam(P(**bad)) == UNSUP, bad
    for n in ("x", "s", "o", "par", "tok"):
        assert beam(P(), **{n: None}) == NULL, n
    assert beam(P(), f=0x6000) == NULL and beam(P(), of=0x6000) == NULL        # finished beams without an end token
    for n in ("x", "s", "o", "par", "tok", "f", "of", "ws"):
        assert beam(P(eos=1), **{n: 0x1004}) == ALIGN, n
    assert beam(P(), ws=None) == WS and beam(P(), wsb=need(ctypes.byref(P())) - 1) == WS
    assert 0 < need(ctypes.byref(P())) < need(ctypes.byref(P(V=50000))) < need(ctypes.byref(P(V=50000, n_out=8)))


def test_reordering_states_refuses_bad_arguments():
    def reorder(at=(0x1000, 0x2000), size=(64, 12), n=None, parent=0x3000, B=2, K=4):
        a, s = (vp * max(len(at), 1))(*at), (ctypes.c_size_t * max(len(size), 1))(*size)
        return pkg.library().lsm_state_reorder(a, s, len(at) if n is None else n, vp(parent), B, K, vp(None))
    assert reorder(parent=None) == NULL and reorder(at=(0x1000, None)) == NULL
    assert pkg.library().lsm_state_reorder(None, None, 1, vp(0x1000), 1, 1, vp(None)) == NULL
    assert reorder(n=0) == SHAPE and reorder(at=(0x1000,) * 65, size=(64,) * 65) == SHAPE
    assert reorder(B=0) == SHAPE and reorder(B=65536) == SHAPE and reorder(K=0) == SHAPE and reorder(K=33) == UNSUP
    assert reorder(size=(64, 0)) == SHAPE and reorder(size=(64, 6)) == SHAPE
    assert reorder(at=(0x1000, 0x2004)) == ALIGN and reorder(parent=0x3004) == ALIGN


def moe_params(size=None, **kw):
    c = dict(n=4, D=64, F=32, E=8, top_k=2, dtype=1, renormalise=1)
    c.update(kw)
    return block._MoeParams(ctypes.sizeof(block._MoeParams) if size is None else size, *c.values())


def moe(p, x=0x1000, r=0x2000, gu=0x3000, d=0x4000, res=0x5000, y=0x6000, ws=0x10000, wsb=1 << 40):
    return pkg.library().lsm_moe_step(ctypes.byref(p), vp(x), vp(r), vp(gu), vp(d), vp(res), vp(y), vp(ws), wsb, vp(None))


def test_mixture_of_experts_refuses_bad_arguments():
    P = moe_params
    need = pkg.library().lsm_moe_step_workspace_bytes
    assert pkg.library().lsm_moe_step(None, *[vp(None)] * 7, 0, vp(None)) == NULL
    for bad in (dict(n=0), dict(D=0), dict(F=0), dict(E=0), dict(top_k=0), dict(top_k=9), dict(size=4)):
        assert moe(P(**bad)) == SHAPE, bad
        assert need(ctypes.byref(P(**bad))) == 0
    for bad in (dict(n=129), dict(E=257), dict(top_k=17, E=32), dict(D=60), dict(F=36), dict(D=65544), dict(F=65544), dict(dtype=2),
                dict(renormalise=2)):
        assert moe(P(**bad)) == UNSUP, bad
    for n in ("x", "r", "gu", "d", "y"):
        assert moe(P(), **{n: None}) == NULL, n
    for n in ("x", "r", "gu", "d", "res", "y", "ws"):
        assert moe(P(), **{n: 0x1004}) == ALIGN, n
    assert moe(P(), ws=None) == WS and moe(P(), wsb=need(ctypes.byref(P())) - 1) == WS
    assert 0 < need(ctypes.byref(P())) < need(ctypes.byref(P(n=8))) < need(ctypes.byref(P(n=8, dtype=0, F=64)))
