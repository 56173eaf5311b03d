"""Workloads of the operators around the token mixer: what feeds it (per-head norm of queries and keys with the rotation by
position, forward and backward) and what follows it when a model decodes (a mixture-of-experts layer for a few tokens; one
step of a beam search with the recurrent states moved along).

``listed()`` names the standing cases, ``draw(rng)`` makes further ones of the same ranges, ``prepare`` / ``run`` set a case
up and make one pass: through the public entry points where ``own`` is true, in elementary torch operations in 32 bits
otherwise.  ``exact`` gives the outputs from the definitions in 64 bits, ``work`` the bytes and operations a pass cannot do
without.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}
LARGEST = torch.finfo(torch.float32).max


# ---- cases -------------------------------------------------------------------------------------------------------

def _qk(name, **kw):
    """Norm and rotation of q and k.  train: forward and backward; norm: "rms" (with a weight per feature) or "l2";
    rot: features rotated; pairs: neighbouring features form a pair (else i and i + rot/2); tokens_first: [B,T,H,d], q and k
    being slices of one fused projection; positions: "index" (0..T-1 in every sequence), "packed" (restarting at random
    places), "cached" (anywhere up to 65535, one per token)."""
    c = dict(name=name, op="qk", train=False, B=1, T=1, H_q=16, H_k=16, d=128, dtype="bf16", norm="rms", rot=128, pairs=False,
             tokens_first=True, positions="index")
    c.update(kw)
    return c


def _moe(name, **kw):
    """Mixture of experts over n tokens of width D: E experts of width F, top_k of them for a token."""
    c = dict(name=name, op="moe", n=1, D=1024, F=1024, E=64, top_k=8, dtype="bf16", renormalise=True, residual=True)
    c.update(kw)
    return c


def _beam(name, **kw):
    """One beam step: n_out of K x V candidates for each of B sequences; pad: logits that follow a row's V; finished: some
    beams have ended; first: the first step, where one beam of each sequence counts; layers: so many layers' states
    [B K, H, d, d] follow their beams (0: selection alone)."""
    c = dict(name=name, op="beam", B=1, K=4, V=32000, n_out=4, dtype="f32", pad=0, finished=False, first=False, layers=0, H=8,
             d=128)
    c.update(kw)
    return c


def listed():
    return [
        # A chat-sized decode batch: one token for each of 4 sequences, 16 heads of 128.  Latency of a launch.
        _qk("qk_decode_b4", B=4, positions="cached"),
        # Prefill of unequal prompts packed on one token axis, grouped keys, the first half of a head rotated.
        _qk("qk_prefill_packed", T=9373, H_q=32, H_k=8, rot=64, positions="packed"),
        # A training step's worth of q and k at the metric shape of the token mixer (B=4, H=16, T=8192).
        _qk("qk_train_t8192", train=True, B=4, T=8192),
        # Unit keys for a delta-rule layer in fp32 with 64-wide heads, a length that is no multiple of anything.
        _qk("qk_train_f32_l2_t2047", train=True, B=4, T=2047, d=64, dtype="f32", norm="l2", rot=64, pairs=True,
            tokens_first=False),
        # One token through the experts of the small model (hidden 1024, 64 experts, 8 active).
        _moe("moe_one_token"),
        # A decode batch of 16 through the larger model's experts (hidden 2048), an expert width that no tile divides.
        _moe("moe_b16", n=16, D=2048, F=1032),
        # A full serving batch: every expert has tokens, some have several tiles of them.
        _moe("moe_b128", n=128, D=2048, F=1536, top_k=6),
        # Few large experts in fp32, the precision for checking a model.
        _moe("moe_f32_b5", n=5, D=1024, F=776, E=8, top_k=2, dtype="f32", renormalise=False, residual=False),
        # Beam search for one request, selection alone: latency.
        _beam("beam_select_b1"),
        # A decode step of 8 requests with 4 beams each and two layers' states; an odd vocabulary.
        _beam("beam_step_b8", B=8, V=50257, dtype="bf16", layers=2),
        # Wide search over a large vocabulary, twice as many candidates as beams: the logits are the work.
        _beam("beam_wide_v131071", B=16, K=16, V=131071, n_out=32, dtype="bf16", pad=1),
        # A serving batch whose states (4 layers of 16 heads, 1 GiB) follow their beams, some beams finished.
        _beam("beam_step_b32", B=32, K=8, V=32003, n_out=8, dtype="bf16", pad=61, finished=True, layers=4, H=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges the listed ones stand for."""
    op = rng.choice(["qk", "qk", "moe", "moe", "beam", "beam"])
    if op == "qk":
        dtype, d, H = rng.choice(["bf16", "bf16", "f32"]), rng.choice([64, 128, 128, 256]), rng.choice([2, 4, 8, 16, 32])
        group = rng.choice([g for g in (1, 1, 2, 4, 8) if H % g == 0])
        most = (1 << 27) // (SIZES[dtype] * d * H)  # half of the largest listed case's bytes, whatever the heads
        tokens = _log_int(rng, 1, most)
        B = 1 if rng.random() < 0.4 else min(tokens, _log_int(rng, 1, 32))
        return _qk("", train=rng.random() < 0.5, B=B, T=max(1, tokens // B), H_q=H, H_k=H // group, d=d, dtype=dtype,
                   norm=rng.choice(["rms", "rms", "l2"]), rot=rng.choice([0, d // 2, d, d]), pairs=rng.random() < 0.3,
                   tokens_first=rng.random() < 0.6, positions=rng.choice(["index", "packed", "cached"]))
    if op == "moe":
        dtype, E = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([8, 16, 32, 64, 128])
        D, F = 8 * _log_int(rng, 32, 375), 8 * _log_int(rng, 16, 350)
        F = max(128, min(F, (1 << 30) // (3 * E * D * SIZES[dtype]) // 8 * 8))
        return _moe("", n=_log_int(rng, 1, 128), D=D, F=F, E=E, top_k=rng.choice([1, 2, 4, 6, 8]), dtype=dtype,
                    renormalise=rng.random() < 0.5, residual=rng.random() < 0.5)
    K = rng.choice([1, 2, 3, 4, 5, 8, 16])
    V = _log_int(rng, 4096, 131072)
    B = _log_int(rng, 1, max(1, min(64, (1 << 25) // (K * V))))
    finished, first = rng.random() < 0.4, rng.random() < 0.2
    if rng.random() < 0.4:
        return _beam("", B=B, K=K, V=V, n_out=rng.choice([K, 2 * K]), dtype=rng.choice(["bf16", "f32"]),
                     pad=rng.choice([0, 0, 3, 64]), finished=finished, first=first)
    H, d = rng.choice([4, 8, 16]), rng.choice([64, 128])
    most = (1 << 30) // (B * K * H * d * d * 4)
    return _beam("", B=B, K=K, V=V, n_out=K, dtype=rng.choice(["bf16", "f32"]), pad=rng.choice([0, 0, 3, 64]),
                 finished=finished, first=first, layers=max(1, min(rng.choice([1, 2, 6, 12]), most)), H=H, d=d)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_qk(c, seed):
    gen, dev, dt = _generator(seed), torch.device("cuda"), DTYPES[c["dtype"]]
    B, T, Hq, Hk, d, rot = (c[n] for n in ("B", "T", "H_q", "H_k", "d", "rot"))

    def heads(H):
        shape = (B, T, H, d) if c["tokens_first"] else (B, H, T, d)
        return torch.randn(shape, generator=gen, device=dev, dtype=dt)
    s = dict(c)
    if c["tokens_first"]:  # q and k as they stand in the output of one projection, the values behind them
        fused = torch.randn(B, T, Hq + 2 * Hk, d, generator=gen, device=dev, dtype=dt)
        s["q"], s["k"] = fused[:, :, :Hq], fused[:, :, Hq:Hq + Hk]
    else:
        s["q"], s["k"] = heads(Hq), heads(Hk)
    s["q_weight"] = s["k_weight"] = None
    if c["norm"] == "rms":
        s["q_weight"] = 1 + 0.2 * torch.randn(d, generator=gen, device=dev)
        s["k_weight"] = 1 + 0.2 * torch.randn(d, generator=gen, device=dev)
    n_pos = 65536 if c["positions"] == "cached" else T
    s["positions"] = None
    if c["positions"] == "cached":
        s["positions"] = torch.randint(0, n_pos, (B, T), generator=gen, device=dev, dtype=torch.int32)
    elif c["positions"] == "packed":
        t = torch.arange(T, device=dev).expand(B, T)
        start = (torch.rand(B, T, generator=gen, device=dev) < 8 / T) | (t == 0)
        s["positions"] = (t - torch.where(start, t, 0).cummax(1).values).to(torch.int32)
    s["cos_sin"] = None
    if rot:
        angle = torch.arange(n_pos, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        s["cos_sin"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    if c["train"]:
        s["d_q_out"], s["d_k_out"] = heads(Hq), heads(Hk)
    return s


def _prepare_moe(c, seed):
    gen, dev, dt = _generator(seed), torch.device("cuda"), DTYPES[c["dtype"]]
    n, D, F, E = (c[k] for k in ("n", "D", "F", "E"))

    def weight(std, *shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=dt).mul_(std)
    return dict(c, x=weight(1.0, n, D), router=weight(2 / D ** 0.5, E, D), w_gate_up=weight(D ** -0.5, E, 2 * F, D),
                w_down=weight(F ** -0.5, E, D, F), skip=weight(1.0, n, D) if c["residual"] else None)


def _prepare_beam(c, seed):
    gen, dev = _generator(seed), torch.device("cuda")
    B, K, V = (c[k] for k in ("B", "K", "V"))
    logits = (3 * torch.randn(B, K, V + c["pad"], generator=gen, device=dev)).to(DTYPES[c["dtype"]])
    logits.masked_fill_(torch.rand(logits.shape, generator=gen, device=dev) < 0.01, -math.inf)  # tokens not allowed here
    scores = -10 * torch.rand(B, K, generator=gen, device=dev)
    if c["first"]:
        scores[:, 1:] = -math.inf
    ended = torch.rand(B, K, generator=gen, device=dev) < 0.15 if c["finished"] else None
    states = [torch.randn(B * K, c["H"], c["d"], c["d"], generator=gen, device=dev) for _ in range(c["layers"])]
    return dict(c, logits=logits[:, :, :V], scores=scores, ended=ended, eos=2 if c["finished"] else None, states=states)


def prepare(case, seed):
    return {"qk": _prepare_qk, "moe": _prepare_moe, "beam": _prepare_beam}[case["op"]](case, seed)


# ---- one pass: the framework's operators -------------------------------------------------------------------------

def _own_qk(s):
    import paper_2503_05447_amd as lsm
    how = dict(cos_sin=s["cos_sin"], positions=s["positions"], q_weight=s["q_weight"], k_weight=s["k_weight"],
               norm=lsm.NORM_RMS if s["norm"] == "rms" else lsm.NORM_L2, eps=1e-6,
               rotation=lsm.ROT_PAIRS if s["pairs"] else lsm.ROT_HALVES, q_scale=s["d"] ** -0.5,
               layout=lsm.LAYOUT_BTHD if s["tokens_first"] else lsm.LAYOUT_BHTD)
    out = lsm.lsm_qk_norm_rope(s["q"], s["k"], **how)
    if not s["train"]:
        return out
    return out, lsm.lsm_qk_norm_rope_bwd(s["q"], s["k"], s["d_q_out"], s["d_k_out"], **how)


def _own_moe(s):
    import paper_2503_05447_amd as lsm
    return lsm.lsm_moe_step(s["x"], s["router"], s["w_gate_up"], s["w_down"], s["top_k"], renormalise=s["renormalise"],
                            residual=s["skip"])


def _own_beam(s):
    import paper_2503_05447_amd as lsm
    scores, parent, token, ended = lsm.lsm_beam_select(s["logits"], s["scores"], s["n_out"], finished=s["ended"], eos=s["eos"])
    if s["states"]:
        lsm.lsm_state_reorder(s["states"], parent)
    return dict(scores=scores, parent=parent, token=token, finished=ended, states=s["states"])


# ---- one pass: the plain forms -----------------------------------------------------------------------------------

def _rotation(s):
    """cos, sin of every token, shaped to go with [.., rot/2] halves of q and k."""
    table = s["cos_sin"] if s["positions"] is None else s["cos_sin"][s["positions"].long()]
    cos, sin = (table if table.dim() == 3 else table[None]).chunk(2, -1)
    return (cos[:, :, None], sin[:, :, None]) if s["tokens_first"] else (cos[:, None], sin[:, None])


def _turn(x, s, back):
    if not s["rot"]:
        return x
    cos, sin = _rotation(s)
    sin = -sin if back else sin
    turned, rest = x[..., :s["rot"]], x[..., s["rot"]:]
    if s["pairs"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = turned.chunk(2, -1)
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1)


def _inverse_length(x, s):
    square = x * x
    return torch.rsqrt((square.mean(-1, keepdim=True) if s["norm"] == "rms" else square.sum(-1, keepdim=True)) + 1e-6)


def _plain_head(x, weight, scale, s):
    xf = x.float()
    n = xf * _inverse_length(xf, s)
    n = n if weight is None else n * weight
    return (scale * _turn(n, s, False)).to(x.dtype)


def _plain_head_gradient(x, weight, scale, g, s):
    xf = x.float()
    r = _inverse_length(xf, s)
    n = xf * r
    u = _turn(scale * g.float(), s, True)
    z = u if weight is None else u * weight
    along = (n * z).mean(-1, keepdim=True) if s["norm"] == "rms" else (n * z).sum(-1, keepdim=True)
    return (r * (z - n * along)).to(x.dtype), None if weight is None else (u * n).sum((0, 1, 2))


def _plain_qk(s):
    qs = s["d"] ** -0.5
    out = _plain_head(s["q"], s["q_weight"], qs, s), _plain_head(s["k"], s["k_weight"], 1.0, s)
    if not s["train"]:
        return out
    dq, dqw = _plain_head_gradient(s["q"], s["q_weight"], qs, s["d_q_out"], s)
    dk, dkw = _plain_head_gradient(s["k"], s["k_weight"], 1.0, s["d_k_out"], s)
    return out, dict(dq=dq, dk=dk, d_q_weight=dqw, d_k_weight=dkw)


def _plain_moe(s):
    x, E, F, k = s["x"].float(), s["E"], s["F"], s["top_k"]
    p = torch.softmax(x @ s["router"].float().t(), -1)
    p, chosen = torch.topk(p, k, -1)
    if s["renormalise"]:
        p = p / p.sum(-1, keepdim=True)
    if s["n"] * k < E:  # the chosen experts' weights for each token
        gate, up = torch.matmul(s["w_gate_up"][chosen].float(), x[:, None, :, None]).squeeze(-1).split(F, -1)
        h = gate * torch.sigmoid(gate) * up * p[..., None]
        y = torch.matmul(s["w_down"][chosen].float(), h[..., None]).squeeze(-1).sum(1)
    else:  # every expert for every token, those not chosen with weight 0
        w = torch.zeros(s["n"], E, device=x.device).scatter_(1, chosen, p)
        both = (s["w_gate_up"].float().view(-1, s["D"]) @ x.t()).view(E, 2 * F, s["n"])
        gate, up = both.split(F, 1)
        h = gate * torch.sigmoid(gate) * up * w.t()[:, None]
        y = torch.bmm(s["w_down"].float(), h).sum(0).t()
    if s["skip"] is not None:
        y = y + s["skip"].float()
    return y.to(s["x"].dtype).contiguous()


def _plain_beam(s):
    B, K, V, n = s["B"], s["K"], s["V"], s["n_out"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x).clamp(max=LARGEST)
    m = x.max(-1, keepdim=True).values
    score = s["scores"][..., None] + ((x - m) - torch.exp(x - m).sum(-1, keepdim=True).log())
    score = torch.where(torch.isnan(score), -math.inf, score)
    if s["ended"] is not None:
        alone = torch.full_like(score, -math.inf)
        alone[..., s["eos"]] = s["scores"]
        score = torch.where(s["ended"][..., None], alone, score)
    score = score.view(B, K * V) + 0.0
    bits = score.view(torch.int32).long()  # whole numbers in the order of the scores, the lowest index first among equals
    order = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits)
    best = torch.topk((order << 32) + (K * V - 1 - torch.arange(K * V, device=x.device)), n, -1).values
    index = K * V - 1 - (best & 0xffffffff)
    parent, token = (index // V).int(), (index % V).int()
    ended = None if s["ended"] is None else s["ended"].gather(1, parent.long()) | (token == s["eos"])
    if s["states"]:
        rows = (torch.arange(B, device=x.device)[:, None] * K + parent).view(-1)
        for m in s["states"]:
            m.copy_(m[rows])
    return dict(scores=score.gather(1, index), parent=parent, token=token, finished=ended, states=s["states"])


def run(state):
    if own:
        return {"qk": _own_qk, "moe": _own_moe, "beam": _own_beam}[state["op"]](state)
    return {"qk": _plain_qk, "moe": _plain_moe, "beam": _plain_beam}[state["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _exact_head(x, weight, scale, s):
    """x / length, times weight, as complex numbers turned by their position's angle."""
    length = x.norm(dim=-1, keepdim=True) ** 2
    y = x / ((length / x.shape[-1] if s["norm"] == "rms" else length) + 1e-6).sqrt()
    if weight is not None:
        y = y * weight
    rot = s["rot"]
    if rot:
        B, T = s["B"], s["T"]
        at = torch.arange(T, device=x.device).expand(B, T) if s["positions"] is None else s["positions"].long()
        table = s["cos_sin"].double()[at]
        z = torch.complex(table[..., :rot // 2], table[..., rot // 2:]).unsqueeze(2 if s["tokens_first"] else 1)
        part = y[..., :rot].unflatten(-1, (-1, 2) if s["pairs"] else (2, -1))
        part = part if s["pairs"] else part.transpose(-1, -2)
        part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * z)
        part = part if s["pairs"] else part.transpose(-1, -2)
        y = torch.cat((part.flatten(-2), y[..., rot:]), -1)
    return scale * y


def _exact_qk(s):
    out, grads = [], {}
    for n, scale in (("q", s["d"] ** -0.5), ("k", 1.0)):
        w = s[n + "_weight"]
        x, w = s[n].double().requires_grad_(), None if w is None else w.double().requires_grad_()
        with torch.enable_grad():
            y = _exact_head(x, w, scale, s)
        out.append(y.detach())
        grads["d_%s_weight" % n] = None
        if s["train"]:
            got = torch.autograd.grad(y, [x] if w is None else [x, w], s["d_%s_out" % n].double())
            grads["d" + n] = got[0]
            if w is not None:
                grads["d_%s_weight" % n] = got[1]
        del x, y
    return (tuple(out), grads) if s["train"] else tuple(out)


def _exact_moe(s):
    x = s["x"].double()
    logits = x @ s["router"].double().t()
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    y = torch.zeros_like(x) if s["skip"] is None else s["skip"].double().clone()
    chosen = torch.argsort(p, dim=1, descending=True, stable=True)[:, :s["top_k"]]
    total = p.gather(1, chosen).sum(1) if s["renormalise"] else torch.ones_like(p[:, 0])
    for expert in chosen.unique().tolist():
        rows = (chosen == expert).any(1).nonzero().squeeze(1)
        both = x[rows] @ s["w_gate_up"][expert].double().t()
        gate, up = both[:, :s["F"]], both[:, s["F"]:]
        h = gate / (1 + torch.exp(-gate)) * up
        y[rows] += (p[rows, expert] / total[rows])[:, None] * (h @ s["w_down"][expert].double().t())
    return y


def _exact_beam(s):
    B, K, V = s["B"], s["K"], s["V"]
    score = s["scores"].double()[..., None] + torch.log_softmax(s["logits"].double(), -1)
    if s["ended"] is not None:
        score[s["ended"]] = -math.inf
        score[..., s["eos"]] = torch.where(s["ended"], s["scores"].double(), score[..., s["eos"]])
    value, index = torch.sort(score.view(B, K * V), dim=1, descending=True, stable=True)
    value, index = value[:, :s["n_out"]], index[:, :s["n_out"]]
    parent, token = index // V, index % V
    ended = None if s["ended"] is None else s["ended"].gather(1, parent) | (token == s["eos"])
    states = [m.view(B, K, -1)[torch.arange(B, device=m.device)[:, None], parent].view(m.shape).double() for m in s["states"]]
    return dict(scores=value, parent=parent, token=token, finished=ended, states=states)


def exact(case, seed):
    return {"qk": _exact_qk, "moe": _exact_moe, "beam": _exact_beam}[case["op"]](prepare(case, seed))


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def _active(n, E, k):
    """Experts that n tokens with k of E experts each are expected to reach."""
    return E * (1 - (1 - k / E) ** n)


def work(case):
    c = case
    if c["op"] == "qk":
        el = c["B"] * c["T"] * (c["H_q"] + c["H_k"]) * c["d"]
        moved = el * SIZES[c["dtype"]] * (5 if c["train"] else 2)
        # the rotation's cosines and sines, once for each token in either direction
        return dict(bytes=moved + c["B"] * c["T"] * 4 * c["rot"] * (2 if c["train"] else 1), flops=el * (23 if c["train"] else 8))
    if c["op"] == "moe":
        per = 3 * c["D"] * c["F"]
        io = c["n"] * c["D"] * (3 if c["residual"] else 2) + c["E"] * c["D"]
        return dict(bytes=SIZES[c["dtype"]] * (per * _active(c["n"], c["E"], c["top_k"]) + io),
                    flops=2.0 * c["n"] * (c["top_k"] * per + c["E"] * c["D"]))
    el = c["B"] * c["K"] * c["V"]
    moved = 2 * 4 * c["layers"] * c["B"] * c["K"] * c["H"] * c["d"] ** 2
    return dict(bytes=el * SIZES[c["dtype"]] + moved + c["B"] * (4 * c["K"] + 12 * c["n_out"]), flops=4.0 * el)
