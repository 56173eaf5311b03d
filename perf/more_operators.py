"""Workloads of the operators that training a Linear-MoE model needs around the token mixer: routing tokens to experts (with its
gradient and the plan that sorts them by expert), the experts' grouped products for many tokens (forward and backward), and
the losses over a large vocabulary that never hold the logits: softmax cross entropy, and distillation from a teacher's top
logits, both with gradients.

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

def _route(name, **kw):
    """n tokens' outputs of a router over E experts, top_k chosen; train: with the gradient; padded: that share of tokens is
    padding (all their outputs -inf: no expert); barred: that share of experts takes no tokens (-inf for every token)."""
    c = dict(name=name, op="route", train=False, n=1, E=64, top_k=8, dtype="f32", renormalise=True, padded=0.0, barred=0.0)
    c.update(kw)
    return c


def _experts(name, **kw):
    """n tokens of width D through E experts of width F, top_k of them for a token; skew: how unevenly the experts are liked
    (standard deviation of their bias, in router outputs of standard deviation 1); dropped: that share of (token, expert)
    pairs is left out; residual: what the result is added to."""
    c = dict(name=name, op="experts", train=False, n=1, D=1024, F=1024, E=64, top_k=8, dtype="bf16", skew=0.3, dropped=0.0,
             residual=True)
    c.update(kw)
    return c


def _loss(name, **kw):
    """n tokens of width D against V rows of an output layer; teacher: 0 for cross entropy with one target a token, else so many
    logits of a teacher; ignored: that share of tokens has no target (prompts, padding); train: with the gradients."""
    c = dict(name=name, op="loss", train=False, n=1, D=1024, V=32000, teacher=0, dtype="bf16", ignored=0.0, temperature=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # Routing of a handful of decoded tokens: latency of the launches.
        _route("route_n4", n=4),
        # A training step's tokens (B=4, T=8192), routed and sorted by expert, and the gradient of the router's outputs.
        _route("route_train_n32768", train=True, n=32768, dtype="bf16"),
        # A packed batch with padding behind the last sequence, an odd number of experts of which some are switched off.
        _route("route_train_n9373_e129", train=True, n=9373, E=129, top_k=6, renormalise=False, padded=0.1, barred=0.05),
        # A few tokens through the experts: as many experts as pairs, so their weights are what is read.
        _experts("experts_n5", n=5),
        # A prompt's tokens, forward alone, an expert width that no tile divides, experts that are liked unevenly.
        _experts("experts_prefill_n2047", n=2047, D=2048, F=1032, skew=0.6),
        # A training step of the small model (hidden 1024, 64 experts, 8 active) on half the metric shape's tokens.
        _experts("experts_train_n16384", train=True, n=16384),
        # Few larger experts in fp32, the precision for checking a model, with a capacity that drops pairs.
        _experts("experts_train_f32_n1500", train=True, n=1500, D=512, F=776, E=8, top_k=2, dtype="f32", dropped=0.05, residual=False),
        # Scoring three tokens: the output layer's weights are read once.
        _loss("ce_score_n3", n=3, V=50257),
        # A training step: an odd vocabulary, a third of the tokens are prompts without a target.
        _loss("ce_train_n8191", train=True, n=8191, D=2048, V=50257, ignored=0.3),
        # The same loss in fp32 with a small model.
        _loss("ce_train_f32_n700", train=True, n=700, D=512, V=32003, dtype="f32"),
        # Scoring a short reply against a teacher's 20 best logits.
        _loss("distill_score_n61", n=61, V=131071, teacher=20, temperature=2.0),
        # A step of distillation from the 64 best logits of each token.
        _loss("distill_train_n4096", train=True, n=4096, V=32000, teacher=64, ignored=0.1, temperature=2.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """A case of the ranges the listed ones stand for."""
    op = rng.choice(["route", "experts", "experts", "loss", "loss", "loss"])
    train, dtype = rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"])
    if op == "route":
        E = rng.choice([8, 16, 32, 60, 64, 64, 127, 128, 160, 256])
        return _route("", train=train, n=_log_int(rng, 1, 32768), E=E, top_k=rng.choice([1, 2, 3, 4, 6, 8]), dtype=dtype,
                      renormalise=rng.random() < 0.5, padded=rng.choice([0.0, 0.0, 0.2]), barred=rng.choice([0.0, 0.0, 0.1]))
    most = 2.5e12 if dtype == "bf16" else 2.5e11  # operations: no more than the largest listed case's
    if op == "experts":
        E, k = rng.choice([4, 8, 16, 32, 64, 64, 128]), rng.choice([1, 2, 4, 6, 8])
        k = min(k, E)
        D, F = 8 * _log_int(rng, 32, 320), 8 * _log_int(rng, 16, 350)
        F = max(128, min(F, (1 << 30) // (3 * E * D * SIZES[dtype]) // 8 * 8))
        n = _log_int(rng, 1, min(16384, int(most / (18 * k * D * F))))
        return _experts("", train=train, n=n, D=D, F=F, E=E, top_k=k, dtype=dtype, skew=rng.choice([0.0, 0.3, 1.0]),
                        dropped=rng.choice([0.0, 0.0, 0.1]), residual=rng.random() < 0.5)
    D, V = 8 * _log_int(rng, 32, 375), _log_int(rng, 2000, 131072)
    n = _log_int(rng, 1, min(16384, int(most / (6 * D * V))))
    return _loss("", train=train, n=n, D=D, V=V, teacher=rng.choice([0, 0, 1, 8, 32, 64, 100]), dtype=dtype,
                 ignored=rng.choice([0.0, 0.2, 0.6]), temperature=rng.choice([1.0, 1.0, 2.0, 0.7]))


# ---- inputs ------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_route(c, seed):
    gen, dev = _generator(seed), torch.device("cuda")
    n, E = c["n"], c["E"]
    logits = torch.randn(n, E, generator=gen, device=dev) + 0.3 * torch.randn(E, generator=gen, device=dev)
    logits[:, torch.rand(E, generator=gen, device=dev) < c["barred"]] = -math.inf
    logits[torch.rand(n, generator=gen, device=dev) < c["padded"]] = -math.inf
    s = dict(c, logits=logits.to(DTYPES[c["dtype"]]))
    if c["train"]:
        s["d_weights"] = torch.randn(n, c["top_k"], generator=gen, device=dev)
    return s


def _prepare_experts(c, seed):
    gen, dev, dt = _generator(seed), torch.device("cuda"), DTYPES[c["dtype"]]
    n, D, F, E, k = (c[name] for name in ("n", "D", "F", "E", "top_k"))

    def normal(std, *shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=dt).mul_(std)
    out = torch.randn(n, E, generator=gen, device=dev) + c["skew"] * torch.randn(E, generator=gen, device=dev)
    value, chosen = torch.sort(out, -1, descending=True)
    weights, chosen = torch.softmax(value[:, :k], -1), chosen[:, :k].int()
    dropped = torch.rand(n, k, generator=gen, device=dev) < c["dropped"]
    return dict(c, x=normal(1.0, n, D), weights=weights.masked_fill(dropped, 0.0), chosen=chosen.masked_fill(dropped, -1),
                w_gate_up=normal(D ** -0.5, E, 2 * F, D), w_down=normal(F ** -0.5, E, D, F),
                skip=normal(1.0, n, D) if c["residual"] else None, d_y=normal(1.0, n, D) if c["train"] else None)


def _prepare_loss(c, seed):
    gen, dev, dt = _generator(seed), torch.device("cuda"), DTYPES[c["dtype"]]
    n, D, V, K = (c[name] for name in ("n", "D", "V", "teacher"))
    s = dict(c, x=torch.randn(n, D, generator=gen, device=dev, dtype=dt),
             w=torch.randn(V, D, generator=gen, device=dev, dtype=dt).mul_(2 * D ** -0.5))
    left_out = torch.rand(n, generator=gen, device=dev) < c["ignored"]
    if K:  # distinct tokens in any order, their logits falling
        step = torch.randint(1, V // K + 1, (n, K), generator=gen, device=dev)
        s["index"] = ((step.cumsum(1) + torch.randint(0, V, (n, 1), generator=gen, device=dev)) % V).int()
        s["index"][left_out] = -1
        s["logits"] = (3 * torch.randn(n, K, generator=gen, device=dev)).sort(-1, descending=True).values
    else:
        s["target"] = torch.randint(0, V, (n,), generator=gen, device=dev, dtype=torch.int32).masked_fill_(left_out, -100)
    if c["train"]:
        s["d_loss"] = (0.5 + torch.rand(n, generator=gen, device=dev)) / n
    return s


def prepare(case, seed):
    return {"route": _prepare_route, "experts": _prepare_experts, "loss": _prepare_loss}[case["op"]](case, seed)


# ---- one pass: the framework's operators -------------------------------------------------------------------------

def _own_route(s):
    import paper_2503_05447_amd as lsm
    weights, chosen = lsm.lsm_moe_route(s["logits"], s["top_k"], renormalise=s["renormalise"])
    offsets, order, place = lsm.lsm_moe_plan(chosen, s["E"])
    out = dict(weights=weights, chosen=chosen, offsets=offsets, order=order, place=place)
    if s["train"]:
        out["d_logits"] = lsm.lsm_moe_route_bwd(s["logits"], chosen, s["d_weights"], renormalise=s["renormalise"])
    return out


def _own_experts(s):
    import paper_2503_05447_amd as lsm
    plan = lsm.lsm_moe_plan(s["chosen"], s["E"])
    if not s["train"]:
        return dict(y=lsm.lsm_moe_experts(s["x"], s["weights"], plan, s["w_gate_up"], s["w_down"], residual=s["skip"]))
    y = lsm.lsm_moe_experts(s["x"], s["weights"], plan, s["w_gate_up"], s["w_down"], residual=s["skip"])
    return dict(lsm.lsm_moe_experts_bwd(s["x"], s["weights"], plan, s["w_gate_up"], s["w_down"], s["d_y"]), y=y)


def _own_loss(s):
    import paper_2503_05447_amd as lsm
    if s["teacher"]:
        what = s["x"], s["w"], s["index"], s["logits"]
        loss, lse = lsm.lsm_linear_distill(*what, temperature=s["temperature"])
        grads = lsm.lsm_linear_distill_bwd(*what, lse, s["d_loss"], temperature=s["temperature"]) if s["train"] else {}
    else:
        what = s["x"], s["w"], s["target"]
        loss, lse = lsm.lsm_linear_cross_entropy(*what, temperature=s["temperature"])
        grads = lsm.lsm_linear_cross_entropy_bwd(*what, lse, s["d_loss"], temperature=s["temperature"]) if s["train"] else {}
    return dict(grads, loss=loss, lse=lse)


# ---- one pass: the plain forms -----------------------------------------------------------------------------------

def _plain_route(s):
    x, E, k = s["logits"].float(), s["E"], s["top_k"]
    value, chosen = torch.sort(x, dim=-1, descending=True, stable=True)
    value, chosen = value[:, :k], chosen[:, :k]
    there = value > -math.inf
    top = torch.where(there[:, :1], value[:, :1], 0.0)
    e = torch.exp(x - top)
    part = torch.exp(value - top)
    total = (part if s["renormalise"] else e).sum(-1, keepdim=True)
    weights = torch.where(there, part / total, 0.0)
    chosen = torch.where(there, chosen, -1)
    expert = torch.where(there, chosen, E).view(-1)
    sorted_by, order = torch.sort(expert, dim=0, stable=True)
    count = (expert[:, None] == torch.arange(E, device=x.device)).sum(0)
    offsets = torch.cat((count.new_zeros(1), count.cumsum(0)))
    at = torch.arange(expert.numel(), device=x.device)
    place = torch.empty_like(at).scatter_(0, order, at)
    out = dict(weights=weights, chosen=chosen.int(), offsets=offsets.int(), order=torch.where(sorted_by < E, order, -1).int(),
               place=torch.where(expert < E, place, -1).int().view_as(chosen))
    if s["train"]:
        d = torch.where(there, s["d_weights"], 0.0)
        along = (weights * d).sum(-1, keepdim=True)
        if s["renormalise"]:
            grad = torch.zeros_like(x)
        else:
            grad = torch.where(there[:, :1], -(e / torch.where(there[:, :1], total, 1.0)) * along, 0.0)
            along = 0.0
        grad = grad.scatter_add(1, chosen.clamp(min=0), weights * (d - along))
        out["d_logits"] = grad.to(s["logits"].dtype)
    return out


def _plain_experts(s):
    x, p, F = s["x"].float(), s["weights"], s["F"]
    y = torch.zeros_like(x) if s["skip"] is None else s["skip"].float()
    if s["train"]:
        d_y, dx, dp = s["d_y"].float(), torch.zeros_like(x), torch.zeros_like(p)
        d_up, d_down = torch.zeros_like(s["w_gate_up"]), torch.zeros_like(s["w_down"])
    if not s["train"] and s["n"] * s["top_k"] <= s["E"]:  # few pairs: their experts' weights, one matrix for each pair
        expert = s["chosen"].clamp(min=0)
        gate, up = torch.matmul(s["w_gate_up"][expert].float(), x[:, None, :, None]).split(F, 2)
        h = gate * torch.sigmoid(gate) * up * torch.where(s["chosen"] < 0, 0.0, p)[..., None, None]
        y = y + torch.matmul(s["w_down"][expert].float(), h).squeeze(-1).sum(1)
        return dict(y=y.to(s["x"].dtype))
    for e in range(s["E"]):
        rows, slot = (s["chosen"] == e).nonzero(as_tuple=True)
        xe, pe = x[rows], p[rows, slot][:, None]
        w_up, w_down = s["w_gate_up"][e].float(), s["w_down"][e].float()
        gate, up = (xe @ w_up.t()).split(F, -1)
        sig = torch.sigmoid(gate)
        h = gate * sig * up
        y = y.index_add(0, rows, pe * (h @ w_down.t()))
        if s["train"]:
            g = d_y[rows]
            t = g @ w_down
            dp[rows, slot] = (t * h).sum(-1)
            dh = pe * t
            da = torch.cat((dh * up * (sig + gate * sig * (1 - sig)), dh * gate * sig), -1)
            d_down[e] = (g.t() @ (pe * h)).to(d_down.dtype)
            d_up[e] = (da.t() @ xe).to(d_up.dtype)
            dx = dx.index_add(0, rows, da @ w_up)
    dt = s["x"].dtype
    if not s["train"]:
        return dict(y=y.to(dt))
    return dict(y=y.to(dt), dx=dx.to(dt), d_weights=dp, d_w_gate_up=d_up, d_w_down=d_down)


def _plain_teacher(s):
    """Entries that are there, their tokens (0 where none) and probabilities."""
    there = (s["index"] >= 0) & (s["index"] < s["V"])
    z = torch.where(there, s["logits"].float() / s["temperature"], -math.inf)
    e = torch.exp(z - z.max(-1, keepdim=True).values.clamp(min=-LARGEST))
    return there, torch.where(there, s["index"], 0).long(), e / e.sum(-1, keepdim=True).clamp(min=1.0)


def _plain_loss(s):
    x, w, scale = s["x"].float(), s["w"].float(), 1.0 / s["temperature"]
    z = (x @ w.t()) * scale
    top = z.max(-1, keepdim=True).values
    lse = top.squeeze(1) + torch.exp(z - top).sum(-1).log()
    if s["teacher"]:
        there, index, p = _plain_teacher(s)
        counts = there.any(-1)
        loss = (p * (torch.log(torch.where(p > 0, p, 1.0)) - z.gather(1, index) + lse[:, None])).sum(-1)
    else:
        counts = (s["target"] >= 0) & (s["target"] < s["V"])
        index = torch.where(counts, s["target"], 0).long()[:, None]
        p = torch.ones_like(lse)[:, None]
        loss = lse - z.gather(1, index).squeeze(1)
    out = dict(loss=torch.where(counts, loss, 0.0), lse=torch.where(counts, lse, 0.0))
    if s["train"]:
        g = torch.exp(z - lse[:, None]).scatter_add_(1, index, -p) * (torch.where(counts, s["d_loss"], 0.0) * scale)[:, None]
        out.update(dx=(g @ w).to(s["x"].dtype), dw=(g.t() @ x).to(s["w"].dtype))
    return out


def run(state):
    if own:
        return {"route": _own_route, "experts": _own_experts, "loss": _own_loss}[state["op"]](state)
    return {"route": _plain_route, "experts": _plain_experts, "loss": _plain_loss}[state["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _exact_route(s):
    """Softmax over the experts and its derivative by automatic differentiation; the sort by counting."""
    n, E, k = s["n"], s["E"], s["top_k"]
    x = s["logits"].double().requires_grad_()
    rank = torch.argsort(x.detach(), dim=1, descending=True, stable=True)[:, :k]
    there = x.detach().gather(1, rank) > -math.inf
    with torch.enable_grad():
        some = torch.where(there[:, :1], x, torch.zeros_like(x))
        share = torch.softmax(some, -1).gather(1, rank)
        share = torch.where(there, share, torch.zeros_like(share))
        if s["renormalise"]:
            share = share / torch.where(there[:, :1], share.sum(-1, keepdim=True), torch.ones_like(share[:, :1]))
    chosen = rank.masked_fill(~there, -1)
    flat = chosen.view(-1)
    groups = [(flat == e).nonzero().squeeze(1) for e in range(E)]
    order = torch.cat(groups)
    place = torch.full_like(flat, -1)
    place[order] = torch.arange(order.numel(), device=flat.device)
    offsets = torch.tensor([0] + [g.numel() for g in groups], device=flat.device).cumsum(0)
    order = torch.cat((order, order.new_full((n * k - order.numel(),), -1)))
    out = dict(weights=share.detach(), chosen=chosen.int(), offsets=offsets.int(), order=order.int(), place=place.view(n, k).int())
    if s["train"]:
        grad, = torch.autograd.grad(share, x, torch.where(there, s["d_weights"].double(), 0.0))
        out["d_logits"] = grad
    return out


def _exact_experts(s):
    x, p = s["x"].double(), s["weights"].double()
    y = torch.zeros_like(x) if s["skip"] is None else s["skip"].double().clone()
    out = {}
    if s["train"]:
        out = dict(dx=torch.zeros_like(x), d_weights=torch.zeros_like(p),
                   d_w_gate_up=torch.zeros(s["w_gate_up"].shape, dtype=torch.float64, device=x.device),
                   d_w_down=torch.zeros(s["w_down"].shape, dtype=torch.float64, device=x.device))
    for e in range(s["E"]):
        pairs = (s["chosen"].view(-1) == e).nonzero().squeeze(1)
        if pairs.numel() == 0:
            continue
        token = pairs // s["top_k"]
        leaves = [t.clone().requires_grad_(s["train"]) for t in
                  (x[token], p.view(-1)[pairs], s["w_gate_up"][e].double(), s["w_down"][e].double())]
        with torch.enable_grad():
            both = torch.matmul(leaves[0], leaves[2].t())
            gate, up = both[:, :s["F"]], both[:, s["F"]:]
            z = torch.matmul(gate / (1 + torch.exp(-gate)) * up, leaves[3].t()) * leaves[1][:, None]
        y.index_add_(0, token, z.detach())
        if s["train"]:
            gx, gp, gu, gd = torch.autograd.grad(z, leaves, s["d_y"].double()[token])
            out["dx"].index_add_(0, token, gx)
            out["d_weights"].view(-1)[pairs] = gp
            out["d_w_gate_up"][e], out["d_w_down"][e] = gu, gd
    return dict(out, y=y)


def _exact_loss(s):
    """Over the tokens that count alone; the derivative of a token's loss by its logits is softmax minus the wanted shares."""
    n, V, tau = s["n"], s["V"], s["temperature"]
    if s["teacher"]:
        there = (s["index"] >= 0) & (s["index"] < V)
        rows = there.any(1).nonzero().squeeze(1)
        there, index = there[rows], s["index"][rows].long().clamp(0, V - 1)
        share = torch.softmax((s["logits"][rows].double() / tau).masked_fill(~there, -math.inf), 1)
    else:
        rows = ((s["target"] >= 0) & (s["target"] < V)).nonzero().squeeze(1)
        index = s["target"][rows].long()[:, None]
        share = torch.ones(rows.numel(), 1, dtype=torch.float64, device=rows.device)
    x, w = s["x"][rows].double(), s["w"].double()
    z = torch.matmul(x, w.t()).div_(tau)
    lse = torch.logsumexp(z, 1)
    entropy = torch.special.xlogy(share, share).sum(1)
    out = dict(loss=torch.zeros(n, dtype=torch.float64, device=x.device), lse=torch.zeros(n, dtype=torch.float64, device=x.device))
    out["loss"][rows] = entropy + lse - (share * z.gather(1, index)).sum(1)
    out["lse"][rows] = lse
    if s["train"]:
        g = z.sub_(lse[:, None]).exp_()
        g.scatter_add_(1, index, -share)
        g.mul_((s["d_loss"].double()[rows] / tau)[:, None])
        dx = torch.zeros(n, s["D"], dtype=torch.float64, device=x.device)
        dx[rows] = torch.matmul(g, w)
        out.update(dx=dx, dw=torch.matmul(g.t(), x))
    return out


def exact(case, seed):
    return {"route": _exact_route, "experts": _exact_experts, "loss": _exact_loss}[case["op"]](prepare(case, seed))


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c, el = case, SIZES[case["dtype"]]
    if c["op"] == "route":
        pairs = c["n"] * c["top_k"]
        moved = c["n"] * c["E"] * el + pairs * 16 + 4 * (c["E"] + 1)  # weights, experts, order and place
        if c["train"]:  # the outputs of the router are there already; the gradients of the weights and of the outputs
            moved += pairs * 4 + c["n"] * c["E"] * el
        return dict(bytes=moved, flops=c["n"] * c["E"] * (8.0 if c["train"] else 4.0))
    if c["op"] == "experts":
        pairs = c["n"] * c["top_k"] * (1 - c["dropped"])
        active = c["E"] * (1 - (1 - c["top_k"] * (1 - c["dropped"]) / c["E"]) ** c["n"])
        per = 3 * c["D"] * c["F"]
        moved = el * (active * per + c["n"] * c["D"] * (3 if c["residual"] else 2)) + 8 * c["n"] * c["top_k"]
        if c["train"]:  # the gradients of y, of x, of the weights of every expert and of the routing weights
            moved += el * (c["E"] * per + 2 * c["n"] * c["D"]) + 4 * c["n"] * c["top_k"]
        return dict(bytes=moved, flops=2.0 * pairs * per * (3 if c["train"] else 1))
    n = c["n"] * (1 - c["ignored"])
    moved = el * (n + c["V"]) * c["D"] + c["n"] * (8 + 8 * max(c["teacher"], 1))
    if c["train"]:
        moved += el * (c["n"] + c["V"]) * c["D"] + 4 * c["n"]
    return dict(bytes=moved, flops=2.0 * n * c["V"] * c["D"] * (3 if c["train"] else 1))
