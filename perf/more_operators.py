"""The dense block in front of the uniformly-sparse output layer, and what the layer learns from beside label lists, as cases that can be timed and compared.

A case is a dict of plain values.  Its "kind" names the operator of one pass:

  gated         the gated block: x = act(e V_gate^T) * (e V_up^T), e the trunk's output, x the layer's activations; keeps both projections for its backward pass
  gated_grad    its backward pass, from the gradient that the layer returns: by e, by V_gate, by V_up
  project_i8    one projection in 8-bit integers: e quantised row by row, its product with a matrix that is held so
  gated_i8      the gated block of a serving process: e quantised, both projections in 8-bit integers
  distill       loss and gradient of the scores against a teacher's best labels and their logits
  policy        loss and gradient of a clipped policy objective with a KL term, for the labels that instances were answered with; their log-probabilities

m labels, d activations, w values of the trunk, batch b; "storage" is the type of e, x and the matrices, all sums are 32 bits.

own = False: every operator in its plain form, elementary torch operations in 32 bits, rounded once at the end.
own = True:  the calls of paper_2306_03725_amd.usl.Layer.
"""
import math

import torch

own = False

TEMPERATURE = 2.0                             # of the distillation
CLIP_LOW, CLIP_HIGH, BETA = 0.2, 0.28, 0.05   # bounds of the policy's ratio below and above 1, weight of its KL term
SILU, GELU = 0, 1                             # the block's activations, as the library numbers them
LIMIT = {"gated": 512 * 768 * 32768, "gated_grad": 512 * 768 * 32768, "project_i8": 1024 * 512 * 65536, "gated_i8": 512 * 768 * 32768,
         "distill": 256 * 500000, "policy": 256 * 500000}   # the largest listed case of a kind, in products or scores


def listed():
    def case(name, kind, **sizes):
        return dict(name=name, kind=kind, **sizes)

    return [
        # one request of a serving process: the rate at which both matrices are read
        case("gated_one", "gated", b=1, w=768, d=32768, act="silu", storage="bf16"),
        # a training step's way up, the batch of the widest bfloat16 configuration
        case("gated_batch", "gated", b=512, w=768, d=32768, act="silu", storage="bf16"),
        # its way back
        case("gated_grad_batch", "gated_grad", b=512, w=768, d=32768, act="silu", storage="bf16"),
        # sizes that are multiples of nothing, in float32
        case("gated_grad_ragged", "gated_grad", b=100, w=509, d=4099, act="gelu", storage="f32"),
        # one request against the widest layer of activations
        case("project_i8_one", "project_i8", b=1, w=512, d=65536, storage="f32"),
        # a batch against it
        case("project_i8_batch", "project_i8", b=1024, w=512, d=65536, storage="bf16"),
        # a handful of requests that came together
        case("gated_i8_few", "gated_i8", b=7, w=768, d=32768, act="silu", storage="bf16"),
        # evaluation of a batch, an odd width
        case("gated_i8_batch", "gated_i8", b=500, w=750, d=32768, act="gelu", storage="bf16"),
        # the middle-sized layer, a teacher's 32 best labels
        case("distill_medium", "distill", m=30938, b=128, n=32),
        # the headline layer and batch, a teacher's 100 best labels
        case("distill_large", "distill", m=500000, b=256, n=100),
        # odd sizes, one answer an instance
        case("policy_ragged", "policy", m=70001, b=100, n=1),
        # the headline layer and batch, answers of up to 10 labels
        case("policy_large", "policy", m=500000, b=256, n=10),
    ]


def draw(rng):
    """One more case: sizes spread over their logarithm, odd ones among them, no larger than the largest listed one of its kind."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["gated", "gated", "gated_grad", "gated_grad", "project_i8", "gated_i8", "distill", "policy"])
    while True:
        case = dict(kind=kind)
        if kind in ("distill", "policy"):
            case.update(m=log_int(1000, 3000000), b=log_int(1, 1024), n=log_int(1, 256 if kind == "distill" else 32))
            size = case["m"] * case["b"]
        else:
            case.update(b=log_int(1, 1024), w=log_int(64, 2048), d=log_int(64, 65536), storage=rng.choice(["f32", "bf16"]))
            if kind != "project_i8":
                case["act"] = rng.choice(["silu", "gelu"])
            if rng.random() < 0.5:   # as widths mostly are
                case.update(w=max(64, case["w"] // 64 * 64), d=max(64, case["d"] // 64 * 64))
            size = case["b"] * case["w"] * case["d"]
        if 30000 <= size <= LIMIT[kind]:
            return case


# ------------------------------------------------------------------------------------------------ inputs

def _act(name):
    return SILU if name == "silu" else GELU


def _lengths(case):
    """The lengths of the instances' lists, in some order: a teacher's best labels, every ninth instance has none; or the labels of an answer."""
    b, n = case["b"], case["n"]
    if case["kind"] == "policy":
        return [1 + i % n for i in range(b)]
    return [0 if i % 9 == 8 else n - 5 * i % (n * 3 // 10 + 1) for i in range(b)]


def prepare(case, seed):
    kind, b = case["kind"], case["b"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kept = torch.bfloat16 if case.get("storage") == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(shape, device="cuda", generator=gen)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def codes(rows, w):
        """A matrix as a serving process holds it: codes whose row has a 127, a scale for each row."""
        q = (normal(rows, w) * (127.0 / 3.5)).round_().clamp_(-127, 127).to(torch.int8)
        q[:, 0] = 127
        return q, (uniform(rows) + 0.5) * (3.5 / 127 * w ** -0.5)

    s = dict(case=case)
    if kind in ("gated", "gated_grad"):
        w, d = case["w"], case["d"]
        s["e"] = normal(b, w).to(kept)
        s["V_gate"], s["V_up"] = (normal(d, w).mul_(w ** -0.5).to(kept) for _ in range(2))
        if kind == "gated":
            s["x"], s["gate"], s["up"] = (empty(b, d, dtype=kept) for _ in range(3))
        else:   # what the forward pass kept, and the gradient that the layer returns
            s["gate"], s["up"] = ((s["e"].float() @ s[v].float().t()).to(kept) for v in ("V_gate", "V_up"))
            s["grad_x"] = normal(b, d).mul_(1.0 / b)
            s["grad_e"], s["grad_V_gate"], s["grad_V_up"] = empty(b, w), empty(d, w), empty(d, w)
    elif kind in ("project_i8", "gated_i8"):
        w, d = case["w"], case["d"]
        s["e"] = (normal(b, w) * (uniform(b, 1) + 0.5)).to(kept)   # tokens of different sizes
        s["e_codes"], s["e_scales"] = empty(b, w, dtype=torch.int8), empty(b)
        for name in ("V",) if kind == "project_i8" else ("V_gate", "V_up"):
            s[name + "_codes"], s[name + "_scales"] = codes(d, w)
        s["x"] = empty(b, d, dtype=kept)
    else:
        m, most = case["m"], case["n"]
        s["out"] = normal(b, m).mul_(1.5)
        lengths = torch.tensor(_lengths(case), dtype=torch.int64, device="cuda")[torch.randperm(b, device="cuda", generator=gen)]
        s["off"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)])
        n = int(s["off"][-1])
        # distinct labels of an instance: a start and steps of its own (m is far more than n of them)
        row = torch.searchsorted(s["off"], torch.arange(n, device="cuda"), right=True) - 1
        step = 1 + (uniform(b) * max(1, m // (most + 1) - 1)).to(torch.int64)
        s["lab"] = (((uniform(b) * m).to(torch.int64)[row] + step[row] * (torch.arange(n, device="cuda") - s["off"][row])) % m).to(torch.int32)
        if kind == "distill":
            s["out"].view(-1).index_add_(0, row * m + s["lab"], normal(n).add_(4.0))   # a student that has learned something
            s["logit"] = normal(n).mul_(2.0).add_(8.0)
        else:
            s["out"].view(-1).index_add_(0, row * m + s["lab"], normal(n).add_(6.0))   # likely answers
            logp = _plain_logp(s["out"], row, s["lab"])
            # the policy that answered and the reference: some answers' ratios lie inside the bounds, some beyond
            s["old_logp"], s["ref_logp"] = logp + 0.25 * normal(n), logp + 0.3 * normal(n)
            s["advantage"] = normal(n)
            s["logp"] = empty(n)
        s["g"], s["loss"] = empty(b, m), empty(1)
    if own:   # the handle that such a program keeps
        from paper_2306_03725_amd import usl
        s["layer"] = usl.Layer(case.get("m", 1), case.get("d", 1), 1, b, case.get("storage", "f32"), torch.cuda.current_stream().cuda_stream)
    return s


# ------------------------------------------------------------------------------------------------ one pass

def _plain_act(gate, act):
    if act == "silu":
        return gate / (1.0 + torch.exp(-gate))
    return 0.5 * gate * (1.0 + torch.erf(gate * math.sqrt(0.5)))


def _plain_slope(gate, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-gate))
        return p * (1.0 + gate * (1.0 - p))
    return 0.5 * (1.0 + torch.erf(gate * math.sqrt(0.5))) + gate * torch.exp(-0.5 * gate * gate) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_codes(e):
    """The values of e in 8-bit integers, as numbers, and the rows' scales."""
    e = e.float()
    scale = (e.abs().amax(1) / 127.0).clamp_(min=2.0 ** -126)
    return torch.round(e / scale[:, None]).clamp_(-127, 127), scale


def _plain_product(q, e_scale, codes, scales):
    """Products of 8-bit numbers, summed exactly: up to 1024 of them at a time stay below 2^24."""
    acc = torch.zeros((q.shape[0], codes.shape[0]), dtype=torch.float64, device="cuda") if q.shape[1] > 1024 else None
    if acc is None:
        acc = q @ codes.float().t()
    else:
        acc.add_(q[:, :1024] @ codes[:, :1024].float().t())
        acc.add_(q[:, 1024:] @ codes[:, 1024:].float().t())
    return acc.float() * (e_scale[:, None] * scales)


def _plain_logp(out, row, lab):
    top = out.amax(1, keepdim=True)
    lse = torch.log(torch.exp(out - top).sum(1).double()) + top[:, 0].double()
    return (out[row, lab.long()].double() - lse[row]).float()


def _rows(s):
    """The instance of every list entry."""
    return torch.searchsorted(s["off"], torch.arange(s["lab"].numel(), device="cuda"), right=True) - 1


def _plain_distill(s):
    out, b, m = s["out"], s["case"]["b"], s["case"]["m"]
    row, at = _rows(s), s["lab"].long()
    t = s["logit"].double() / TEMPERATURE
    top = torch.full((b,), -math.inf, dtype=torch.float64, device="cuda").scatter_reduce_(0, row, t, "amax")
    p = torch.exp(t - top[row])
    total = torch.zeros(b, dtype=torch.float64, device="cuda").index_add_(0, row, p)
    p, log_p = p / total[row], t - top[row] - torch.log(total[row])
    best = out.amax(1, keepdim=True)
    q = torch.exp((out - best) / TEMPERATURE)
    mass = q.sum(1, keepdim=True)
    log_q = (out[row, at].double() - best[row, 0].double()) / TEMPERATURE - torch.log(mass[row, 0].double())
    scale = 1.0 / b
    q *= scale * TEMPERATURE / mass
    q *= (s["off"].diff() > 0)[:, None]
    q.view(-1).index_add_(0, row * m + at, (-scale * TEMPERATURE * p).float())
    return dict(g=q, loss=(scale * TEMPERATURE ** 2 * (p * (log_p - log_q)).sum()).float().view(1))


def _plain_policy(s):
    out, b, m = s["out"], s["case"]["b"], s["case"]["m"]
    row, at = _rows(s), s["lab"].long()
    best = out.amax(1, keepdim=True)
    q = torch.exp(out - best)
    mass = q.sum(1, keepdim=True)
    logp = out[row, at].double() - best[row, 0].double() - torch.log(mass[row, 0].double())
    a = s["advantage"].double()
    ratio = torch.exp(logp - s["old_logp"].double())
    free, bound = ratio * a, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * a
    back = torch.exp(s["ref_logp"].double() - logp)
    scale = 1.0 / s["lab"].numel()
    loss = scale * (BETA * (back - (s["ref_logp"].double() - logp) - 1.0) - torch.minimum(free, bound)).sum()
    c = scale * (BETA * (1.0 - back) - torch.where(free <= bound, free, 0.0))   # of the loss by the log-probability
    total = torch.zeros(b, dtype=torch.float64, device="cuda").index_add_(0, row, c)
    q *= -(total[:, None] / mass.double()).float()
    q.view(-1).index_add_(0, row * m + at, c.float())
    return dict(g=q, logp=logp.float(), loss=loss.float().view(1))


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "distill":
        return _plain_distill(s)
    if kind == "policy":
        return _plain_policy(s)
    kept = s["e"].dtype
    if kind == "gated":
        gate, up = (s["e"].float() @ s[v].float().t() for v in ("V_gate", "V_up"))
        return dict(x=(_plain_act(gate, case["act"]) * up).to(kept), gate=gate.to(kept), up=up.to(kept))
    if kind == "gated_grad":
        gate, up = s["gate"].float(), s["up"].float()
        by_gate, by_up = s["grad_x"] * up * _plain_slope(gate, case["act"]), s["grad_x"] * _plain_act(gate, case["act"])
        e = s["e"].float()
        return dict(grad_e=by_gate @ s["V_gate"].float() + by_up @ s["V_up"].float(), grad_V_gate=by_gate.t() @ e, grad_V_up=by_up.t() @ e)
    q, scale = _plain_codes(s["e"])
    if kind == "project_i8":
        return dict(h=_plain_product(q, scale, s["V_codes"], s["V_scales"]).to(kept))
    gate, up = (_plain_product(q, scale, s[v + "_codes"], s[v + "_scales"]) for v in ("V_gate", "V_up"))
    return dict(x=(_plain_act(gate, case["act"]) * up).to(kept))


def run(s):
    if not own:
        return _plain(s)
    case, layer = s["case"], s["layer"]
    kind, b, w = case["kind"], case["b"], case.get("w")
    if kind == "gated":
        layer.gated_block(s["e"], s["V_gate"], s["V_up"], w, _act(case["act"]), s["x"], s["gate"], s["up"], b)
        return dict(x=s["x"], gate=s["gate"], up=s["up"])
    if kind == "gated_grad":
        layer.gated_block_backward(s["grad_x"], s["e"], s["V_gate"], s["V_up"], s["gate"], s["up"], w, _act(case["act"]), s["grad_e"], s["grad_V_gate"],
                                   s["grad_V_up"], b)
        return dict(grad_e=s["grad_e"], grad_V_gate=s["grad_V_gate"], grad_V_up=s["grad_V_up"])
    if kind in ("project_i8", "gated_i8"):
        layer.quantize_i8(s["e"], b, w, s["e_codes"], s["e_scales"])
        if kind == "project_i8":
            layer.project_i8(s["e_codes"], s["e_scales"], s["V_codes"], s["V_scales"], w, s["x"], b)
            return dict(h=s["x"])
        layer.gated_block_i8(s["e_codes"], s["e_scales"], s["V_gate_codes"], s["V_gate_scales"], s["V_up_codes"], s["V_up_scales"], w, _act(case["act"]),
                             s["x"], b)
        return dict(x=s["x"])
    if kind == "distill":
        layer.distill_loss_grad(s["out"], s["off"], s["lab"], s["logit"], TEMPERATURE, 1.0 / b, s["g"], s["loss"], b)
        return dict(g=s["g"], loss=s["loss"])
    layer.policy_loss_grad(s["out"], s["off"], s["lab"], s["old_logp"], s["ref_logp"], s["advantage"], CLIP_LOW, CLIP_HIGH, BETA, 1.0 / s["lab"].numel(),
                           s["g"], s["logp"], s["loss"], b)
    return dict(g=s["g"], logp=s["logp"], loss=s["loss"])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind, b, es = case["kind"], case["b"], 2 if case.get("storage") == "bf16" else 4
    if kind in ("distill", "policy"):
        n = sum(_lengths(case))
        return dict(bytes=8 * b * case["m"] + 8 * (b + 1) + n * (8 if kind == "distill" else 20), flops=5 * b * case["m"])
    w, d = case["w"], case["d"]
    if kind == "gated":
        return dict(bytes=es * (b * w + 2 * d * w + 3 * b * d), flops=4 * b * w * d)
    if kind == "gated_grad":
        return dict(bytes=b * d * (4 + 2 * es) + b * w * (4 + es) + d * w * (8 + 2 * es), flops=8 * b * w * d)
    matrices = 1 if kind == "project_i8" else 2
    return dict(bytes=es * b * w + matrices * d * (w + 4) + es * b * d, flops=2 * matrices * b * w * d)


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definitions

def _phi(v):
    """The normal distribution's function."""
    return torch.special.erfc(-v / math.sqrt(2.0)) / 2


def exact(case, seed):
    s = prepare(case, seed)
    kind, b = case["kind"], case["b"]
    if kind in ("gated", "gated_grad"):
        e, V, U = s["e"].double(), s["V_gate"].double(), s["V_up"].double()
        a = torch.matmul(V, e.t()).t() if kind == "gated" else s["gate"].double()
        u = torch.matmul(U, e.t()).t() if kind == "gated" else s["up"].double()
        value = a * torch.sigmoid(a) if case["act"] == "silu" else a * _phi(a)
        if kind == "gated":
            return dict(x=value * u, gate=a, up=u)
        if case["act"] == "silu":   # (a p)' = p + a p (1 - p)
            slope = torch.sigmoid(a) + value * torch.sigmoid(-a)
        else:
            slope = _phi(a) + a * torch.pow(2 * math.pi, torch.tensor(-0.5, dtype=torch.float64, device="cuda")) * torch.exp(-a.square() / 2)
        g = s["grad_x"].double()
        ga, gu = g * u * slope, g * value
        return dict(grad_e=torch.matmul(torch.cat([ga, gu], 1), torch.cat([V, U], 0)), grad_V_gate=torch.matmul(e.t(), ga).t(), grad_V_up=torch.matmul(e.t(), gu).t())
    if kind in ("project_i8", "gated_i8"):
        e = s["e"].double()
        q = torch.empty_like(e)
        scale = torch.empty(b, dtype=torch.float64, device="cuda")
        for i in range(b):   # the scale is a number of 32 bits, and so is the quotient that is rounded to a code
            unit = torch.clamp((e[i].abs().max() / 127).float(), min=2.0 ** -126)
            scale[i] = unit.double()
            q[i] = torch.clamp(torch.round((e[i] / unit.double()).float()), -127, 127).double()

        def product(name):
            return torch.matmul(s[name + "_codes"].double() * s[name + "_scales"].double()[:, None], (q * scale[:, None]).t()).t()

        if kind == "project_i8":
            return dict(h=product("V"))
        a = product("V_gate")
        return dict(x=(a * torch.sigmoid(a) if case["act"] == "silu" else a * _phi(a)) * product("V_up"))
    g = torch.zeros((b, case["m"]), dtype=torch.float64, device="cuda")
    off, loss, logp = s["off"].tolist(), 0.0, []
    for i in range(b):
        here = slice(off[i], off[i + 1])
        at = s["lab"][here].long()
        if at.numel() == 0:
            continue
        log_q = torch.log_softmax(s["out"][i].double() / (TEMPERATURE if kind == "distill" else 1.0), 0)
        if kind == "distill":
            log_p = torch.log_softmax(s["logit"][here].double() / TEMPERATURE, 0)
            g[i] = torch.exp(log_q)
            g[i].index_add_(0, at, -torch.exp(log_p))
            g[i] *= TEMPERATURE / b
            loss += float((torch.exp(log_p) * (log_p - log_q[at])).sum()) * TEMPERATURE ** 2 / b
        else:
            lp, adv = log_q[at], s["advantage"][here].double()
            ratio, gap = torch.exp(lp - s["old_logp"][here].double()), s["ref_logp"][here].double() - lp
            stopped = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
            held = torch.where(stopped, torch.where(adv > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW), ratio)
            loss += float((BETA * (torch.expm1(gap) - gap) - held * adv).sum()) / s["lab"].numel()
            slope = -BETA * torch.expm1(gap) - torch.where(stopped, 0.0, ratio * adv)
            g[i] = -slope.sum() * torch.exp(log_q)
            g[i].index_add_(0, at, slope)
            g[i] /= s["lab"].numel()
            logp.append(lp)
    loss = torch.tensor([loss], dtype=torch.float64, device="cuda")
    return dict(g=g, loss=loss) if kind == "distill" else dict(g=g, logp=torch.cat(logp), loss=loss)
