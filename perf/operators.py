"""Performance cases of the operators that run, serve, score and train on a pruned layer.

A user who has pruned a feed-forward layer runs it (gated feed-forward: its output is the X of the next Gram), trains it on
to recover what was lost (the same with its backward pass), serves the kept rows in 8-bit integers, and measures the model
by the log probabilities it gives to held-out tokens.  Sizes are those of the repository's layers before and after pruning
(2048 x 8192 keeping 4096, 7168 x 28672 keeping 14336, the odd widths 5461 and 1365 of its narrowed layers) and generic
ones; `draw` spreads more over the same ranges.

Fields.  kind "gated": n tokens, d inputs, f neurons, type, act; rows "in" (weights d x f, as the solver holds them) or
"out" (f x d); train: forward and backward, else forward alone.  kind "int": n tokens, d1 inputs, m outputs, type of the
activations and the result, bias.  kind "score": n rows of `vocab` logits, type, top alternatives, masked: columns at the end
that are minus infinity (padding of the vocabulary), train: gradient of log probability and entropy too.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_DEV = "cuda:0"


def _gated(name, **kw):
    return dict({"name": name} if name else {}, kind="gated", **dict(dict(type="bf16", act="silu", rows="in", train=False), **kw))


def _int(name, **kw):
    return dict({"name": name} if name else {}, kind="int", **dict(dict(type="bf16", bias=False), **kw))


def _score(name, **kw):
    return dict({"name": name} if name else {}, kind="score", **dict(dict(type="bf16", top=0, masked=0, train=False), **kw))


def listed():
    return [
        # one token through a layer of 8192 neurons that keeps 4096: the latency of a call counts
        _gated("gated_token", n=1, d=2048, f=4096),
        # a few sequences decoded together, the large layer with half its neurons, weights stored output by output
        _gated("gated_batch", n=16, d=7168, f=14336, rows="out"),
        # a prompt through a layer narrowed to an odd width
        _gated("gated_prompt_odd", n=777, d=2048, f=5461, rows="out", act="gelu"),
        # calibration segments through a whole layer: the activations that the Gram of the down projection takes
        _gated("gated_calibration", n=16384, d=2048, f=8192),
        # a training step on the large layer after pruning
        _gated("gated_train", n=4096, d=7168, f=14336, train=True),
        # the same in float32 on a small odd layer
        _gated("gated_train_odd_f32", n=2048, d=1365, f=3001, type="f32", act="gelu_tanh", train=True),
        # one token through the kept rows of the large down projection
        _int("int_token", n=1, d1=14336, m=7168),
        # a few sequences decoded together, narrowed widths, float32 in and out
        _int("int_batch_odd", n=24, d1=5461, m=1365, type="f32", bias=True),
        # a long prompt through the large down projection
        _int("int_prompt", n=8192, d1=14336, m=7168),
        # tokens being decoded: probability of the drawn token and its alternatives
        _score("score_decode", n=4, vocab=131072, type="f32", top=8),
        # held-out text: perplexity, entropy and alternatives; the vocabulary is padded
        _score("score_held_out", n=4096, vocab=50304, top=5, masked=47),
        # the loss of a training step with an entropy term
        _score("score_train", n=8192, vocab=32000, train=True),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], even over its logarithm, every third rounded to a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(64, v // 64 * 64) if v >= 64 and rng.random() < 1 / 3 else v


def _draw(rng):
    kind = rng.choice(("gated", "gated", "gated", "int", "int", "score", "score"))
    if kind == "gated":
        return _gated(None, n=_spread(rng, 1, 16384), d=_spread(rng, 256, 7168), f=_spread(rng, 256, 14336), type=rng.choice(("bf16", "bf16", "f32")),
                      act=rng.choice(("silu", "gelu", "gelu_tanh", "relu")), rows=rng.choice(("in", "out")), train=rng.random() < 0.4)
    if kind == "int":
        return _int(None, n=_spread(rng, 1, 8192), d1=_spread(rng, 256, 14336), m=_spread(rng, 256, 7168), type=rng.choice(("bf16", "bf16", "f32")),
                    bias=rng.random() < 0.5)
    train = rng.random() < 0.5
    return _score(None, n=_spread(rng, 1, 8192), vocab=_spread(rng, 4096, 131072), type=rng.choice(("bf16", "f32")), top=0 if train else rng.randrange(0, 21),
                  masked=rng.choice((0, 0, rng.randrange(1, 1000))), train=train)


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for key in w:
            most[c["kind"], key] = max(most.get((c["kind"], key), 0), w[key])
    while True:
        c = _draw(rng)
        w = work(c)
        slow = 4 if c["kind"] == "gated" and c["type"] == "f32" else 1      # float32 costs about that much more
        if all(slow * w[key] <= most[c["kind"], key] for key in w):
            return c


def work(case):
    b = _BYTES[case["type"]]
    n = case["n"]
    if case["kind"] == "gated":
        d, f = case["d"], case["f"]
        moved, flops = b * (n * d + 2 * d * f + n * f), 4 * n * d * f
        if case["train"]:      # the gradient of h in, those of X and of both weights out
            moved, flops = moved + b * (n * f + n * d + 2 * d * f), 3 * flops
        return {"bytes": moved, "flops": flops}
    if case["kind"] == "int":
        d1, m = case["d1"], case["m"]
        return {"bytes": b * n * (d1 + m) + m * d1 + 4 * m * (2 if case["bias"] else 1), "flops": 2 * n * d1 * m}
    v = case["vocab"]
    moved, flops = b * n * v + n * (8 + 12 + 12 * case["top"]), 6 * n * v
    if case["train"]:
        moved, flops = 2 * moved, 2 * flops
    return {"bytes": moved, "flops": flops}


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=_DEV)

    dt, n = _DT[case["type"]], case["n"]
    state = dict(case=case)
    if case["kind"] == "gated":
        d, f = case["d"], case["f"]
        scale = torch.exp(0.5 * normal(d))      # hidden states: channels of uneven size
        state["X"] = (normal(n, d) * scale).to(dt)
        for name in ("Wg", "Wu"):
            state[name] = (normal(d, f) if case["rows"] == "in" else normal(f, d)).mul_(1.2 / math.sqrt(d)).to(dt)
            if case["rows"] == "out":
                state[name] = state[name].t()      # d x f, each neuron's weights side by side
        if case["train"]:
            state["dH"] = normal(n, f).mul_(1e-3).to(dt)
    elif case["kind"] == "int":
        d1, m = case["d1"], case["m"]
        scale = torch.exp(normal(d1))      # products of activations: uneven neurons, as the layers to be pruned have them
        state["X"] = (normal(n, d1) * scale).to(dt)
        w = normal(m, d1).mul_(0.02)
        state["w_scale"] = w.abs().amax(1) / 127
        state["Wq"] = torch.zeros(m, -(-d1 // 16) * 16, dtype=torch.int8, device=_DEV)      # rows of whole 16 bytes
        state["Wq"][:, :d1] = torch.round(w / state["w_scale"][:, None]).to(torch.int8)
        state["bias"] = normal(m) if case["bias"] else None
    else:
        v = case["vocab"]
        state["logits"] = normal(n, v).mul_(2.5).to(dt)
        if case["masked"]:
            state["logits"][:, v - case["masked"]:] = -math.inf
        t = torch.randint(0, v - case["masked"], (n,), generator=gen, device=_DEV)
        state["logits"][torch.arange(n, device=_DEV), t] += 6.0      # a model that has learned something
        skip = torch.rand(n, generator=gen, device=_DEV) < 0.1      # tokens of the prompt, which count for nothing
        state["targets"] = torch.where(skip & (n > 1), torch.full_like(t, -1), t)
        if case["train"]:
            state["dlogp"] = torch.full((n,), -1.0 / n, device=_DEV)
            state["dentropy"] = torch.full((n,), -0.01 / n, device=_DEV)
    return state


# --------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    form = {"gated": (_gated_plain, _gated_own), "int": (_int_plain, _int_own), "score": (_score_plain, _score_own)}[case["kind"]]
    return form[1 if own else 0](state, case)


def _gated_own(state, case):
    import paper_2403_12983_amd as osscar
    act = {"silu": osscar.OSSCAR_ACT_SILU, "gelu": osscar.OSSCAR_ACT_GELU, "gelu_tanh": osscar.OSSCAR_ACT_GELU_TANH, "relu": osscar.OSSCAR_ACT_RELU}[case["act"]]
    X, Wg, Wu = state["X"], state["Wg"], state["Wu"]
    if not case["train"]:
        return {"H": osscar.osscar_gated_forward(X, Wg, Wu, act)}
    H, G, U = osscar.osscar_gated_forward(X, Wg, Wu, act, save=True)
    dX, dWg, dWu = osscar.osscar_gated_backward(X, Wg, Wu, state["dH"], act, G=G, U=U)
    return {"H": H, "dX": dX, "dWg": dWg, "dWu": dWu}


def _int_own(state, case):
    import paper_2403_12983_amd as osscar
    return {"Y": osscar.osscar_int_product(state["X"], state["Wq"], state["w_scale"], bias=state["bias"], out_dtype=_DT[case["type"]])}


def _score_own(state, case):
    import paper_2403_12983_amd as osscar
    logits, targets = state["logits"], state["targets"]
    got = osscar.osscar_logprobs(logits, targets, top=case["top"])
    out = {"logp": got.logp, "entropy": got.entropy}
    if case["top"]:
        out.update(top_index=got.top_index, top_logp=got.top_logp)
    if case["train"]:
        out["dlogits"] = osscar.osscar_logprobs_backward(logits, targets, got.lse, state["dlogp"], entropy=got.entropy, dentropy=state["dentropy"])
    return out


_SQRT_HALF, _TANH_C = math.sqrt(0.5), math.sqrt(2 / math.pi)


def _act(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    if act == "gelu":
        return 0.5 * g * (1 + torch.erf(g * _SQRT_HALF))
    if act == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(_TANH_C * (g + 0.044715 * g * g * g)))
    return torch.clamp_min(g, 0)


def _act_slope(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return s * (1 + g * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(g * _SQRT_HALF)) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_TANH_C * (g + 0.044715 * g * g * g))
        return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * _TANH_C * (1 + 3 * 0.044715 * g * g)
    return (g > 0).to(g.dtype)


def _gated_plain(state, case):
    dt, act = _DT[case["type"]], case["act"]
    X, Wg, Wu = state["X"].float(), state["Wg"].float(), state["Wu"].float()
    g, u = X @ Wg, X @ Wu
    a = _act(g, act)
    out = {"H": (a * u).to(dt)}
    if case["train"]:
        dH = state["dH"].float()
        du = dH * a
        dg = dH * u * _act_slope(g, act)
        out.update(dX=(dg @ Wg.t() + du @ Wu.t()).to(dt), dWg=(X.t() @ dg).to(dt), dWu=(X.t() @ du).to(dt))
        if case["rows"] == "out":
            out.update(dWg=out["dWg"].t().contiguous().t(), dWu=out["dWu"].t().contiguous().t())
    return out


def _int_plain(state, case):
    x = state["X"].float()
    s = x.abs().amax(1, keepdim=True) / 127
    q = torch.clamp(torch.round(x / s), -127, 127)
    q = torch.where(s > 0, q, torch.zeros_like(q))
    y = (q @ state["Wq"][:, :case["d1"]].float().t()) * s * state["w_scale"]
    return {"Y": (y + state["bias"] if case["bias"] else y).to(_DT[case["type"]])}


def _top(z, k):
    """The k largest of each row and where they are; of equal ones the first."""
    bits = (z + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64) << 32      # ordered as the numbers are
    key = key | (0xFFFFFFFF - torch.arange(z.shape[1], device=z.device))
    return 0xFFFFFFFF - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)


def _score_plain(state, case):
    z, t = state["logits"].float(), state["targets"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    S = e.sum(1, keepdim=True)
    log_S = torch.log(S)
    lse = m + log_S
    entropy = log_S + torch.where(e > 0, (m - z) * e, torch.zeros_like(e)).sum(1, keepdim=True) / S
    given = t.clamp_min(0)[:, None]
    counts = (t >= 0)[:, None]
    logp = torch.where(counts, torch.gather(z, 1, given) - lse, torch.zeros_like(lse))
    out = {"logp": logp[:, 0], "entropy": entropy[:, 0]}
    if case["top"]:
        index = _top(z, case["top"])
        out.update(top_index=index, top_logp=torch.gather(z, 1, index) - lse)
    if case["train"]:
        p = e / S
        dlogp = torch.where(counts, state["dlogp"][:, None], torch.zeros_like(lse))
        dz = -p * (dlogp + state["dentropy"][:, None] * torch.where(p > 0, z - lse + entropy, torch.zeros_like(p)))
        out["dlogits"] = dz.scatter_add(1, given, dlogp).to(_DT[case["type"]])
    return out


# --------------------------------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _gated_exact, "int": _int_exact, "score": _score_exact}[case["kind"]](s, case)


def _gated_exact(s, case):
    X, Wg, Wu = s["X"].double(), s["Wg"].double().contiguous(), s["Wu"].double().contiguous()
    g, u = torch.matmul(X, Wg), torch.matmul(X, Wu)
    if case["act"] == "silu":
        sig = 1 / (1 + torch.exp(-g))
        a, slope = g * sig, sig + g * sig * (1 - sig)
    elif case["act"] == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        a, slope = g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    elif case["act"] == "gelu_tanh":
        w = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)      # (1 + tanh(w / 2)) / 2 is the logistic function of w
        sig = 1 / (1 + torch.exp(-w))
        a, slope = g * sig, sig + g * sig * (1 - sig) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)
    else:
        slope = (g > 0).double()
        a = g * slope
    out = {"H": a * u}
    if case["train"]:
        dH = s["dH"].double()
        dg, du = dH * u * slope, dH * a
        out["dX"] = torch.matmul(dg, Wg.t().contiguous()) + torch.matmul(du, Wu.t().contiguous())
        Xt = X.t().contiguous()
        out["dWg"], out["dWu"] = torch.matmul(Xt, dg), torch.matmul(Xt, du)
    return out


def _int_exact(s, case):
    x = s["X"].double()
    scale = x.abs().max(dim=1).values / 127
    unit = torch.where(scale > 0, scale, torch.ones_like(scale))
    q = torch.round(x / unit[:, None])
    w = s["Wq"][:, :case["d1"]].double() * s["w_scale"].double()[:, None]
    y = torch.matmul(q * scale[:, None], w.t().contiguous())
    return {"Y": y + s["bias"].double() if case["bias"] else y}


def _score_exact(s, case):
    n, t = case["n"], s["targets"]
    parts = []
    for rows in torch.arange(n, device=_DEV).split(1024):
        z = s["logits"][rows].double()
        lp = torch.log_softmax(z, 1)
        p = torch.exp(lp)
        plogp = torch.where(p > 0, p * lp, torch.zeros_like(p))
        entropy = -plogp.sum(1)
        given = t[rows]
        ok = given >= 0
        at = (torch.arange(len(rows), device=_DEV)[ok], given[ok])
        logp = torch.zeros(len(rows), dtype=torch.float64, device=_DEV)
        logp[ok] = lp[at]
        out = {"logp": logp, "entropy": entropy}
        if case["top"]:
            order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out.update(top_index=order, top_logp=torch.gather(lp, 1, order))
        if case["train"]:
            dlogp = torch.where(ok, s["dlogp"][rows].double(), torch.zeros(len(rows), dtype=torch.float64, device=_DEV))
            hot = torch.zeros_like(z)
            hot[at] = 1.0
            out["dlogits"] = dlogp[:, None] * (hot - p) - s["dentropy"][rows].double()[:, None] * (plogp + p * entropy[:, None])
        parts.append(out)
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
