"""The operators around the experts of a block, as cases that can be timed: the scored router, the norms before and after
a block with the block's gate and residual, and the projections beside the layer (bias, activation and residual in the product).

`run` computes a case in its plain form (elementary torch operations) or, where `own` is true, through this framework's calls.
Widths are those of workloads/synth.py (256, 896, 1536 and 2048 wide tokens, FFN widths 4864, 8960 and 11008, outlier channels
of the long prompts) or generic.
"""
import math

import torch

own = False

MAX_TOKENS = 8192
LARGEST_LINEAR = 4096 * 2048 * 11008          # multiply-adds of the largest product
LARGEST_NORM = 8192 * 2048                    # elements of the largest norm
WIDTHS = [256, 896, 1536, 2048]


def _route(name, T, d, E, k, *, scoring="softmax", groups=1, topk_groups=1, select_bias=False, logit_bias=False, renorm=True,
           scale=1.0, w="float32", logits=False, outliers=False):
    return dict(name=name, op="route", T=T, d=d, E=E, k=k, scoring=scoring, groups=groups, topk_groups=topk_groups,
                select_bias=select_bias, logit_bias=logit_bias, renorm=renorm, scale=scale, w=w, logits=logits, outliers=outliers)


def _norm(name, T, d, *, post=False, post_gain=False, pre_gain=True, gate="none", gate_tokens=1, gate_dtype="bfloat16",
          sigmoid=False, residual="bfloat16", scale=1.0):
    return dict(name=name, op="norm", T=T, d=d, post=post, post_gain=post_gain, pre_gain=pre_gain, gate=gate,
                gate_tokens=gate_tokens, gate_dtype=gate_dtype, sigmoid=sigmoid, residual=residual, scale=scale)


def _linear(name, T, K, N, *, bits=16, bias=False, act="none", residual=False, out="bfloat16"):
    return dict(name=name, op="linear", T=T, K=K, N=N, bits=bits, bias=bias, act=act, residual=residual, out=out)


def listed():
    return [
        # one user's decode step: one token to two of 16 experts
        _route("route-1", 1, 2048, 16, 2),
        # a small decode batch, 64 experts in 8 groups of which four may be used, a bias that balances them
        _route("route-37-groups", 37, 1536, 64, 6, scoring="sigmoid", groups=8, topk_groups=4, select_bias=True, scale=2.5, w="bfloat16"),
        # a prompt of odd length with outlier channels; probabilities over all experts as weights, logits kept for the balance loss
        _route("route-1003-softmax", 1003, 896, 60, 4, logit_bias=True, renorm=False, logits=True, outliers=True),
        # a long batched prompt
        _route("route-8192-groups", 8192, 2048, 64, 8, scoring="sigmoid", groups=8, topk_groups=4, select_bias=True, scale=2.5),
        # one user's decode step: the block's output joins the residual stream, the next block's input is its norm
        _norm("norm-1", 1, 2048),
        # a prompt of odd length: norms on both sides of a block, a gate for each token, residual stream in 32 bits
        _norm("norm-333-sandwich", 333, 1536, post=True, post_gain=True, gate="token", sigmoid=True, residual="float32"),
        # one gate row for every sequence of 512 tokens (conditioned blocks), scaled
        _norm("norm-2047-sequences", 2047, 896, gate="channel", gate_tokens=512, gate_dtype="float32", scale=0.5),
        # a long batched prompt, norms on both sides and a gain for each channel of the block's output
        _norm("norm-8192-sandwich", 8192, 2048, post=True, post_gain=True, gate="channel", gate_tokens=0),
        # one user's decode step: queries, keys and values of one token, with their bias
        _linear("linear-1-qkv", 1, 2048, 2560, bias=True),
        # a small decode batch through a wide projection held as INT8 codes, onto the residual stream
        _linear("linear-8-int8", 8, 11008, 2048, bits=8, residual=True),
        # a prompt of odd length through the first half of a connector (GELU)
        _linear("linear-333-gelu", 333, 1536, 8960, bias=True, act="gelu"),
        # a long batched prompt through the widest projection
        _linear("linear-4096", 4096, 2048, 11008, bias=True, act="silu"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "norm", "linear"])
    T = _log_int(rng, 1, MAX_TOKENS)
    if op == "route":
        d = rng.choice(WIDTHS) if rng.random() < 0.5 else 8 * rng.randint(8, 256)
        groups = rng.choice([1, 1, 2, 4, 8])
        E = rng.randint(2, 64) if groups == 1 else groups * rng.randint(2, 64 // groups)
        topk_groups = rng.randint(1, groups)
        k = rng.randint(1, min(8, topk_groups * (E // groups)))
        c = _route("", T, d, E, k, scoring=rng.choice(["softmax", "sigmoid"]), groups=groups, topk_groups=topk_groups,
                   select_bias=rng.choice([True, False]), logit_bias=rng.choice([True, False]), renorm=rng.choice([True, False]),
                   scale=rng.choice([1.0, 2.5]), w=rng.choice(["float32", "bfloat16"]), logits=rng.choice([True, False]),
                   outliers=rng.choice([True, False]))
    elif op == "norm":
        d = rng.choice(WIDTHS) if rng.random() < 0.5 else 8 * _log_int(rng, 8, 1024)
        T = min(T, LARGEST_NORM // d)
        post = rng.choice([True, False])
        gate = rng.choice(["none", "token", "channel", "full"])
        c = _norm("", T, d, post=post, post_gain=post and rng.choice([True, False]), pre_gain=rng.choice([True, False]), gate=gate,
                  gate_tokens=rng.choice([0, _log_int(rng, 2, 4096)]) if gate == "channel" else 1,
                  gate_dtype=rng.choice(["bfloat16", "float32"]), sigmoid=rng.choice([True, False]),
                  residual=rng.choice(["bfloat16", "float32"]), scale=rng.choice([1.0, 0.5]))
    else:
        K = rng.choice(WIDTHS) if rng.random() < 0.5 else 16 * _log_int(rng, 8, 688)
        N = rng.choice([256, 896, 1536, 2048, 2560, 4864, 8960, 11008]) if rng.random() < 0.5 else _log_int(rng, 16, 11008)
        T = max(1, min(T, LARGEST_LINEAR // (K * N)))
        c = _linear("", T, K, N, bits=rng.choice([16, 16, 8, 4]), bias=rng.choice([True, False]),
                    act=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), residual=rng.choice([True, False]),
                    out=rng.choice(["bfloat16", "float32"]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _randn(seed, tag, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1009 + tag) & (2 ** 62 - 1))
    return torch.randn(shape, generator=g, device="cuda")


def _randint(seed, tag, lo, hi, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1009 + tag) & (2 ** 62 - 1))
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int8)


def _pack4(q):
    """4-bit codes as mote_rtn_quant stores them: eight elements of a row in a 32-bit word, element 2p in nibble p and
    element 2p + 1 in nibble 4 + p, each as code + 8."""
    n, m = q.shape
    u = (q + 8).to(torch.uint8).view(n, m // 8, 4, 2).permute(0, 1, 3, 2).reshape(n, m // 2, 2)
    return (u[..., 0] | (u[..., 1] << 4)).contiguous()


def _inputs(c, seed):
    """What the user's program has in hand, made from the seed alone."""
    if c["op"] == "route":
        x = _randn(seed, 1, c["T"], c["d"])
        if c["outliers"]:                                   # 1 % of the channels, twenty times as large
            n = max(1, round(0.01 * c["d"]))
            x[:, _randn(seed, 2, c["d"]).argsort()[:n]] *= 20.0
        return dict(x=x.bfloat16(), Wr=(_randn(seed, 3, c["E"], c["d"]) * 0.02).to(getattr(torch, c["w"])),
                    logit_bias=_randn(seed, 4, c["E"]) * 0.5 if c["logit_bias"] else None,
                    select_bias=_randn(seed, 5, c["E"]) * 0.02 if c["select_bias"] else None)
    if c["op"] == "norm":
        T, d = c["T"], c["d"]
        rows = 1 if c["gate_tokens"] == 0 else -(-T // c["gate_tokens"])
        shape = {"none": None, "token": (T, 1), "channel": (rows, d), "full": (T, d)}[c["gate"]]
        return dict(y=(_randn(seed, 1, T, d) * 0.7).bfloat16(), residual=(_randn(seed, 2, T, d) * 4.0).to(getattr(torch, c["residual"])),
                    post_gain=1.0 + 0.1 * _randn(seed, 3, d) if c["post_gain"] else None,
                    pre_gain=1.0 + 0.1 * _randn(seed, 4, d) if c["pre_gain"] else None,
                    gate=_randn(seed, 5, *shape).to(getattr(torch, c["gate_dtype"])) if shape else None)
    T, K, N = c["T"], c["K"], c["N"]
    s = dict(x=_randn(seed, 1, T, K).bfloat16(), bias=_randn(seed, 3, N) * 0.5 if c["bias"] else None,
             residual=(_randn(seed, 4, T, N) * 2.0).bfloat16() if c["residual"] else None, scale=None)
    if c["bits"] == 16:
        s["W"] = (_randn(seed, 2, N, K) * 0.02).bfloat16()
    else:                                                    # round-to-nearest codes and a scale for each row
        top = 127 if c["bits"] == 8 else 7
        s["codes"] = _randint(seed, 2, -top, top, N, K)
        s["W"] = s["codes"] if c["bits"] == 8 else _pack4(s["codes"])
        s["scale"] = (0.06 + 0.02 * torch.rand(N, generator=torch.Generator("cuda").manual_seed(seed + 7), device="cuda")) / top
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:                                                  # the weights as a program holds them between calls
        import paper_2506_14435_b200 as mote
        s["mote"] = mote
        if case["op"] == "route":
            s["op"] = mote.MoteRouter(s["Wr"], case["k"], scoring=case["scoring"], logit_bias=s["logit_bias"],
                                      select_bias=s["select_bias"], n_groups=case["groups"], topk_groups=case["topk_groups"],
                                      renorm=case["renorm"], scale=case["scale"])
        elif case["op"] == "norm":
            s["op"] = mote.MoteBlockNorm(case["d"], post_norm=case["post"], post_gain=s["post_gain"], pre_gain=s["pre_gain"],
                                         scale=case["scale"], gate_sigmoid=case["sigmoid"], gate_tokens=case["gate_tokens"])
        else:
            s["op"] = mote.MoteLinear(s["W"], bits=case["bits"], scale=s["scale"], bias=s["bias"], act=case["act"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if own:
        mote = state["mote"]
        if c["op"] == "route":
            idx, w, logits = mote.mote_route_scored(state["op"], state["x"], want_logits=c["logits"])
            return [idx, w, logits] if c["logits"] else [idx, w]
        if c["op"] == "norm":
            return list(mote.mote_block_norm(state["op"], state["y"], state["residual"], gate=state["gate"]))
        return mote.mote_linear(state["op"], state["x"], residual=state["residual"], out_dtype=getattr(torch, c["out"]))
    return {"route": _plain_route, "norm": _plain_norm, "linear": _plain_linear}[c["op"]](c, state)


def _plain_route(c, s):
    # in 64 bits: which of two close scores is larger must not depend on the order of a sum
    T, E, G, k = c["T"], c["E"], c["groups"], c["k"]
    logits = s["x"].double() @ s["Wr"].double().t()
    if s["logit_bias"] is not None:
        logits = logits + s["logit_bias"].double()
    if c["scoring"] == "softmax":
        e = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
        score = e / e.sum(dim=1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    choice = score if s["select_bias"] is None else score + s["select_bias"].double()
    if G > 1:
        by_group = choice.view(T, G, E // G).sort(dim=2, descending=True, stable=True).values[:, :, :2].sum(dim=2)
        order = by_group.sort(dim=1, descending=True, stable=True).indices
        kept = torch.zeros(T, G, dtype=torch.bool, device=choice.device).scatter_(1, order[:, :c["topk_groups"]], True)
        choice = choice.masked_fill(~kept.repeat_interleave(E // G, dim=1), -math.inf)
    idx = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(dim=1, keepdim=True).clamp_min(1e-20)
    out = [idx.to(torch.int32), (w * c["scale"]).float()]
    return out + [logits.float()] if c["logits"] else out


def _rms(v, eps=1e-6):
    return v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + eps)


def _plain_norm(c, s):
    v = s["y"].float()
    if c["post"]:
        v = _rms(v)
        if s["post_gain"] is not None:
            v = v * s["post_gain"]
    if s["gate"] is not None:
        g = s["gate"].float()
        if c["sigmoid"]:
            g = 1.0 / (1.0 + torch.exp(-g))
        if c["gate"] == "channel":
            g = g[:1] if c["gate_tokens"] == 0 else g[torch.arange(c["T"], device=g.device) // c["gate_tokens"]]
        v = v * g
    res = (s["residual"].float() + c["scale"] * v).to(s["residual"].dtype)
    n = _rms(res.float())
    if s["pre_gain"] is not None:
        n = n * s["pre_gain"]
    return [res, n.bfloat16()]


def _plain_linear(c, s):
    w = s["W"].float() if c["bits"] == 16 else s["codes"].float()
    z = s["x"].float() @ w.t()
    if s["scale"] is not None:
        z = z * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    if c["act"] == "relu":
        z = z.clamp_min(0.0)
    elif c["act"] == "silu":
        z = z / (1.0 + torch.exp(-z))
    elif c["act"] == "gelu":
        z = 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    elif c["act"] == "gelu_tanh":
        z = 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if s["residual"] is not None:
        z = z + s["residual"].float()
    return z.to(getattr(torch, c["out"]))


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "route":
        # ranks instead of sorts: an expert is taken if fewer than k of the eligible ones come before it
        z = torch.einsum("td,ed->te", s["x"].double(), s["Wr"].double())
        z = z if s["logit_bias"] is None else z + s["logit_bias"].double()[None]
        p = torch.softmax(z, dim=1) if c["scoring"] == "softmax" else torch.sigmoid(z)
        v = p if s["select_bias"] is None else p + s["select_bias"].double()[None]
        if c["groups"] > 1:
            per = c["E"] // c["groups"]
            best = v.unflatten(1, (c["groups"], per)).topk(2, dim=2).values.sum(dim=2)
            least = best.topk(c["topk_groups"], dim=1).values[:, -1:]
            v = torch.where((best >= least).repeat_interleave(per, dim=1), v, torch.full_like(v, -math.inf))
        w = p.gather(1, v.topk(c["k"], dim=1).indices)
        w = c["scale"] * (w / w.sum(dim=1, keepdim=True) if c["renorm"] else w)
        return [None, w, z] if c["logits"] else [None, w]
    if c["op"] == "norm":
        y, r = s["y"].double(), s["residual"].double()
        if c["post"]:
            y = y / torch.sqrt(y.pow(2).sum(1, keepdim=True) / c["d"] + 1e-6)
            y = y if s["post_gain"] is None else torch.einsum("td,d->td", y, s["post_gain"].double())
        if s["gate"] is not None:
            g = torch.sigmoid(s["gate"].double()) if c["sigmoid"] else s["gate"].double()
            if c["gate"] == "channel" and c["gate_tokens"]:
                g = g.repeat_interleave(c["gate_tokens"], dim=0)[:c["T"]]
            y = y * g
        r = r + y * c["scale"]
        n = r / torch.sqrt(r.pow(2).sum(1, keepdim=True) / c["d"] + 1e-6)
        return [r, n if s["pre_gain"] is None else n * s["pre_gain"].double()]
    w = s["W"].double() if c["bits"] == 16 else torch.einsum("nk,n->nk", s["codes"].double(), s["scale"].double())
    z = torch.nn.functional.linear(s["x"].double(), w, None if s["bias"] is None else s["bias"].double())
    f = torch.nn.functional
    z = {"none": lambda v: v, "relu": f.relu, "silu": f.silu, "gelu": f.gelu,
         "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[c["act"]](z)
    return z if s["residual"] is None else z + s["residual"].double()


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "route":
        T, d, E = c["T"], c["d"], c["E"]
        return dict(bytes=2.0 * T * d + (4 if c["w"] == "float32" else 2) * E * d + 8.0 * T * c["k"] + (4.0 * T * E if c["logits"] else 0.0),
                    flops=2.0 * T * d * E)
    if c["op"] == "norm":
        n = float(c["T"]) * c["d"]
        r = 4 if c["residual"] == "float32" else 2
        rows = 1 if c["gate_tokens"] == 0 else -(-c["T"] // c["gate_tokens"])
        gate = {"none": 0, "token": c["T"], "channel": rows * c["d"], "full": n}[c["gate"]] * (4 if c["gate_dtype"] == "float32" else 2)
        return dict(bytes=n * (2 + r + r + 2) + gate + 4.0 * c["d"] * (c["post_gain"] + c["pre_gain"]), flops=0.0)
    T, K, N = float(c["T"]), c["K"], c["N"]
    return dict(bytes=2.0 * T * K + N * K * c["bits"] / 8.0 + T * N * ((4 if c["out"] == "float32" else 2) + (2 if c["residual"] else 0)),
                flops=2.0 * T * K * N)
