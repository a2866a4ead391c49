"""Cases, plain forms and framework calls of the operators around an expert layer: the residual-adding RMS norm
with an 8-bit output and its gradient, the router and its gradient, the gated activation with an 8-bit output, and
the 8-bit integer matrix product with a scale per token and per channel, dense and per expert.

`own` chooses what `run` does: False, the plain form in elementary torch operations on 32-bit values; True, the
framework's operators.  Values held in 8 bits are returned as the values they stand for, in bf16."""
import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
TINY = 2.0 ** -100      # rows whose largest magnitude is below this quantise to zeros


def listed():
    return [
        # the hidden state of one generated token on its way into an 8-bit product: latency counts
        {"name": "norm_one_token", "op": "norm", "rows": 1, "d": 4096, "dtype": "bf16", "out": "int8", "residual": True, "pad": 0},
        # a long prompt's (or a large batch's) hidden states
        {"name": "norm_prompt", "op": "norm", "rows": 16384, "d": 4096, "dtype": "bf16", "out": "int8", "residual": True, "pad": 0},
        # a training micro-batch with a ragged number of tokens
        {"name": "norm_gradient", "op": "norm_backward", "rows": 12289, "d": 2048, "dtype": "bf16", "residual": True, "pad": 0},
        # a decode batch over many experts, chosen within groups with a balancing bias
        {"name": "route_decode", "op": "route", "rows": 48, "experts": 256, "k": 8, "dtype": "f32", "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "group_best": 2, "renormalise": True},
        # eight ranks' tokens of a fine-grained layer, a ragged number of them
        {"name": "route_layer", "op": "route", "rows": 65521, "experts": 64, "k": 6, "dtype": "bf16", "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "group_best": 1, "renormalise": True},
        # the same layer's step back to the router's logits
        {"name": "route_gradient", "op": "route_backward", "rows": 65521, "experts": 64, "k": 6, "dtype": "bf16", "score": "softmax", "renormalise": False},
        # one generated token through a wide gate and up projection: the weights are streamed once
        {"name": "matmul_one_token", "op": "matmul", "rows": 1, "k": 4096, "n": 28672, "experts": 0, "dtype": "bf16", "pad": 0},
        # a prompt of odd length through the same projection: the largest product
        {"name": "matmul_prompt", "op": "matmul", "rows": 7919, "k": 4096, "n": 28672, "experts": 0, "dtype": "bf16", "pad": 0},
        # a decode batch spread over many experts, a handful of rows each, some with none
        {"name": "experts_decode", "op": "matmul", "rows": 96, "k": 2048, "n": 8192, "experts": 16, "dtype": "bf16", "pad": 0},
        # the rows of a fine-grained layer's local experts, ragged counts
        {"name": "experts_layer", "op": "matmul", "rows": 49152, "k": 2048, "n": 2816, "experts": 8, "dtype": "bf16", "pad": 0},
        # the gated activation between an expert's two products: a decode batch and a prompt
        {"name": "swiglu_decode", "op": "swiglu", "rows": 37, "f": 1408, "dtype": "bf16", "pad": 0},
        {"name": "swiglu_prompt", "op": "swiglu", "rows": 8192, "f": 14336, "dtype": "bf16", "pad": 0},
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, even in its logarithm."""
    while True:
        v = int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
        if v != 3072:
            return min(max(v, lo), hi)


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "route", "route_backward", "matmul", "matmul", "swiglu"])
    if op in ("norm", "norm_backward"):
        d = _between(rng, 64, 8192)
        if rng.random() < 0.7:
            d = (d + 7) // 8 * 8 if (d + 7) // 8 * 8 != 3072 else 3080
        c = {"op": op, "rows": _between(rng, 1, max(1, (16384 if op == "norm" else 8192) * 4096 // max(d, 4096))), "d": d,
             "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "residual": rng.random() < 0.8, "pad": rng.choice([0, 0, 0, 8])}
        if op == "norm":
            c["out"] = rng.choice(["int8", "same"])
        return c
    if op in ("route", "route_backward"):
        score = rng.choice(["softmax", "sigmoid"])
        groups = rng.choice([1, 1, 4, 8])
        e = _between(rng, 8, 384) if groups == 1 else groups * rng.randint(2, 48)
        c = {"op": op, "rows": _between(rng, 1, 65521 * 64 // max(e, 64)), "experts": e, "k": rng.randint(1, min(8, e // groups)),
             "dtype": rng.choice(["bf16", "f32"]), "score": score, "renormalise": rng.random() < 0.6}
        if op == "route":
            c.update(bias=score == "sigmoid" and rng.random() < 0.6, groups=groups, top_groups=rng.randint(1, groups))
            c["group_best"] = 2 if c["bias"] and groups > 1 else 1
        return c
    if op == "swiglu":
        f = _between(rng, 64, 14336)
        if rng.random() < 0.7:
            f = (f + 7) // 8 * 8 if (f + 7) // 8 * 8 != 3072 else 3080
        return {"op": op, "rows": _between(rng, 1, 8192), "f": f, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "pad": rng.choice([0, 0, 8])}
    experts = rng.choice([0, 0, 0, 4, 8, 16, 32, 64])
    k = 16 * (_between(rng, 128, 8192) // 16)
    k = k if k != 3072 else 3088
    n = _between(rng, 64, 16384 if experts < 16 else 4096)
    rows = _between(rng, 1, 8192)
    return {"op": op, "rows": rows, "k": k, "n": n, "experts": experts, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "pad": rng.choice([0, 0, 0, 16])}


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, pad=0, scale=1.0):
    """Normal values; with pad, a view of rows that lie further apart than they are long."""
    full = torch.randn((*shape[:-1], shape[-1] + pad), generator=g, device="cuda", dtype=torch.float32)
    return full.mul_(scale).to(dtype)[..., :shape[-1]]


def _bytes8(g, shape, spread, pad=0):
    full = torch.empty((*shape[:-1], shape[-1] + pad), dtype=torch.int8, device="cuda")
    flat = full.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        part = flat[lo:lo + (1 << 26)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda").mul_(spread).round_().clamp_(-127, 127))
    return full[..., :shape[-1]]


def prepare(case, seed):
    g, op, s = _generator(seed), case["op"], dict(case)
    dev, dt = "cuda", DTYPES[case["dtype"]]
    if op in ("norm", "norm_backward"):
        t, d = case["rows"], case["d"]
        s["weight"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=dev)).to(dt)
        # hidden states: a few channels much larger than the others
        channel = torch.exp(0.5 * torch.randn(d, generator=g, device=dev))
        s["x"] = _normal(g, (t, d), dt, case["pad"])
        s["residual_in"] = (_normal(g, (t, d), torch.float32) * channel).to(dt) if case["residual"] else None
        if op == "norm":
            s["residual_out"] = torch.empty((t, d), dtype=dt, device=dev) if case["residual"] else None
            s["rstd"] = torch.empty(t, device=dev)
            if case["out"] == "int8":
                s.update(q=torch.empty((t, d), dtype=torch.int8, device=dev), scale=torch.empty(t, device=dev), values=torch.empty((t, d), dtype=torch.bfloat16, device=dev))
            else:
                s["y"] = torch.empty((t, d), dtype=dt, device=dev)
        else:
            s["dy"] = _normal(g, (t, d), dt, case["pad"])
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS)
            s["dx"], s["dweight"] = torch.empty((t, d), dtype=dt, device=dev), torch.empty(d, device=dev)
            s["workspace"] = torch.empty(8 << 20, dtype=torch.float32, device=dev)
    elif op in ("route", "route_backward"):
        t, e, k = case["rows"], case["experts"], case["k"]
        popular = 0.5 * torch.randn(e, generator=g, device=dev)
        s["logits"] = (torch.randn((t, e), generator=g, device=dev) + popular).to(dt)
        if op == "route":
            s["bias_values"] = torch.round(100 * torch.randn(e, generator=g, device=dev)) * 0.001 if case["bias"] else None
            s["expert"], s["gate"] = torch.empty((t, k), dtype=torch.int32, device=dev), torch.empty((t, k), device=dev)
            s["counts"] = torch.empty(e, dtype=torch.int32, device=dev)
        else:
            s["expert"] = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32).contiguous()
            s["dgate"] = torch.randn((t, k), generator=g, device=dev)
            s["dlogits"] = torch.empty((t, e), dtype=dt, device=dev)
    elif op == "swiglu":
        t, f = case["rows"], case["f"]
        s["gate_up"] = _normal(g, (t, 2 * f), dt, case["pad"])
        s.update(q=torch.empty((t, f), dtype=torch.int8, device=dev), scale=torch.empty(t, device=dev), values=torch.empty((t, f), dtype=torch.bfloat16, device=dev))
    else:
        m, k, n, e = case["rows"], case["k"], case["n"], case["experts"]
        s["a"] = _bytes8(g, (m, k), 32.0, case["pad"])
        s["a_scale"] = 0.01 + 0.02 * torch.rand(m, generator=g, device=dev)
        s["b"] = _bytes8(g, (max(e, 1), n, k), 36.0)
        s["b_scale"] = (0.5 + torch.rand((max(e, 1), n), generator=g, device=dev)) / (36.0 * k ** 0.5)
        s["output"] = torch.empty((m, n), dtype=dt, device=dev)
        s["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
        s["counts"] = None
        if e:
            share = np.random.default_rng(seed).permutation(1.0 / np.arange(1, e + 1) ** 0.5)
            counts = np.random.default_rng(seed + 1).multinomial(m, share / share.sum())
            s["counts"] = torch.from_numpy(counts.astype(np.int32)).to(dev)
            s["most"] = int(counts.max())
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _quantised(y):
    most = y.abs().amax(1, keepdim=True)
    none = most < TINY
    scale = torch.where(none, 0.0, most / 127.0)
    inverse = torch.where(none, 0.0, 127.0 / most)
    q = torch.clamp(torch.round(y * inverse), -127, 127).to(torch.int8)
    return {"values": (q.float() * scale).to(torch.bfloat16), "scale": scale.squeeze(1)}


def _plain_norm(s):
    dt, out = DTYPES[s["dtype"]], {}
    h = s["x"]
    if s["residual"]:
        h = (s["x"].float() + s["residual_in"].float()).to(dt)
        out["residual"] = h
    hf = h.float()
    rstd = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
    y = hf * rstd * s["weight"].float()
    out["rstd"] = rstd.squeeze(1)
    out.update(_quantised(y) if s["out"] == "int8" else {"y": y.to(dt)})
    return out


def _plain_norm_backward(s):
    rstd = s["rstd"].unsqueeze(1)
    dy, xhat = s["dy"].float(), s["x"].float() * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
    if s["residual"]:
        dx = dx + s["residual_in"].float()
    return {"dx": dx.to(DTYPES[s["dtype"]]), "dweight": (dy * xhat).sum(0)}


def _plain_route(s):
    t, e, k, ng = s["rows"], s["experts"], s["k"], s["groups"]
    logits = s["logits"].float()
    sigmoid = s["score"] == "sigmoid"
    score = torch.reciprocal(1.0 + torch.exp(-logits)) if sigmoid else None
    choice = score + s["bias_values"] if s["bias"] else logits      # scores rise with their logits
    if ng > 1:
        best = torch.sort(choice.view(t, ng, e // ng), dim=2, descending=True)[0][:, :, :s["group_best"]].sum(2)
        taken = torch.sort(best, dim=1, descending=True, stable=True)[1][:, :s["top_groups"]]
        inside = torch.zeros((t, ng), dtype=torch.bool, device=choice.device).scatter_(1, taken, True)
        choice = torch.where(inside.repeat_interleave(e // ng, 1), choice, float("-inf"))
    expert = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    if sigmoid:
        gate = score.gather(1, expert)
    else:
        p = torch.exp(logits - logits.amax(1, keepdim=True))
        gate = p.gather(1, expert) / p.sum(1, keepdim=True)
    if s["renormalise"]:
        gate = gate / gate.sum(1, keepdim=True)
    counts = torch.zeros(e, dtype=torch.int32, device=gate.device)
    counts.index_add_(0, expert.reshape(-1), torch.ones(t * k, dtype=torch.int32, device=gate.device))
    return {"expert": expert.to(torch.int32), "gate": gate, "counts": counts}


def _plain_route_backward(s):
    logits, at, dgate = s["logits"].float(), s["expert"].long(), s["dgate"]
    if s["score"] == "softmax":
        p = torch.exp(logits - logits.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        slope = p
    else:
        p = torch.reciprocal(1.0 + torch.exp(-logits))
        slope = p * (1.0 - p)
    if s["renormalise"]:
        chosen = p.gather(1, at)
        total = chosen.sum(1, keepdim=True)
        dgate = (dgate - (dgate * chosen).sum(1, keepdim=True) / total) / total
    dscore = torch.zeros_like(p).scatter_(1, at, dgate)
    if s["score"] == "softmax":
        dscore = dscore - (dscore * p).sum(1, keepdim=True)
    return {"dlogits": (slope * dscore).to(DTYPES[s["dtype"]])}


def _plain_swiglu(s):
    f = s["f"]
    g, u = s["gate_up"][:, :f].float(), s["gate_up"][:, f:].float()
    return _quantised(g * torch.reciprocal(1.0 + torch.exp(-g)) * u)


def _plain_matmul(s):
    a, b, dt = s["a"].float(), s["b"].float(), DTYPES[s["dtype"]]
    if not s["experts"]:
        y = torch.matmul(a, b[0].t()) * s["a_scale"].unsqueeze(1) * s["b_scale"][0]
        return {"output": y.to(dt)}
    counts, m, e = s["counts"].long(), s["rows"], s["experts"]
    expert = torch.repeat_interleave(torch.arange(e, device=a.device), counts, output_size=m)
    place = torch.arange(m, device=a.device) - (counts.cumsum(0) - counts)[expert]
    rows = torch.zeros((e, s["most"], s["k"]), device=a.device)
    rows[expert, place] = a
    y = torch.bmm(rows, b.transpose(1, 2))[expert, place] * s["a_scale"].unsqueeze(1) * s["b_scale"][expert]
    return {"output": y.to(dt)}


PLAIN = {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "route": _plain_route, "route_backward": _plain_route_backward,
         "swiglu": _plain_swiglu, "matmul": _plain_matmul}


# ------------------------------------------------------------------------------------------------ the framework's calls

def _values(s):
    torch.mul(s["q"], s["scale"].unsqueeze(1), out=s["values"])
    return {"values": s["values"], "scale": s["scale"]}


def _own(s):
    from paper_2607_19539_b200 import ops
    op = s["op"]
    if op == "norm":
        quant = s["out"] == "int8"
        ops.moe_ovl_add_norm(x=s["x"], residual=s["residual_in"], weight=s["weight"], eps=EPS, residual_out=s["residual_out"], rstd=s["rstd"],
                             y=None if quant else s["y"], q=s["q"] if quant else None, scale=s["scale"] if quant else None)
        out = {"residual": s["residual_out"]} if s["residual"] else {}
        return {**out, "rstd": s["rstd"], **(_values(s) if quant else {"y": s["y"]})}
    if op == "norm_backward":
        ops.moe_ovl_add_norm_backward(dy=s["dy"], h=s["x"], weight=s["weight"], rstd=s["rstd"], d_residual=s["residual_in"], dx=s["dx"], dweight=s["dweight"],
                                      workspace=s["workspace"])
        return {"dx": s["dx"], "dweight": s["dweight"]}
    if op == "route":
        ops.moe_ovl_route(logits=s["logits"], expert=s["expert"], gate=s["gate"], counts=s["counts"], bias=s["bias_values"], score=ops.SCORES[s["score"]],
                          num_groups=s["groups"], top_groups=s["top_groups"], group_best=s["group_best"], renormalise=s["renormalise"])
        return {"expert": s["expert"], "gate": s["gate"], "counts": s["counts"]}
    if op == "route_backward":
        ops.moe_ovl_route_backward(logits=s["logits"], expert=s["expert"], dgate=s["dgate"], dlogits=s["dlogits"], score=ops.SCORES[s["score"]],
                                   renormalise=s["renormalise"])
        return {"dlogits": s["dlogits"]}
    if op == "swiglu":
        ops.moe_ovl_swiglu_quant(gate_up=s["gate_up"], q=s["q"], scale=s["scale"])
        return _values(s)
    ops.moe_ovl_quant_matmul(a=s["a"], a_scale=s["a_scale"], b=s["b"], b_scale=s["b_scale"], out=s["output"], expert_counts=s["counts"], status=s["status"])
    return {"output": s["output"]}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


def work(case):
    op, size = case["op"], {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    t = case["rows"]
    if op == "norm":
        d = case["d"]
        return {"bytes": t * d * (size * (3 if case["residual"] else 1) + (1 if case["out"] == "int8" else size)) + d * size + 8 * t, "flops": 8 * t * d}
    if op == "norm_backward":
        d = case["d"]
        return {"bytes": t * d * size * (4 if case["residual"] else 3) + d * (size + 4) + 4 * t, "flops": 12 * t * d}
    if op in ("route", "route_backward"):
        e, k = case["experts"], case["k"]
        return {"bytes": t * e * size * (1 if op == "route" else 2) + 8 * t * k + 4 * e, "flops": 8 * t * e}
    if op == "swiglu":
        return {"bytes": t * case["f"] * (2 * size + 1) + 4 * t, "flops": 10 * t * case["f"]}
    k, n, e = case["k"], case["n"], min(max(case["experts"], 1), t)
    return {"bytes": t * k + e * n * k + t * n * size + 4 * (t + e * n), "flops": 2 * t * n * k}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_quantised(y):
    most = y.abs().max(dim=1).values
    step = most / 127
    q = torch.where(most[:, None] < TINY, torch.zeros_like(y), y / torch.clamp(step, min=1e-300)[:, None]).round()
    return {"values": q * step[:, None], "scale": step}


def _exact_route(s):
    lg = s["logits"].double().cpu().numpy()
    t, e = lg.shape
    ng, k = s["groups"], s["k"]
    sig = 1 / (1 + np.exp(-lg))
    want = sig + s["bias_values"].double().cpu().numpy() if s["bias"] else lg.copy()
    if ng > 1:
        by_group = np.sort(want.reshape(t, ng, e // ng), axis=2)[:, :, -s["group_best"]:].sum(2)
        order = np.argsort(-by_group, axis=1, kind="stable")[:, s["top_groups"]:]
        left_out = np.zeros((t, ng), bool)
        np.put_along_axis(left_out, order, True, 1)
        want[np.repeat(left_out, e // ng, axis=1)] = -np.inf
    idx = np.argsort(-want, axis=1, kind="stable")[:, :k]
    if s["score"] == "sigmoid":
        gate = np.take_along_axis(sig, idx, 1)
    else:
        z = np.exp(lg - lg.max(1, keepdims=True))
        gate = np.take_along_axis(z / z.sum(1, keepdims=True), idx, 1)
    if s["renormalise"]:
        gate = gate / gate.sum(1, keepdims=True)
    return {"expert": None, "gate": gate, "counts": None}


def _exact_route_backward(s):
    z = s["logits"].double().requires_grad_()
    p = torch.softmax(z, 1) if s["score"] == "softmax" else torch.sigmoid(z)
    gate = p.gather(1, s["expert"].long())
    if s["renormalise"]:
        gate = gate / gate.sum(1, keepdim=True)
    (gate * s["dgate"].double()).sum().backward()
    return {"dlogits": z.grad}


def _exact_norm_backward(s):
    # with the rstd that is given, as a constant of the call: d(h rstd w) by the norm's definition in 64 bits
    h, dy, w, r = s["x"].double(), s["dy"].double(), s["weight"].double(), s["rstd"].double()[:, None]
    n = h.shape[1]
    inner = ((dy * w) * h).sum(1, keepdim=True)
    dx = dy * w * r - h * r ** 3 * inner / n
    if s["residual"]:
        dx = dx + s["residual_in"].double()
    return {"dx": dx, "dweight": ((dy * h) * r).sum(0)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        out, h = {}, s["x"].double()
        if case["residual"]:
            out["residual"] = h + s["residual_in"].double()
            h = out["residual"].to(DTYPES[case["dtype"]]).double()     # the norm is the stored sum's
        r = 1 / torch.sqrt((h ** 2).sum(1) / case["d"] + EPS)
        y = s["weight"].double() * h * r[:, None]
        out["rstd"] = r
        return {**out, **(_exact_quantised(y) if case["out"] == "int8" else {"y": y})}
    if op == "norm_backward":
        return _exact_norm_backward(s)
    if op == "route":
        return _exact_route(s)
    if op == "route_backward":
        return _exact_route_backward(s)
    if op == "swiglu":
        g, u = s["gate_up"].double().chunk(2, dim=1)
        return _exact_quantised(g * u * torch.sigmoid(g))
    if not case["experts"]:
        y = s["a"].double() @ s["b"][0].double().t()
        return {"output": y * s["a_scale"].double()[:, None] * s["b_scale"][0].double()}
    parts, lo = [], 0
    for i, c in enumerate(s["counts"].tolist()):
        y = s["a"][lo:lo + c].double() @ s["b"][i].double().t()
        parts.append(y * s["a_scale"][lo:lo + c, None].double() * s["b_scale"][i].double())
        lo += c
    return {"output": torch.cat(parts)}
