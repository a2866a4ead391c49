"""Cases, plain forms and framework calls of the operators for training experts and for experts in 8-bit floats: the products
grouped by expert with both gradients, the 8-bit floating-point product with a scale per block of 128 and the quantiser
that makes its operands, and the norm of a list of gradients with clipping by it.

`own` chooses what `run` does: False, the plain form in elementary torch operations on 32-bit values; True, the
framework's operators.  Values held in 8 bits are returned as the values they stand for, in bf16."""
import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
F8 = torch.float8_e4m3fn
BLOCK = 128
LARGEST = 448.0         # of e4m3
TINY = 2.0 ** -100      # blocks whose largest magnitude is below this quantise to zeros
EPS = 1e-6


def listed():
    return [
        # a decode batch through the first product of many experts, a handful of rows each, some with none: weights are streamed
        {"name": "experts_decode", "op": "grouped", "rows": 96, "k": 2048, "n": 8192, "experts": 16, "dtype": "bf16", "out": "bf16", "transposed": False, "pad": 0},
        # the rows of a fine-grained layer's local experts in training, forward: gate and up projection, ragged counts
        {"name": "experts_forward", "op": "grouped", "rows": 49152, "k": 2048, "n": 2816, "experts": 8, "dtype": "bf16", "out": "bf16", "transposed": False, "pad": 0},
        # the same step back to the rows, by the weights as they are stored, in the other 16-bit type
        {"name": "experts_input_gradient", "op": "grouped", "rows": 49152, "k": 2816, "n": 2048, "experts": 8, "dtype": "f16", "out": "f16", "transposed": True, "pad": 0},
        # and to the weights, in 32 bits for the optimizer
        {"name": "experts_weight_gradient", "op": "grouped_backward", "rows": 49152, "k": 2048, "n": 2816, "experts": 8, "dtype": "bf16", "out": "f32", "pad": 0},
        # one generated token through a wide gate and up projection
        {"name": "block_one_token", "op": "block_matmul", "rows": 1, "k": 4096, "n": 28672, "experts": 0, "out": "bf16", "pad": 0},
        # a prompt of odd length through the same projection: the largest product
        {"name": "block_prompt", "op": "block_matmul", "rows": 7919, "k": 4096, "n": 28672, "experts": 0, "out": "bf16", "pad": 0},
        # a fine-grained layer's second product, ragged counts
        {"name": "block_experts", "op": "block_matmul", "rows": 49152, "k": 1408, "n": 2048, "experts": 8, "out": "bf16", "pad": 0},
        # hidden states of a decode batch on their way into an 8-bit product
        {"name": "quant_decode", "op": "block_quant", "rows": 37, "k": 4096, "experts": 0, "dtype": "bf16", "gated": False, "tiles": False, "pad": 0},
        # the gated activation between an expert's two products, a prompt's rows
        {"name": "quant_gated_prompt", "op": "block_quant", "rows": 8192, "k": 14336, "experts": 0, "dtype": "bf16", "gated": True, "tiles": False, "pad": 0},
        # a layer's 32-bit weights after an optimizer step, once more in 8 bits
        {"name": "quant_weights", "op": "block_quant", "rows": 2816, "k": 2048, "experts": 8, "dtype": "f32", "gated": False, "tiles": True, "pad": 0},
        # the gradients of a layer's small parts: norm weights, a bias, a router
        {"name": "clip_small", "op": "clip", "layers": 1, "d": 2048, "f": 0, "experts": 64, "dtype": "f32", "max_norm": 0.05},
        # the gradients of some whole layers: norm weights and routers in 32 bits, experts in 16
        {"name": "clip_layers", "op": "clip", "layers": 6, "d": 2048, "f": 1408, "experts": 8, "dtype": "bf16", "max_norm": 1.0},
    ]


def _between(rng, lo, hi):
    """A whole number of lo..hi, even in its logarithm."""
    return min(max(int(round(np.exp(rng.uniform(np.log(lo), np.log(hi))))), lo), hi)


def draw(rng):
    op = rng.choice(["grouped", "grouped", "grouped_backward", "block_matmul", "block_matmul", "block_quant", "clip"])
    if op in ("grouped", "grouped_backward"):
        experts = rng.choice([1, 4, 8, 16, 32, 64])
        k, n = (8 * _between(rng, 8, 512) for _ in range(2))
        while experts * n * k > 1 << 28:
            n, k = (max(8, v // 16 * 8) for v in (n, k))
        c = {"op": op, "rows": _between(rng, 1, 32768), "k": k, "n": n, "experts": experts, "dtype": rng.choice(["bf16", "f16"]), "pad": rng.choice([0, 0, 8])}
        c["out"] = rng.choice([c["dtype"], "f32"])
        if op == "grouped":
            c["transposed"] = rng.random() < 0.5
        return c
    if op == "block_matmul":
        experts = rng.choice([0, 0, 4, 8, 16, 32])
        return {"op": op, "rows": _between(rng, 1, 8192), "k": 16 * _between(rng, 8, 512), "n": _between(rng, 64, 16384 if experts == 0 else 4096),
                "experts": experts, "out": rng.choice(["bf16", "bf16", "f16", "f32"]), "pad": rng.choice([0, 0, 16])}
    if op == "block_quant":
        kind = rng.choice(["rows", "rows", "gated", "tiles"])
        k = _between(rng, 64, 14336)
        if rng.random() < 0.7:
            k = (k + 7) // 8 * 8
        c = {"op": op, "rows": _between(rng, 1, 8192), "k": k, "experts": 0, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "gated": kind == "gated",
             "tiles": kind == "tiles", "pad": rng.choice([0, 0, 8])}
        if kind == "tiles":
            c["experts"] = rng.choice([1, 2, 8])
            c["rows"] = _between(rng, 1, 4096)
            c["k"] = min(c["k"], 4096)
            c["pad"] = 0
        return c
    return {"op": op, "layers": rng.randint(1, 6), "d": _between(rng, 64, 2048), "f": rng.choice([0, _between(rng, 32, 1408)]), "experts": rng.choice([4, 8, 64]) if rng.random() < 0.3 else 8,
            "dtype": rng.choice(["bf16", "f16", "f32"]), "max_norm": rng.choice([0.1, 1.0, 1e6])}


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, dtype, pad=0, scale=1.0):
    """Normal values; with pad, a view of rows that lie further apart than they are long."""
    full = torch.empty((*shape[:-1], shape[-1] + pad), dtype=dtype, device="cuda")
    flat = full.view(-1)
    for lo in range(0, flat.numel(), 1 << 27):
        part = flat[lo:lo + (1 << 27)]
        values = torch.randn(part.numel(), generator=g, device="cuda").mul_(scale)
        part.copy_(values.clamp_(-LARGEST, LARGEST) if dtype is F8 else values)
    return full[..., :shape[-1]]


def _counts(rows, experts, seed):
    """Rows per expert: some experts are asked for more often than others."""
    share = np.random.default_rng(seed).permutation(1.0 / np.arange(1, experts + 1) ** 0.5)
    return np.random.default_rng(seed + 1).multinomial(rows, share / share.sum())


def _shapes(case):
    """The parameters of the layers: norm weight, router and its bias in 32 bits; first and second products of every expert."""
    d, f, e = case["d"], case["f"], case["experts"]
    layer = [((d,), "f32"), ((e, d), "f32"), ((e,), "f32")]
    if f:
        layer += [((e, 2 * f, d), case["dtype"]), ((e, d, f), case["dtype"])]
    return layer * case["layers"]


def prepare(case, seed):
    g, op, s = _generator(seed), case["op"], dict(case)
    dev = "cuda"
    if op == "clip":
        # gradients: small, each tensor with a size of its own
        sizes = np.random.default_rng(seed).uniform(-9.0, -5.0, len(_shapes(case)))
        s["grads"] = [_normal(g, shape, DTYPES[t], scale=float(np.exp(z))) for (shape, t), z in zip(_shapes(case), sizes)]
        s["clipped"] = [torch.empty_like(t) for t in s["grads"]]
        s["norm"] = torch.empty(1, device=dev)
        s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
        return s
    s["status"] = torch.zeros(4, dtype=torch.int32, device=dev)
    rows, k, experts = case["rows"], case["k"], case["experts"]
    if op == "block_quant":
        shape = (rows, 2 * k if case["gated"] else k)
        blocks = (k + BLOCK - 1) // BLOCK
        if case["tiles"]:
            s["x"] = _normal(g, (experts, *shape), DTYPES[case["dtype"]], scale=k ** -0.5)
            s["q"], s["scale"] = torch.empty((experts, rows, k), dtype=F8, device=dev), torch.empty((experts, (rows + BLOCK - 1) // BLOCK, blocks), device=dev)
        else:
            s["x"] = _normal(g, shape, DTYPES[case["dtype"]], case["pad"])
            # hidden states: a few channels much larger than the others
            s["x"].mul_(torch.exp(0.5 * torch.randn(shape[1], generator=g, device=dev)).to(s["x"].dtype))
            s["q"], s["scale"] = torch.empty((rows, k), dtype=F8, device=dev), torch.empty((rows, blocks), device=dev)
        s["values"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=dev)
        return s
    n = case["n"]
    if op == "block_matmul":
        blocks = (k + BLOCK - 1) // BLOCK
        s["a"] = _normal(g, (rows, k), F8, case["pad"], scale=150.0)
        s["a_scale"] = torch.exp(0.5 * torch.randn((rows, blocks), generator=g, device=dev)) / 150
        s["b"] = _normal(g, (max(experts, 1), n, k), F8, scale=110.0)
        s["b_scale"] = (0.5 + torch.rand((max(experts, 1), (n + BLOCK - 1) // BLOCK, blocks), generator=g, device=dev)) / (110 * k ** 0.5)
        s["output"] = torch.empty((rows, n), dtype=DTYPES[case["out"]], device=dev)
    elif op == "grouped":
        dt = DTYPES[case["dtype"]]
        s["a"] = _normal(g, (rows, k), dt, case["pad"])
        s["b"] = _normal(g, (experts, k, n) if case["transposed"] else (experts, n, k), dt, scale=k ** -0.5)
        s["output"] = torch.empty((rows, n), dtype=DTYPES[case["out"]], device=dev)
    else:
        dt = DTYPES[case["dtype"]]
        s["dy"] = _normal(g, (rows, n), dt, case["pad"], scale=0.02)
        s["x"] = _normal(g, (rows, k), dt, case["pad"])
        s["dweight"] = torch.empty((experts, n, k), dtype=DTYPES[case["out"]], device=dev)
        s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    s["counts"] = None
    if experts:
        counts = _counts(rows, experts, seed)
        s["counts"] = torch.from_numpy(counts.astype(np.int32)).to(dev)
        s["most"] = int(counts.max())
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _places(s):
    """For every row its expert and its place among the expert's rows."""
    counts, dev = s["counts"].long(), s["counts"].device
    expert = torch.repeat_interleave(torch.arange(s["experts"], device=dev), counts, output_size=s["rows"])
    return expert, torch.arange(s["rows"], device=dev) - (counts.cumsum(0) - counts)[expert]


def _by_expert(s, x, expert, place):
    out = torch.zeros((s["experts"], s["most"], x.shape[1]), device=x.device)
    out[expert, place] = x.float()
    return out


def _plain_grouped(s):
    expert, place = _places(s)
    b = s["b"].float()
    y = torch.bmm(_by_expert(s, s["a"], expert, place), b if s["transposed"] else b.transpose(1, 2))
    return {"output": y[expert, place].to(DTYPES[s["out"]])}


def _plain_grouped_backward(s):
    expert, place = _places(s)
    dw = torch.bmm(_by_expert(s, s["dy"], expert, place).transpose(1, 2), _by_expert(s, s["x"], expert, place))
    return {"dweight": dw.to(DTYPES[s["out"]])}


def _spread(scale, rows, k, tall):
    """A block's scale for each of its values."""
    scale = scale.repeat_interleave(BLOCK, -1)[..., :k]
    return scale.repeat_interleave(BLOCK, -2)[..., :rows, :] if tall else scale


def _plain_block_matmul(s):
    a = s["a"].float() * _spread(s["a_scale"], s["rows"], s["k"], False)
    b = s["b"].float() * _spread(s["b_scale"], s["n"], s["k"], True)
    if not s["experts"]:
        return {"output": torch.matmul(a, b[0].t()).to(DTYPES[s["out"]])}
    expert, place = _places(s)
    return {"output": torch.bmm(_by_expert(s, a, expert, place), b.transpose(1, 2))[expert, place].to(DTYPES[s["out"]])}


def _plain_block_quant(s):
    # in 64 bits: 16-bit values often lie half-way between two steps, and which way they go must not hang on a rounded quotient
    k, tall = s["k"], s["tiles"]
    v = s["x"].double()
    if s["gated"]:
        v = v[:, :k] / (1.0 + torch.exp(-v[:, :k])) * v[:, k:]
    rows = v.shape[-2]
    pad = torch.nn.functional.pad(v, (0, -k % BLOCK, 0, -rows % BLOCK if tall else 0)).abs()
    most = pad.unflatten(-1, (-1, BLOCK)).amax(-1)
    if tall:
        most = most.unflatten(-2, (-1, BLOCK)).amax(-2)
    none = most < TINY
    scale = torch.where(none, 0.0, most / LARGEST)
    divisor = torch.where(none, float("inf"), most)
    q = (v * LARGEST / _spread(divisor, rows, k, tall)).to(F8)
    return {"values": (q.double() * _spread(scale, rows, k, tall)).to(torch.bfloat16), "scale": scale.float()}


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["grads"]:
        total = total + (t.float() * t.float()).sum(dtype=torch.float64)
    norm = torch.sqrt(total).float().reshape(1)
    factor = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    return {"norm": norm, "clipped": [(t.float() * factor).to(t.dtype) for t in s["grads"]]}


PLAIN = {"grouped": _plain_grouped, "grouped_backward": _plain_grouped_backward, "block_matmul": _plain_block_matmul, "block_quant": _plain_block_quant,
         "clip": _plain_clip}


# ------------------------------------------------------------------------------------------------ the framework's calls

def _own(s):
    from paper_2607_19539_b200 import ops
    op = s["op"]
    if op == "grouped":
        ops.moe_ovl_grouped_matmul(a=s["a"], b=s["b"], out=s["output"], expert_counts=s["counts"], transposed=s["transposed"], status=s["status"])
        return {"output": s["output"]}
    if op == "grouped_backward":
        ops.moe_ovl_grouped_matmul_backward(dy=s["dy"], x=s["x"], dweight=s["dweight"], expert_counts=s["counts"], status=s["status"], workspace=s["workspace"])
        return {"dweight": s["dweight"]}
    if op == "block_matmul":
        ops.moe_ovl_block_matmul(a=s["a"], a_scale=s["a_scale"], b=s["b"], b_scale=s["b_scale"], out=s["output"], expert_counts=s["counts"], status=s["status"])
        return {"output": s["output"]}
    if op == "block_quant":
        ops.moe_ovl_block_quant(x=s["x"], q=s["q"], scale=s["scale"], gated=s["gated"], tiles=s["tiles"])
        scale = _spread(s["scale"], s["q"].shape[-2], s["k"], s["tiles"])
        return {"values": torch.mul(s["q"].float(), scale, out=s["values"]), "scale": s["scale"]}
    ops.moe_ovl_grad_norm(grads=s["grads"], norm=s["norm"], workspace=s["workspace"])
    ops.moe_ovl_clip_grads(grads=s["grads"], norm=s["norm"], max_norm=s["max_norm"], eps=EPS, out=s["clipped"])
    return {"norm": s["norm"], "clipped": s["clipped"]}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


def work(case):
    op = case["op"]
    if op == "clip":
        sizes = [(int(np.prod(shape)), SIZES[t]) for shape, t in _shapes(case)]
        return {"bytes": 2 * sum(n * b for n, b in sizes) + 4, "flops": 3 * sum(n for n, _ in sizes)}
    rows, k, e = case["rows"], case["k"], case["experts"]
    blocks = (k + BLOCK - 1) // BLOCK
    if op == "block_quant":
        v = rows * k * max(e, 1)
        scales = max(e, 1) * (-(-rows // BLOCK) if case["tiles"] else rows) * blocks
        return {"bytes": v * (SIZES[case["dtype"]] * (2 if case["gated"] else 1) + 1) + 4 * scales, "flops": (10 if case["gated"] else 3) * v}
    n, used, out = case["n"], min(max(e, 1), rows), SIZES[case["out"]]
    if op == "block_matmul":
        return {"bytes": rows * k + used * n * k + rows * n * out + 4 * blocks * (rows + used * -(-n // BLOCK)), "flops": 2 * rows * n * k}
    size = SIZES[case["dtype"]]
    if op == "grouped":
        return {"bytes": size * (rows * k + used * n * k) + rows * n * out + 4 * e, "flops": 2 * rows * n * k}
    return {"bytes": size * rows * (n + k) + e * n * k * out + 4 * e, "flops": 2 * rows * n * k}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _e4m3(v):
    """The nearest number of four significant bits, or multiple of 2^-9 below 2^-6; ties to even."""
    exponent = torch.clamp(torch.floor(torch.log2(torch.clamp(v.abs(), min=1e-300))), min=-6)
    step = torch.exp2(exponent - 3)
    return torch.clamp(torch.round(v / step) * step, -LARGEST, LARGEST)


def _exact_block_quant(s):
    values, scales = [], []
    for x in (s["x"] if s["tiles"] else s["x"].unsqueeze(0)):
        v = x.double()
        if s["gated"]:
            g, u = v.chunk(2, dim=1)
            v = g * torch.sigmoid(g) * u
        height = BLOCK if s["tiles"] else 1
        step = torch.empty((-(-v.shape[0] // height), -(-s["k"] // BLOCK)), dtype=torch.float64, device=v.device)
        out = torch.empty_like(v)
        for j in range(step.shape[1]):
            cols = slice(j * BLOCK, min((j + 1) * BLOCK, s["k"]))
            most = v[:, cols].abs().max(dim=1).values
            if height > 1:
                most = torch.stack([p.max() for p in most.split(height)])
            step[:, j] = torch.where(most < TINY, torch.zeros_like(most), most / LARGEST)
            each = step[:, j].repeat_interleave(height)[:v.shape[0], None]
            whole = most.repeat_interleave(height)[:v.shape[0], None]
            out[:, cols] = torch.where(each > 0, _e4m3(v[:, cols] * LARGEST / torch.clamp(whole, min=1e-300)), torch.zeros_like(v[:, cols])) * each
        values.append(out)
        scales.append(step)
    if s["tiles"]:
        return {"values": torch.stack(values), "scale": torch.stack(scales)}
    return {"values": values[0], "scale": scales[0]}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norm = torch.sqrt(sum((t.double() ** 2).sum() for t in s["grads"]))
        factor = min(1.0, case["max_norm"] / (float(norm) + EPS))
        return {"norm": norm.reshape(1), "clipped": [t.double() * factor for t in s["grads"]]}
    if op == "block_quant":
        return _exact_block_quant(s)
    lo, parts = 0, []
    counts = [case["rows"]] if s["counts"] is None else s["counts"].tolist()
    for e, c in enumerate(counts):
        at = slice(lo, lo + c)
        lo += c
        if op == "grouped_backward":
            parts.append(s["dy"][at].double().t() @ s["x"][at].double())
            continue
        a, b = s["a"][at].double(), s["b"][e].double()
        if op == "block_matmul":
            for j in range(s["a_scale"].shape[1]):
                cols = slice(j * BLOCK, (j + 1) * BLOCK)
                a[:, cols] *= s["a_scale"][at, j:j + 1].double()
                for i in range(s["b_scale"].shape[1]):
                    b[i * BLOCK:(i + 1) * BLOCK, cols] *= s["b_scale"][e, i, j].double()
        parts.append(a @ b if op == "grouped" and case["transposed"] else a @ b.t())
    return {"dweight": torch.stack(parts)} if op == "grouped_backward" else {"output": torch.cat(parts)}
