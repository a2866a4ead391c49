"""A whole expert layer around the library's operators, with all experts on this GPU: norm of the residual sum, router, experts
in 8-bit integers or in 8-bit floats with a scale per block, gate-weighted sum.  What lies between the operators (the router's projection, sorting
rows by expert, the weighted sum) is plain torch.  `expert_ffn` is the experts' part for training: its products and their gradients are operators
under torch's autograd, and `clip_gradients` clips what a backward pass has left.

The same routing also feeds the bf16 experts of moe_ovl_expert_return (`routed_rows` gives its arguments), and

    python -m paper_2607_19539_b200.layer

runs all of them on random weights, prints how far they are apart, and takes a training step.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import binding as B, ops


def quantise_channels(w: torch.Tensor):
    """Weights [..., channels, k] in 8 bits with a scale per channel: (int8, float32 [..., channels])."""
    scale = w.float().abs().amax(-1) / 127
    q = torch.round(w.float() / scale.clamp_min(1e-30).unsqueeze(-1)).clamp_(-127, 127).to(torch.int8)
    return q, scale


@dataclass
class RoutedRows:
    """Rows (token, slot) in the order of their experts, tokens ascending inside an expert; rows whose slot is empty come last."""
    order: torch.Tensor       # [T * k] flat (token, slot) index of every row
    token: torch.Tensor       # [T * k] int32
    gate: torch.Tensor        # [T * k]
    counts: torch.Tensor      # [experts] int32


def routed_rows(expert: torch.Tensor, gate: torch.Tensor, counts: torch.Tensor) -> RoutedRows:
    k = expert.shape[1]
    flat = expert.reshape(-1)
    order = torch.sort(torch.where(flat >= 0, flat, counts.shape[0]), stable=True)[1]
    return RoutedRows(order, (order // k).to(torch.int32), gate.reshape(-1)[order], counts)


class QuantExpertLayer:
    """norm_weight [d]; router [experts, d]; w1 [experts, 2F, d] (gate rows, then up rows) and w2 [experts, d, F] in bf16, kept in 8 bits.
    Buffers are sized for `max_tokens` and reused by every call on the current stream; `status[0]` is not 0 when a bounded wait inside a product
    gave up, and the outputs since then are not to be used (nothing waits for it here: look after a synchronize of your own)."""

    eight = torch.int8              # what rows and weights are held in

    def __init__(self, norm_weight, router, w1, w2, *, top_k: int, max_tokens: int, eps: float = 1e-6, score: int = ops.SCORE_SOFTMAX, bias=None,
                 num_groups: int = 1, top_groups: int = 1, group_best: int = 1, renormalise: bool = True, gate_scale: float = 1.0):
        self.norm_weight, self.router, self.eps, self.k = norm_weight, router, eps, top_k
        self.experts, self.d, self.f = w2.shape
        if w1.shape != (self.experts, 2 * self.f, self.d) or router.shape != (self.experts, self.d):
            raise B.MoeOvlError(B.ERR_INVALID_ARG, "QuantExpertLayer: w1 has to be [experts, 2F, d], w2 [experts, d, F], router [experts, d]")
        self.hold(w1, w2)
        self.choice = dict(score=score, bias=bias, num_groups=num_groups, top_groups=top_groups, group_best=group_best, renormalise=renormalise,
                           gate_scale=gate_scale)
        dev, t, rows = w1.device, max_tokens, max_tokens * top_k
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        self.y, self.q, self.scale = new(t, self.d, dtype=w1.dtype), new(t, self.d, dtype=self.eight), new(*self.scales(t, self.d))
        self.expert, self.gate, self.counts = new(t, top_k, dtype=torch.int32), new(t, top_k), new(self.experts, dtype=torch.int32)
        self.gate_up, self.hidden, self.hidden_scale = new(rows, 2 * self.f, dtype=w1.dtype), new(rows, self.f, dtype=self.eight), new(*self.scales(rows, self.f))
        self.rows_out = new(rows, self.d, dtype=w1.dtype)
        self.status = torch.zeros(4, dtype=torch.int32, device=dev)

    def scales(self, rows: int, k: int) -> tuple:
        """The shape of the scales of rows of k values."""
        return (rows,)

    def hold(self, w1, w2) -> None:
        """Keeps the experts' weights in 8 bits."""
        self.w1, self.s1 = quantise_channels(w1)
        self.w2, self.s2 = quantise_channels(w2)

    def norm(self, x, residual, residual_out) -> None:
        """The normed rows, as they are and in 8 bits, into self.y, self.q and self.scale."""
        t = x.shape[0]
        ops.moe_ovl_add_norm(x=x, residual=residual, weight=self.norm_weight, eps=self.eps, residual_out=residual_out, y=self.y[:t], q=self.q[:t],
                             scale=self.scale[:t])

    def route(self, x, residual=None, residual_out=None) -> RoutedRows:
        """Norm (bf16 for the router, 8 bits for the experts) and choice; self.y, self.q and self.scale hold the normed rows."""
        t = x.shape[0]
        self.norm(x, residual, residual_out)
        logits = self.y[:t] @ self.router.t()
        ops.moe_ovl_route(logits=logits, expert=self.expert[:t], gate=self.gate[:t], counts=self.counts, **self.choice)
        return routed_rows(self.expert[:t], self.gate[:t], self.counts)

    def experts_of(self, r: RoutedRows):
        """The routed rows through their experts in 8 bits: [rows, d] in the order of `r`."""
        n, token = r.token.shape[0], r.token
        ops.moe_ovl_quant_matmul(a=self.q[token], a_scale=self.scale[token], b=self.w1, b_scale=self.s1, out=self.gate_up[:n], expert_counts=r.counts,
                                 status=self.status)
        ops.moe_ovl_swiglu_quant(gate_up=self.gate_up[:n], q=self.hidden[:n], scale=self.hidden_scale[:n])
        ops.moe_ovl_quant_matmul(a=self.hidden[:n], a_scale=self.hidden_scale[:n], b=self.w2, b_scale=self.s2, out=self.rows_out[:n],
                                 expert_counts=r.counts, status=self.status)
        return self.rows_out[:n]

    def __call__(self, x, residual=None, residual_out=None):
        """x [T, d] (+ residual) -> the layer's output [T, d]; residual_out, where given, becomes the sum that the next layer adds to."""
        t = x.shape[0]
        r = self.route(x, residual, residual_out)
        y = self.experts_of(r)
        by_slot = torch.empty_like(r.order)
        by_slot[r.order] = torch.arange(r.order.shape[0], device=x.device)
        gate = self.gate[:t].unsqueeze(-1)
        rows = y[by_slot].view(t, self.k, self.d).float()
        return torch.where(self.expert[:t].unsqueeze(-1) >= 0, rows * gate, 0.0).sum(1).to(x.dtype)      # an empty slot's row was never written


def quantise_blocks(w: torch.Tensor):
    """Weights [..., channels, k] in 8-bit floats with a scale per 128 x 128: (float8_e4m3fn, float32 [..., ceil(channels / 128), ceil(k / 128)])."""
    w = w.detach().contiguous()
    q = torch.empty(w.shape, dtype=ops.FLOAT8, device=w.device)
    scale = torch.empty((*w.shape[:-2], -(-w.shape[-2] // ops.BLOCK), -(-w.shape[-1] // ops.BLOCK)), device=w.device)
    ops.moe_ovl_block_quant(x=w, q=q, scale=scale, tiles=True)
    return q, scale


class BlockExpertLayer(QuantExpertLayer):
    """The same layer with its experts in 8-bit floats: a scale per 128 values of a row and per 128 x 128 weights.  d and F have to be multiples of 16."""

    eight = ops.FLOAT8

    def scales(self, rows: int, k: int) -> tuple:
        return (rows, -(-k // ops.BLOCK))

    def hold(self, w1, w2) -> None:
        if self.d % 16 or self.f % 16:
            raise B.MoeOvlError(B.ERR_UNSUPPORTED, "BlockExpertLayer: d and F have to be multiples of 16")
        self.w1, self.s1 = quantise_blocks(w1)
        self.w2, self.s2 = quantise_blocks(w2)

    def norm(self, x, residual, residual_out) -> None:
        t = x.shape[0]
        ops.moe_ovl_add_norm(x=x, residual=residual, weight=self.norm_weight, eps=self.eps, residual_out=residual_out, y=self.y[:t])
        ops.moe_ovl_block_quant(x=self.y[:t], q=self.q[:t], scale=self.scale[:t])

    def experts_of(self, r: RoutedRows):
        n, token = r.token.shape[0], r.token
        rows = self.q.view(torch.uint8)[token].view(ops.FLOAT8)     # torch gathers bytes
        ops.moe_ovl_block_matmul(a=rows, a_scale=self.scale[token], b=self.w1, b_scale=self.s1, out=self.gate_up[:n], expert_counts=r.counts, status=self.status)
        ops.moe_ovl_block_quant(x=self.gate_up[:n], q=self.hidden[:n], scale=self.hidden_scale[:n], gated=True)
        ops.moe_ovl_block_matmul(a=self.hidden[:n], a_scale=self.hidden_scale[:n], b=self.w2, b_scale=self.s2, out=self.rows_out[:n], expert_counts=r.counts,
                                 status=self.status)
        return self.rows_out[:n]


class ExpertProduct(torch.autograd.Function):
    """rows @ weight[e]^T for the rows of every expert, with both gradients by the operators.  Rows behind the last expert's give zeros, and get them.  The counts are looked at
    again on the way back: they have to be what they were."""

    @staticmethod
    def forward(ctx, rows, weight, counts, status):
        ctx.save_for_backward(rows, weight, counts)
        ctx.status = status             # not saved: the caller may clear it in between
        out = torch.zeros((rows.shape[0], weight.shape[1]), dtype=rows.dtype, device=rows.device)
        ops.moe_ovl_grouped_matmul(a=rows, b=weight, out=out, expert_counts=counts, status=status)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (rows, weight, counts), status = ctx.saved_tensors, ctx.status
        dout = dout.contiguous()
        if dout.data_ptr() % 16:
            dout = dout.clone()         # a piece of another tensor's gradient begins anywhere
        drows = dweight = None
        if ctx.needs_input_grad[0]:
            drows = torch.zeros_like(rows)
            ops.moe_ovl_grouped_matmul(a=dout, b=weight, out=drows, expert_counts=counts, transposed=True, status=status)
        if ctx.needs_input_grad[1]:
            dweight = torch.empty_like(weight)
            workspace = torch.empty(ops.moe_ovl_grouped_matmul_workspace_bytes(weight.shape[0]), dtype=torch.uint8, device=rows.device)
            ops.moe_ovl_grouped_matmul_backward(dy=dout, x=rows, dweight=dweight, expert_counts=counts, status=status, workspace=workspace)
        return drows, dweight, None, None


def expert_ffn(rows, w1, w2, counts, status):
    """Rows grouped by expert ([n, d], counts [experts] int32) through their experts, for training: w1 [experts, 2F, d] (gate rows, then up rows), w2 [experts, d, F].
    d and F have to be multiples of 8, and rows and weights begin on 16 bytes.  `status`: 4 int32 that the caller clears once; look at it after a synchronize of your own.  Gradients of gradients are refused.  Where a
    step is captured into a graph, no eager step's result may live any more: torch would tie the leaves' gradients to that step's stream, which no capture can wait for."""
    counts = counts.clone()             # the router's buffer may hold the next batch's by the time of the backward pass
    gate, up = ExpertProduct.apply(rows, w1, counts, status).float().chunk(2, dim=1)
    hidden = (torch.nn.functional.silu(gate) * up).to(rows.dtype)
    return ExpertProduct.apply(hidden, w2, counts, status)


def clip_gradients(parameters, max_norm: float, eps: float = 1e-6) -> torch.Tensor:
    """Scales the gradients of the parameters (or of one) that have one, so that their norm is max_norm at most; returns the norm before, on the gradients' device (where
    there are none, 0 on the first parameter's)."""
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else list(parameters)
    grads = [p.grad for p in parameters if p.grad is not None]
    if not grads:
        return torch.zeros(1, device=parameters[0].device if parameters else None)
    norm = torch.empty(1, device=grads[0].device)
    workspace = torch.empty(ops.moe_ovl_grad_norm_workspace_bytes(len(grads)), dtype=torch.uint8, device=norm.device)
    ops.moe_ovl_grad_norm(grads=grads, norm=norm, workspace=workspace)
    ops.moe_ovl_clip_grads(grads=grads, norm=norm, max_norm=max_norm, eps=eps)
    return norm


def bf16_experts(layer: QuantExpertLayer, r: RoutedRows, tokens: int, w1, w2, mode: int = B.MODE_AUTO):
    """The same routing through moe_ovl_expert_return: one source rank, every expert local, bf16 weights.  Every slot has to be taken."""
    dev, n = w1.device, r.token.shape[0]
    ctx = B.MoeOvl(B.make_config(device=dev.index, num_src_ranks=1, self_rank=0, tokens_per_rank=tokens, num_local_experts=layer.experts,
                                 top_k=layer.k, d_model=layer.d, d_ffn=layer.f, max_rows=n))
    ret = torch.empty((1, tokens * min(layer.k, layer.experts), layer.d), dtype=torch.bfloat16, device=dev)
    out = torch.empty((tokens, layer.d), dtype=torch.bfloat16, device=dev)
    ctx.moe_ovl_expert_return(x=layer.y[r.token], expert_counts=r.counts, src_rank=torch.zeros_like(r.token), src_token=r.token, gate=r.gate,
                              w1=w1, w2=w2, ret=ret, out=out, mode=mode, consumer_sm_count=0)
    code, detail = ctx.moe_ovl_query_status()
    if code != B.OK:
        raise B.MoeOvlError(code, f"moe_ovl_expert_return (detail {detail:#x})")
    return out


def random_layer(tokens: int, d: int, f: int, experts: int, top_k: int, seed: int = 0, device="cuda:0", kind=QuantExpertLayer, **choice):
    """Random weights of that size: (layer, x, residual, w1, w2)."""
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *shape, scale=1.0: (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)  # noqa: E731
    w1, w2 = normal(experts, 2 * f, d, scale=d ** -0.5), normal(experts, d, f, scale=f ** -0.5)
    layer = kind(1 + normal(d, scale=0.1), normal(experts, d, scale=d ** -0.5), w1, w2, top_k=top_k, max_tokens=tokens, **choice)
    return layer, normal(tokens, d), normal(tokens, d), w1, w2


def main() -> None:
    tokens = 2048
    layer, x, residual, w1, w2 = random_layer(tokens, d=2048, f=1408, experts=64, top_k=6)
    residual_out = torch.empty_like(x)
    out = layer(x, residual, residual_out)
    ref = bf16_experts(layer, routed_rows(layer.expert, layer.gate, layer.counts), tokens, w1, w2)
    block = random_layer(tokens, d=2048, f=1408, experts=64, top_k=6, kind=BlockExpertLayer)[0]

    def distance(out):
        far = (out.double() - ref.double()).norm(dim=1) / ref.double().norm(dim=1)
        return f"relative distance per token median {float(far.median()):.4f}, largest {float(far.max()):.4f}"

    print(f"{tokens} tokens, 64 experts, top 6, rows per expert {int(layer.counts.min())} .. {int(layer.counts.max())}: 8-bit experts against bf16 experts, {distance(out)}; "
          f"in 8-bit floats {distance(block(x, residual, residual_out))}")
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for name, each in (("8-bit integers", layer), ("8-bit floats", block)):
        for _ in range(3):
            each(x, residual, residual_out)
        begin.record()
        for _ in range(10):
            each(x, residual, residual_out)
        end.record()
        torch.cuda.synchronize()
        print(f"layer in {name} {begin.elapsed_time(end) / 10:.3f} ms per call, the torch steps between the operators included")

    r = routed_rows(layer.expert, layer.gate, layer.counts)
    rows, w1, w2 = layer.y[r.token], w1.requires_grad_(), w2.requires_grad_()
    for step in range(4):
        begin.record()
        w1.grad = w2.grad = None
        expert_ffn(rows, w1, w2, r.counts, layer.status).backward(torch.full_like(rows, 1e-3))
        norm = clip_gradients([w1, w2], 1.0)
        end.record()
    torch.cuda.synchronize()
    print(f"experts' training step (forward, backward, clipping; {rows.shape[0]} rows in bf16) {begin.elapsed_time(end):.3f} ms, gradient norm {float(norm):.3f} before clipping, "
          f"status {layer.status.tolist()}")


if __name__ == "__main__":
    main()
