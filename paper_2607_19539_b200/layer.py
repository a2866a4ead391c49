"""A whole expert layer around the library's operators, with all experts on this GPU: norm of the residual sum, router, experts
in 8-bit integers, gate-weighted sum.  What lies between the operators (the router's projection, sorting rows by expert,
the weighted sum) is plain torch.

The same routing also feeds the bf16 experts of moe_ovl_expert_return (`routed_rows` gives its arguments), and

    python -m paper_2607_19539_b200.layer

runs both on random weights and prints how far they are apart.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

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

    def __init__(self, norm_weight, router, w1, w2, *, top_k: int, max_tokens: int, eps: float = 1e-6, score: int = ops.SCORE_SOFTMAX, bias=None,
                 num_groups: int = 1, top_groups: int = 1, group_best: int = 1, renormalise: bool = True, gate_scale: float = 1.0):
        self.norm_weight, self.router, self.eps, self.k = norm_weight, router, eps, top_k
        self.experts, self.d, self.f = w2.shape
        if w1.shape != (self.experts, 2 * self.f, self.d) or router.shape != (self.experts, self.d):
            raise B.MoeOvlError(B.ERR_INVALID_ARG, "QuantExpertLayer: w1 has to be [experts, 2F, d], w2 [experts, d, F], router [experts, d]")
        self.w1, self.s1 = quantise_channels(w1)
        self.w2, self.s2 = quantise_channels(w2)
        self.choice = dict(score=score, bias=bias, num_groups=num_groups, top_groups=top_groups, group_best=group_best, renormalise=renormalise,
                           gate_scale=gate_scale)
        dev, t, rows = w1.device, max_tokens, max_tokens * top_k
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        self.y, self.q, self.scale = new(t, self.d, dtype=w1.dtype), new(t, self.d, dtype=torch.int8), new(t)
        self.expert, self.gate, self.counts = new(t, top_k, dtype=torch.int32), new(t, top_k), new(self.experts, dtype=torch.int32)
        self.gate_up, self.hidden, self.hidden_scale = new(rows, 2 * self.f, dtype=w1.dtype), new(rows, self.f, dtype=torch.int8), new(rows)
        self.rows_out = new(rows, self.d, dtype=w1.dtype)
        self.status = torch.zeros(4, dtype=torch.int32, device=dev)

    def route(self, x, residual=None, residual_out=None) -> RoutedRows:
        """Norm (bf16 for the router, 8 bits for the experts) and choice; self.y, self.q and self.scale hold the normed rows."""
        t = x.shape[0]
        ops.moe_ovl_add_norm(x=x, residual=residual, weight=self.norm_weight, eps=self.eps, residual_out=residual_out, y=self.y[:t], q=self.q[:t],
                             scale=self.scale[:t])
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


def random_layer(tokens: int, d: int, f: int, experts: int, top_k: int, seed: int = 0, device="cuda:0", **choice):
    """Random weights of that size: (layer, x, residual, w1, w2)."""
    g = torch.Generator(device=device).manual_seed(seed)
    normal = lambda *shape, scale=1.0: (torch.randn(shape, generator=g, device=device) * scale).to(torch.bfloat16)  # noqa: E731
    w1, w2 = normal(experts, 2 * f, d, scale=d ** -0.5), normal(experts, d, f, scale=f ** -0.5)
    layer = QuantExpertLayer(1 + normal(d, scale=0.1), normal(experts, d, scale=d ** -0.5), w1, w2, top_k=top_k, max_tokens=tokens, **choice)
    return layer, normal(tokens, d), normal(tokens, d), w1, w2


def main() -> None:
    tokens = 2048
    layer, x, residual, w1, w2 = random_layer(tokens, d=2048, f=1408, experts=64, top_k=6)
    residual_out = torch.empty_like(x)
    out = layer(x, residual, residual_out)
    ref = bf16_experts(layer, routed_rows(layer.expert, layer.gate, layer.counts), tokens, w1, w2)
    far = (out.double() - ref.double()).norm(dim=1) / ref.double().norm(dim=1)
    print(f"{tokens} tokens, 64 experts, top 6: 8-bit experts against bf16 experts, relative distance per token "
          f"median {float(far.median()):.4f}, largest {float(far.max()):.4f}; rows per expert {int(layer.counts.min())} .. {int(layer.counts.max())}")
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(3):
        layer(x, residual, residual_out)
    begin.record()
    for _ in range(10):
        layer(x, residual, residual_out)
    end.record()
    torch.cuda.synchronize()
    print(f"8-bit layer {begin.elapsed_time(end) / 10:.3f} ms per call, the torch steps between the operators included")


if __name__ == "__main__":
    main()
