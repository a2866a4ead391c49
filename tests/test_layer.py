"""The expert layer built of the operators: wired as its formula says, and close to the library's bf16 experts.

8 bits with a scale per row or channel have a step of max / 127, so a rounding error of max / (127 sqrt(12)) (rms).  Of d values of
rms 1, normal ones have max <= 4.5 (the rows and weights: 1.0 % each, twice), products of two (the hidden values) max <= 14 (3.2 %).  Errors of
different values are independent, so the relative distance of an output row is about sqrt(4 * 1.0^2 + 3.2^2) = 3.8 %; the bound is twice that."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import binding as B, layer as L, ops  # noqa: E402

gpu = pytest.mark.gpu


def layer64(layer, x, residual, w1, w2):
    """The layer in 64 bits on its own choice of experts, without 8-bit rounding; the norm's output is rounded as it is stored."""
    h = (x.float() + residual.float()).to(x.dtype).double()
    y = (h / torch.sqrt((h * h).mean(1, keepdim=True) + layer.eps) * layer.norm_weight.double()).to(x.dtype).double()
    t = x.shape[0]
    out = torch.zeros((t, layer.d), dtype=torch.float64, device=x.device)
    for s in range(layer.k):
        for e in range(layer.experts):
            at = (layer.expert[:t, s] == e).nonzero().squeeze(1)
            gu = y[at] @ w1[e].double().t()
            g, u = gu.chunk(2, dim=1)
            out[at] += layer.gate[at, s].double()[:, None] * ((g * torch.sigmoid(g) * u) @ w2[e].double().t())
    return out


@gpu
@pytest.mark.parametrize("tokens,d,f,experts,k,choice", [
    (1, 256, 128, 8, 2, {}), (37, 512, 384, 16, 4, {}), (300, 256, 256, 8, 2, dict(score=ops.SCORE_SIGMOID, gate_scale=2.5)),
    (129, 512, 256, 32, 6, dict(score=ops.SCORE_SIGMOID, num_groups=8, top_groups=3, group_best=2)), (1111, 256, 640, 4, 4, dict(renormalise=False))])
def test_layer_against_64_bits_and_bf16_experts(tokens, d, f, experts, k, choice):
    layer, x, residual, w1, w2 = L.random_layer(tokens, d, f, experts, k, seed=tokens, **choice)
    if choice.get("group_best") == 2:
        layer.choice["bias"] = torch.linspace(-0.1, 0.1, experts, device="cuda")
    residual_out = torch.empty_like(x)
    out = layer(x, residual, residual_out)
    assert torch.equal(residual_out, (x.float() + residual.float()).to(x.dtype)) and not layer.status.any()
    want = layer64(layer, x, residual, w1, w2)
    far = (out.double() - want).norm(dim=1) / want.norm(dim=1)
    assert float(far.max()) <= 0.076, float(far.max())
    assert int(layer.counts.sum()) == tokens * k
    again = torch.empty_like(x)
    assert torch.equal(layer(x, residual, again), out)             # the same bits
    bf16 = L.bf16_experts(layer, L.routed_rows(layer.expert[:tokens], layer.gate[:tokens], layer.counts), tokens, w1, w2)
    far = (out.double() - bf16.double()).norm(dim=1) / bf16.double().norm(dim=1)
    assert float(far.max()) <= 0.076 + 0.01, float(far.max())       # and the bf16 path's own rounding


@gpu
def test_layer_with_masked_experts():
    """A bias of -inf leaves fewer experts than slots: empty slots add nothing, though their rows are never computed."""
    layer, x, residual, w1, w2 = L.random_layer(50, 256, 128, 8, 4, seed=5)
    layer.choice["bias"] = torch.tensor([0.0, float("-inf"), 0.0, float("-inf"), float("-inf"), float("-inf"), float("nan"), 0.0], device="cuda")
    layer.rows_out.fill_(float("nan"))
    out = layer(x, residual)
    assert bool((layer.expert[:, 3] == -1).all()) and int(layer.counts.sum()) == 150
    want = layer64(layer, x, residual, w1, w2)
    assert float(((out.double() - want).norm(dim=1) / want.norm(dim=1)).max()) <= 0.076


@gpu
def test_layer_refuses_weights_that_do_not_fit():
    layer, x, residual, w1, w2 = L.random_layer(4, 256, 128, 8, 2)
    with pytest.raises(B.MoeOvlError) as e:
        L.QuantExpertLayer(layer.norm_weight, layer.router, w1[:, :200], w2, top_k=2, max_tokens=4)
    assert e.value.code == B.ERR_INVALID_ARG


def test_quantise_channels_on_the_host():
    w = torch.tensor([[[1.0, -2.0, 0.5], [0.0, 0.0, 0.0]]])
    q, s = L.quantise_channels(w)
    assert q.tolist() == [[[64, -127, 32], [0, 0, 0]]] and torch.allclose(s, torch.tensor([[2 / 127, 0.0]]))


def test_routed_rows_on_the_host():
    expert = torch.tensor([[2, 0], [0, -1], [1, 2]], dtype=torch.int32)
    gate = torch.tensor([[0.6, 0.4], [1.0, 0.0], [0.7, 0.3]])
    r = L.routed_rows(expert, gate, torch.tensor([2, 1, 2], dtype=torch.int32))
    assert r.order.tolist() == [1, 2, 4, 0, 5, 3] and r.token.tolist() == [0, 1, 2, 0, 2, 1]
    assert torch.equal(r.gate, torch.tensor([0.4, 1.0, 0.7, 0.6, 0.3, 0.0]))
