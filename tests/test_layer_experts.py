"""The expert layer in 8-bit floats, and the experts' products under autograd.

8-bit floats have four significant bits: a value is off by a relative 2^-4 at most, uniformly distributed over a step, so by 2^-4 / sqrt(3) = 3.6 % (rms) where
its significand is smallest and 1.8 % where it is largest, 2.6 % over all.  An output is a product of rows, first weights, hidden values (of a product of two: twice the error of
rows and first weights), second weights: sqrt(2 * 2 * 2.6^2 + 2.6^2 + 2.6^2) = 6.4 % of the row's norm if the errors are independent; the bound is twice that."""
import pytest

from paper_2607_19539_b200 import binding as B

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import layer as L, ops  # noqa: E402

from tests.test_layer import layer64  # noqa: E402

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("tokens,d,f,experts,k,choice", [
    (1, 256, 128, 8, 2, {}), (37, 512, 384, 16, 4, {}), (300, 256, 272, 8, 2, dict(score=ops.SCORE_SIGMOID, gate_scale=2.5)), (1111, 272, 640, 4, 4, dict(renormalise=False))])
def test_block_layer_against_64_bits(tokens, d, f, experts, k, choice):
    layer, x, residual, w1, w2 = L.random_layer(tokens, d, f, experts, k, seed=tokens, kind=L.BlockExpertLayer, **choice)
    residual_out = torch.empty_like(x)
    out = layer(x, residual, residual_out)
    assert torch.equal(residual_out, (x.float() + residual.float()).to(x.dtype)) and not layer.status.any()
    want = layer64(layer, x, residual, w1, w2)
    far = (out.double() - want).norm(dim=1) / want.norm(dim=1)
    assert float(far.max()) <= 0.128, float(far.max())
    again = torch.empty_like(x)
    assert torch.equal(layer(x, residual, again), out)             # the same bits


@gpu
def test_block_layer_with_masked_experts():
    layer, x, residual, w1, w2 = L.random_layer(50, 256, 128, 8, 4, seed=5, kind=L.BlockExpertLayer)
    layer.choice["bias"] = torch.tensor([0.0, float("-inf"), 0.0, float("-inf"), float("-inf"), float("-inf"), float("nan"), 0.0], device="cuda")
    layer.rows_out.fill_(float("nan"))
    layer.gate_up.fill_(float("nan"))
    out = layer(x, residual)
    want = layer64(layer, x, residual, w1, w2)
    assert float(((out.double() - want).norm(dim=1) / want.norm(dim=1)).max()) <= 0.128


@gpu
def test_block_layer_refuses_what_its_products_do():
    with pytest.raises(B.MoeOvlError) as e:
        L.random_layer(4, 264, 128, 8, 2, kind=L.BlockExpertLayer)
    assert e.value.code == B.ERR_UNSUPPORTED


@gpu
def test_expert_ffn_gradients():
    """Against autograd in 64 bits on the same bf16 inputs.  Rounding to bf16 (2^-9 rms / sqrt(3) of a value, 2^-8 at most) happens to the first product, the hidden values, their
    gradients and the outputs: at most six roundings in a row, 6 * 2^-8 of the norms."""
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(torch.bfloat16)  # noqa: E731
    n, d, f, counts = 230, 136, 72, [50, 0, 130, 20]
    rows, w1, w2, dout = normal(n, d), normal(4, 2 * f, d, scale=d ** -0.5), normal(4, d, f, scale=f ** -0.5), normal(n, d)
    status, dc = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor(counts, dtype=torch.int32, device="cuda")
    leaves = [t.clone().requires_grad_() for t in (rows, w1, w2)]
    out = L.expert_ffn(*leaves, dc, status)
    out.backward(dout)
    wide = [t.double().requires_grad_() for t in (rows, w1, w2)]
    parts, lo = [], 0
    for e, c in enumerate(counts):
        gate, up = (wide[0][lo:lo + c] @ wide[1][e].t()).chunk(2, dim=1)
        parts.append((torch.nn.functional.silu(gate) * up) @ wide[2][e].t())
        lo += c
    want = torch.cat(parts)
    want.backward(dout[:lo].double())
    assert not out[lo:].any() and not leaves[0].grad[lo:].any() and not leaves[1].grad[1].any() and not status.any()
    for got, ref in [(out.detach()[:lo], want.detach())] + [(a.grad, b.grad) for a, b in zip(leaves, wide)]:
        assert float((got.double() - ref).norm() / ref.norm()) <= 6 * 2.0 ** -8
    norm = L.clip_gradients(leaves[1:], 0.25)
    before = float(torch.sqrt(sum((t.grad ** 2).sum() for t in wide[1:])))
    after = float(torch.sqrt(sum((t.grad.double() ** 2).sum() for t in leaves[1:])))
    assert abs(float(norm) - before) <= 6 * 2.0 ** -8 * before and abs(after - 0.25) <= 2.0 ** -8 * 0.25


@gpu
def test_expert_product_asks_for_the_gradients_that_are_wanted():
    g = torch.Generator(device="cuda").manual_seed(4)
    rows, w = torch.randn(40, 64, generator=g, device="cuda").half(), torch.randn(2, 24, 64, generator=g, device="cuda").half()
    status, counts = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor([10, 30], dtype=torch.int32, device="cuda")
    for i in range(2):
        leaves = [rows.clone(), w.clone()]
        leaves[i].requires_grad_()
        L.ExpertProduct.apply(*leaves, counts, status).float().sum().backward()
        assert leaves[i].grad is not None and leaves[1 - i].grad is None


def test_clip_gradients_without_any():
    assert L.clip_gradients([torch.nn.Parameter(torch.zeros(3))], 1.0).tolist() == [0.0]


def test_clip_gradients_of_one_parameter():
    class Seen(Exception):
        pass

    def norm_of(n):
        raise Seen(n)

    p, real = torch.nn.Parameter(torch.zeros(3, 5)), ops.moe_ovl_grad_norm_workspace_bytes
    p.grad = torch.ones(3, 5)
    ops.moe_ovl_grad_norm_workspace_bytes = norm_of
    try:
        for parameters in (p, [p], iter([p])):
            with pytest.raises(Seen) as e:
                L.clip_gradients(parameters, 1.0)
            assert e.value.args == (1,)                            # one gradient, not one per row
    finally:
        ops.moe_ovl_grad_norm_workspace_bytes = real


def training_leaves(n, d, f, experts, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(torch.bfloat16)  # noqa: E731
    leaves = [normal(n, d).requires_grad_(), normal(experts, 2 * f, d, scale=d ** -0.5).requires_grad_(), normal(experts, d, f, scale=f ** -0.5).requires_grad_()]
    return leaves, normal(n, d), torch.zeros(4, dtype=torch.int32, device="cuda")


@gpu
def test_status_may_be_cleared_between_the_passes():
    leaves, dout, status = training_leaves(40, 64, 32, 2, 5)
    counts = torch.tensor([15, 25], dtype=torch.int32, device="cuda")
    out = L.expert_ffn(*leaves, counts, status)
    want = torch.autograd.grad(out, leaves, dout, retain_graph=True)
    status.zero_()
    counts.fill_(7)                                                # the next batch's: the gradients are of this one
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves, dout), want))


@gpu
def test_gradients_of_gradients_are_refused():
    leaves, dout, status = training_leaves(40, 64, 32, 2, 6)
    counts = torch.tensor([15, 25], dtype=torch.int32, device="cuda")
    for i in range(2):
        got, = torch.autograd.grad(L.ExpertProduct.apply(*leaves[:2], counts, status).float().square().sum(), leaves[i], create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            got.float().sum().backward()


@gpu
def test_training_without_rows():
    leaves, dout, status = training_leaves(0, 64, 32, 2, 7)
    out = L.expert_ffn(*leaves, torch.zeros(2, dtype=torch.int32, device="cuda"), status)
    out.backward(dout)
    assert out.shape == (0, 64) and leaves[0].grad.shape == (0, 64) and not leaves[1].grad.any() and not leaves[2].grad.any() and not status.any()
    assert float(L.clip_gradients(leaves, 1.0)) == 0.0 and not leaves[1].grad.any()


@gpu
def test_training_step_in_a_graph():
    leaves, dout, status = training_leaves(230, 136, 72, 4, 8)
    counts = torch.tensor([50, 0, 130, 20], dtype=torch.int32, device="cuda")

    def step():
        for t in leaves:
            t.grad = None
        out = L.expert_ffn(*leaves, counts, status)
        out.backward(dout)
        return out.detach(), L.clip_gradients(leaves, 0.25)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    kept = [*captured, *(t.grad for t in leaves)]
    for now in ([50, 0, 130, 20], [0, 229, 0, 1], [0, 0, 0, 0]):
        counts.copy_(torch.tensor(now, dtype=torch.int32))
        for t in kept:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(got, [*eager, *(t.grad for t in leaves)])) and not status.any()
