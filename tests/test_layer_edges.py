"""The expert layer's edges: gradients that begin anywhere, parameters without any, and what the layer in 8-bit floats keeps."""
import pytest

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import layer as L, ops  # noqa: E402

from tests.test_layer_experts import training_leaves  # noqa: E402

gpu = pytest.mark.gpu


@gpu
def test_clip_gradients_without_any_is_on_the_parameters_device():
    p = torch.nn.Parameter(torch.zeros(3, device="cuda"))
    for parameters in (p, [p], iter([p])):
        norm = L.clip_gradients(parameters, 1.0)
        assert norm.device == p.device and norm.dtype is torch.float32 and norm.tolist() == [0.0]
    assert L.clip_gradients([], 1.0).tolist() == [0.0]


@gpu
@pytest.mark.parametrize("product", [False, True])
def test_gradients_that_begin_anywhere(product):
    """What arrives on the way back is a piece of another tensor's gradient, contiguous, behind one value: not on 16 bytes.  The gradients are those of the same values on a boundary."""
    leaves, dout, status = training_leaves(40, 64, 32, 2, 9)
    counts = torch.tensor([15, 25], dtype=torch.int32, device="cuda")
    out = L.ExpertProduct.apply(*leaves[:2], counts, status) if product else L.expert_ffn(*leaves, counts, status)
    used = leaves[:2] if product else leaves
    want = torch.autograd.grad(out, used, dout, retain_graph=True)
    first = torch.zeros(1, dtype=out.dtype, device="cuda")
    got = torch.autograd.grad(torch.cat([first, out.flatten()]), used, torch.cat([first, dout.flatten()]))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and not status.any()


@gpu
def test_block_layer_keeps_its_own_buffers():
    """q and scale are the normed rows in 8-bit floats, and every buffer is there before the first call and used by all."""
    layer, x, residual, w1, w2 = L.random_layer(50, 256, 272, 8, 4, seed=5, kind=L.BlockExpertLayer)
    names = ("y", "q", "scale", "expert", "gate", "counts", "gate_up", "hidden", "hidden_scale", "rows_out", "status")
    at = {n: getattr(layer, n).data_ptr() for n in names}
    assert layer.q.dtype is layer.hidden.dtype is ops.FLOAT8 and layer.scale.shape == (50, 2) and layer.hidden.shape == (200, 272) and layer.hidden_scale.shape == (200, 3)
    first = layer(x[:37], residual[:37])
    q, scale = torch.empty((37, 256), dtype=ops.FLOAT8, device="cuda"), torch.empty((37, 2), device="cuda")
    ops.moe_ovl_block_quant(x=layer.y[:37], q=q, scale=scale)
    assert torch.equal(layer.q[:37].view(torch.uint8), q.view(torch.uint8)) and torch.equal(layer.scale[:37], scale)
    hidden, hidden_scale = torch.empty((148, 272), dtype=ops.FLOAT8, device="cuda"), torch.empty((148, 3), device="cuda")
    ops.moe_ovl_block_quant(x=layer.gate_up[:148], q=hidden, scale=hidden_scale, gated=True)
    assert torch.equal(layer.hidden[:148].view(torch.uint8), hidden.view(torch.uint8)) and torch.equal(layer.hidden_scale[:148], hidden_scale)
    layer(x, residual)
    assert torch.equal(layer(x[:37], residual[:37]), first) and at == {n: getattr(layer, n).data_ptr() for n in names} and not layer.status.any()
    assert layer(x[:0], residual[:0]).shape == (0, 256)
