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
