"""The operators around the expert layer at the edges of what they accept: values half-way between two steps, logits at the ends of
their type, the widest rows, the longest matrices, waits that give up while copies are under way.

U, FLOOR and the comparison are those of test_ops; a tolerance that is not derived there is derived at its test.
"""
import math

import pytest

from paper_2607_19539_b200 import binding as B

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import ops  # noqa: E402

from tests.test_ops import BF16, F16, F32, FLOOR, U, call_route, check_product, close, gen, make8, norm64, norm_backward64, normal  # noqa: E402, F401

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", [33, 40, 4096, 4099])
def test_quantised_halves_and_scales(d, dtype):
    """A value of half the row's largest is 63.5 steps: an even 64, whatever rstd is.  With a largest magnitude of 2^j the step's inverse
    127 / 2^j is exact, and so is its product with 2^(j - 1).  The scale is the quotient max|v| / 127 itself, rounded once."""
    g = gen(d)
    rows = 64
    h = torch.rand((rows, d), generator=g, device="cuda") * 0.4
    half = torch.rand((rows, d), generator=g, device="cuda") < 0.3
    h = torch.where(half, 0.5, h)
    h[:, 0] = 1.0
    sign = torch.where(torch.rand((rows, d), generator=g, device="cuda") < 0.5, -1.0, 1.0)
    power = 2.0 ** torch.randint(-6, 7, (rows, 1), generator=g, device="cuda").float()
    x = (h * sign * power).to(dtype)
    q, scale, rstd = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ops.moe_ovl_add_norm(x=x, weight=torch.ones(d, dtype=dtype, device="cuda"), q=q, scale=scale, rstd=rstd)
    at_half = x.float().abs() == power / 2
    assert int(at_half.sum()) > rows and bool((q[at_half].abs() == 64).all()) and bool((q[:, 0].abs() == 127).all())
    assert torch.equal(q.sign(), torch.where(q == 0, 0, x.float().sign()).to(torch.int8))
    most = power.squeeze(1) * rstd                          # exact: a power of two
    assert torch.equal(scale, (most.double() / 127).float())
