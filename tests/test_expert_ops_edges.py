"""Edges of the operators for training experts and for experts in 8-bit floats: values that do not fit among their neighbours, the longest sums, gates far below
zero, gradients that begin anywhere.  Tolerances are derived at each test; U is half a unit in the last place."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import ops  # noqa: E402

from tests.test_expert_ops import F8, INF, NAN, check_grouped, e4m3, norm_of, status, whole  # noqa: E402
from tests.test_ops import BF16, F16, F32, U, close, gen, normal  # noqa: E402

gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ norm of gradients

# 32 positive terms in 32 bits and one more addition, the rest in 64, then a root (half of that) and a rounding
NORM_OFF = (33 / 2 + 1) * 2.0 ** -24 * 1.01


def gradient_lists(g, t):
    """The tensor in lists of one block's run, of a cluster, of two kernels, and of more tensors than a short list holds."""
    yield [t]
    yield [normal(g, (40000,), F32), t]
    yield [normal(g, (300001,), BF16), t, normal(g, (7,), F16)]
    yield [normal(g, (i,), F32) for i in range(40)] + [t]


def norm64(grads):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))


def starting(g, n, dtype, shift):
    """n normal values that begin `shift` values behind a boundary of 16 bytes."""
    return normal(g, (n + shift,), dtype)[shift:]


@gpu
@pytest.mark.parametrize("value", [NAN, INF, -INF, 1e20, 1e-25])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_grad_norm_of_one_value_unlike_the_others(dtype, value):
    """One NaN, infinity, large or small value among ordinary ones: only the thread whose share it is leaves the range of 32 bits.  The clipped gradients are what the norm says."""
    if dtype is F16 and abs(value) == 1e20:
        value = 65504.0
    g = gen(3)
    for n in (2048, 16384, 100001):
        for shift in (0, 1):
            base = starting(g, n, dtype, shift)
            for at in (0, 1, 5, 9, 257, 1000, n // 2, n - 1):
                t = base.clone() if shift == 0 else torch.cat([base[:1], base])[1:]
                t[at] = value
                for grads in gradient_lists(g, t):
                    norm, want = norm_of(grads), norm64(grads)
                    if math.isfinite(want):
                        assert abs(float(norm) - want) <= NORM_OFF * want, (n, shift, at, len(grads), float(norm), want)
                        continue
                    assert math.isnan(want) == math.isnan(float(norm)) and (math.isnan(want) or float(norm) == INF), (n, shift, at, len(grads), float(norm))
                    out = [torch.full_like(x, 7.5) for x in grads]
                    ops.moe_ovl_clip_grads(grads=grads, norm=norm, max_norm=1.0, out=out)
                    for x, o in zip(grads, out):
                        assert bool(o.isnan().all()) if math.isnan(want) else torch.equal(o.isnan(), x.isinf()) and not o.nan_to_num().any()


@gpu
@pytest.mark.parametrize("dtype,small,large", [(BF16, 1e-17, 1e-2), (F32, 1e-17, 1e-2), (F32, 1e-30, 1.0), (BF16, 1.0, 1e20), (F32, 1.0, 1e20), (BF16, -0.0, 1.0), (F16, -0.0, 1.0), (F32, -0.0, 1.0)])
def test_grad_norm_of_columns_unlike_each_other(dtype, small, large):
    """Whole columns of another magnitude, as experts and channels that are hardly used have: some threads' shares leave the range of 32 bits, their neighbours' do not."""
    for rows, cols in ((16, 1024), (8, 2048), (100, 264), (33, 1001)):
        for first in (cols // 2, 8, cols - 3):
            t = torch.full((rows, cols), large, dtype=dtype, device="cuda")
            t[:, :first] = small
            for grads in gradient_lists(gen(5), t):
                norm, want = float(norm_of(grads)), norm64(grads)
                assert abs(norm - want) <= NORM_OFF * want, (rows, cols, first, len(grads), norm, want)


@gpu
def test_clip_grads_without_a_limit():
    """max_norm may be infinite: the gradients stay as they are, but for a norm that is infinite (factor 0) or NaN."""
    for values, want in (([1.0, 2.0], [1.0, 2.0]), ([1.0, INF, -2.0], [0.0, NAN, 0.0]), ([1.0, NAN], [NAN, NAN]), ([0.0, 0.0], [0.0, 0.0])):
        for eps in (0.0, 1e-6):
            t, w = torch.tensor(values, device="cuda"), torch.tensor(want, device="cuda")
            norm, out = norm_of([t]), torch.full_like(t, 7.5)
            ops.moe_ovl_clip_grads(grads=[t], norm=norm, max_norm=INF, eps=eps, out=[out])
            ops.moe_ovl_clip_grads(grads=[t], norm=norm, max_norm=INF, eps=eps)
            assert all(torch.equal(o.isnan(), w.isnan()) and torch.equal(o.nan_to_num(), w.nan_to_num()) for o in (out, t))


# ------------------------------------------------------------------------------------------------ 16-bit products

@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m", [1, 20, 64, 129, 300])
def test_longest_sums_in_16_bits(m, dtype, transposed):
    """The longest k, all terms of one sign.  A matrix instruction cuts its 16 products and the sum so far to 24 bits of the largest, 33 * 2^-23 of the magnitudes at most; a sum ends after 4096
    of k, 256 instructions, and the up to 4096 of them are added in 32 bits, 2^-24 each (and as many parts as a cluster has CTAs): 1.25e-3, and the output's rounding."""
    k, n, period = 1 << 24, 8, 1 << 20
    g = gen(m)
    pattern = lambda rows: (0.5 + 0.5 * torch.rand((rows, period), generator=g, device="cuda")).mul_(2.0 ** -6).to(dtype)  # noqa: E731
    pa, pb = pattern(m), pattern(n)
    a, b = pa.repeat(1, k // period), pb.repeat(1, k // period)
    b = b.t().contiguous() if transposed else b
    out, st = torch.empty((m, n), dtype=dtype, device="cuda"), status()
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, transposed=transposed, status=st)
    want = sum(pa[:, c:c + 65536].double() @ pb[:, c:c + 65536].double().t() for c in range(0, period, 65536)) * (k // period)
    assert not st.any()
    close(out, want, ((256 * 33 * 2.0 ** -23) + (4096 + 8) * 2.0 ** -24 + U[dtype]) * want)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("k", [4088, 4096, 4104, 8192, 8200, 12352])
def test_sums_of_some_pieces(k, transposed):
    """Whole numbers, whose sums are exact however they are cut: one piece of 4096, two, three, and a little more, on tiles of every width."""
    g = gen(k)
    for counts in ([1], [13], [30, 0, 2], [64], [130], [100, 0, 129, 1], [300, 700], [40] * 9):
        m, n = sum(counts), 264
        for dtype in (BF16, F16):
            a, b = whole(g, (m, k), dtype, 2), whole(g, (len(counts), k, n) if transposed else (len(counts), n, k), dtype, 2)
            check_grouped(a, b, counts, transposed, dtype)
    a, b = whole(g, (33, k), BF16, 2), whole(g, (k, 20000) if transposed else (20000, k), BF16, 2)        # more tiles than SMs
    check_grouped(a[:13], b, None, transposed, BF16)
    check_grouped(a, b, None, transposed, BF16)


# ------------------------------------------------------------------------------------------------ quantiser

@gpu
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_block_quant_gates_far_below_zero(dtype, shift):
    """A gate far below zero leaves little of a value, but of a large one enough: exp(-87.4) is the last one whose reciprocal is a normal number.  Gate and value in 32 bits: the exponent is off by
    |g| / ln 2 * 2^-24 twice (its factor and its rounding), the rest by 2^-20."""
    k = 256
    gates = [-1.0, -80.0, -86.5, -87.0, -87.5, -88.0, -88.5, -89.0, -90.0, -95.0, -100.0, -120.0, -140.0, -155.0, -160.0, -250.0, -1000.0, -1e30]
    ups = [1.0, -1e-3, 1e30, 1e36, -3e38]
    rows = len(gates) * len(ups)
    x = torch.zeros((rows, 2 * k + 8), dtype=dtype, device="cuda")[:, shift:2 * k + shift]
    g = torch.tensor(gates).repeat_interleave(len(ups))[:, None]
    u = torch.tensor(ups).repeat(len(gates))[:, None]
    spread = torch.linspace(0.25, 1.0, k)[None]
    x[:, :k], x[:, k:] = (g * torch.where(torch.arange(k) % 3 == 0, 1.0, 0.99)).to("cuda"), (u * spread).to("cuda")
    x[:, 5] = 0.0
    x[1::2, 40:60], x[1::2, k + 40:k + 60] = 2.0, 3.0                      # ordinary ones beside them
    q, scale = torch.empty((rows, k), dtype=F8, device="cuda"), torch.empty((rows, 2), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale, gated=True)
    gate, up = x[:, :k].double(), x[:, k:].double()
    v = gate * torch.exp(gate.clamp_max(0)) / (1 + torch.exp(-gate.abs())) * up
    most = v.abs().unflatten(1, (2, 128)).amax(2)
    off = gate.abs().amax(1, keepdim=True).clamp_max(250.0) * 2.0 ** -23 + 2.0 ** -20
    sure, none = most >= 2.0 ** -100 * (1 + off), most < 2.0 ** -100 * (1 - off)
    assert not scale[none].any() and bool(((scale.double() - most / 448).abs() <= (2 * off + 2.0 ** -23) * most / 448)[sure].all())
    t = (v.unflatten(1, (2, 128)) * 448 / most.clamp_min(1e-300)[..., None]).flatten(1)
    got, whole = q.double(), sure.repeat_interleave(128, 1)
    assert bool(((got >= e4m3(t - 2 * off * t.abs())) & (got <= e4m3(t + 2 * off * t.abs())))[whole].all()) and not got[none.repeat_interleave(128, 1)].any()
