"""The operators for training experts and for experts in 8-bit floats, against plain implementations in 64 bits.

Where the tolerances come from.  Small whole numbers (up to 8 in magnitude, products up to 64, at most 2^18 of them in a sum) are exact in the operands and
in 32-bit sums whatever their order, and powers of two as scales keep them exact: such products have to be equal to the 64-bit result rounded once.
Of other values a matrix instruction adds up to 32 products to a sum, each cut to no fewer than 24 bits of the largest: at most 33 * 2^-23 of the sum of magnitudes S per instruction, K / 16 of
them (32 in 8 bits).  So K / 16 * 33 * 2^-23 * S, and the last rounding; scales add three products of 2^-24 and an addition per block of 128, which is less than one instruction's share.
U is half a unit in the last place, FLOOR half the distance of the values below f16's normal range."""
import ctypes
import math
import warnings

import pytest

from paper_2607_19539_b200 import binding as B

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import ops  # noqa: E402

from tests.test_ops import BF16, F16, F32, FLOOR, U, close, gen, guarded, normal, untouched  # noqa: E402

gpu = pytest.mark.gpu
F8 = torch.float8_e4m3fn
INF, NAN = float("inf"), float("nan")


def whole(g, shape, dtype, most=8, pad=0):
    """Whole numbers of -most .. most."""
    full = torch.randint(-most, most + 1, (*shape[:-1], shape[-1] + pad), generator=g, device="cuda").float().to(dtype)
    return full[..., :shape[-1]]


def status():
    return torch.zeros(4, dtype=torch.int32, device="cuda")


def device_counts(counts):
    return None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")


def spans(counts, rows):
    """First and last row of every expert, cut at the rows there are."""
    out, lo = [], 0
    for c in ([rows] if counts is None else counts):
        hi = min(lo + max(c, 0), rows)
        out.append((lo, hi))
        lo = hi
    return out


def product64(a, b, counts, transposed=False):
    b = b if b.dim() == 3 else b[None]
    out = torch.zeros((a.shape[0], b.shape[2] if transposed else b.shape[1]), dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate(spans(counts, a.shape[0])):
        w = b[e].double()
        out[lo:hi] = a[lo:hi].double() @ (w if transposed else w.t())
    return out


def slack(k, s):
    return k / 16 * 33 * 2.0 ** -23 * s


# ------------------------------------------------------------------------------------------------ 16-bit products

def check_grouped(a, b, counts, transposed, out_dtype, pad=0, shift=0, exact=True, stream=None):
    m, n = a.shape[0], b.shape[-1] if transposed else b.shape[-2]
    out, full = guarded(m, n, out_dtype, pad, shift)
    st = status()
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, expert_counts=device_counts(counts), transposed=transposed, status=st, stream=stream)
    want = product64(a, b, counts, transposed)
    covered = spans(counts, m)[-1][1]
    if exact:
        assert torch.equal(out[:covered], want[:covered].to(out_dtype))
    else:
        s = product64(a.abs(), b.abs(), counts, transposed)
        close(out[:covered], want[:covered], U[out_dtype] * want[:covered].abs() + slack(a.shape[1], s[:covered]) + FLOOR[out_dtype])
    assert untouched(full, out) and not st.any()
    if covered < m:
        assert bool((out[covered:].float() == 7.5).all())


SHAPES = [(1, 1, 8), (1, 5, 40), (2, 127, 64), (3, 128, 72), (16, 129, 256), (17, 304, 400), (31, 64, 1024), (33, 257, 1000), (64, 1000, 512), (65, 130, 136),
          (127, 256, 640), (128, 512, 4096), (129, 384, 1280), (200, 77, 16), (257, 513, 520), (500, 2050, 1032), (1025, 768, 264), (1, 4096, 8192),
          (2000, 1500, 200), (4097, 640, 128)]


@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_grouped_matmul_of_one_matrix(m, n, k, dtype, transposed):
    g = gen(m + n)
    a = whole(g, (m, k), dtype, pad=8 if m % 3 == 0 else 0)
    b = whole(g, (k, n) if transposed else (n, k), dtype, pad=(-n % 8 if transposed else 0) + (16 if n % 3 == 0 else 0))
    check_grouped(a, b, None, transposed, F32, pad=5 if m % 2 else 0, shift=1 if n % 2 else 0)
    check_grouped(a, b[None], None, transposed, dtype, pad=3 if n % 2 else 0)


COUNTS = [([5], 136, 256), ([0, 3, 0], 256, 128), ([1] * 40, 96, 272), ([0, 0, 0, 17], 128, 512), ([100, 1, 0, 33, 250], 640, 1024),
          ([700, 300, 0, 513], 304, 208), ([3, 0, 2] * 30, 384, 640), ([1000] * 5, 512, 512), ([0] * 1023 + [7], 16, 64), ([2] * 700, 24, 48), ([63, 64, 65, 1, 128], 200, 72)]


@gpu
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("counts,n,k", COUNTS)
def test_grouped_matmul(counts, n, k, transposed):
    m, e = sum(counts), len(counts)
    for dtype in (BF16, F16):
        g = gen(m + n)
        a, b = whole(g, (m, k), dtype), whole(g, (e, k, n) if transposed else (e, n, k), dtype)
        check_grouped(a, b, counts, transposed, dtype)
        check_grouped(a, b, counts, transposed, F32, pad=3)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_grouped_matmul_of_normal_values(transposed):
    g = gen(5)
    counts = [300, 0, 17, 512, 1]
    for dtype in (BF16, F16):
        for k in (136, 2048):
            a, b = normal(g, (830, k), dtype), normal(g, (5, k, 264) if transposed else (5, 264, k), dtype, k ** -0.5)
            check_grouped(a, b, counts, transposed, F32, exact=False)
            check_grouped(a, b, counts, transposed, dtype, exact=False)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_grouped_matmul_counts_that_do_not_add_up(transposed):
    g = gen(4)
    a, b = whole(g, (90, 256), BF16), whole(g, (4, 256, 144) if transposed else (4, 144, 256), BF16)
    for counts in ([20, 0, 30, 11], [50, 60, 70, 2147483647], [2147483647] * 4, [-5, 40, -2147483648, 10], [0, 0, 0, 0]):
        check_grouped(a, b, counts, transposed, F32)


@gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_grouped_matmul_keeps_what_is_not_a_number_to_itself(transposed):
    """Rows of one expert, weights of another, columns behind the last and rows behind the sum hold NaN and infinities: only their own outputs do."""
    g = gen(11)
    counts, k, n = [40, 70, 0, 30], 72, 136
    a = whole(g, (160, k), BF16, pad=8)
    a._base[:, k:] = NAN
    a[140:] = NAN
    a[45] = INF
    b = whole(g, (4, k, n) if transposed else (4, n, k), BF16, pad=8)
    b._base[..., -8:] = NAN
    b[2] = NAN
    out, st = torch.zeros((160, n), device="cuda"), status()
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, expert_counts=device_counts(counts), transposed=transposed, status=st)
    want = product64(a, b, counts, transposed)
    rows = [r for r in range(140) if r != 45]
    assert torch.equal(out[rows], want[rows].float()) and not bool(out[45].isfinite().any()) and not out[140:].any()


@gpu
def test_grouped_matmul_of_experts_that_lie_apart():
    """Matrices cut out of larger ones, and those of every second expert."""
    g = gen(12)
    full = whole(g, (6, 200, 320), BF16)
    a = whole(g, (50, 128), BF16)
    check_grouped(a, full[::2, 8:144, 64:192], [20, 0, 30], False, F32)
    a = whole(g, (50, 136), BF16)
    check_grouped(a, full[::2, 8:144, 64:192], [20, 0, 30], True, F32)
    check_grouped(a[:, :128], full[1:4].transpose(0, 1)[:, :, :128].transpose(0, 1), [50, 0, 0], False, F32)


@gpu
def test_grouped_matmul_rounds_once_and_overflows_to_infinity():
    a = torch.full((2, 64), 200.0, dtype=F16, device="cuda")
    b = torch.full((8, 64), 200.0, dtype=F16, device="cuda")
    b[1] = -200
    b[2] = 0.001
    out, wide, st = torch.empty((2, 8), dtype=F16, device="cuda"), torch.empty((2, 8), device="cuda"), status()
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, status=st)
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=wide, status=st)
    assert out[0, 0] == INF and out[0, 1] == -INF and wide[0, 0] == 64 * 40000.0 and torch.equal(out, wide.to(F16))


# ------------------------------------------------------------------------------------------------ their gradient

def gradient64(dy, x, counts):
    return torch.stack([dy[lo:hi].double().t() @ x[lo:hi].double() for lo, hi in spans(counts, dy.shape[0])])


def workspace(experts):
    return torch.full((ops.moe_ovl_grouped_matmul_workspace_bytes(experts),), 0xA5, dtype=torch.uint8, device="cuda")


def check_backward(dy, x, counts, out_dtype, exact=True, accumulate=False, pad=0):
    e, n, k = 1 if counts is None else len(counts), dy.shape[1], x.shape[1]
    full = torch.full((e + 2, n + 1, k + pad), 7.5, dtype=out_dtype, device="cuda")
    dw = full[1:e + 1, :n, :k]
    want = gradient64(dy, x, counts)
    if accumulate:
        before = whole(gen(e), (e, n, k), out_dtype)
        dw.copy_(before)
        want = want + before.double()
    st = status()
    ops.moe_ovl_grouped_matmul_backward(dy=dy, x=x, dweight=dw if counts is not None else dw[0], expert_counts=device_counts(counts), status=st,
                                        workspace=workspace(e), accumulate=accumulate)
    if exact:
        assert torch.equal(dw, want.to(out_dtype))
    else:
        m = max(hi - lo for lo, hi in spans(counts, dy.shape[0]))
        close(dw, want, U[out_dtype] * want.abs() + slack(m + 64, gradient64(dy.abs(), x.abs(), counts)) + FLOOR[out_dtype])
    keep = full.clone()
    keep[1:e + 1, :n, :k] = 7.5
    assert bool((keep == 7.5).all()) and not st.any()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("m,n,k", [(1, 8, 8), (1, 136, 264), (7, 40, 1000), (16, 128, 128), (63, 64, 72), (64, 256, 256), (65, 520, 136), (129, 1032, 640), (1000, 2048, 1032),
                                   (5000, 24, 16), (333, 4096, 256)])
def test_grouped_backward_of_one_matrix(m, n, k, dtype):
    g = gen(m + n)
    dy, x = whole(g, (m, n), dtype, pad=8 if m % 2 else 0), whole(g, (m, k), dtype, pad=16 if m % 3 else 0)
    check_backward(dy, x, None, F32, pad=1 if m % 2 else 0)
    check_backward(dy, x, None, dtype)
    check_backward(dy, x, None, F32, accumulate=True)


@gpu
@pytest.mark.parametrize("counts,n,k", COUNTS)
def test_grouped_backward(counts, n, k):
    m = sum(counts)
    for dtype in (BF16, F16):
        g = gen(m + n)
        dy, x = whole(g, (m, n), dtype), whole(g, (m, k), dtype)
        check_backward(dy, x, counts, F32)
        check_backward(dy, x, counts, dtype, accumulate=True)


@gpu
def test_grouped_backward_of_columns_that_are_no_multiple():
    """Odd n and k of matrices whose rows begin on 16 bytes; what lies between the rows is not a number."""
    g = gen(2)
    dy, x = whole(g, (150, 131), BF16, pad=5), whole(g, (150, 77), BF16, pad=3)
    dy._base[:, 131:] = NAN
    x._base[:, 77:] = INF
    check_backward(dy, x, [70, 0, 80], F32)


@gpu
def test_grouped_backward_of_normal_values():
    g = gen(3)
    for dtype in (BF16, F16):
        dy, x = normal(g, (3000, 264), dtype, 0.02), normal(g, (3000, 520), dtype)
        check_backward(dy, x, [1000, 0, 1777, 223], F32, exact=False)
        check_backward(dy, x, [1000, 0, 1777, 223], dtype, exact=False)


@gpu
def test_grouped_backward_does_not_look_at_other_rows():
    """The rows of other experts and those behind the last are NaN or infinite on both sides: an expert's own gradient is not."""
    g = gen(6)
    counts = [30, 33, 0, 1, 40, 64]
    for one in (0, 1, 3, 4, 5):
        dy, x = torch.full((200, 72), NAN, dtype=BF16, device="cuda"), torch.full((200, 136), INF, dtype=BF16, device="cuda")
        lo, hi = spans(counts, 200)[one]
        dy[lo:hi], x[lo:hi] = whole(g, (hi - lo, 72), BF16), whole(g, (hi - lo, 136), BF16)
        dw, st = torch.full((6, 72, 136), 9.0, device="cuda"), status()
        ops.moe_ovl_grouped_matmul_backward(dy=dy, x=x, dweight=dw, expert_counts=device_counts(counts), status=st, workspace=workspace(6))
        assert torch.equal(dw[one], gradient64(dy, x, counts)[one].float()) and not dw[2].any()


@gpu
def test_grouped_backward_counts_that_do_not_add_up_and_no_rows():
    g = gen(4)
    dy, x = whole(g, (90, 40), BF16), whole(g, (90, 136), BF16)
    for counts in ([20, 0, 30, 11], [50, 60, 70, 2147483647], [2147483647] * 4, [-5, 40, -2147483648, 10], [0, 0, 0, 0]):
        check_backward(dy, x, counts, F32)
    check_backward(dy[:0], x[:0], [0, 0], F32)
    check_backward(dy[:0], x[:0], None, BF16)
    check_backward(dy[:0], x[:0], [3, 0], F32, accumulate=True)


@gpu
def test_products_and_gradients_are_each_others():
    """sum(dout * f(a, b)) moved along random directions of a and of b, by the formula's gradients: the product is linear in each, so that differences have no error of their own.  Whole
    numbers throughout, exact in 32 bits."""
    g = gen(8)
    counts, k, n = [20, 0, 45, 5], 64, 40
    a, b, dout = whole(g, (70, k), BF16, 2), whole(g, (4, n, k), BF16, 2), whole(g, (70, n), BF16, 2)
    va, vb = whole(g, a.shape, BF16, 1), whole(g, b.shape, BF16, 1)
    st, dc = status(), device_counts(counts)

    def loss(a, b):
        out = torch.empty((70, n), device="cuda")
        ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, expert_counts=dc, status=st)
        return float((out.double() * dout.double()).sum())

    da, db = torch.empty((70, k), device="cuda"), torch.empty((4, n, k), device="cuda")
    ops.moe_ovl_grouped_matmul(a=dout, b=b, out=da, expert_counts=dc, transposed=True, status=st)
    ops.moe_ovl_grouped_matmul_backward(dy=dout, x=a, dweight=db, expert_counts=dc, status=st, workspace=workspace(4))
    assert loss(a + va, b) - loss(a - va, b) == 2 * float((da.double() * va.double()).sum())
    assert loss(a, b + vb) - loss(a, b - vb) == 2 * float((db.double() * vb.double()).sum())


# ------------------------------------------------------------------------------------------------ quantiser

def e4m3(v):
    """The nearest of e4m3 in 64 bits, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(1e-300))).clamp_min(-6) - 3)
    return (torch.round(v / step) * step).clamp(-448, 448)


def per_value(scale, shape, tiles):
    s = scale.double().repeat_interleave(128, -1)[..., :shape[-1]]
    return s.repeat_interleave(128, -2)[..., :shape[-2], :] if tiles else s


def largest64(v, tiles):
    p = torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 128, 0, -v.shape[-2] % 128 if tiles else 0)).unflatten(-1, (-1, 128)).amax(-1)
    return p.unflatten(-2, (-1, 128)).amax(-2) if tiles else p


def check_quant(x, gated=False, tiles=False, pad=0, shift=0):
    k = x.shape[-1] // 2 if gated else x.shape[-1]
    shape = (*x.shape[:-1], k)
    if x.dim() == 2:
        q8, full = guarded(x.shape[0], k, torch.int8, pad, shift)
        q = q8.view(F8)
    else:
        q = torch.empty(shape, dtype=F8, device="cuda")
    blocks = -(-k // 128)
    scale = torch.full((*shape[:-2], -(-shape[-2] // 128) if tiles else shape[-2], blocks), -1.0, device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale, gated=gated, tiles=tiles)
    v = x.double()
    if gated:
        gate, up = v[:, :k], v[:, k:]
        v = gate * torch.sigmoid(gate) * up
    most = largest64(v, tiles)
    spread = per_value(most, shape, tiles)
    t = torch.where(spread < 2.0 ** -100, 0.0, v * 448 / spread.clamp_min(1e-300))
    want = torch.where(most < 2.0 ** -100, 0.0, most / 448)
    # the gate is an exponential, a sum, a division and two products in 32 bits: within 2^-20, and the maximum with it; a 32-bit v itself loses 2^-23 of
    # its quotient; 16-bit ones nothing
    off = 2.0 ** -18 if gated else 2.0 ** -22 if x.dtype is F32 else 0.0
    close(scale, want, (2.0 ** -24 + off) * want)
    got = q.double()
    assert bool(((got >= e4m3(t - off * t.abs())) & (got <= e4m3(t + off * t.abs()))).all())
    if x.dim() == 2:
        assert untouched(full, q8)
    return q, scale


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("k", [1, 7, 8, 64, 100, 127, 128, 129, 136, 255, 256, 1000, 1408, 4096, 4099])
def test_block_quant(k, dtype):
    for case, (rows, pad, shift) in enumerate([(1, 0, 0), (3, 8, 0), (5, 3, 1), (131, 0, 0)]):
        g = gen(k * 10 + case)
        x, _ = guarded(rows, k, dtype, pad, shift)
        x.copy_(normal(g, (rows, k), dtype, 3.0))
        check_quant(x, pad=pad, shift=shift)
        check_quant(x, tiles=True, pad=pad, shift=shift)
        x, _ = guarded(rows, 2 * k, dtype, pad, shift)
        x.copy_(normal(g, (rows, 2 * k), dtype, 2.0))
        check_quant(x, gated=True, pad=pad, shift=shift)


@gpu
def test_block_quant_tiles_of_several_matrices():
    g = gen(1)
    for dtype in (BF16, F32):
        check_quant(normal(g, (3, 200, 264), dtype), tiles=True)
        check_quant(normal(g, (6, 130, 400), dtype)[::2, 1:, 3:300], tiles=True)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_block_quant_halves(dtype):
    """Values that lie exactly between two steps go to the even one, whatever the block's maximum: 7, 448 / 3 and the like are not powers of two."""
    steps = torch.arange(0, 127, device="cuda").to(torch.uint8).view(F8).double()
    mid = (steps[:-1] + steps[1:]) / 2
    for most in (448.0, 7.0, 1.75, 3.5, 14.0, 56.0, 0.875):
        x = torch.zeros((1, 128), dtype=torch.float64, device="cuda")
        x[0, :126] = mid * most / 448
        x[0, 127] = most
        x = x.to(dtype)
        q, scale = check_quant(x)
        assert float(q[0, 127]) == 448


@gpu
def test_block_quant_blocks_out_of_the_ordinary():
    """Zeros, values below the range of the scale, one large value, NaN, infinity, the type's ends: each block by itself."""
    x = torch.zeros((9, 256), device="cuda")
    x[:, 128:] = 1.0
    x[1, :128] = 2.0 ** -101
    x[2, 5] = 1e30
    x[3, 7] = NAN
    x[4, 9] = INF
    x[5, :128] = torch.finfo(F32).max
    x[6, :128] = -torch.finfo(F32).max
    x[6, 0] = 1.0
    x[7, 3] = 2.0 ** -100
    x[8, 3] = -INF
    q, scale = torch.empty((9, 256), dtype=F8, device="cuda"), torch.empty((9, 2), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale)
    q = q.float()
    assert bool((q[:, 128:] == 448).all()) and bool((scale[:, 1] == torch.tensor(1.0) / 448).all())
    assert not q[0, :128].any() and scale[0, 0] == 0 and not q[1, :128].any() and scale[1, 0] == 0
    assert q[2, 5] == 448 and q[2, :128].abs().sum() == 448
    for r in (3, 4, 8):
        assert not q[r, :128].any() and bool(scale[r, 0].isnan())
    assert bool((q[5, :128] == 448).all()) and q[6, 1] == -448 and q[6, 0] == 0 and bool(scale[5:7, 0].isfinite().all())
    assert q[7, 3] == 448 and scale[7, 0] > 0
    ops.moe_ovl_block_quant(x=x[:0], q=torch.empty((0, 256), dtype=F8, device="cuda"), scale=torch.empty((0, 2), device="cuda"))


@gpu
def test_block_quant_gate_at_its_ends():
    """Large negative gates give zero, large positive ones the product; infinities make NaN scales, not wrong values."""
    x = torch.ones((4, 256), device="cuda")
    x[0, :128] = -1000.0
    x[1, :128] = 1000.0
    x[2, 3] = NAN
    x[3, 3] = -INF
    q, scale = torch.empty((4, 128), dtype=F8, device="cuda"), torch.empty((4, 1), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale, gated=True)
    assert not q[0].float().any() and scale[0, 0] == 0 and bool((q[1].float() == 448).all()) and abs(float(scale[1, 0]) * 448 - 1000) < 1e-3
    assert bool(scale[2, 0].isnan()) and bool(scale[3, 0].isnan()) and not q[2:].float().any()      # -inf * 0 is not a number


# ------------------------------------------------------------------------------------------------ 8-bit floats

def block64(a, sa, b, sb, counts):
    b, sb = (b, sb) if b.dim() == 3 else (b[None], sb[None])
    av = a.double() * per_value(sa, a.shape, False)
    out = torch.zeros((a.shape[0], b.shape[1]), dtype=torch.float64, device="cuda")
    for e, (lo, hi) in enumerate(spans(counts, a.shape[0])):
        out[lo:hi] = av[lo:hi] @ (b[e].double() * per_value(sb[e], b[e].shape, True)).t()
    return out


def block_operands(g, m, n, k, experts=None, pad_a=0, pad_b=0, exact=True):
    """Whole numbers with powers of two as scales, or normal values with any."""
    lead = () if experts is None else (experts,)
    blocks = -(-k // 128)
    scales = lambda *s: torch.exp2(torch.randint(-2, 3, s, generator=g, device="cuda").float()) if exact else torch.rand(s, generator=g, device="cuda")  # noqa: E731
    values = lambda s, pad: whole(g, s, F8, pad=pad) if exact else normal(g, (*s[:-1], s[-1] + pad), F32, 60.0).clamp(-448, 448).to(F8)[..., :s[-1]]  # noqa: E731
    return values((m, k), pad_a), scales(m, blocks), values((*lead, n, k), pad_b), scales(*lead, -(-n // 128), blocks)


def check_block(a, sa, b, sb, counts, out_dtype, exact=True, pad=0, shift=0):
    m, n, k = a.shape[0], b.shape[-2], a.shape[1]
    out, full = guarded(m, n, out_dtype, pad, shift)
    st = status()
    ops.moe_ovl_block_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, expert_counts=device_counts(counts), status=st)
    want = block64(a, sa, b, sb, counts)
    covered = spans(counts, m)[-1][1]
    if exact:
        assert torch.equal(out[:covered], want[:covered].to(out_dtype))
    else:
        mag = lambda t: t.float().abs().to(F8)  # noqa: E731
        s = block64(mag(a), sa, mag(b), sb, counts)
        close(out[:covered], want[:covered], U[out_dtype] * want[:covered].abs() + slack(k + 128, s[:covered]) + FLOOR[out_dtype])
    assert untouched(full, out) and not st.any()
    if covered < m:
        assert bool((out[covered:].float() == 7.5).all())


@gpu
@pytest.mark.parametrize("m,n,k", [(1, 1, 16), (1, 5, 48), (2, 127, 128), (3, 128, 144), (16, 129, 256), (17, 300, 400), (31, 64, 1024), (33, 257, 2048), (64, 1000, 512),
                                   (65, 130, 272), (127, 256, 640), (128, 512, 4096), (129, 384, 1280), (200, 77, 16), (257, 513, 1040), (500, 2050, 1040), (1025, 768, 528),
                                   (1, 4096, 8192), (2000, 1500, 400), (4097, 640, 256), (300, 6000, 128)])
def test_block_matmul(m, n, k):
    g = gen(m + n)
    a, sa, b, sb = block_operands(g, m, n, k, pad_a=16 if m % 3 == 0 else 0, pad_b=32 if n % 3 == 0 else 0)
    check_block(a, sa, b, sb, None, F32, pad=5 if m % 2 else 0, shift=1 if n % 2 else 0)
    check_block(a, sa, b[None], sb[None], None, BF16)
    check_block(a, sa, b, sb, None, F16, pad=1)


@gpu
@pytest.mark.parametrize("counts,n,k", COUNTS)
def test_block_matmul_experts(counts, n, k):
    m, e, k = sum(counts), len(counts), (k + 15) // 16 * 16
    g = gen(m + n)
    a, sa, b, sb = block_operands(g, m, n, k, e)
    check_block(a, sa, b, sb, counts, F32)
    check_block(a, sa, b, sb, counts, BF16, pad=3)


@gpu
def test_block_matmul_of_normal_values():
    g = gen(5)
    for m, counts in ((7, None), (40, None), (300, None), (830, [300, 0, 17, 512, 1]), (30, [3, 20, 0, 2, 5])):
        for k in (144, 2048):
            a, sa, b, sb = block_operands(g, m, 264, k, None if counts is None else 5, exact=False)
            for dtype in (F32, BF16):
                check_block(a, sa, b, sb, counts, dtype, exact=False)


@gpu
def test_block_matmul_counts_that_do_not_add_up():
    g = gen(4)
    for rows in (90, 700):
        a, sa, b, sb = block_operands(g, rows, 140, 256, 4)
        for counts in ([20, 0, 30, 11], [50, 60, 70, 2147483647], [2147483647] * 4, [-5, 40, -2147483648, 10], [0, 0, 0, 0]):
            check_block(a, sa, b, sb, counts, F32)


@gpu
def test_block_matmul_keeps_what_is_not_a_number_to_itself():
    g = gen(7)
    for m, counts in ((60, [20, 5, 0, 30]), (600, [300, 70, 0, 200])):
        a, sa, b, sb = block_operands(g, m, 200, 144, 4, pad_a=16)
        a._base.view(torch.uint8)[:, 144:] = 0x7f
        covered = sum(counts)
        sa[covered:] = NAN
        sa[3, 1] = NAN
        sa[4, 0] = INF
        sb[2] = NAN
        out, st = torch.zeros((m, 200), device="cuda"), status()
        ops.moe_ovl_block_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, expert_counts=device_counts(counts), status=st)
        rows = [r for r in range(covered) if r not in (3, 4)]
        assert torch.equal(out[rows], block64(a, sa, b, sb, counts)[rows].float())
        assert bool(out[3].isnan().all()) and not bool(out[4].isfinite().any()) and not out[covered:].any()


@gpu
def test_block_matmul_of_quantised_values():
    """Quantiser and product together against the product of the values themselves: each operand is off by a step's half, 2^-4 of the value (or of the smallest normal one, 2^-6 of 448)."""
    g = gen(9)
    m, n, k = 130, 200, 400
    x, w = normal(g, (m, k), BF16), normal(g, (n, k), F32)
    qa, sa = check_quant(x)
    qb, sb = check_quant(w, tiles=True)
    out, st = torch.empty((m, n), device="cuda"), status()
    a8, b8 = torch.empty((m, k), dtype=F8, device="cuda"), torch.empty((n, k), dtype=F8, device="cuda")
    a8.copy_(qa), b8.copy_(qb)
    ops.moe_ovl_block_matmul(a=a8, a_scale=sa, b=b8, b_scale=sb, out=out, status=st)
    xa, wb = x.double().abs(), w.double().abs()
    ra, rb = xa / 16 + per_value(sa, x.shape, False) * 2.0 ** -10, wb / 16 + per_value(sb, w.shape, True) * 2.0 ** -10
    bound = ra @ wb.t() + xa @ rb.t() + ra @ rb.t()
    close(out, x.double() @ w.double().t(), bound * 1.0001)


# ------------------------------------------------------------------------------------------------ norm of gradients

def norm_of(grads):
    norm = torch.full((1,), -1.0, device="cuda")
    ops.moe_ovl_grad_norm(grads=grads, norm=norm, workspace=torch.full((ops.moe_ovl_grad_norm_workspace_bytes(len(grads)),), 0xFF, dtype=torch.uint8, device="cuda"))
    return norm


def check_clip(grads, max_norm, eps=1e-6):
    norm = norm_of(grads)
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    # 32 positive terms in 32 bits and one more addition, the rest in 64, then a root (half of that) and a rounding
    assert abs(float(norm) - want) <= (33 / 2 + 1) * 2.0 ** -24 * want * 1.01
    factor = torch.clamp(torch.tensor(max_norm, device="cuda") / (norm + eps), max=1.0)
    expected = [(t.float() * factor).to(t.dtype) for t in grads]
    out = [torch.full_like(t, 7.5) for t in grads]
    ops.moe_ovl_clip_grads(grads=grads, norm=norm, max_norm=max_norm, eps=eps, out=out)
    for o, w in zip(out, expected):
        assert torch.equal(o, w)
    ops.moe_ovl_clip_grads(grads=grads, norm=norm, max_norm=max_norm, eps=eps)
    for t, w in zip(grads, expected):
        assert torch.equal(t, w)


@gpu
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9])
def test_clip_grads_of_many_sizes(max_norm):
    g = gen(1)
    sizes = [0, 1, 2, 3, 7, 8, 9, 31, 255, 256, 257, 8191, 8192, 8193, 16384, 100001]
    check_clip([normal(g, (n,), (BF16, F16, F32)[i % 3], 0.1) for i, n in enumerate(sizes * 3)], max_norm)
    check_clip([normal(g, (5,), F32)], max_norm)
    for n in (131072, 131073, 262144, 262145):      # eight and sixteen chunks, and one value more
        check_clip([normal(g, (n,), F32)], max_norm)
        check_clip([normal(g, (n - 40000,), BF16), normal(g, (40000,), F16)], max_norm)
    check_clip([normal(g, (3, 0), F32)], max_norm)
    check_clip([], max_norm)


@gpu
def test_clip_grads_more_tensors_than_a_launch_holds():
    g = gen(2)
    flat = normal(g, (2500 * 41,), BF16)
    grads, at = [], 0
    for i in range(2500):                   # pieces of one buffer, beginning anywhere
        n = (i * 7) % 41
        grads.append(flat[at:at + n])
        at += n
    keep = flat[at:].clone()
    check_clip(grads, 1.0)
    assert torch.equal(flat[at:], keep)


@gpu
def test_clip_grads_into_buffers_that_begin_elsewhere():
    g = gen(3)
    for dtype in (BF16, F16, F32):
        src, dst = normal(g, (30007,), dtype), torch.full((30011,), 7.5, dtype=dtype, device="cuda")
        for a, b, n in ((0, 1, 30000), (1, 1, 20001), (3, 2, 9000), (5, 5, 1)):
            grads, out = [src[a:a + n]], [dst[b:b + n]]
            dst.fill_(7.5)
            norm = norm_of(grads)
            ops.moe_ovl_clip_grads(grads=grads, norm=norm, max_norm=0.25, out=out)
            factor = torch.clamp(torch.tensor(0.25, device="cuda") / (norm + 1e-6), max=1.0)
            assert torch.equal(out[0], (grads[0].float() * factor).to(dtype))
            assert bool((dst[:b] == 7.5).all()) and bool((dst[b + n:] == 7.5).all())


@gpu
def test_grad_norm_beyond_the_range_of_32_bit_squares():
    for value, dtype in ((1e30, F32), (1e-30, F32), (3e38, F32), (1e-40, F32), (1e30, BF16), (2.0 ** -24, F16), (65504.0, F16)):
        t = torch.zeros(20000, dtype=dtype, device="cuda")
        t[::7] = value
        want = math.sqrt(float((t.double() ** 2).sum()))
        got = float(norm_of([t, torch.zeros(9, device="cuda")]))
        assert got == INF if want > 3.5e38 else abs(got - want) <= 2e-6 * want + 1e-45, (value, dtype, got, want)
    assert float(norm_of([torch.zeros(1000, device="cuda")])) == 0.0
    assert float(norm_of([torch.zeros(1000, device="cuda"), torch.tensor([INF, 1.0], device="cuda")])) == INF
    assert math.isnan(float(norm_of([torch.zeros(1000, device="cuda"), torch.tensor([INF, NAN], dtype=BF16, device="cuda")])))


@gpu
def test_clip_grads_by_a_norm_that_is_no_number():
    t = torch.tensor([1.0, INF, -2.0], device="cuda")
    ops.moe_ovl_clip_grads(grads=[t], norm=norm_of([t]), max_norm=1.0)
    assert t[0] == 0 and bool(t[1].isnan()) and t[2] == 0
    t = torch.tensor([1.0, NAN, -2.0], device="cuda")
    ops.moe_ovl_clip_grads(grads=[t], norm=norm_of([t]), max_norm=1.0)
    assert bool(t.isnan().all())


@gpu
def test_clip_grads_of_zeros_and_into_themselves():
    t = torch.zeros(100, device="cuda")
    for max_norm, eps in ((0.0, 0.0), (1.0, 0.0), (0.0, 1e-6)):
        ops.moe_ovl_clip_grads(grads=[t], norm=norm_of([t]), max_norm=max_norm, eps=eps)
        assert not t.any()
    t = torch.full((100,), 3.0, dtype=BF16, device="cuda")
    ops.moe_ovl_clip_grads(grads=[t], norm=norm_of([t]), max_norm=15.0, eps=0.0, out=[t])
    assert bool((t == 1.5).all())


@gpu
def test_clip_grads_of_other_layouts():
    g = gen(4)
    a, b = normal(g, (33, 65), F32), normal(g, (4, 6, 10), BF16)
    check_clip([a.t(), b.permute(2, 0, 1)], 0.3)


# ------------------------------------------------------------------------------------------------ what they share

class Training:
    """One pass of an expert layer, forward and backward, with clipped gradients, all by the operators; the activation is torch's."""

    def __init__(s, rows=300, d=256, f=136, counts=(90, 0, 130, 60), seed=0):
        g = gen(seed)
        s.e, s.d, s.f = len(counts), d, f
        s.x, s.dy = normal(g, (rows, d), BF16), normal(g, (rows, d), BF16, 0.1)
        s.w1, s.w2 = normal(g, (s.e, 2 * f, d), BF16, d ** -0.5), normal(g, (s.e, d, f), BF16, f ** -0.5)
        s.counts, s.rows = device_counts(counts), rows
        new = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
        s.gu, s.h, s.y, s.dh, s.dgu, s.dx = new(rows, 2 * f), new(rows, f), new(rows, d), new(rows, f), new(rows, 2 * f), new(rows, d)
        s.dw1, s.dw2, s.norm = new(s.e, 2 * f, d, dtype=F32), new(s.e, d, f, dtype=F32), new(1, dtype=F32)
        s.q, s.scale = new(rows, f, dtype=F8), new(rows, -(-f // 128), dtype=F32)
        s.q2, s.scale2 = new(s.e, d, f, dtype=F8), new(s.e, -(-d // 128), -(-f // 128), dtype=F32)
        s.y8 = new(rows, d)
        s.st, s.ws = status(), workspace(s.e)
        s.ws2 = torch.zeros(ops.moe_ovl_grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")

    def run(s, x, stream=None):
        o = dict(expert_counts=s.counts, status=s.st, stream=stream)
        ops.moe_ovl_grouped_matmul(a=x, b=s.w1, out=s.gu, **o)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            gate, up = s.gu[:, :s.f].float(), s.gu[:, s.f:].float()
            sig = torch.sigmoid(gate)
            s.h.copy_(gate * sig * up)
        ops.moe_ovl_grouped_matmul(a=s.h, b=s.w2, out=s.y, **o)
        ops.moe_ovl_grouped_matmul(a=s.dy, b=s.w2, out=s.dh, transposed=True, **o)
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            dh = s.dh.float()
            s.dgu[:, :s.f].copy_(dh * up * sig * (1 + gate * (1 - sig)))
            s.dgu[:, s.f:].copy_(dh * gate * sig)
        ops.moe_ovl_grouped_matmul(a=s.dgu, b=s.w1, out=s.dx, transposed=True, **o)
        ops.moe_ovl_grouped_matmul_backward(dy=s.dgu, x=x, dweight=s.dw1, workspace=s.ws, **o)
        ops.moe_ovl_grouped_matmul_backward(dy=s.dy, x=s.h, dweight=s.dw2, workspace=s.ws, **o)
        ops.moe_ovl_grad_norm(grads=[s.dw1, s.dw2], norm=s.norm, workspace=s.ws2, stream=stream)
        ops.moe_ovl_clip_grads(grads=[s.dw1, s.dw2], norm=s.norm, max_norm=0.5, stream=stream)
        ops.moe_ovl_block_quant(x=s.gu, q=s.q, scale=s.scale, gated=True, stream=stream)
        ops.moe_ovl_block_quant(x=s.w2, q=s.q2, scale=s.scale2, tiles=True, stream=stream)
        if s.f % 16 == 0:
            ops.moe_ovl_block_matmul(a=s.q, a_scale=s.scale, b=s.q2, b_scale=s.scale2, out=s.y8, **o)
        return [t.clone() for t in (s.y, s.dx, s.dw1, s.dw2, s.norm, s.q.view(torch.uint8), s.scale, s.y8)]


@gpu
def test_streams_and_graph_capture():
    """All of them on another stream, and captured once and replayed with new inputs: the same bits as direct calls."""
    a, b = Training(f=144), Training(f=144)
    x2 = normal(gen(99), a.x.shape, BF16)
    direct, direct2 = a.run(a.x), a.run(x2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pass
    other = b.run(b.x, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for got, want in zip([b.y, b.dx, b.dw1, b.dw2, b.norm], direct):
        assert torch.equal(got, want)
    del other
    c = Training(f=144)
    x = c.x.clone()
    c.run(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.run(x)
    for new, want in ((a.x, direct), (x2, direct2), (a.x, direct)):
        x.copy_(new)
        graph.replay()
        for got, w in zip(out, want):
            assert torch.equal(got, w)
    assert not c.st.any()


@gpu
def test_two_streams_at_once():
    """Two training passes side by side, each with workspaces and a status of its own, give the bits of each alone."""
    a, b = Training(seed=1), Training(rows=700, counts=(0, 300, 100, 299), seed=2)
    want = [a.run(a.x)[:5], b.run(b.x)[:5]]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s in zip((a, b), streams):
            t.run(t.x, stream=s)
    torch.cuda.synchronize()
    for t, w in zip((a, b), want):
        for got, ref in zip([t.y, t.dx, t.dw1, t.dw2, t.norm], w):
            assert torch.equal(got, ref)
        assert not t.st.any()


@gpu
def test_values_at_the_ends_of_the_types():
    """Subnormal operands, exact in products and sums: 16-bit floats and e4m3 (2^-9), and the largest values."""
    st = status()
    for dtype, small, large in ((F16, 2.0 ** -24, 2.0 ** 10), (BF16, 2.0 ** -133, 2.0 ** 100), (F16, 65504.0, 2.0 ** -8), (BF16, 2.0 ** 127, 2.0 ** -120)):
        a = torch.zeros((3, 64), dtype=dtype, device="cuda")
        a[0], a[1, ::2], a[2, 7] = small, -small, small
        b = torch.full((8, 64), large, dtype=dtype, device="cuda")
        for transposed, w in ((False, b), (True, b.t().contiguous())):
            out = torch.empty((3, 8), device="cuda")
            ops.moe_ovl_grouped_matmul(a=a, b=w, out=out, transposed=transposed, status=st)
            assert torch.equal(out, product64(a, w, None, transposed).float())
    for m in (3, 200):
        a, b = torch.zeros((m, 256), dtype=F8, device="cuda"), torch.full((130, 256), 448.0, device="cuda").to(F8)
        a.view(torch.uint8)[0], a.view(torch.uint8)[1, ::3], a.view(torch.uint8)[2] = 1, 0x87, 0x7e          # 2^-9, -7 * 2^-9, 448
        sa, sb = torch.full((m, 2), 2.0 ** 40, device="cuda"), torch.full((2, 2), 2.0 ** -60, device="cuda")
        check_block(a, sa, b, sb, None, F32)


@gpu
def test_experts_that_interleave():
    """Matrices whose rows lie between each other's (k or n first in memory): read from there, and written there."""
    g = gen(21)
    counts, n, k = [20, 0, 33], 72, 136
    a = whole(g, (53, k), BF16)
    b = whole(g, (n, 3, k), BF16).transpose(0, 1)                                 # [3, n, k]
    check_grouped(a, b, counts, False, F32)
    check_grouped(a, whole(g, (k, 3, n), BF16).transpose(0, 1), counts, True, F32)
    dy = whole(g, (53, n), BF16)
    full, st = torch.full((n, 3, k), 7.5, device="cuda"), status()
    ops.moe_ovl_grouped_matmul_backward(dy=dy, x=a, dweight=full.transpose(0, 1), expert_counts=device_counts(counts), status=st, workspace=workspace(3))
    assert torch.equal(full.transpose(0, 1), gradient64(dy, a, counts).float())
    a8, sa, b8, sb = block_operands(g, 53, n, 144, 3)
    check_block(a8, sa, b8.transpose(0, 1).contiguous().transpose(0, 1), sb, counts, F32)
    x = normal(g, (200, 3, 256), F32).transpose(0, 1)
    q, scale = torch.empty((200, 3, 256), dtype=F8, device="cuda").transpose(0, 1), torch.empty((3, 2, 2), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale, tiles=True)
    flat = torch.empty((3, 200, 256), dtype=F8, device="cuda")
    again = torch.empty_like(scale)
    ops.moe_ovl_block_quant(x=x.contiguous(), q=flat, scale=again, tiles=True)
    assert torch.equal(q.contiguous().view(torch.uint8), flat.view(torch.uint8)) and torch.equal(scale, again)


@gpu
def test_offsets_beyond_32_bits():
    """Rows and matrices that lie so far apart that element and byte offsets pass 32 bits."""
    g = gen(22)
    far, k, n = 1_500_000_016, 64, 72

    def spread(shape, dtype, strides):
        full = torch.empty(sum((d - 1) * s for d, s in zip(shape, strides)) + 1, dtype=dtype, device="cuda")
        return full.as_strided(shape, strides)

    a, out = spread((3, k), BF16, (far, 1)), spread((3, n), BF16, (far, 1))
    a.copy_(whole(g, (3, k), BF16))
    b = spread((3, n, k), BF16, (2 * far, k, 1))
    b.copy_(whole(g, (3, n, k), BF16))
    counts, st = device_counts([1, 0, 2]), status()
    ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, expert_counts=counts, status=st)
    assert torch.equal(out, product64(a, b, [1, 0, 2]).to(BF16))
    dy = whole(g, (3, n), BF16)
    ops.moe_ovl_grouped_matmul_backward(dy=dy, x=a, dweight=b, expert_counts=counts, status=st, workspace=workspace(3))      # written where the weights were
    assert torch.equal(b, gradient64(dy, a, [1, 0, 2]).to(BF16)) and not st.any()
    del b
    x = spread((3, 2 * 144), BF16, (far, 1))
    x.copy_(normal(g, (3, 2 * 144), BF16))
    q, scale = spread((3, 144), F8, (far, 1)), torch.empty((3, 2), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale, gated=True)
    near, again = torch.empty((3, 144), dtype=F8, device="cuda"), torch.empty_like(scale)
    ops.moe_ovl_block_quant(x=x.contiguous(), q=near, scale=again, gated=True)
    assert torch.equal(q.contiguous().view(torch.uint8), near.view(torch.uint8)) and torch.equal(scale, again)
    w, sw = whole(g, (n, 144), F8), torch.ones((1, 2), device="cuda")
    ops.moe_ovl_block_matmul(a=q, a_scale=scale, b=w, b_scale=sw, out=out, status=st)
    dense = torch.empty((3, n), dtype=BF16, device="cuda")
    ops.moe_ovl_block_matmul(a=near, a_scale=scale, b=w, b_scale=sw, out=dense, status=st)
    assert torch.equal(out, dense)
    del a, out, x, q
    big = torch.zeros(2 ** 31 + 77, dtype=BF16, device="cuda")
    big[-5:], big[2 ** 31 - 3] = 3.0, 4.0
    assert abs(float(norm_of([big])) - math.sqrt(5 * 9 + 16)) < 1e-5
    ops.moe_ovl_clip_grads(grads=[big], norm=torch.ones(1, device="cuda"), max_norm=0.5, eps=0.0)
    assert big[-5:].tolist() == [1.5] * 5 and big[2 ** 31 - 3] == 2.0 and float(big.sum(dtype=torch.float64)) == 9.5


@gpu
def test_most_rows():
    """2^31 - 1 rows: the last ones are found, multiplied, and end where the experts' counts say."""
    rows, e = 2 ** 31 - 1, 2
    counts = device_counts([rows - 70, 60])
    x = torch.zeros((rows, 8), dtype=F16, device="cuda")
    x[-70:-10, 0] = torch.arange(60, device="cuda").half()
    x[-10:] = NAN
    x[5, 1] = 2.0
    w, st = torch.zeros((e, 1, 8), dtype=F16, device="cuda"), status()
    w[0], w[1] = 1.0, 3.0
    out = torch.zeros((rows, 1), dtype=F16, device="cuda")
    ops.moe_ovl_grouped_matmul(a=x, b=w, out=out, expert_counts=counts, status=st)
    assert torch.equal(out[-70:-10, 0], 3 * torch.arange(60, device="cuda").half()) and not out[-10:].any() and out[5] == 2.0
    dw = torch.empty((e, 8, 8), device="cuda")
    ops.moe_ovl_grouped_matmul_backward(dy=x, x=x, dweight=dw, expert_counts=counts, status=st, workspace=workspace(e))
    assert not st.any()
    want = torch.zeros((e, 8, 8), device="cuda")
    want[0, 1, 1], want[1, 0, 0] = 4.0, float((torch.arange(60) ** 2).sum())
    assert torch.equal(dw, want)
    del out
    q, scale = torch.empty((rows, 8), dtype=F8, device="cuda"), torch.empty((rows, 1), device="cuda")
    ops.moe_ovl_block_quant(x=x, q=q, scale=scale)
    assert scale[5, 0] == torch.tensor(2.0) / 448 and scale[-11, 0] == torch.tensor(59.0) / 448 and bool(scale[-10:].isnan().all()) and not scale[6:1000].any()
    assert q[-11].float().tolist() == [448.0] + [0.0] * 7


@gpu
def test_same_bits_every_time():
    t = Training(rows=5000, d=512, f=256, counts=(1700, 0, 3000, 300))
    first = t.run(t.x)
    for _ in range(3):
        for got, want in zip(t.run(t.x), first):
            assert torch.equal(got, want)


@gpu
def test_bounded_waits_run_out():
    """Test hook: no tile is loaded.  Every wait gives up, the status says so, and the next call on a cleared status is right."""
    g = gen(8)
    give_up = dict(wait_timeout_us=3000, flags=ops.FLAG_MATMUL_TEST_NO_LOADS)
    for m, counts in ((3, None), (700, None), (300, [100, 0, 200]), (20, [10, 10]), (2000, [900, 1100])):
        e = 1 if counts is None else len(counts)
        for transposed in (False, True):
            a, b = whole(g, (m, 512), BF16), whole(g, (e, 512, 1000) if transposed else (e, 1000, 512), BF16)
            out, st = torch.empty((m, 1000), dtype=BF16, device="cuda"), status()
            ops.moe_ovl_grouped_matmul(a=a, b=b, out=out, status=st, expert_counts=device_counts(counts), transposed=transposed, **give_up)
            torch.cuda.synchronize()
            assert int(st[0]) == B.ERR_TIMEOUT
            check_grouped(a, b, counts, transposed, F32)
        dy, st = whole(g, (m, 1000), BF16), status()
        ops.moe_ovl_grouped_matmul_backward(dy=dy, x=a, dweight=torch.empty((e, 1000, 512), device="cuda"), status=st, expert_counts=device_counts(counts), workspace=workspace(e),
                                            **give_up)
        torch.cuda.synchronize()
        assert int(st[0]) == B.ERR_TIMEOUT
        check_backward(dy, a, counts, F32)
        a, sa, b, sb = block_operands(g, m, 1000, 512, e if counts is not None else None)
        st = status()
        ops.moe_ovl_block_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=torch.empty((m, 1000), device="cuda"), status=st, expert_counts=device_counts(counts), **give_up)
        torch.cuda.synchronize()
        assert int(st[0]) == B.ERR_TIMEOUT
        check_block(a, sa, b, sb, counts, F32)


@gpu
def test_refusals_of_the_python_calls():
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    st, c4 = status(), torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(a=z(6, 64), b=z(4, 32, 64), out=z(6, 32), status=st, expert_counts=c4)
    ops.moe_ovl_grouped_matmul(**ok)
    for wrong in (dict(a=z(6, 72)), dict(a=z(6, 64, dtype=F16)), dict(a=z(6, 64, dtype=F32)), dict(b=z(4, 64, 32)), dict(b=z(32, 64)), dict(expert_counts=None),
                  dict(expert_counts=c4.long()), dict(expert_counts=c4[:3]), dict(out=z(6, 33)), dict(out=z(6, 32, dtype=F16)), dict(status=st[:3]), dict(a=z(6, 64).cpu()),
                  dict(a=z(64, 6).t()), dict(b=z(4, 64, 32).transpose(1, 2)), dict(out=z(32, 6).t()), dict(transposed=True)):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_grouped_matmul(**{**ok, **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    for wrong in (dict(a=z(6, 65)[:, 1:]), dict(a=z(6, 68)[:, :64]), dict(b=z(4, 32, 68)[..., :64])):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_grouped_matmul(**{**ok, **wrong})
        assert err.value.code == B.ERR_UNSUPPORTED
    ok = dict(dy=z(6, 32), x=z(6, 64), dweight=z(4, 32, 64, dtype=F32), status=st, expert_counts=c4, workspace=workspace(4))
    ops.moe_ovl_grouped_matmul_backward(**ok)
    for wrong in (dict(dy=z(7, 32)), dict(x=z(6, 64, dtype=F16)), dict(dweight=z(4, 64, 32)), dict(dweight=z(4, 32, 64, dtype=F16)), dict(expert_counts=None),
                  dict(dweight=z(1, 32, 64).expand(4, 32, 64)), dict(workspace=workspace(4)[::2])):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_grouped_matmul_backward(**{**ok, **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    for wrong in (dict(workspace=workspace(3)), dict(workspace=torch.zeros(2048, dtype=torch.uint8, device="cuda")[64:])):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_grouped_matmul_backward(**{**ok, **wrong})
        assert err.value.code == B.ERR_WORKSPACE
    ok = dict(x=z(6, 256), q=z(6, 256, dtype=F8), scale=z(6, 2, dtype=F32))
    ops.moe_ovl_block_quant(**ok)
    for wrong in (dict(x=z(6, 257)), dict(q=z(6, 256, dtype=torch.int8)), dict(scale=z(6, 3, dtype=F32)), dict(scale=z(6, 2)), dict(tiles=True), dict(gated=True), dict(x=z(6, 0)),
                  dict(x=z(6, 256, dtype=torch.float64)), dict(x=z(2, 3, 256)), dict(x=z(256, 6).t())):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_block_quant(**{**ok, **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    ok = dict(a=z(6, 64, dtype=F8), a_scale=z(6, 1, dtype=F32), b=z(4, 32, 64, dtype=F8), b_scale=z(4, 1, 1, dtype=F32), out=z(6, 32), status=st, expert_counts=c4)
    ops.moe_ovl_block_matmul(**ok)
    for wrong in (dict(a=z(6, 64, dtype=torch.float8_e5m2)), dict(b=z(4, 32, 64)), dict(a_scale=z(6, dtype=F32)), dict(b_scale=z(4, 1, 2, dtype=F32)), dict(out=z(6, 32, dtype=F8)),
                  dict(expert_counts=None)):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_block_matmul(**{**ok, **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    with pytest.raises(B.MoeOvlError) as err:
        ops.moe_ovl_block_matmul(**{**ok, "a": z(6, 72, dtype=F8)[:, :64]})
    assert err.value.code == B.ERR_UNSUPPORTED
    t, norm, ws = z(10, dtype=F32), z(1, dtype=F32), z(ops.moe_ovl_grad_norm_workspace_bytes(2), dtype=torch.uint8)
    ops.moe_ovl_grad_norm(grads=[t], norm=norm, workspace=ws)
    for wrong in (dict(grads=[t, t]), dict(grads=[t[::2]]), dict(grads=[t.cpu()]), dict(grads=[t.double()]), dict(norm=z(2, dtype=F32)), dict(norm=z(1))):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_grad_norm(**{**dict(grads=[t], norm=norm, workspace=ws), **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    with pytest.raises(B.MoeOvlError) as err:
        ops.moe_ovl_grad_norm(grads=[t], norm=norm, workspace=ws[:8])
    assert err.value.code == B.ERR_WORKSPACE
    for wrong in (dict(out=[]), dict(out=[t[:9]]), dict(out=[z(10)]), dict(max_norm=-1.0), dict(max_norm=NAN), dict(eps=-1.0)):
        with pytest.raises(B.MoeOvlError) as err:
            ops.moe_ovl_clip_grads(**{**dict(grads=[t], norm=norm, max_norm=1.0), **wrong})
        assert err.value.code == B.ERR_INVALID_ARG, wrong
    w = z(4, 32, 64).requires_grad_()
    with pytest.warns(UserWarning, match="records nothing"):
        ops.moe_ovl_grouped_matmul(a=z(6, 64), b=w, out=z(6, 32), status=st, expert_counts=c4)
    with torch.no_grad(), warnings.catch_warnings():
        warnings.simplefilter("error")
        ops.moe_ovl_grouped_matmul(a=z(6, 64), b=w, out=z(6, 32), status=st, expert_counts=c4)


# ------------------------------------------------------------------------------------------------ without a GPU

def refused(name, kind, good, wrong, code=B.ERR_INVALID_ARG):
    """Calls with one field changed each; none of them reaches a device."""
    fields = [f for f, _ in kind._fields_]
    for change in wrong:
        values = {**dict.fromkeys(fields, 0), **good, **change}
        args = kind(*[values[f] for f in fields])
        if "struct_size" not in change:
            args.struct_size = ctypes.sizeof(kind)
        assert getattr(B.load(), name)(ctypes.byref(args)) == code, change


def test_refusals_of_the_c_calls():
    p = 1 << 20
    for name in ("moe_ovl_grouped_matmul", "moe_ovl_grouped_matmul_backward", "moe_ovl_block_quant", "moe_ovl_block_matmul", "moe_ovl_grad_norm", "moe_ovl_clip_grads"):
        assert getattr(B.load(), name)(None) == B.ERR_INVALID_ARG
    common = [dict(struct_size=8), dict(device=-1), dict(rows=-1), dict(n=0), dict(k=0), dict(num_experts=-1), dict(flags=2), dict(wait_timeout_us=-1), dict(expert_counts=0),
              dict(num_experts=0), dict(status=0), dict(status=p + 2), dict(expert_counts=p + 1)]
    good = dict(rows=9, n=64, k=64, num_experts=2, a=p, b=p, expert_counts=p, out=p, status=p, a_stride=64, b_stride=64, b_expert_stride=4096, out_stride=64)
    refused("moe_ovl_grouped_matmul", ops.GroupedMatmulArgs, good, common + [dict(dtype=2), dict(dtype=3), dict(out_dtype=1), dict(out_dtype=5), dict(transposed=2), dict(a=0), dict(b=0),
            dict(out=0), dict(a=p + 1), dict(out=p + 1), dict(a_stride=63), dict(b_stride=63), dict(out_stride=63), dict(b_expert_stride=0)])
    refused("moe_ovl_grouped_matmul", ops.GroupedMatmulArgs, good, [dict(num_experts=1025), dict(n=1 << 25), dict(k=1 << 25, a_stride=1 << 25), dict(a=p + 8), dict(b=p + 2), dict(a_stride=68),
            dict(b_stride=65), dict(b_expert_stride=4100), dict(a_stride=1 << 31), dict(out_stride=1 << 31), dict(b_expert_stride=1 << 39)], B.ERR_UNSUPPORTED)
    good = dict(rows=9, n=64, k=64, num_experts=2, out_dtype=2, dy=p, x=p, expert_counts=p, dweight=p, status=p, workspace=p, workspace_bytes=4096, dy_stride=64, x_stride=64, dweight_stride=64,
                dweight_expert_stride=4096)
    refused("moe_ovl_grouped_matmul_backward", ops.GroupedMatmulBackwardArgs, good, common + [dict(dtype=2), dict(out_dtype=1), dict(accumulate=2), dict(dy=0), dict(x=0), dict(dweight=0),
            dict(dy=p + 1), dict(dweight=p + 2), dict(dy_stride=63), dict(x_stride=63), dict(dweight_stride=63), dict(dweight_expert_stride=0)])
    refused("moe_ovl_grouped_matmul_backward", ops.GroupedMatmulBackwardArgs, good, [dict(num_experts=1025), dict(n=1 << 25), dict(dy=p + 8), dict(x=p + 2), dict(dy_stride=68),
            dict(x_stride=1 << 31), dict(dweight_expert_stride=1 << 39)], B.ERR_UNSUPPORTED)
    refused("moe_ovl_grouped_matmul_backward", ops.GroupedMatmulBackwardArgs, good, [dict(workspace=0), dict(workspace=p + 64), dict(workspace_bytes=519)], B.ERR_WORKSPACE)
    good = dict(rows=9, depth=1, k=64, x=p, q=p, scale=p, x_stride=64, q_stride=64)
    refused("moe_ovl_block_quant", ops.BlockQuantArgs, good, [dict(struct_size=8), dict(device=-1), dict(depth=0), dict(depth=2), dict(rows=-1), dict(k=0), dict(dtype=3), dict(gated=2),
            dict(tiles=2), dict(gated=1, tiles=1, x_stride=128), dict(flags=1), dict(x=0), dict(q=0), dict(scale=0), dict(scale=p + 1), dict(x=p + 1), dict(x_stride=63), dict(q_stride=63),
            dict(gated=1), dict(tiles=1, depth=2)])
    refused("moe_ovl_block_quant", ops.BlockQuantArgs, good, [dict(k=1 << 25), dict(x_stride=1 << 31), dict(tiles=1, rows=65536 * 128), dict(tiles=1, depth=65536, x_far=64, q_far=64)],
            B.ERR_UNSUPPORTED)
    good = dict(rows=9, n=64, k=64, num_experts=2, a=p, a_scale=p, b=p, b_scale=p, expert_counts=p, out=p, status=p, a_stride=64, b_stride=64, b_expert_stride=4096, out_stride=64)
    refused("moe_ovl_block_matmul", ops.BlockMatmulArgs, good, common + [dict(out_dtype=3), dict(a=0), dict(a_scale=0), dict(b=0), dict(b_scale=0), dict(out=0), dict(a_scale=p + 2), dict(out=p + 1),
            dict(a_stride=63), dict(b_stride=63), dict(out_stride=63), dict(b_expert_stride=0)])
    refused("moe_ovl_block_matmul", ops.BlockMatmulArgs, good, [dict(num_experts=1025), dict(n=1 << 25), dict(a=p + 8), dict(b=p + 1), dict(a_stride=72), dict(b_stride=72),
            dict(b_expert_stride=4104), dict(out_stride=1 << 31), dict(b_expert_stride=1 << 40)], B.ERR_UNSUPPORTED)
    at, sizes, kinds = (ctypes.c_uint64 * 2)(p, p + 64), (ctypes.c_int64 * 2)(4, 8), (ctypes.c_int32 * 2)(0, 2)
    address = ctypes.addressof
    good = dict(num_tensors=2, grads=address(at), sizes=address(sizes), dtypes=address(kinds), norm=p, workspace=p, workspace_bytes=1 << 16, max_norm=1.0)
    bad = [dict(struct_size=8), dict(device=-1), dict(num_tensors=-1), dict(flags=1), dict(norm=0), dict(norm=p + 2), dict(grads=0), dict(sizes=0), dict(dtypes=0),
           dict(dtypes=address((ctypes.c_int32 * 2)(0, 3))), dict(sizes=address((ctypes.c_int64 * 2)(4, -1))), dict(grads=address((ctypes.c_uint64 * 2)(p, 0))),
           dict(grads=address((ctypes.c_uint64 * 2)(p + 1, p)))]
    keep = [(ctypes.c_int32 * 2)(0, 3), (ctypes.c_int64 * 2)(4, -1), (ctypes.c_uint64 * 2)(p, 0), (ctypes.c_uint64 * 2)(p + 1, p), (ctypes.c_int64 * 2)(4, 1 << 43)]
    bad[9:] = [dict(dtypes=address(keep[0])), dict(sizes=address(keep[1])), dict(grads=address(keep[2])), dict(grads=address(keep[3]))]
    refused("moe_ovl_grad_norm", ops.GradsArgs, good, bad)
    refused("moe_ovl_grad_norm", ops.GradsArgs, good, [dict(workspace=0), dict(workspace_bytes=100), dict(workspace=p + 4)], B.ERR_WORKSPACE)
    refused("moe_ovl_clip_grads", ops.GradsArgs, good, bad + [dict(max_norm=-1.0), dict(max_norm=NAN), dict(eps=-1.0), dict(eps=NAN), dict(out=address(keep[2]))])
    for name in ("moe_ovl_grad_norm", "moe_ovl_clip_grads"):
        refused(name, ops.GradsArgs, good, [dict(sizes=address(keep[4]))], B.ERR_UNSUPPORTED)


def test_workspaces_and_limits():
    assert ops.moe_ovl_grouped_matmul_workspace_bytes(0) == ops.moe_ovl_grouped_matmul_workspace_bytes(1) == 260
    assert ops.moe_ovl_grouped_matmul_workspace_bytes(ops.MAX_GROUPS) == 260 * ops.MAX_GROUPS
    assert ops.moe_ovl_grad_norm_workspace_bytes(0) == ops.moe_ovl_grad_norm_workspace_bytes(960) < ops.moe_ovl_grad_norm_workspace_bytes(961)
    for call, n, code in ((ops.moe_ovl_grouped_matmul_workspace_bytes, -1, B.ERR_INVALID_ARG), (ops.moe_ovl_grouped_matmul_workspace_bytes, 1025, B.ERR_UNSUPPORTED),
                          (ops.moe_ovl_grad_norm_workspace_bytes, -1, B.ERR_INVALID_ARG), (ops.moe_ovl_grad_norm_workspace_bytes, 65537, B.ERR_UNSUPPORTED)):
        with pytest.raises(B.MoeOvlError) as err:
            call(n)
        assert err.value.code == code


def test_dense_layouts():
    t = torch.empty(4, 6, 10)
    assert all(map(ops._dense, (t, t.permute(2, 0, 1), t[:, :, :1][:1, :1], t[:0], torch.empty(5, 1, 3).transpose(0, 1))))
    assert not any(map(ops._dense, (t[:, ::2], t[..., :9], t[:1].expand(2, 6, 10))))
