"""The operators around the expert layer at the edges of what they accept: values half-way between two steps, logits at the ends of
their type, the widest rows, the longest matrices, waits that give up while copies are under way.

U, FLOOR and the comparison are those of test_ops; a tolerance that is not derived there is derived at its test.
"""
import math
import warnings

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


def usable64(logits):
    """Logits as the router uses them, in 64 bits: +inf is the largest finite value, NaN is -inf."""
    z = logits.double()
    return torch.where(z.isnan(), -math.inf, z).clamp_max(3.4028234663852886e38)


@gpu
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("e,k", [(40, 6), (5, 2), (300, 8), (1024, 4)])
def test_route_gradient_of_rows_at_the_ends_of_the_type(e, k, dtype, score, renorm):
    """Rows that a mask fills with the type's lowest value, far-away rows, ties of infinities, rows with nothing left."""
    g = gen(e + k)
    low, inf = torch.finfo(dtype).min, math.inf
    far = -1e4 if dtype is F16 else -1e10
    z = normal(g, (16, e), dtype)
    z[0] = low
    z[1] = far
    z[2, 1] = z[2, 3] = inf
    z[3] = -inf
    z[4] = float("nan")
    z[5, 2:] = low
    z[6, 2:] = -inf
    z[7] = -low
    z[8] = -far
    z[9] = far + normal(g, (e,), F32, abs(far) * 1e-2).to(dtype)
    z[10, ::2] = low
    z[11, 4] = -low
    z[12, 0] = inf
    z[12, 1:] = -inf
    expert, gate, _ = call_route(z, k, score=score, renorm=renorm)
    assert bool(gate.isfinite().all())
    dgate = torch.randn((16, k), generator=g, device="cuda")
    out = torch.empty_like(z)
    ops.moe_ovl_route_backward(logits=z, expert=expert, dgate=dgate, dlogits=out, score=ops.SCORES[score], renormalise=renorm)
    # the definition, with rows that are masked throughout giving 0
    u = usable64(z)
    live = expert >= 0
    at = expert.long().clamp_min(0)
    if score == "softmax":
        top = u.amax(1, keepdim=True)
        p = torch.where(u > -inf, torch.exp(u - torch.where(top > -inf, top, 0.0)), 0.0)
        total = p.sum(1, keepdim=True)
        p = torch.where(total > 0, p / total, 0.0)
        slope = torch.ones_like(p)
    else:
        p, slope = torch.sigmoid(u), torch.sigmoid(-u)
    s, d = torch.where(live, p.gather(1, at), 0.0), dgate.double()
    if renorm:
        if score == "softmax":                              # of the chosen logits
            c = torch.where(live, u.gather(1, at), -inf)
            top = c.amax(1, keepdim=True)
            s = torch.where(c > -inf, torch.exp(c - torch.where(top > -inf, top, 0.0)), 0.0)
        # scores that 32 bits do not hold are 0, and gates of a row without a sum are 0
        s = torch.where(s < 2.0 ** -126, 0.0, s)
        total = s.sum(1, keepdim=True)
        s = torch.where(total > 0, s / total, 0.0)
    dot = (d * s).sum(1, keepdim=True) if renorm or score == "softmax" else 0.0
    mine = s * (d - dot) * slope.gather(1, at)
    want = torch.where(live, mine, 0.0)
    dense = torch.zeros_like(u)
    if score == "softmax" and not renorm:
        dense = -p * dot
    for j in range(k):
        rows = live[:, j].nonzero().squeeze(1)
        dense[rows, at[rows, j]] = want[rows, j]
    size = (d.abs() * s).sum(1, keepdim=True)
    bound = 1e-5 * (p * size if score == "softmax" and not renorm else torch.zeros_like(p))
    reach = 1e-5 * s * (d.abs() + size) * slope.gather(1, at)
    for j in range(k):
        rows = live[:, j].nonzero().squeeze(1)
        bound[rows, at[rows, j]] += reach[rows, j]
    assert bool(out.isfinite().all())
    close(out, dense, U[dtype] * dense.abs() + bound + FLOOR[dtype] + 1e-37)   # 1e-37: scores below the normal range


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_sigmoid_gradient_of_large_logits(dtype, renorm):
    """s (1 - s) of logits from -30 to 30 to its own relative accuracy.  Both factors come of one exp to 2 ulp, a sum, a quotient and a product; with
    the quotient by the sum of up to 8 scores, the sum over them and four products less than 60 roundings of 2^-24 = 3.6e-6, of the
    magnitudes (1 - s) w (|d| + sum |d| w); 1e-5 as in test_ops."""
    g = gen(13)
    for e, k in ((5, 2), (64, 8), (300, 4)):
        z = ((torch.rand((50, e), generator=g, device="cuda") * 60 - 30)).to(dtype)
        expert = torch.stack([torch.randperm(e, generator=g, device="cuda")[:k] for _ in range(50)]).to(torch.int32)
        dgate = torch.randn((50, k), generator=g, device="cuda")
        out = torch.empty_like(z)
        ops.moe_ovl_route_backward(logits=z, expert=expert, dgate=dgate, dlogits=out, score=ops.SCORE_SIGMOID, renormalise=renorm)
        at, d = expert.long(), dgate.double()
        l = z.double().gather(1, at)
        w, slope = torch.sigmoid(l), torch.sigmoid(-l)
        dot = size = torch.zeros((50, 1), dtype=torch.float64, device="cuda")
        if renorm:
            w = w / w.sum(1, keepdim=True)
            dot, size = (w * d).sum(1, keepdim=True), (w * d).abs().sum(1, keepdim=True)
        want, bound = torch.zeros_like(z, dtype=torch.float64), torch.zeros_like(z, dtype=torch.float64)
        want.scatter_(1, at, w * (d - dot) * slope)
        bound.scatter_(1, at, w * (d.abs() + size) * slope)
        close(out, want, U[dtype] * want.abs() + 1e-5 * bound + 1e-37)


@gpu
def test_route_gradient_of_a_softmax_in_32_bits():
    """Two experts far apart, the nearer one chosen: dlogits of the other is -s0 s1 d with s0 = exp(l0 - l1) to 2 ulp (2.4e-7), s1 = 1 and at most six
    roundings of 2^-24 (3.6e-7); 8e-7.  The difference is exact: both logits are multiples of 1/8."""
    rows = 640
    z = torch.zeros((rows, 2), device="cuda")
    z[:, 0] = -torch.arange(rows, device="cuda") / 8
    expert = torch.ones((rows, 1), dtype=torch.int32, device="cuda")
    dgate = 1 + torch.rand((rows, 1), generator=gen(3), device="cuda")
    out = torch.empty_like(z)
    ops.moe_ovl_route_backward(logits=z, expert=expert, dgate=dgate, dlogits=out, renormalise=False)
    p = torch.softmax(z.double(), 1)
    far = p[:, 0] < 2.0 ** -25                              # there s1 rounds to 1
    want = -p[:, 0] * p[:, 1] * dgate.double()[:, 0]
    close(out[far, 0], want[far], 8e-7 * want[far].abs())
    close(out[far, 1], -want[far], 1.2e-7 * dgate.double()[far, 0])


@gpu
@pytest.mark.parametrize("m,n,k,counts", [(3, 1000, 2048, None), (1, 512, 8192, None), (20, 256, 512, [10, 10]), (64, 4096, 4096, None), (700, 1024, 512, None),
                                          (300, 512, 512, [100, 0, 200]), (5, 28672, 1024, None), (2048, 4096, 4096, None), (1200, 2048, 2048, [900, 300])])
def test_quant_matmul_waits_that_give_up_with_copies_under_way(m, n, k, counts):
    """Calls whose waits give up at once, because their status says so already or because of a limit of 1 us, between calls that have to be
    right: a kernel that gave up leaves when its copies have landed, so the next one's shared and tensor memory is its own."""
    g = gen(m + n)
    e = 1 if counts is None else len(counts)
    a, b = make8(g, (m, k)), make8(g, (e, n, k))
    sa, sb = torch.rand(m, generator=g, device="cuda") * 1e-3, torch.rand((e, n), generator=g, device="cuda")
    dc = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    want, clear = torch.empty((m, n), dtype=BF16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    call = lambda out, status, **kw: ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, expert_counts=dc, status=status, **kw)  # noqa: E731
    call(want, clear)
    full = torch.full((m + 2, n), 7.5, dtype=BF16, device="cuda")
    out = torch.empty_like(want)
    for turn in range(12):
        aborted = torch.tensor([0, 1, 0, 0], dtype=torch.int32, device="cuda")
        call(full[1:m + 1], aborted)
        call(out, clear)
        assert torch.equal(out, want)
        late = torch.zeros(4, dtype=torch.int32, device="cuda")
        call(full[1:m + 1], late, wait_timeout_us=1)
        call(out, clear)
        assert torch.equal(out, want) and int(late[0]) in (0, B.ERR_TIMEOUT)
        assert bool((full[0] == 7.5).all()) and bool((full[m + 1] == 7.5).all())
    assert not clear.any()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d,pad", [(32761, 0), (32762, 0), (32765, 0), (32766, 0), (32767, 0), (32768, 1), (32768, 9), (32763, 5)])
def test_norm_and_gradient_of_the_widest_rows_that_begin_anywhere(d, pad, dtype):
    """Aligned bases, rows that are no multiple of 16 bytes apart, up to the widest: each row can touch one pack more than it fills."""
    g = gen(d + pad)
    for rows in (3, 310):
        wide = lambda t=dtype: torch.full((rows, d + pad), 7, dtype=t, device="cuda")  # noqa: E731
        x, r, h, y, q, dy, dx = wide(), wide(), wide(), wide(), wide(torch.int8), wide(), wide()
        cut = lambda m: m[:, :d]  # noqa: E731
        scale, rstd, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(d, device="cuda")
        for m in (x, r, dy):
            cut(m).copy_(normal(g, (rows, d), dtype))
        w = normal(g, (d,), dtype) + 1
        ops.moe_ovl_add_norm(x=cut(x), residual=cut(r), weight=w, residual_out=cut(h), y=cut(y), q=cut(q), scale=scale, rstd=rstd)
        assert torch.equal(cut(h), (cut(x).float() + cut(r).float()).to(dtype))
        v, rs = norm64(cut(h), w, 1e-6)
        close(rstd, rs, 4e-6 * rs)
        close(cut(y), v, (U[dtype] + 6e-6) * v.abs() + FLOOR[dtype])
        close(cut(q).double() * scale.double()[:, None], v, 0.502 * v.abs().amax(1, keepdim=True) / 127)
        ws = torch.empty(ops.moe_ovl_add_norm_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
        ops.moe_ovl_add_norm_backward(dy=cut(dy), h=cut(h), weight=w, rstd=rstd, d_residual=cut(r), dx=cut(dx), dweight=dw, workspace=ws)
        want, dw_want, size, dw_size = norm_backward64(cut(dy), cut(h), w, rstd, cut(r))
        close(cut(dx), want, U[dtype] * want.abs() + 1e-5 * size + FLOOR[dtype])
        close(dw, dw_want, 1e-5 * dw_size + 1e-30)
        for m in (h, y, q, dx):
            assert pad == 0 or bool((m[:, d:] == 7).all())


@gpu
def test_quant_matmul_one_channel_of_every_expert():
    """Experts of one channel each, cut out of larger ones: the distance of their rows is the experts'."""
    g = gen(21)
    a, whole = make8(g, (60, 64)), make8(g, (6, 10, 64))
    sa, sb = torch.rand(60, generator=g, device="cuda"), torch.rand((6, 1), generator=g, device="cuda")
    check_product(a, sa, whole[:, 3:4], sb, F32, [10, 0, 20, 5, 5, 20])
    check_product(a, sa, whole[2, 3:4], sb[0], F32)


def long_matrix(rows, cols, dtype, value):
    """All one value, but for eight rows at either end."""
    m = torch.full((rows, cols), value, dtype=dtype, device="cuda")
    ends = torch.arange(1, 17, device="cuda").view(16, 1).expand(16, cols).to(dtype)
    m[:8], m[-8:] = ends[:8], ends[8:]
    return m


def check_long(got, middle, ends):
    """got [rows]: `middle` all over, `ends` in the eight rows at either end; in parts, for the comparison's own memory."""
    assert torch.equal(got[:8], ends[:8]) and torch.equal(got[-8:], ends[8:])
    for part in got[8:-8].split(1 << 28):
        assert bool((part == middle).all())


MOST_ROWS = 2 ** 31 - 1


@gpu
def test_row_operators_of_the_longest_matrices():
    """As many rows as their count can say: one step behind the last row passes 2^31.  One column each; every row's result is that of a
    short matrix with the same value."""
    x = long_matrix(MOST_ROWS, 1, BF16, 3.0)
    short = torch.cat([x[:8], x[-8:], torch.full((1, 1), 3.0, dtype=BF16, device="cuda")])
    w = torch.full((1,), 1.5, dtype=BF16, device="cuda")

    def norm(m):
        rstd, y = torch.zeros(m.shape[0], device="cuda"), torch.zeros_like(m)
        ops.moe_ovl_add_norm(x=m, weight=w, eps=0.5, y=y, rstd=rstd)
        return y, rstd

    y, rstd = norm(x)
    ys, rs = norm(short)
    check_long(rstd, rs[16], rs[:16])
    check_long(y[:, 0], ys[16, 0], ys[:16, 0])
    dx = torch.zeros_like(x)
    ops.moe_ovl_add_norm_backward(dy=y, h=x, weight=w, rstd=rstd, dx=dx)
    ds = torch.zeros_like(short)
    ops.moe_ovl_add_norm_backward(dy=ys, h=short, weight=w, rstd=rs, dx=ds)
    check_long(dx[:, 0], ds[16, 0], ds[:16, 0])
    del y, dx, rstd
    scale, q = torch.zeros(MOST_ROWS, device="cuda"), torch.zeros((MOST_ROWS, 1), dtype=torch.int8, device="cuda")
    gate_up = x.expand(MOST_ROWS, 2).contiguous()
    ops.moe_ovl_swiglu_quant(gate_up=gate_up, q=q, scale=scale)
    ss, qs = torch.zeros(17, device="cuda"), torch.zeros((17, 1), dtype=torch.int8, device="cuda")
    ops.moe_ovl_swiglu_quant(gate_up=short.expand(17, 2).contiguous(), q=qs, scale=ss)
    check_long(scale, ss[16], ss[:16])
    check_long(q[:, 0], qs[16, 0], qs[:16, 0])


@gpu
def test_router_of_the_most_rows():
    x = long_matrix(MOST_ROWS, 1, BF16, 3.0)
    expert, gate = torch.full((MOST_ROWS, 1), -9, dtype=torch.int32, device="cuda"), torch.zeros((MOST_ROWS, 1), device="cuda")
    counts = torch.zeros(1, dtype=torch.int32, device="cuda")
    ops.moe_ovl_route(logits=x, expert=expert, gate=gate, counts=counts, score=ops.SCORE_SIGMOID, renormalise=False)
    short = torch.cat([x[:8], x[-8:], torch.full((1, 1), 3.0, dtype=BF16, device="cuda")])
    _, gs, _ = call_route(short, 1, score="sigmoid", renorm=False)
    check_long(gate[:, 0], gs[16, 0], gs[:16, 0])
    assert int(counts) == MOST_ROWS and all(not bool(part.any()) for part in expert[:, 0].split(1 << 28))
    dx = torch.full_like(x, 7.0)
    ops.moe_ovl_route_backward(logits=x, expert=expert, dgate=gate, dlogits=dx, score=ops.SCORE_SIGMOID, renormalise=False)
    ds = torch.zeros_like(short)
    ops.moe_ovl_route_backward(logits=short, expert=torch.zeros((17, 1), dtype=torch.int32, device="cuda"), dgate=gs, dlogits=ds, score=ops.SCORE_SIGMOID,
                               renormalise=False)
    check_long(dx[:, 0], ds[16, 0], ds[:16, 0])


@gpu
@pytest.mark.parametrize("long_a", [True, False])
def test_quant_matmul_of_the_longest_matrices(long_a):
    """As many tokens, or channels, as their count can say."""
    big, one = long_matrix(MOST_ROWS, 16, torch.int8, 3), torch.ones((1, 16), dtype=torch.int8, device="cuda")
    scale, unit = torch.full((MOST_ROWS,), 0.5, device="cuda"), torch.ones(1, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    out = torch.zeros((MOST_ROWS, 1) if long_a else (1, MOST_ROWS), dtype=BF16, device="cuda")
    if long_a:
        ops.moe_ovl_quant_matmul(a=big, a_scale=scale, b=one, b_scale=unit, out=out, status=status)
    else:
        ops.moe_ovl_quant_matmul(a=one, a_scale=unit, b=big, b_scale=scale, out=out, status=status)
    assert not status.any()
    check_long(out.view(-1), 24.0, torch.arange(1, 17, device="cuda").to(BF16) * 8)


@gpu
def test_a_gradient_is_not_lost_without_a_word():
    """Outputs are the caller's buffers and carry no gradient: an input that requires one is warned about, unless gradients are off."""
    g = gen(17)
    x, w, q = normal(g, (5, 64), BF16), normal(g, (64,), BF16), torch.empty((5, 64), dtype=torch.int8, device="cuda")
    y, s, half = torch.empty_like(x), torch.ones(5, device="cuda"), torch.empty((5, 32), dtype=torch.int8, device="cuda")
    expert, gate, status = torch.empty((5, 2), dtype=torch.int32, device="cuda"), torch.empty((5, 2), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    b, sb, out = make8(g, (8, 64)), torch.ones(8, device="cuda"), torch.empty((5, 8), device="cuda")
    grad = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [
        lambda f: ops.moe_ovl_add_norm(x=f(x), weight=w, y=y), lambda f: ops.moe_ovl_add_norm(x=x, weight=f(w), y=y),
        lambda f: ops.moe_ovl_add_norm(x=x, residual=f(x), weight=w, y=y, q=q, scale=s), lambda f: ops.moe_ovl_swiglu_quant(gate_up=f(x), q=half, scale=s),
        lambda f: ops.moe_ovl_route(logits=f(x), expert=expert, gate=gate),
        lambda f: ops.moe_ovl_quant_matmul(a=q, a_scale=f(s), b=b, b_scale=sb, out=out, status=status),
        lambda f: ops.moe_ovl_quant_matmul(a=q, a_scale=s, b=b, b_scale=f(sb), out=out, status=status),
    ]
    for call in calls:
        with pytest.warns(UserWarning, match="autograd"):
            call(grad)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            call(lambda t: t)
            with torch.no_grad():
                call(grad)
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", [40, 2050, 4096, 4099])
def test_quantised_values_are_rounded_products(d, dtype):
    """With weights of 1, a value over its row's largest is that of the inputs, and rstd is no part of it: in 8 bits it is the 32-bit product with the
    32-bit quotient 127 / max, rounded to a whole number, ties to even.  Both roundings are defined, so the values are equal."""
    g = gen(d + 1)
    x = normal(g, (700, d), dtype)
    q, scale = torch.empty((700, d), dtype=torch.int8, device="cuda"), torch.empty(700, device="cuda")
    most = x.float().abs().amax(1, keepdim=True)
    want = torch.round(x.float() * (torch.full_like(most, 127.0) / most)).to(torch.int8)
    for y in (None, torch.empty_like(x)):
        ops.moe_ovl_add_norm(x=x, weight=torch.ones(d, dtype=dtype, device="cuda"), y=y, q=q, scale=scale)
        assert torch.equal(q, want)
